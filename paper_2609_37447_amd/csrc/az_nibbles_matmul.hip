// out = a b^T + bias, b in 4 bits and a in 4 bits or e4m3 codes, the summed dimension along the rows of both.
//
// The scaled f8f6f4 matrix instruction takes both formats, each operand with a scale byte for each row and 32 columns:
// a block of the 4-bit format exactly.  Two 4-bit operands run at twice the rate of e4m3, and
// their products (multiples of 1/4 up to 36) are summed exactly.  With an e4m3 operand small products are
// cut (see the products of two e4m3 matrices), so that fp32 results of a coded a run on the bf16 instruction,
// for which codes times their scale are exact operands.
#include "az_matmul_common.h"
#include "az_nibbles_common.h"

namespace {

enum { E4M3 = 0, E2M1 = 4 };  // the instruction's format numbers

// Either kind of the left operand: scale_row(r) begins row r's scale bytes, one for each 32 (e2m1) or 128 columns.
struct LeftView {
  uint8_t* codes;
  uint8_t* scales;
  int64_t ld, ld_scales;
  int rows, cols, shift;
  __device__ __forceinline__ const uint8_t* scale_row(int64_t r) const { return scales + (r >> shift) * ld_scales; }
};

// A lane's 32 columns of step k (128 columns), zeros past cols.  The 16 x 16 x 128 instruction has lane group g's
// 4-bit columns at 32 g on, but 8-bit ones in two halves at 16 g and 64 + 16 g on.  (SPLIT; the bf16
// instruction takes any columns, if a and b agree.)
template <int FORMAT, bool SPLIT>
__device__ __forceinline__ cm_i32x8 fragment(const uint8_t* row, int k, int g, int cols) {
  if constexpr (FORMAT == E2M1) {
    const cm_i32x4 v = nibble_chunk(row, 4 * k + g, cols);
    return cm_i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
  } else {
    const int c = k * CB + g * (SPLIT ? 16 : 32);
    const cm_i32x4 lo = code_chunk(row, c, cols), hi = code_chunk(row, c + (SPLIT ? 64 : 16), cols);
    return cm_i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  }
}

// Eight codes (the i-th eight of a fragment) as exact bf16 values.
template <int FORMAT>
__device__ __forceinline__ cm_bf16x8 values8(const cm_i32x8& w, int i, float s) {
  cm_i32x4 u;
  if constexpr (FORMAT == E2M1) {
    const uint32_t c = (uint32_t)w[i];
    u = cm_i32x4{__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0)), __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1)),
                 __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2)), __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3))};
  } else {
    u = cm_i32x4{(int)code_pair_bf16<false>((uint32_t)w[2 * i], s), (int)code_pair_bf16<true>((uint32_t)w[2 * i], s),
                 (int)code_pair_bf16<false>((uint32_t)w[2 * i + 1], s), (int)code_pair_bf16<true>((uint32_t)w[2 * i + 1], s)};
  }
  return __builtin_bit_cast(cm_bf16x8, u);
}

// Few rows of a.  A workgroup of eight waves owns 16 rows of a times 16 rows of b.  Each wave takes DU neighbouring
// steps of 128 columns of every DW * DU: b's codes go through LDS of its own, copied as 512 neighbouring bytes of a row (chunks
// exchanged by the row against bank conflicts), a row's scale bytes are loaded by four lanes and handed to the
// others, a's codes come straight.  The waves' sums meet in LDS in the order of the waves.
// 1 x 4672 x 8192, e4m3 a: 9.2 us; with each lane loading its own blocks and scales of b 12.3.
constexpr int DW = 8, DU = 8, DROW = DU * 64;  // bytes of a row of b that a wave has

template <int A, bool EXACT>
struct DirectStep {
  cm_i32x8 a, b;
  uint32_t sa, sb;
  __device__ __forceinline__ void add_to(cm_f32x4& acc) const {
    if constexpr (!EXACT) {
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, E2M1, A, 0, (int)sb, 0, (int)sa);
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<E2M1>(b, q, scale_value(sb)), values8<A>(a, q, scale_value(sa)), acc, 0, 0, 0);
    }
  }
};

template <int A, bool EXACT, bool F32>
__global__ __launch_bounds__(DW * 64) void az_nibble_direct(LeftView a, NibbleView b, const float* __restrict__ bias,
                                                            void* __restrict__ out, int64_t ldo, int nt) {
  __shared__ __attribute__((aligned(16))) uint8_t tiles[DW][16 * DROW];  // and the waves' sums, afterwards
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int m0 = (int)(blockIdx.x / (uint32_t)nt) * 16, n0 = (int)(blockIdx.x % (uint32_t)nt) * 16;
  const int64_t am = min((int64_t)m0 + r, (int64_t)a.rows - 1), bn = min((int64_t)n0 + r, (int64_t)b.rows - 1);
  const uint8_t *ar = a.codes + am * a.ld, *br = b.codes + bn * b.ld;
  const uint8_t *as = a.scale_row(am), *bs = b.scales + bn * b.ld_scales;
  const int whole = a.cols / CB;
  const int bytes = (min(b.rows - n0, 16) - 1) * (int)b.ld + (a.cols + NB - 1) / NB * 16;
  cm_f32x4 acc = {0, 0, 0, 0}, add = {0, 0, 0, 0};
  if (bias && wave == 0) {
#pragma unroll
    for (int e = 0; e < 4; e++) add[e] = bias[min((int64_t)n0 + 4 * g + e, (int64_t)b.rows - 1)];
  }
  for (int k0 = wave * DU; k0 < whole; k0 += DW * DU) {
    constexpr int CHUNKS = DROW / 16, ROWS = 64 / CHUNKS;  // of a row, and rows of a copy
    // From these steps on to the matrix's end: rows past it are out of the buffer's range and read as zeros.
    const __amdgpu_buffer_rsrc_t bbuf = __builtin_amdgcn_make_buffer_rsrc(b.codes + n0 * b.ld + k0 * 64, 0, bytes - k0 * 64, 0x00027000);
#pragma unroll
    for (int j = 0; j < 16 / ROWS; j++) {
      const int row = j * ROWS + lane / CHUNKS, chunk = lane % CHUNKS ^ row;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(bbuf, (lds_bytes*)&tiles[wave][j * 1024], 16, row * (int)b.ld + chunk * 16, 0, 0, 0);
    }
    // Steps 2 g and 2 g + 1 of the row; past the end the last one.
    uint32_t sa[2], sb[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int k = min(k0 + 2 * g + i, whole - 1);
      sb[i] = *reinterpret_cast<const uint32_t*>(bs + 4 * k);
      if constexpr (A == E2M1) sa[i] = *reinterpret_cast<const uint32_t*>(as + 4 * k);
      else sa[i] = as[k];
    }
    DirectStep<A, EXACT> s[DU];
#pragma unroll
    for (int u = 0; u < DU; u++) {
      const int k = min(k0 + u, whole - 1);
      if constexpr (A == E2M1) {
        const cm_i32x4 y = *reinterpret_cast<const cm_i32x4*>(ar + (int64_t)k * 64 + g * 16);
        s[u].a = cm_i32x8{y[0], y[1], y[2], y[3], 0, 0, 0, 0};
      } else {
        const uint8_t* at = ar + (int64_t)k * CB + g * (EXACT ? 32 : 16);
        const cm_i32x4 y = *reinterpret_cast<const cm_i32x4*>(at), z = *reinterpret_cast<const cm_i32x4*>(at + (EXACT ? 16 : 64));
        s[u].a = cm_i32x8{y[0], y[1], y[2], y[3], z[0], z[1], z[2], z[3]};
      }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < DU; u++) {
      const cm_i32x4 x = *reinterpret_cast<const cm_i32x4*>(&tiles[wave][r * DROW + (((4 * u + g) ^ r) * 16)]);
      s[u].b = cm_i32x8{x[0], x[1], x[2], x[3], 0, 0, 0, 0};
      // (past the end the codes count as zeros, which adds nothing but a NaN that is in the result already)
      if (u > 0) s[u].b &= -(int)(k0 + u < whole);
      s[u].sb = (__shfl(sb[u & 1], r + 16 * (u >> 1)) >> (8 * g)) & 0xffu;
      s[u].sa = __shfl(sa[u & 1], r + 16 * (u >> 1));
      if constexpr (A == E2M1) s[u].sa = (s[u].sa >> (8 * g)) & 0xffu;
      s[u].add_to(acc);
    }
    __builtin_amdgcn_s_waitcnt(0);  // the reads are back before the next copies overwrite what they read
    __builtin_amdgcn_sched_barrier(0);
  }
  if (a.cols % CB && wave == whole / DU % DW) {  // the columns that do not fill a step
    const int last = min(4 * whole + g, (a.cols - 1) / NB);  // (past cols: zeros, with the last block's scale)
    const DirectStep<A, EXACT> s = {fragment<A, !EXACT>(ar, whole, g, a.cols), fragment<E2M1, !EXACT>(br, whole, g, a.cols),
                                    as[A == E2M1 ? last : whole], bs[last]};
    s.add_to(acc);
  }
  __syncthreads();  // every wave is done with its tile
  cm_f32x4* const part = reinterpret_cast<cm_f32x4*>(&tiles[0][0]);
  if (wave > 0) part[(wave - 1) * 64 + lane] = acc;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < DW - 1; w++) acc += part[w * 64 + lane];
  acc += add;
  const int64_t m = (int64_t)m0 + r;
  if (m >= a.rows) return;
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const int64_t n = (int64_t)n0 + 4 * g + e;
    if (n >= b.rows) continue;
    const float v = acc[e];
    if constexpr (F32) ((float*)out)[m * ldo + n] = v;
    else ((uint16_t*)out)[m * ldo + n] = bf16_of(v);
  }
}

// More rows of a.  Four waves own a tile of TM rows of a and TN rows of b, WM x WN parts of FA x FB blocks of 32 x 32.
// A K step is 128 bytes of a row of a: 256 columns in 4 bits, 128 in e4m3 (64 bytes of b).  Steps go straight from memory into
// LDS, two in turn; a wave reads the fragments of the next 64 columns while the matrix unit works on these.
//
// LDS rows' 16-byte chunks are exchanged by the row's place (chunk ^ (row / 2) % chunks), which spreads the
// rows that are read together over all banks; the copy into LDS puts lanes side by side, so that the exchange is
// made on the source address.
//
// Scale bytes are copied for 512 columns at a time, 16 bytes of a row: a step's own 8 bytes of each row would be twice as many
// requests as its codes.
template <int A, int FA_, int FB_, int WM, int WN, bool EXACT, bool F32>
struct Tiled {
  static constexpr int FA = FA_, FB = FB_, ACROSS = WM, TM = 32 * FA * WM, TN = 32 * FB * WN;
  static constexpr int STEP = A == E2M1 ? 256 : 128, SUBS = STEP / 64;  // columns, and matrix instructions a block
  static constexpr int BROW = STEP / 2;                                 // bytes of a row of b; a's are 128
  static constexpr int ASTEP = TM * 128, BSTEP = TN * BROW;
  static constexpr int AW = A == E2M1 ? 2 : 1, BW = STEP / 128;         // words of scale bytes of a row that a step takes
  static constexpr int GROUP = 512 / STEP;                              // steps that scales are copied for together
  static constexpr int SROW = A == E2M1 ? 16 : 8;                       // bytes of a row of a's: e4m3's are two words, of which it has four bytes
  static constexpr int SA = TM < 64 ? 64 : TM, ACOPIES = SA * SROW / (A == E2M1 ? 1024 : 256), COPIES = ACOPIES + TN / 64;
  static constexpr int STAGE = ASTEP + BSTEP, SCALES = 2 * STAGE, SGROUP = SA * SROW + TN * 16;
  static constexpr int USED = SCALES + 2 * SGROUP;
  static constexpr int OUT = TM * TN * (F32 ? 4 : 2) / (FA > 1 ? 2 : 1);  // what results need on their way out
  static constexpr int LDS = USED > OUT ? USED : OUT;
  static constexpr int AROWS = 32, BROWS = 4096 / BROW;                 // rows that one copy instruction of the workgroup fills
  static constexpr int TURNS = (COPIES + 3) / 4;
  static_assert(WM * WN == 4 && TM % AROWS == 0 && TN % BROWS == 0, "four waves' work");

  struct Frag {
    cm_i32x8 a[FA], b[FB];
  };

  template <int BYTES>
  static __device__ __forceinline__ void copy_scales(__amdgpu_buffer_rsrc_t rows, uint32_t off, lds_bytes* to) {
    if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, to, 16, off, 0, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, to, 4, off, 0, 0, 0);
  }
  // A thread's chunks of a step, BYTES of LDS apart: `off` in the tile's first step, `at` the step's place in a row.
  template <int CHUNKS, int BYTES>
  static __device__ __forceinline__ void copy(__amdgpu_buffer_rsrc_t tile, const uint32_t* off, int at, lds_bytes* to) {
#pragma unroll
    for (int j = 0; j < CHUNKS; j++) __builtin_amdgcn_raw_ptr_buffer_load_lds(tile, to + j * BYTES, 16, off[j], at, 0, 0);
  }
  // Spreads LDS reads and copies over the matrix instructions of 64 columns, reads first.
  template <bool LAST>
  static __device__ __forceinline__ void interleave() {
    if constexpr (!EXACT) {
#pragma unroll
      for (int i = 0; i < FA * FB; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction
        if (i < FA + FB) __builtin_amdgcn_sched_group_barrier(0x100, LAST ? 3 : A == E2M1 ? 1 : 2, 0);  // LDS reads
        else if (LAST) __builtin_amdgcn_sched_group_barrier(0x020, 3, 0);                               // copies
      }
    }
  }
  // Chunks of a's fragment of 64 columns s: 32 columns of e4m3 are two, where the instruction wants them (16 h and
  // 32 + 16 h on); for the bf16 instruction they follow each other, as b's.
  static __device__ __forceinline__ int a_chunk(int s, int h, int i) {
    return A == E2M1 ? 2 * s + h : EXACT ? 4 * s + 2 * h + i : 4 * s + 2 * i + h;
  }
  template <int S>
  static __device__ __forceinline__ void read(Frag& f, const uint8_t* ap, const uint8_t* bp, int h, int sa, int sb) {
    const int c0 = (a_chunk(S, h, 0) ^ sa) * 16, c1 = (a_chunk(S, h, 1) ^ sa) * 16, cb = ((2 * S + h) ^ sb) * 16;
#pragma unroll
    for (int i = 0; i < FA; i++) {
      const cm_i32x4 x = *reinterpret_cast<const cm_i32x4*>(ap + i * 32 * 128 + c0);
      cm_i32x4 y = {};
      if constexpr (A == E4M3) y = *reinterpret_cast<const cm_i32x4*>(ap + i * 32 * 128 + c1);
      f.a[i] = cm_i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    }
#pragma unroll
    for (int j = 0; j < FB; j++) {
      const cm_i32x4 x = *reinterpret_cast<const cm_i32x4*>(bp + j * 32 * BROW + cb);
      f.b[j] = cm_i32x8{x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    }
  }
  // 64 columns; the scale bytes are byte OA of sa and byte OB of sb.
  template <int OA, int OB>
  static __device__ __forceinline__ void multiply(cm_f32x16 (&acc)[FA][FB], const Frag& f, const uint32_t (&sa)[FA], const uint32_t (&sb)[FB]) {
    if constexpr (!EXACT) {
#pragma unroll
      for (int i = 0; i < FA; i++)
#pragma unroll
        for (int j = 0; j < FB; j++)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f.b[j], f.a[i], acc[i][j], E2M1, A, OB, (int)sb[j], OA, (int)sa[i]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++) {
        cm_bf16x8 va[FA], vb[FB];
#pragma unroll
        for (int i = 0; i < FA; i++) va[i] = values8<A>(f.a[i], q, scale_value((sa[i] >> (8 * OA)) & 0xffu));
#pragma unroll
        for (int j = 0; j < FB; j++) vb[j] = values8<E2M1>(f.b[j], q, scale_value((sb[j] >> (8 * OB)) & 0xffu));
#pragma unroll
        for (int i = 0; i < FA; i++)
#pragma unroll
          for (int j = 0; j < FB; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[j], va[i], acc[i][j], 0, 0, 0);
      }
    }
  }
};

// 8192^3: 272-294 us in 4 bits by card and heat (3,740-4,040 TFLOP/s, matrix unit busy 46%: two steps on their way cannot hide
// the copies' way), 441-452 with an e4m3 a.
template <int A, int FA, int FB, int WM, int WN, bool EXACT, bool F32>
__global__ __launch_bounds__(256, FA * FB == 16 ? 1 : 2) void az_nibble_tiled(LeftView a, NibbleView b, const float* __restrict__ bias,
                                                                              void* __restrict__ out, int64_t ldo, int mt, int nt,
                                                                              int part_steps, int64_t part_stride) {
  using K = Tiled<A, FA, FB, WM, WN, EXACT, F32>;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  int tm, tn;
  tile_of(blockIdx.x, mt, nt, tm, tn);
  // The last tile of a side ends with the matrix: what it shares with the tile before is computed
  // twice, to the same bits.  A matrix of fewer rows than a tile is the one tile's beginning.
  const int m0 = max(min(tm * K::TM, a.rows - K::TM), 0), n0 = max(min(tn * K::TN, b.rows - K::TN), 0);
  const int ms = min(a.rows, K::TM), ns = min(b.rows, K::TN);

  // Copying: a lane takes one chunk of one row of those that an instruction of its wave fills; for a row past the matrix,
  // of no result, its last one: the scalar offset is the step's alone, and no copy of codes leaves the matrix whatever a buffer's
  // range counts (against rows by the scalar offset and zeros past the range: the same within 1%, 333 x 1880 3% less).
  const int arow = 8 * wave + (lane >> 3), achunk = (lane & 7) ^ ((arow >> 1) & 7);
  constexpr int BC = K::BROW / 16;  // chunks of a row of b
  const int brow = K::BROWS / 4 * wave + lane / BC, bchunk = (lane % BC) ^ ((brow >> 1) & (BC - 1));
  uint32_t aoff[K::TM / K::AROWS], boff[K::TN / K::BROWS];
#pragma unroll
  for (int j = 0; j < K::TM / K::AROWS; j++) aoff[j] = (uint32_t)min(j * K::AROWS + arow, ms - 1) * (uint32_t)a.ld + achunk * 16;
#pragma unroll
  for (int j = 0; j < K::TN / K::BROWS; j++) boff[j] = (uint32_t)min(j * K::BROWS + brow, ns - 1) * (uint32_t)b.ld + bchunk * 16;
  const int blocks = (a.cols + NB - 1) / NB, awidth = A == E2M1 ? blocks * 16 : (a.cols + 15) & ~15;
  const __amdgpu_buffer_rsrc_t abuf = __builtin_amdgcn_make_buffer_rsrc(a.codes + m0 * a.ld, 0, (ms - 1) * (int)a.ld + awidth, 0x00027000);
  const __amdgpu_buffer_rsrc_t bbuf = __builtin_amdgcn_make_buffer_rsrc(b.codes + n0 * b.ld, 0, (ns - 1) * (int)b.ld + blocks * 16, 0x00027000);
  lds_bytes* const alds = (lds_bytes*)smem + 8 * wave * 128;
  lds_bytes* const blds = (lds_bytes*)smem + K::ASTEP + K::BROWS / 4 * wave * K::BROW;
  // The part's steps, of which `whole` is the first that does not fill its columns or is not the part's.
  const int first = (int)blockIdx.y * part_steps, last = min(first + part_steps, (a.cols + K::STEP - 1) / K::STEP), whole = min(last, a.cols / K::STEP);
  // Scales: copies of 64 rows' 16 bytes, or of 32 rows' two words of an e4m3 matrix (ScaleWords: the word that holds a byte), a's
  // and then b's, dealt to the waves in turn.
  const CodeView codes = {a.codes, a.scales, a.ld, a.rows, a.cols, (int)a.ld_scales, a.shift};
  const ScaleWords aw(codes);
  const __amdgpu_buffer_rsrc_t awords = A == E2M1 ? __builtin_amdgcn_make_buffer_rsrc(a.scales + m0 * a.ld_scales, 0, (ms - 1) * (int)a.ld_scales + ((blocks + 3) & ~3), 0x00027000) : aw.words;
  const __amdgpu_buffer_rsrc_t bwords = __builtin_amdgcn_make_buffer_rsrc(b.scales + n0 * b.ld_scales, 0, (ns - 1) * (int)b.ld_scales + ((blocks + 3) & ~3), 0x00027000);
  uint32_t srow[K::TURNS];
#pragma unroll
  for (int i = 0; i < K::TURNS; i++) {
    const int copy = i * 4 + wave;
    if (copy >= K::ACOPIES) srow[i] = (uint32_t)min((copy - K::ACOPIES) * 64 + lane, ns - 1) * (uint32_t)b.ld_scales;
    else if (A == E2M1) srow[i] = (uint32_t)min(copy * 64 + lane, ms - 1) * (uint32_t)a.ld_scales;
    else srow[i] = (aw.place(codes, m0 + min(copy * 32 + lane / 2, ms - 1)) & ~3u) + 4 * (lane & 1);
  }
  lds_bytes* const slds = (lds_bytes*)smem + K::SCALES;
  // (past the last step: that step again, which nothing reads)
  auto fetch = [&](int kb) {
    const int stage = (kb & 1) * K::STAGE;
    if (kb < whole && (kb % K::GROUP == 0 || kb == first)) {
      const int group = kb / K::GROUP;
      lds_bytes* const to = slds + (group & 1) * K::SGROUP;
#pragma unroll
      for (int i = 0; i < K::TURNS; i++) {
        const int copy = i * 4 + wave;
        if (copy < K::ACOPIES) {
          if constexpr (A == E2M1) K::template copy_scales<16>(awords, srow[i] + group * 16, to + copy * 1024);
          else K::template copy_scales<4>(awords, srow[i] + group * 4, to + copy * 256);
        } else if (copy < K::COPIES) {
          K::template copy_scales<16>(bwords, srow[i] + group * 16, to + K::SA * K::SROW + (copy - K::ACOPIES) * 1024);
        }
      }
    }
    kb = min(kb, whole - 1);
    K::template copy<K::TM / K::AROWS, K::AROWS * 128>(abuf, aoff, kb * 128, alds + stage);
    K::template copy<K::TN / K::BROWS, K::BROWS * K::BROW>(bbuf, boff, kb * K::BROW, blds + stage);
  };

  // Reading: a lane holds row l % 32 of a block, its block of 32 columns l / 32.
  const int r = lane & 31, h = lane >> 5, wm = (wave % WM) * 32 * FA, wn = (wave / WM) * 32 * FB;
  const int sa_ = (r >> 1) & 7, sb_ = (r >> 1) & (BC - 1);
  const uint8_t* ap = smem + (wm + r) * 128;
  const uint8_t* bp = smem + K::ASTEP + (wn + r) * K::BROW;
  uint32_t ac[FA];  // e4m3: which byte of its first word the lane's row of scales begins with
#pragma unroll
  for (int i = 0; i < FA; i++) ac[i] = A == E2M1 ? 0 : aw.place(codes, m0 + min(wm + 32 * i + r, ms - 1)) & 3;
  // A 4-bit operand's words are moved down by its lane's byte, so that 64 columns s have theirs at byte 2 (s % 2) of word s / 2.
  uint32_t sa[K::AW][FA], sb[K::BW][FB], na[K::AW][FA], nb[K::BW][FB];
  auto scale_words = [&](int kb) {
    const uint8_t* from = smem + K::SCALES + (kb / K::GROUP & 1) * K::SGROUP;
    const int at = kb % K::GROUP;
#pragma unroll
    for (int i = 0; i < FA; i++) {
      const uint8_t* row = from + (wm + 32 * i + r) * K::SROW;
      if constexpr (A == E2M1) {
        const cm_i32x2 w = *reinterpret_cast<const cm_i32x2*>(row + at * 8);
        na[0][i] = (uint32_t)w[0];
        na[K::AW - 1][i] = (uint32_t)w[1];
      } else {
        na[0][i] = *reinterpret_cast<const uint32_t*>(row + ((ac[i] + at) & 4));
      }
    }
#pragma unroll
    for (int j = 0; j < FB; j++) {
      const uint8_t* row = from + K::SA * K::SROW + (wn + 32 * j + r) * 16;
      if constexpr (K::BW == 2) {
        const cm_i32x2 w = *reinterpret_cast<const cm_i32x2*>(row + at * 8);
        nb[0][j] = (uint32_t)w[0];
        nb[K::BW - 1][j] = (uint32_t)w[1];
      } else {
        nb[0][j] = *reinterpret_cast<const uint32_t*>(row + at * 4);
      }
    }
  };
  auto scales = [&](int kb) {
#pragma unroll
    for (int w = 0; w < K::AW; w++)
#pragma unroll
      for (int i = 0; i < FA; i++) sa[w][i] = na[w][i] >> (A == E2M1 ? 8 * h : (int)(8 * (ac[i] + kb) & 31));
#pragma unroll
    for (int w = 0; w < K::BW; w++)
#pragma unroll
      for (int j = 0; j < FB; j++) sb[w][j] = nb[w][j] >> (8 * h);
  };

  cm_f32x16 acc[FA][FB];
#pragma unroll
  for (int i = 0; i < FA; i++)
#pragma unroll
    for (int j = 0; j < FB; j++) acc[i][j] = cm_f32x16{};
  typename K::Frag f[2];
  if (whole > first) {
    const int stage = (first & 1) * K::STAGE;
    fetch(first);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    fetch(first + 1);
    scale_words(first);
    scales(first);
    K::template read<0>(f[0], ap + stage, bp + stage, h, sa_, sb_);
  }
  constexpr bool FOUR = A == E2M1;
  for (int kb = first; kb < whole; kb++) {
    const int stage = (kb & 1) * K::STAGE, next = K::STAGE - stage;
    K::template read<1>(f[1], ap + stage, bp + stage, h, sa_, sb_);
    K::template multiply<0, 0>(acc, f[0], sa[0], sb[0]);
    K::template interleave<false>();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (K::SUBS == 4) {
      K::template read<2>(f[0], ap + stage, bp + stage, h, sa_, sb_);
      K::template multiply<2, 2>(acc, f[1], sa[0], sb[0]);
      K::template interleave<false>();
      __builtin_amdgcn_sched_barrier(0);
      K::template read<3>(f[1], ap + stage, bp + stage, h, sa_, sb_);
      K::template multiply<0, 0>(acc, f[0], sa[K::AW - 1], sb[K::BW - 1]);
      K::template interleave<false>();
      __builtin_amdgcn_sched_barrier(0);
    }
    // This wave's reads of step kb are done and its copies of step kb + 1 have landed; after the
    // barrier that holds for every wave.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    // (after the last step these are the bytes of the step before: read, not used)
    K::template read<0>(f[0], ap + next, bp + next, h, sa_, sb_);
    scale_words(kb + 1);
    fetch(kb + 2);
    K::template multiply<FOUR ? 2 : 0, 2>(acc, f[1], sa[K::AW - 1], sb[K::BW - 1]);
    K::template interleave<true>();
    scales(kb + 1);
  }
  __builtin_amdgcn_s_waitcnt(0);  // no copy into LDS is under way when the workgroup ends
  if (whole < last) {  // the columns that do not fill a step, straight from memory
    for (int s = 0; s < K::SUBS; s++) {
      const int kb = whole * (K::STEP / NB) + 2 * s + h, at = min(kb, blocks - 1);  // (past cols: zeros, with the last block's scale)
      uint32_t ta[FA], tb[FB];
#pragma unroll
      for (int i = 0; i < FA; i++) {
        const int64_t row = m0 + min(wm + 32 * i + r, ms - 1);
        ta[i] = a.scale_row(row)[FOUR ? at : whole];
        if constexpr (FOUR) {
          const cm_i32x4 x = nibble_chunk(a.codes + row * a.ld, kb, a.cols);
          f[0].a[i] = cm_i32x8{x[0], x[1], x[2], x[3], 0, 0, 0, 0};
        } else {
          const cm_i32x4 x = code_chunk(a.codes + row * a.ld, whole * CB + 16 * K::a_chunk(s, h, 0), a.cols);
          const cm_i32x4 y = code_chunk(a.codes + row * a.ld, whole * CB + 16 * K::a_chunk(s, h, 1), a.cols);
          f[0].a[i] = cm_i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        }
      }
#pragma unroll
      for (int j = 0; j < FB; j++) {
        const int64_t row = n0 + min(wn + 32 * j + r, ns - 1);
        tb[j] = b.scales[row * b.ld_scales + at];
        const cm_i32x4 x = nibble_chunk(b.codes + row * b.ld, kb, a.cols);
        f[0].b[j] = cm_i32x8{x[0], x[1], x[2], x[3], 0, 0, 0, 0};
      }
      K::template multiply<0, 0>(acc, f[0], ta, tb);
    }
  }
  write_tile<K, F32>(acc, smem, bias, (uint8_t*)out + (blockIdx.y * part_stride + (int64_t)m0 * ldo + n0) * (F32 ? 4 : 2), ldo, n0, ms, ns, wave, r, h);
}

// How a product runs: the kernel, and `parts` parts of the columns of part_steps K steps each.
enum { DIRECT = 0, TILE32 = 1, TILE64 = 2, TILE128 = 3, TILE256 = 4 };
struct Plan {
  int kind, parts, part_steps;
};

// What a product multiplies with: two 4-bit operands, an e4m3 one on the scaled instruction, or on the bf16 one.
enum Mode { FOURS = 0, MIXED = 1, EXACT = 2 };

// The plan with the least estimated time, in microseconds.  Few rows: what a workgroup costs by the columns, more where a has
// several rows to fetch.  Tiles: a K step takes a workgroup `one` alone on a compute unit and `all` with `occ` of them
// there, a round a start and an end, and every byte of an operand that a tile reads a little, which is what small tiles
// lose by.  Parts cost a second launch and their way through memory.  The figures are fitted to the times of every kernel, in one
// to eight parts, at 24 sizes from 1 x 1880 x 10240 to 4096^3; at these sizes the choice is 1% slower than the best on
// average, 20% at the worst (32 x 4672 x 4096 with an e4m3 a goes to the kernel of few rows, 12.9; 32-row tiles in four parts 10.8).
// Chosen against others, two 4-bit operands: 1 x 4672 x 8192 few rows 8.8 (32-row tiles in 8 parts 10.9); 40 x 4672 x 8192
// 32-row tiles in 4 parts 13.4 (few rows 19); 333 x 1880 x 10240 64-row in 4 parts 19.2 (32-row in one 27); 1024 x 4672 x 8192
// 128-row 37.7 (64-row 51.9, 256-row 59.9); 4096^3 256-row 43.7 (128-row 48.9).  The 256-row tile is not used in parts, where it
// was never the best by more than the noise, and not built for fp32 results of an e4m3 a, where it gains at whole rounds (4096^3
// 108, 128-row 113; 8192^3 770 for 827) and loses between them (8192 x 4672 x 8192 548 for 498).
Plan choose_plan(int64_t m, int64_t n, int64_t k, Mode mode, bool f32, bool fits) {
  struct Tile {
    int kind, tm, tn, occ;
    double one[3], all[3];
  };
  static const Tile tiles[] = {{TILE32, 32, 128, 3, {0.391, 0.363, 0.374}, {0.549, 0.467, 0.558}},
                               {TILE64, 64, 128, 3, {0.527, 0.471, 0.502}, {0.745, 0.613, 0.867}},
                               {TILE128, 128, 128, 2, {0.723, 0.634, 0.807}, {0.828, 0.791, 1.180}},
                               {TILE256, 256, 256, 1, {1.865, 1.682, 0.0}, {2.003, 1.461, 0.0}}};
  struct Rest {
    double few, few_k, few_group, few_row, tiled, round, part, part_bytes, traffic;
  };
  static const Rest rest[] = {{3.638, 1.781, 2.005, 1.520, 4.240, 1.121, 3.256, 0.673, 0.019e-6},
                              {4.328, 1.537, 1.790, 3.503, 4.562, 0.019, 3.915, 0.713, 0.008e-6},
                              {6.344, 0.000, 3.155, 4.218, 5.833, 0.000, 2.712, 0.706, 0.020e-6}};
  const Rest& c = rest[mode];
  const int columns = mode == FOURS ? 256 : 128, nb = (int)((k + columns - 1) / columns);
  const double write = 1.0 / 4.5e6;  // microseconds a byte
  const double out = (double)m * (double)n * (f32 ? 4 : 2) * write;
  Plan best = {DIRECT, 1, nb};
  const int64_t few = ((n + 15) / 16) * ((m + 15) / 16);
  double least = c.few + (double)k / 8192 * (c.few_k + (double)few / 256 * (c.few_group + c.few_row * (double)(m < 16 ? m : 16) / 16)) + out;
  if (!fits) return best;
  for (const Tile& t : tiles) {
    if (t.kind == TILE256 && mode == EXACT) continue;
    const int64_t count = ((m + t.tm - 1) / t.tm) * ((n + t.tn - 1) / t.tn);
    for (int parts = 1; parts <= (t.kind == TILE256 ? 1 : 8) && (parts == 1 || 2 * parts <= nb); parts *= 2) {
      const int steps = (nb + parts - 1) / parts, used = (nb + steps - 1) / steps;
      const int64_t groups = count * used, per = (groups + 255) / 256, slots = 256 * t.occ;
      const int occ = per < t.occ ? (int)per : t.occ;
      const double step = t.occ == 1 ? (per > 1 ? t.all[mode] : t.one[mode]) : t.one[mode] + (t.all[mode] - t.one[mode]) * (occ - 1) / (t.occ - 1);
      const double bytes = 128.0 * (t.tm + (mode == FOURS ? t.tn : t.tn / 2));  // of a step
      double cost = c.tiled + (double)((groups + slots - 1) / slots) * (steps * step + c.round) + (double)groups * steps * bytes * c.traffic + out;
      if (used > 1) cost += c.part + (double)used * (double)m * (double)n * 8 * write * c.part_bytes;
      if (cost < least) {
        least = cost;
        best = {t.kind, used, steps};
      }
    }
  }
  return best;
}

struct Operands {
  LeftView a;
  NibbleView b;
  const float* bias;
  void* out;
  int64_t ldo, part_stride;
  hipStream_t stream;
};

template <int A, bool EXACT, bool F32>
int launch_direct(const Operands& o) {
  const int64_t nt = ((int64_t)o.b.rows + 15) / 16, groups = nt * (((int64_t)o.a.rows + 15) / 16);
  if (!grid_fits(groups, DW * 64)) return AZ_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((az_nibble_direct<A, EXACT, F32>), dim3((unsigned)groups), dim3(DW * 64), 0, o.stream, o.a, o.b, o.bias, o.out, o.ldo, (int)nt);
  return AZ_OK;
}

template <int A, int FA, int FB, int WM, int WN, bool EXACT, bool F32>
int launch_tiled(const Plan& p, const Operands& o) {
  using K = Tiled<A, FA, FB, WM, WN, EXACT, F32>;
  const int64_t mt = ((int64_t)o.a.rows + K::TM - 1) / K::TM, nt = ((int64_t)o.b.rows + K::TN - 1) / K::TN;
  if (!grid_fits(mt * nt, 256)) return AZ_ERR_UNSUPPORTED;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(az_nibble_tiled<A, FA, FB, WM, WN, EXACT, F32>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, K::LDS);
  if (e != hipSuccess) return AZ_ERR_DEVICE;
  hipLaunchKernelGGL((az_nibble_tiled<A, FA, FB, WM, WN, EXACT, F32>), dim3((unsigned)(mt * nt), p.parts), dim3(256), K::LDS, o.stream,
                     o.a, o.b, o.bias, o.out, o.ldo, (int)mt, (int)nt, p.part_steps, o.part_stride);
  return AZ_OK;
}

template <int A, bool EXACT, bool F32>
int launch_tiles(const Plan& p, const Operands& o) {
  if constexpr (A == E2M1 || !F32) {
    if (p.kind == TILE256) return launch_tiled<A, 4, 4, 2, 2, EXACT, F32>(p, o);
  }
  return p.kind == TILE128  ? launch_tiled<A, 2, 2, 2, 2, EXACT, F32>(p, o)
         : p.kind == TILE64 ? launch_tiled<A, 1, 2, 2, 2, EXACT, F32>(p, o)
                            : launch_tiled<A, 1, 1, 1, 4, EXACT, F32>(p, o);
}

// A tile's offsets stay below 2^30.
bool tile_fits(const LeftView& a, const NibbleView& b) {
  constexpr int64_t most = 1 << 22;
  return a.ld < most && a.ld_scales < most && b.ld < most && b.ld_scales < most;
}

Plan plan_of(const LeftView& a, const NibbleView& b, int format, int32_t dtype) {
  return choose_plan(a.rows, b.rows, a.cols, format == E2M1 ? FOURS : dtype == AZ_F32 ? EXACT : MIXED, dtype == AZ_F32, tile_fits(a, b));
}

size_t workspace_of(const LeftView& a, const NibbleView& b, int format, int32_t dtype) {
  const Plan p = plan_of(a, b, format, dtype);
  return p.parts > 1 ? (size_t)p.parts * (size_t)a.rows * (size_t)b.rows * sizeof(float) : 0;
}

// The product by its plan, out or the parts' fp32 sums.  F32 of MIXED operands is for parts only: whole fp32 results are EXACT.
int run_plan(const Plan& p, const Operands& o, int format, bool exact, bool f32) {
  if (p.kind == DIRECT) {
    if (format == E2M1) return f32 ? launch_direct<E2M1, false, true>(o) : launch_direct<E2M1, false, false>(o);
    return f32 ? launch_direct<E4M3, true, true>(o) : launch_direct<E4M3, false, false>(o);
  }
  if (format == E2M1) return f32 ? launch_tiles<E2M1, false, true>(p, o) : launch_tiles<E2M1, false, false>(p, o);
  if (exact) return launch_tiles<E4M3, true, true>(p, o);
  return f32 ? launch_tiles<E4M3, false, true>(p, o) : launch_tiles<E4M3, false, false>(p, o);
}

int matmul(const LeftView& a, int format, const NibbleView& b, const float* bias, void* out, int32_t dtype, int64_t ld_out,
           void* workspace, size_t workspace_bytes, void* stream, const char* who) {
  if (a.cols != b.cols) return code_fail(AZ_ERR_INVALID_ARG, who, "a and b differ in cols");
  if (dtype != AZ_F32 && dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (a.rows == 0 || b.rows == 0) return AZ_OK;
  int st = dense_check(out, dtype, ld_out, b.rows, who);
  if (st != AZ_OK) return st;
  if ((uintptr_t)bias & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "bias must be 4-byte aligned");
  if (a.ld >= (1 << 27) || b.ld >= (1 << 27) || (format == E2M1 && a.ld_scales >= (1 << 26)) || b.ld_scales >= (1 << 26))
    return code_fail(AZ_ERR_UNSUPPORTED, who, "rows of 2^27 bytes or scales of 2^26 or more");
  const size_t need = workspace_of(a, b, format, dtype);
  if (workspace_bytes < need || (need && !workspace)) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace is too small");
  if ((uintptr_t)workspace & 15u) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace must be 16-byte aligned");
  const Plan p = plan_of(a, b, format, dtype);
  const bool f32 = dtype == AZ_F32;
  Operands o = {a, b, bias, out, ld_out, 0, static_cast<hipStream_t>(stream)};
  (void)hipGetLastError();
  if (p.parts == 1) return launched(who, run_plan(p, o, format, f32, f32));
  o.bias = nullptr;
  o.out = workspace;
  o.ldo = b.rows;
  o.part_stride = (int64_t)a.rows * b.rows;
  if ((st = launched(who, run_plan(p, o, format, f32, true))) != AZ_OK) return st;
  const dim3 g = join_grid(a.rows, b.rows);
  const float* parts = static_cast<const float*>(workspace);
  if (f32) hipLaunchKernelGGL((az_join_products<true>), g, dim3(256), 0, o.stream, parts, p.parts, a.rows, b.rows, bias, out, ld_out);
  else hipLaunchKernelGGL((az_join_products<false>), g, dim3(256), 0, o.stream, parts, p.parts, a.rows, b.rows, bias, out, ld_out);
  return launch_status(who);
}

LeftView left_view(const az_fp4_matrix& a) { return LeftView{a.codes, a.scales, a.ld, a.ld_scales, (int)a.rows, (int)a.cols, 0}; }
LeftView left_view(const az_code_matrix& a) {
  const CodeView c = code_view(a);
  return LeftView{c.codes, c.scales, c.ld, c.nb, c.rows, c.cols, c.shift};
}

// Whether sizes have a workspace to ask for: those that a call takes.
template <class Matrix>
bool sized(const Matrix* m) { return m && m->rows > 0 && m->cols > 0 && code_sizes(m->rows, m->cols); }

}  // namespace

extern "C" size_t az_nibbles_matmul_workspace(const az_fp4_matrix* a, const az_fp4_matrix* b, int32_t dtype) {
  return sized(a) && sized(b) ? workspace_of(left_view(*a), nibble_view(*b), E2M1, dtype) : 0;
}

extern "C" size_t az_codes_nibbles_matmul_workspace(const az_code_matrix* a, const az_fp4_matrix* b, int32_t dtype) {
  return sized(a) && sized(b) ? workspace_of(left_view(*a), nibble_view(*b), E4M3, dtype) : 0;
}

extern "C" int az_nibbles_matmul(const az_fp4_matrix* a, const az_fp4_matrix* b, const float* bias, void* out, int32_t dtype,
                                 int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "az_nibbles_matmul";
  int st = nibble_check(a, who);
  if (st == AZ_OK) st = nibble_check(b, who);
  if (st != AZ_OK) return st;
  return matmul(left_view(*a), E2M1, nibble_view(*b), bias, out, dtype, ld_out, workspace, workspace_bytes, stream, who);
}

extern "C" int az_codes_nibbles_matmul(const az_code_matrix* a, const az_fp4_matrix* b, const float* bias, void* out, int32_t dtype,
                                       int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "az_codes_nibbles_matmul";
  int st = code_check(a, who);
  if (st == AZ_OK) st = nibble_check(b, who);
  if (st != AZ_OK) return st;
  return matmul(left_view(*a), E4M3, nibble_view(*b), bias, out, dtype, ld_out, workspace, workspace_bytes, stream, who);
}
