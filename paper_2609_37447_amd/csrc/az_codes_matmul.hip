// out = a b^T + bias of two coded matrices, both with the summed dimension along
// their rows.
//
// bf16 results run on the scaled f8f6f4 matrix instruction (K = 128, one scale byte
// per row and 128 columns: exactly a block, so that scales cost no arithmetic).  It
// aligns the products of a group of 8 to the largest and cuts what lies 13 bits below, which costs
// about 1.5e-5 of the result's norm (at most 2^-10 of the sum of the products' sizes): nothing beside
// a bf16 rounding (2e-3), but visible in fp32.  fp32 results therefore run on the bf16 instruction, for which
// codes times their scale are exact operands and products exact fp32 terms.
//
// In both, D's rows are the n of b and its columns the m of a, so that a lane holds
// four neighbouring n of one m and stores them together.
#include "az_matmul_common.h"

namespace {

// 32 consecutive codes of a row for K step kb, the operand of a lane (row l % 16,
// columns 32 (l / 16) on).
__device__ __forceinline__ cm_i32x8 row_fragment(const uint8_t* row, int k0, int cols) {
  const cm_i32x4 lo = code_chunk(row, k0, cols), hi = code_chunk(row, k0 + 16, cols);
  return cm_i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// Eight codes (words 2i, 2i + 1 of a fragment) as exact bf16 values.
__device__ __forceinline__ cm_bf16x8 fragment_bf16(const cm_i32x8& w, int i, float s) {
  const cm_i32x4 u = {(int)code_pair_bf16<false>((uint32_t)w[2 * i], s), (int)code_pair_bf16<true>((uint32_t)w[2 * i], s),
                      (int)code_pair_bf16<false>((uint32_t)w[2 * i + 1], s), (int)code_pair_bf16<true>((uint32_t)w[2 * i + 1], s)};
  return __builtin_bit_cast(cm_bf16x8, u);
}

// Few rows of a.  A workgroup of eight waves owns 16 rows of a times 16 rows of b.  Each wave takes
// every eighth K step, two steps on their way together, through LDS of its own: the copies read whole
// 128-byte lines (loads straight into the operands' places would take 64 bytes of each of 16 rows:
// 1 x 4672 x 8192 13.2 us instead of 11.2).  The waves' sums meet in LDS in the order of the waves.
// Bound by b's bytes and their latency; four steps at once, or sixteen waves, were no faster.
constexpr int DW = 8, DU = 2;

struct DirectStep {
  cm_i32x8 a, b;
  uint32_t sa, sb;
  template <bool EXACT>
  __device__ __forceinline__ void add_to(cm_f32x4& acc) const {
    if constexpr (!EXACT) {
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, acc, 0, 0, 0, (int)sb, 0, (int)sa);
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fragment_bf16(b, q, scale_value(sb)), fragment_bf16(a, q, scale_value(sa)), acc, 0, 0, 0);
    }
  }
};

// 16 rows of a step, straight into 2 KB of LDS: a lane one chunk of row lane / 8 (`off` bytes in) and
// of the row eight below, whose chunks are exchanged by 4 more.
__device__ __forceinline__ void direct_copy(__amdgpu_buffer_rsrc_t rows, const uint32_t (&off)[2], int at, lds_bytes* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, to, 16, off[0], at, 0, 0);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, to + 1024, 16, off[1], at, 0, 0);
}

// EXACT: products on the bf16 instruction, fp32 out; otherwise on the e4m3 one, bf16 out.
// 1 x 4672 x 8192: 10.5 us (3.6 TB/s of b); 64 x 1880 x 10240: 15, with b fetched once for each 16 rows of a.
template <bool EXACT>
__global__ __launch_bounds__(DW * 64) void az_matmul_direct(CodeView a, CodeView b, const float* __restrict__ bias,
                                                            void* __restrict__ out, int64_t ldo, int nt) {
  __shared__ __attribute__((aligned(16))) uint8_t tiles[DW][DU][2][16 * CB];  // and the waves' sums, afterwards
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int m0 = (int)(blockIdx.x / (uint32_t)nt) * 16, n0 = (int)(blockIdx.x % (uint32_t)nt) * 16;
  const int whole = a.cols / CB, width = (a.cols + 15) & ~15;
  const int am = min(m0 + r, a.rows - 1), bn = min(n0 + r, b.rows - 1);
  const uint8_t *as = a.scales + (int64_t)(am >> a.shift) * a.nb, *bs = b.scales + (int64_t)(bn >> b.shift) * b.nb;
  // Chunks are exchanged by the row, as in the tiles below; for a row past the matrix, of no result, its last one is read.
  const int crow = lane >> 3, chunk = (lane & 7) ^ ((crow >> 1) & 7), ms = min(a.rows - m0, 16), ns = min(b.rows - n0, 16);
  uint32_t aoff[2], boff[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    aoff[i] = (uint32_t)min(crow + 8 * i, ms - 1) * (uint32_t)a.ld + (chunk ^ 4 * i) * 16;
    boff[i] = (uint32_t)min(crow + 8 * i, ns - 1) * (uint32_t)b.ld + (chunk ^ 4 * i) * 16;
  }
  const __amdgpu_buffer_rsrc_t abuf = __builtin_amdgcn_make_buffer_rsrc(a.codes + m0 * a.ld, 0, (ms - 1) * (int)a.ld + width, 0x00027000);
  const __amdgpu_buffer_rsrc_t bbuf = __builtin_amdgcn_make_buffer_rsrc(b.codes + n0 * b.ld, 0, (ns - 1) * (int)b.ld + width, 0x00027000);
  const int sw = (r >> 1) & 7, c0 = (g ^ sw) * 16, c1 = ((g + 4) ^ sw) * 16;  // (any columns do, if a and b agree)
  cm_f32x4 acc = {0, 0, 0, 0};
  for (int kb = wave; kb < whole; kb += DW * DU) {
    DirectStep s[DU];
#pragma unroll
    for (int u = 0; u < DU; u++) {
      const int k = min(kb + u * DW, whole - 1);
      direct_copy(abuf, aoff, k * CB, (lds_bytes*)&tiles[wave][u][0][0]);
      direct_copy(bbuf, boff, k * CB, (lds_bytes*)&tiles[wave][u][1][0]);
      s[u].sa = as[k];
      s[u].sb = bs[k];
    }
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < DU; u++) {
      const uint8_t *ta = &tiles[wave][u][0][r * CB], *tb = &tiles[wave][u][1][r * CB];
      const cm_i32x4 a0 = *reinterpret_cast<const cm_i32x4*>(ta + c0), a1 = *reinterpret_cast<const cm_i32x4*>(ta + c1);
      const cm_i32x4 b0 = *reinterpret_cast<const cm_i32x4*>(tb + c0), b1 = *reinterpret_cast<const cm_i32x4*>(tb + c1);
      s[u].a = cm_i32x8{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
      s[u].b = cm_i32x8{b0[0], b0[1], b0[2], b0[3], b1[0], b1[1], b1[2], b1[3]};
      // (past the end the last step was read again: its codes count as zeros, which adds nothing but
      // a NaN that is in the result already)
      if (u > 0) s[u].b &= -(int)(kb + u * DW < whole);
      s[u].add_to<EXACT>(acc);
    }
    __builtin_amdgcn_s_waitcnt(0);  // the reads are back before the next copies overwrite what they read
    __builtin_amdgcn_sched_barrier(0);
  }
  if (whole < a.nb && wave == whole % DW) {  // the columns that do not fill a step
    const int k0 = whole * CB + g * 32;
    const DirectStep s = {row_fragment(a.codes + am * a.ld, k0, a.cols), row_fragment(b.codes + bn * b.ld, k0, a.cols), as[whole], bs[whole]};
    s.add_to<EXACT>(acc);
  }
  __syncthreads();  // every wave is done with its tiles
  cm_f32x4* const part = reinterpret_cast<cm_f32x4*>(&tiles[0][0][0][0]);
  if (wave > 0) part[(wave - 1) * 64 + lane] = acc;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < DW - 1; w++) acc += part[w * 64 + lane];
  const int m = m0 + r;
  if (m >= a.rows) return;
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const int n = n0 + 4 * g + e;
    if (n >= b.rows) continue;
    const float v = acc[e] + (bias ? bias[n] : 0.0f);
    if constexpr (EXACT) ((float*)out)[m * ldo + n] = v;
    else ((uint16_t*)out)[m * ldo + n] = bf16_of(v);
  }
}

// More rows of a.  Four waves own a tile of TM rows of a and TN rows of b, WM x WN parts of FA x FB
// blocks of 32 x 32.  K steps of 128 columns go straight from memory into LDS, two steps in
// turn (four were no faster); a wave reads fragments of half a step (64 columns) while the
// matrix unit works on the half before.
//
// LDS rows are 128 bytes, their 16-byte chunks exchanged by the row's place (chunk ^ (row /
// 2) % 8), which spreads the 16 rows that are read together over all banks.  The copy into
// LDS puts lanes side by side, so that the exchange is made on the source address.
template <int FA_, int FB_, int WM, int WN, bool EXACT>
struct Tiled {
  static constexpr int FA = FA_, FB = FB_, ACROSS = WM, TM = 32 * FA * WM, TN = 32 * FB * WN;
  static constexpr int ASTEP = TM * CB, BSTEP = TN * CB;  // LDS bytes of an operand's step
  static constexpr int SCALES = ASTEP + BSTEP;  // where a word of scale bytes for each row of a, then of b, begins
  static constexpr int SA = TM < 64 ? 64 : TM;  // words of a (a wave copies 64)
  static constexpr int STAGE = SCALES + (SA + TN) * 4;
  static constexpr int LDS = 2 * STAGE;
  static constexpr int ROWS = 32;               // rows that one copy instruction of the workgroup fills
  static_assert(WM * WN == 4 && (SA + TN) % 64 == 0 && TM % ROWS == 0 && TN % ROWS == 0, "four waves' work");

  struct Frag {
    cm_i32x8 a[FA], b[FB];
  };

  // A thread's chunks of a step, one of each ROWS rows: `off` in the tile's first step, `at` the step's
  // place in a row.
  template <int CHUNKS>
  static __device__ __forceinline__ void copy(__amdgpu_buffer_rsrc_t tile, const uint32_t* off, int at, lds_bytes* to) {
#pragma unroll
    for (int j = 0; j < CHUNKS; j++) __builtin_amdgcn_raw_ptr_buffer_load_lds(tile, to + j * ROWS * CB, 16, off[j], at, 0, 0);
  }
  static __device__ __forceinline__ void scale_words(__amdgpu_buffer_rsrc_t words, lds_bytes* to, uint32_t at) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(words, to, 4, at, 0, 0, 0);
  }
  // Spreads half a step's LDS reads (of the next half's fragments) and loads over its matrix
  // instructions, reads first, so that they are back before the half ends.
  static __device__ __forceinline__ void interleave() {
    if constexpr (!EXACT) {
#pragma unroll
      for (int i = 0; i < FA * FB; i++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction
        if (i < FA + FB) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);  // LDS reads
        else __builtin_amdgcn_sched_group_barrier(0x020, 3, 0);  // copies
      }
    }
  }
  static __device__ __forceinline__ cm_i32x8 fragment(const uint8_t* lo, const uint8_t* hi) {
    const cm_i32x4 x = *reinterpret_cast<const cm_i32x4*>(lo), y = *reinterpret_cast<const cm_i32x4*>(hi);
    return cm_i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  }
  static __device__ __forceinline__ void read(Frag& f, const uint8_t* a0, const uint8_t* a1, const uint8_t* b0, const uint8_t* b1) {
#pragma unroll
    for (int i = 0; i < FA; i++) f.a[i] = fragment(a0 + i * 32 * CB, a1 + i * 32 * CB);
#pragma unroll
    for (int j = 0; j < FB; j++) f.b[j] = fragment(b0 + j * 32 * CB, b1 + j * 32 * CB);
  }
  static __device__ __forceinline__ void multiply(cm_f32x16 (&acc)[FA][FB], const Frag& f, const uint32_t (&sa)[FA], const uint32_t (&sb)[FB]) {
    if constexpr (!EXACT) {
#pragma unroll
      for (int i = 0; i < FA; i++)
#pragma unroll
        for (int j = 0; j < FB; j++)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f.b[j], f.a[i], acc[i][j], 0, 0, 0, (int)sb[j], 0, (int)sa[i]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++) {
        cm_bf16x8 va[FA], vb[FB];
#pragma unroll
        for (int i = 0; i < FA; i++) va[i] = fragment_bf16(f.a[i], q, scale_value(sa[i]));
#pragma unroll
        for (int j = 0; j < FB; j++) vb[j] = fragment_bf16(f.b[j], q, scale_value(sb[j]));
#pragma unroll
        for (int i = 0; i < FA; i++)
#pragma unroll
          for (int j = 0; j < FB; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[j], va[i], acc[i][j], 0, 0, 0);
      }
    }
  }
};

// 8192^3: 460-489 us (2,250-2,390 TFLOP/s); 333 x 1880 x 10240 with exact products, four parts: 28 us.
template <int FA, int FB, int WM, int WN, bool EXACT, bool F32>
__global__ __launch_bounds__(256, FA * FB == 16 ? 1 : 2) void az_matmul_tiled(CodeView a, CodeView b, const float* __restrict__ bias,
                                                                              void* __restrict__ out, int64_t ldo, int mt, int nt,
                                                                              int part_steps, int64_t part_stride) {
  using K = Tiled<FA, FB, WM, WN, EXACT>;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  int tm, tn;
  tile_of(blockIdx.x, mt, nt, tm, tn);
  // The last tile of a side ends with the matrix: what it shares with the tile before is computed
  // twice, to the same bits.  A matrix of fewer rows than a tile is the one tile's beginning.
  const int m0 = max(min(tm * K::TM, a.rows - K::TM), 0), n0 = max(min(tn * K::TN, b.rows - K::TN), 0);
  const int ms = min(a.rows, K::TM), ns = min(b.rows, K::TN);

  // Copying: wave w of instruction j takes rows 32 j + 8 w .. + 7, a lane one chunk of one row; for a
  // row past the matrix, of no result, its last one, so that no copy of codes leaves the matrix whatever a
  // buffer's range counts.
  const int crow = 8 * wave + (lane >> 3), chunk = (lane & 7) ^ ((crow >> 1) & 7);
  uint32_t aoff[K::TM / 32], boff[K::TN / 32];
#pragma unroll
  for (int j = 0; j < K::TM / 32; j++) aoff[j] = (uint32_t)min(32 * j + crow, ms - 1) * (uint32_t)a.ld + chunk * 16;
#pragma unroll
  for (int j = 0; j < K::TN / 32; j++) boff[j] = (uint32_t)min(32 * j + crow, ns - 1) * (uint32_t)b.ld + chunk * 16;
  const int width = (a.cols + 15) & ~15;
  const __amdgpu_buffer_rsrc_t abuf = __builtin_amdgcn_make_buffer_rsrc(a.codes + m0 * a.ld, 0, (ms - 1) * (int)a.ld + width, 0x00027000);
  const __amdgpu_buffer_rsrc_t bbuf = __builtin_amdgcn_make_buffer_rsrc(b.codes + n0 * b.ld, 0, (ns - 1) * (int)b.ld + width, 0x00027000);
  lds_bytes* const lds0 = (lds_bytes*)smem + 8 * wave * CB;
  // The part's steps, of which `whole` is the first that does not fill its columns or is not the part's.
  const int first = (int)blockIdx.y * part_steps, last = min(first + part_steps, a.nb), whole = min(last, a.cols / CB);
  // Scales: words of a, then of b, 64 a wave and turn.
  const ScaleWords aw(a), bw(b);
  constexpr int TURNS = ((K::SA + K::TN) / 64 + 3) / 4;
  uint32_t srow[TURNS];
#pragma unroll
  for (int i = 0; i < TURNS; i++) {
    const int w = i * 256 + t;
    srow[i] = w < K::SA ? aw.place(a, m0 + min(w, ms - 1)) : bw.place(b, n0 + min(w - K::SA, ns - 1));
  }
  lds_bytes* const slds = (lds_bytes*)smem + K::SCALES + wave * 64 * 4;
  // (past the last step: that step again, which nothing reads)
  auto fetch = [&](int kb) {
    const int stage = (kb & 1) * K::STAGE;
    kb = min(kb, whole - 1);
    K::template copy<K::TM / 32>(abuf, aoff, kb * CB, lds0 + stage);
    K::template copy<K::TN / 32>(bbuf, boff, kb * CB, lds0 + stage + K::ASTEP);
#pragma unroll
    for (int i = 0; i < TURNS; i++)
      if ((K::SA + K::TN) % 256 == 0 || i * 4 + wave < (K::SA + K::TN) / 64)
        K::scale_words(i * 4 + wave < K::SA / 64 ? aw.words : bw.words, slds + stage + i * 1024, (srow[i] + kb) & ~3u);
  };

  // Reading: a lane holds row l % 32 of a block, columns 32 (l / 32) + 64 s on of half s.
  const int r = lane & 31, h = lane >> 5, wm = (wave % WM) * 32 * K::FA, wn = (wave / WM) * 32 * K::FB;
  const int sw = (r >> 1) & 7;
  const uint8_t* ap = smem + (wm + r) * CB;
  const uint8_t* bp = smem + K::ASTEP + (wn + r) * CB;
  const int at[2][2] = {{((2 * h) ^ sw) * 16, ((2 * h + 1) ^ sw) * 16}, {((2 * h + 4) ^ sw) * 16, ((2 * h + 5) ^ sw) * 16}};
  // Scales: the byte that counts is moved down to the lowest, which is the one that the instruction
  // takes; a shift goes by its amount's low five bits, so that (place + kb) % 4 costs nothing.
  uint32_t ac[K::FA], bc[K::FB];  // eight times the places of the lane's rows' scales
#pragma unroll
  for (int i = 0; i < K::FA; i++) ac[i] = 8 * aw.place(a, m0 + min(wm + 32 * i + r, ms - 1));
#pragma unroll
  for (int j = 0; j < K::FB; j++) bc[j] = 8 * bw.place(b, n0 + min(wn + 32 * j + r, ns - 1));
  uint32_t sa[K::FA], sb[K::FB], na[K::FA], nb[K::FB];
  auto scale_words = [&](int kb) {
    const uint32_t* from = reinterpret_cast<const uint32_t*>(smem + (kb & 1) * K::STAGE + K::SCALES) + r;
#pragma unroll
    for (int i = 0; i < K::FA; i++) na[i] = from[wm + 32 * i];
#pragma unroll
    for (int j = 0; j < K::FB; j++) nb[j] = from[K::SA + wn + 32 * j];
  };
  auto scales = [&](int kb) {
    constexpr uint32_t ONE = EXACT ? 0xffu : ~0u;
#pragma unroll
    for (int i = 0; i < K::FA; i++) sa[i] = (na[i] >> ((ac[i] + 8 * kb) & 31)) & ONE;
#pragma unroll
    for (int j = 0; j < K::FB; j++) sb[j] = (nb[j] >> ((bc[j] + 8 * kb) & 31)) & ONE;
  };

  cm_f32x16 acc[K::FA][K::FB];
#pragma unroll
  for (int i = 0; i < K::FA; i++)
#pragma unroll
    for (int j = 0; j < K::FB; j++) acc[i][j] = cm_f32x16{};
  typename K::Frag f0, f1;
  if (whole > first) {
    const int stage = (first & 1) * K::STAGE;
    fetch(first);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    fetch(first + 1);
    scale_words(first);
    scales(first);
    K::read(f0, ap + stage + at[0][0], ap + stage + at[0][1], bp + stage + at[0][0], bp + stage + at[0][1]);
  }
  for (int kb = first; kb < whole; kb++) {
    const int stage = (kb & 1) * K::STAGE, next = K::STAGE - stage;
    K::read(f1, ap + stage + at[1][0], ap + stage + at[1][1], bp + stage + at[1][0], bp + stage + at[1][1]);
    K::multiply(acc, f0, sa, sb);
    K::interleave();
    __builtin_amdgcn_sched_barrier(0);
    // This wave's reads of step kb are done and its copies of step kb + 1 have landed; after the
    // barrier that holds for every wave.
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    // (after the last step these are the bytes of the step before: read, not used)
    K::read(f0, ap + next + at[0][0], ap + next + at[0][1], bp + next + at[0][0], bp + next + at[0][1]);
    scale_words(kb + 1);
    fetch(kb + 2);
    K::multiply(acc, f1, sa, sb);
    K::interleave();
    scales(kb + 1);
  }
  __builtin_amdgcn_s_waitcnt(0);  // no copy into LDS is under way when the workgroup ends
  if (whole < last) {  // the columns that do not fill a step, straight from memory
#pragma unroll
    for (int i = 0; i < K::FA; i++) sa[i] = a.scales[(int64_t)((m0 + min(wm + 32 * i + r, ms - 1)) >> a.shift) * a.nb + whole];
#pragma unroll
    for (int j = 0; j < K::FB; j++) sb[j] = b.scales[(int64_t)((n0 + min(wn + 32 * j + r, ns - 1)) >> b.shift) * b.nb + whole];
#pragma unroll
    for (int s = 0; s < 2; s++) {
#pragma unroll
      for (int i = 0; i < K::FA; i++) f0.a[i] = row_fragment(a.codes + (m0 + min(wm + 32 * i + r, ms - 1)) * a.ld, whole * CB + 64 * s + 32 * h, a.cols);
#pragma unroll
      for (int j = 0; j < K::FB; j++) f0.b[j] = row_fragment(b.codes + (n0 + min(wn + 32 * j + r, ns - 1)) * b.ld, whole * CB + 64 * s + 32 * h, a.cols);
      K::multiply(acc, f0, sa, sb);
    }
  }
  write_tile<K, F32>(acc, smem, bias, (uint8_t*)out + (blockIdx.y * part_stride + (int64_t)m0 * ldo + n0) * (F32 ? 4 : 2), ldo, n0, ms, ns, wave, r, h);
}

// How a product runs: the kernel, and `parts` parts of the columns of part_steps K steps each.
enum { DIRECT = 0, TILE32 = 1, TILE64 = 2, TILE128 = 3, TILE256 = 4 };
struct Plan {
  int kind, parts, part_steps;
};

// The plan with the least estimated time, in microseconds.  A tile kernel's K step takes a
// workgroup `one` alone on a compute unit (bound by the step's own chain of copies, LDS reads and
// the barrier) and `all` with `occ` of them there; both were measured, for bf16 results and for
// the exact products of fp32 ones.  What parts cost is their way through memory and a second
// launch.  Measured, chosen against others: 16 x 1880 x 10240 by the kernel of few rows 8.3 (32-row
// tiles in 8 parts 13.5); 64 x 4672 x 8192 in 32-row tiles and 8 parts 16.7 (128-row, 8 parts 18.0,
// 32-row in one part 35); 320 x 1880 x 10240 in 64-row tiles and 8 parts 26 (128-row, one part 68); 2048 x
// 4672 x 8192 in 256-row tiles 92 (64-row 100, 128-row 110); 4096^3 in 256-row tiles 59 (128-row 68).  The
// model is off where two plans are within 10%: 1024 x 4672 x 8192 goes to 64-row tiles, 61 (128-row 55,
// 256-row 90), and 512 x 4672 x 8192 to two parts of them, 42 (one part 41).
Plan choose_plan(int64_t m, int64_t n, int64_t k, bool exact, bool fits) {
  struct Tile {
    int kind, tm, tn, occ;
    double one, all, one_exact, all_exact;
  };
  static const Tile tiles[] = {{TILE32, 32, 128, 3, 0.53, 0.70, 0.55, 0.80},
                               {TILE64, 64, 128, 3, 0.60, 0.87, 0.63, 1.35},
                               {TILE128, 128, 128, 2, 0.69, 0.90, 0.80, 1.50},
                               {TILE256, 256, 256, 1, 1.45, 1.72, 2.75, 3.30}};
  const int nb = (int)((k + CB - 1) / CB);
  const double write = 1.0 / 4.5e6;  // microseconds a byte
  const double out = (double)m * (double)n * (exact ? 4 : 2) * write;
  auto rounds = [](int64_t groups, int64_t slots) { return (double)((groups + slots - 1) / slots); };
  Plan best = {DIRECT, 1, nb};
  // eight waves take every eighth step each
  double least = 3.0 + rounds((n + 15) / 16 * ((m + 15) / 16), 256) * (nb / 8.0 * 0.55 + 0.6) + out;
  if (!fits) return best;
  for (const Tile& t : tiles) {
    const int64_t count = ((m + t.tm - 1) / t.tm) * ((n + t.tn - 1) / t.tn);
    const double one = exact ? t.one_exact : t.one, all = exact ? t.all_exact : t.all;
    for (int parts = 1; parts <= 8 && (parts == 1 || 2 * parts <= nb); parts *= 2) {
      const int64_t groups = count * parts, per = (groups + 255) / 256;
      const int steps = (nb + parts - 1) / parts;
      const int occ = per < t.occ ? (int)per : t.occ;
      const double step = t.occ == 1 ? (per > 1 ? all : one) : one + (all - one) * (occ - 1) / (t.occ - 1);
      double cost = 4.0 + rounds(groups, 256 * t.occ) * (steps * step + 2.0) + out;
      if (parts > 1) cost += 3.5 + (double)parts * (double)m * (double)n * 8 * write;
      if (cost < least) {
        least = cost;
        best = {t.kind, (nb + steps - 1) / steps, steps};
      }
    }
  }
  return best;
}

struct Operands {
  CodeView a, b;
  const float* bias;
  void* out;
  int64_t ldo, part_stride;
  hipStream_t stream;
};

template <bool EXACT>
int launch_direct(const Operands& o) {
  const int64_t nt = ((int64_t)o.b.rows + 15) / 16, groups = nt * (((int64_t)o.a.rows + 15) / 16);
  if (!grid_fits(groups, DW * 64)) return AZ_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((az_matmul_direct<EXACT>), dim3((unsigned)groups), dim3(DW * 64), 0, o.stream, o.a, o.b, o.bias, o.out, o.ldo, (int)nt);
  return AZ_OK;
}

template <int FA, int FB, int WM, int WN, bool EXACT, bool F32>
int launch_tiled(const Plan& p, const Operands& o) {
  using K = Tiled<FA, FB, WM, WN, EXACT>;
  const int64_t mt = ((int64_t)o.a.rows + K::TM - 1) / K::TM, nt = ((int64_t)o.b.rows + K::TN - 1) / K::TN;
  if (!grid_fits(mt * nt, 256)) return AZ_ERR_UNSUPPORTED;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(az_matmul_tiled<FA, FB, WM, WN, EXACT, F32>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, K::LDS);
  if (e != hipSuccess) return AZ_ERR_DEVICE;
  hipLaunchKernelGGL((az_matmul_tiled<FA, FB, WM, WN, EXACT, F32>), dim3((unsigned)(mt * nt), p.parts), dim3(256), K::LDS, o.stream,
                     o.a, o.b, o.bias, o.out, o.ldo, (int)mt, (int)nt, p.part_steps, o.part_stride);
  return AZ_OK;
}

template <bool EXACT, bool F32>
int launch_tiles(const Plan& p, const Operands& o) {
  const int st = p.kind == TILE256   ? launch_tiled<4, 4, 2, 2, EXACT, F32>(p, o)
                 : p.kind == TILE128 ? launch_tiled<2, 2, 2, 2, EXACT, F32>(p, o)
                 : p.kind == TILE64  ? launch_tiled<1, 2, 2, 2, EXACT, F32>(p, o)
                                     : launch_tiled<1, 1, 1, 4, EXACT, F32>(p, o);
  return launched("az_codes_matmul", st);
}

// A tile's offsets stay below 2^30.
bool tile_fits(int64_t lda, int64_t ldb) { return lda < (1 << 22) && ldb < (1 << 22); }

}  // namespace

extern "C" size_t az_codes_matmul_workspace(const az_code_matrix* a, const az_code_matrix* b, int32_t dtype) {
  if (!a || !b || a->rows <= 0 || b->rows <= 0 || a->cols <= 0 || b->cols <= 0) return 0;
  if (!code_sizes(a->rows, a->cols) || !code_sizes(b->rows, b->cols)) return 0;
  const Plan p = choose_plan(a->rows, b->rows, a->cols, dtype == AZ_F32, tile_fits(a->ld, b->ld));
  return p.parts > 1 ? (size_t)p.parts * (size_t)a->rows * (size_t)b->rows * sizeof(float) : 0;
}

extern "C" int az_codes_matmul(const az_code_matrix* a, const az_code_matrix* b, const float* bias, void* out,
                               int32_t dtype, int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "az_codes_matmul";
  int st = code_check(a, who);
  if (st == AZ_OK) st = code_check(b, who);
  if (st != AZ_OK) return st;
  if (a->cols != b->cols) return code_fail(AZ_ERR_INVALID_ARG, who, "a and b differ in cols");
  if (dtype != AZ_F32 && dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (a->rows == 0 || b->rows == 0) return AZ_OK;
  if ((st = dense_check(out, dtype, ld_out, b->rows, who)) != AZ_OK) return st;
  if ((uintptr_t)bias & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "bias must be 4-byte aligned");
  // 16 rows in the 32 bits of a buffer's range
  if (a->ld >= (1 << 27) || b->ld >= (1 << 27)) return code_fail(AZ_ERR_UNSUPPORTED, who, "rows of 2^27 bytes or more");
  const size_t need = az_codes_matmul_workspace(a, b, dtype);
  if (workspace_bytes < need || (need && !workspace)) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace is too small");
  if ((uintptr_t)workspace & 15u) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace must be 16-byte aligned");
  const Plan p = choose_plan(a->rows, b->rows, a->cols, dtype == AZ_F32, tile_fits(a->ld, b->ld));
  Operands o = {code_view(*a), code_view(*b), bias, out, ld_out, 0, static_cast<hipStream_t>(stream)};
  (void)hipGetLastError();
  if (p.kind == DIRECT) return launched(who, dtype == AZ_F32 ? launch_direct<true>(o) : launch_direct<false>(o));
  if (p.parts > 1) {
    o.bias = nullptr;
    o.out = workspace;
    o.ldo = b->rows;
    o.part_stride = a->rows * b->rows;
    if ((st = dtype == AZ_F32 ? launch_tiles<true, true>(p, o) : launch_tiles<false, true>(p, o)) != AZ_OK) return st;
    const dim3 g = join_grid(a->rows, b->rows);
    const float* parts = static_cast<const float*>(workspace);
    if (dtype == AZ_F32)
      hipLaunchKernelGGL((az_join_products<true>), g, dim3(256), 0, o.stream, parts, p.parts, (int)a->rows, (int)b->rows, bias, out, ld_out);
    else
      hipLaunchKernelGGL((az_join_products<false>), g, dim3(256), 0, o.stream, parts, p.parts, (int)a->rows, (int)b->rows, bias, out, ld_out);
    return launch_status(who);
  }
  return dtype == AZ_F32 ? launch_tiles<true, true>(p, o) : launch_tiles<false, false>(p, o);
}
