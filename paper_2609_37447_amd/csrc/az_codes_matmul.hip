// out = a b^T + bias of two coded matrices, both with the summed dimension along
// their rows.
//
// bf16 results run on the scaled f8f6f4 matrix instruction (K = 128, one scale byte
// per row and 128 columns: exactly a block, so that scales cost no arithmetic).  It
// aligns the products of a group to the largest and cuts what lies below, which costs
// about 1.5e-5 of the result's norm: nothing beside a bf16 rounding (2e-3), but
// visible in fp32.  fp32 results therefore run on the bf16 instruction, for which
// codes times their scale are exact operands and products exact fp32 terms.
//
// In both, D's rows are the n of b and its columns the m of a, so that a lane holds
// four neighbouring n of one m and stores them together.
#include "az_codes_common.h"

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

// A workgroup of NW waves owns 16 FM rows of a times 16 FN rows of b.  Each wave takes
// every NW-th K step straight from memory to registers; the partial sums meet in LDS in
// the order of the waves.
template <int FM, int FN, int NW, bool F32>
__global__ __launch_bounds__(NW * 64) void az_matmul_direct(CodeView a, CodeView b, const float* __restrict__ bias,
                                                            void* __restrict__ out, int64_t ldo) {
  __shared__ cm_f32x4 part[NW > 1 ? (NW - 1) * FM * FN * 64 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int m0 = blockIdx.y * 16 * FM, n0 = blockIdx.x * 16 * FN;
  cm_f32x4 acc[FM][FN];
  const uint8_t *ar[FM], *br[FN], *as[FM], *bs[FN];
#pragma unroll
  for (int i = 0; i < FM; i++) {
    const int row = min(m0 + 16 * i + r, a.rows - 1);
    ar[i] = a.codes + row * a.ld;
    as[i] = a.scales + (int64_t)(row >> a.shift) * a.nb;
  }
#pragma unroll
  for (int j = 0; j < FN; j++) {
    const int row = min(n0 + 16 * j + r, b.rows - 1);
    br[j] = b.codes + row * b.ld;
    bs[j] = b.scales + (int64_t)(row >> b.shift) * b.nb;
  }
#pragma unroll
  for (int i = 0; i < FM; i++)
#pragma unroll
    for (int j = 0; j < FN; j++) acc[i][j] = cm_f32x4{0, 0, 0, 0};
  for (int kb = wave; kb < a.nb; kb += NW) {
    const int k0 = kb * CB + g * 32;
    cm_i32x8 fa[FM], fb[FN];
    uint32_t sa[FM], sb[FN];
#pragma unroll
    for (int i = 0; i < FM; i++) { fa[i] = row_fragment(ar[i], k0, a.cols); sa[i] = as[i][kb]; }
#pragma unroll
    for (int j = 0; j < FN; j++) { fb[j] = row_fragment(br[j], k0, a.cols); sb[j] = bs[j][kb]; }
    if constexpr (!F32) {
#pragma unroll
      for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa[i], acc[i][j], 0, 0, 0, (int)sb[j], 0, (int)sa[i]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++) {
        cm_bf16x8 va[FM], vb[FN];
#pragma unroll
        for (int i = 0; i < FM; i++) va[i] = fragment_bf16(fa[i], q, scale_value(sa[i]));
#pragma unroll
        for (int j = 0; j < FN; j++) vb[j] = fragment_bf16(fb[j], q, scale_value(sb[j]));
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
          for (int j = 0; j < FN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb[j], va[i], acc[i][j], 0, 0, 0);
      }
    }
  }
  if constexpr (NW > 1) {
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) part[((wave - 1) * FM * FN + i * FN + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < NW - 1; w++)
#pragma unroll
      for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) acc[i][j] += part[(w * FM * FN + i * FN + j) * 64 + lane];
  }
#pragma unroll
  for (int i = 0; i < FM; i++) {
    const int m = m0 + 16 * i + r;
    if (m >= a.rows) continue;
#pragma unroll
    for (int j = 0; j < FN; j++) {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int n = n0 + 16 * j + 4 * g + e;
        if (n >= b.rows) continue;
        const float v = acc[i][j][e] + (bias ? bias[n] : 0.0f);
        if constexpr (F32) ((float*)out)[m * ldo + n] = v;
        else ((uint16_t*)out)[m * ldo + n] = bf16_of(v);
      }
    }
  }
}

// Which tile a workgroup takes.  Workgroups go to the eight XCDs in turn, each with an
// L2 of its own: an XCD gets a run of neighbouring tiles, in groups of eight rows of
// tiles, so that the panels that its tiles share are read once into its L2.
__device__ __forceinline__ void tile_of(uint32_t id, int mt, int nt, int& tm, int& tn) {
  const uint32_t total = (uint32_t)mt * (uint32_t)nt;
  const uint32_t xcd = id & 7u, per = total >> 3, more = total & 7u;
  const uint32_t at = xcd * per + min(xcd, more) + (id >> 3);
  const uint32_t group = 8u * (uint32_t)nt, g = at / group, in = at - g * group;
  const uint32_t high = min(8u, (uint32_t)mt - 8u * g);
  tm = (int)(8u * g + in % high);
  tn = (int)(in / high);
}

typedef __attribute__((address_space(3))) uint8_t lds_bytes;

// Large products.  Four waves own a square tile of 64 W rows of each operand, a wave a
// quarter of it (W x W blocks of 32 x 32).  K steps of 128 columns go straight from memory
// into LDS, two steps in turn; a wave reads fragments of half a step (64 columns) while
// the matrix unit works on the half before.
//
// LDS rows are 128 bytes, their 16-byte chunks exchanged by the row's place (chunk ^ (row /
// 2) % 8), which spreads the 16 rows that are read together over all banks.  The copy into
// LDS puts lanes side by side, so that the exchange is made on the source address.
template <int W, int NW, bool F32>
struct Tiled {
  static constexpr int T = 64 * W;           // rows of a and of b of a tile
  static constexpr int STEP = T * CB;        // LDS bytes of one operand's step
  static constexpr int SCALES = 2 * STEP;    // where a word of scale bytes for each row of a, then of b, begins
  static constexpr int STAGE = 2 * STEP + 2 * T * 4;
  static constexpr int ROWS = 8 * NW;        // rows that one copy instruction of the workgroup fills
  static constexpr int CHUNKS = T / ROWS;
  static constexpr int FA = W, FB = 4 * W / NW;  // 32-row blocks of a wave

  struct Frag {
    cm_i32x8 a[FA], b[FB];
  };

  // A thread's chunks of a step, one of each ROWS rows: `off` within the step's first rows, `at`
  // the step's place in the tile.
  static __device__ __forceinline__ void copy(__amdgpu_buffer_rsrc_t tile, int ld, uint32_t off, int at, lds_bytes* to) {
#pragma unroll
    for (int j = 0; j < CHUNKS; j++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(tile, to + j * ROWS * CB, 16, off, at + j * ROWS * ld, 0, 0);
  }
  // Spreads half a step's LDS reads (of the next half's fragments) and loads over its matrix
  // instructions, reads first, so that they are back before the half ends.
  static __device__ __forceinline__ void interleave() {
    if constexpr (!F32) {
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
    if constexpr (!F32) {
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

// Scale bytes of a matrix as aligned words.  Row r's byte of step kb is byte (start + kb) & 3 of
// the word that holds it, start = place(r).
struct ScaleWords {
  __amdgpu_buffer_rsrc_t words;
  uint32_t skip;
  __device__ __forceinline__ explicit ScaleWords(const CodeView& m) {
    skip = (uint32_t)((uintptr_t)m.scales & 3u);
    const uint32_t rows = (uint32_t)((m.rows - 1) >> m.shift) + 1u;
    words = __builtin_amdgcn_make_buffer_rsrc(m.scales - skip, 0, (int)((skip + rows * (uint32_t)m.nb + 3u) & ~3u), 0x00027000);
  }
  __device__ __forceinline__ uint32_t place(const CodeView& m, int row) const { return skip + (uint32_t)(row >> m.shift) * (uint32_t)m.nb; }
};

template <int W, int NW, bool F32>
__global__ __launch_bounds__(64 * NW, W == 4 && NW == 4 ? 1 : 2) void az_matmul_tiled(CodeView a, CodeView b, const float* __restrict__ bias,
                                                                       void* __restrict__ out, int64_t ldo, int mt, int nt) {
  using K = Tiled<W, NW, F32>;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  int tm, tn;
  tile_of(blockIdx.x, mt, nt, tm, tn);
  // The last tile of a side ends with the matrix (which has at least a tile's rows): what it
  // shares with the tile before is computed twice, to the same bits.
  const int m0 = min(tm * K::T, a.rows - K::T), n0 = min(tn * K::T, b.rows - K::T);

  // Copying: wave w of instruction j takes rows 32 j + 8 w .. + 7, a lane one chunk of one row.
  const int crow = 8 * wave + (lane >> 3), chunk = (lane & 7) ^ ((crow >> 1) & 7);
  const uint32_t aoff = (uint32_t)crow * (uint32_t)a.ld + chunk * 16, boff = (uint32_t)crow * (uint32_t)b.ld + chunk * 16;
  const __amdgpu_buffer_rsrc_t abuf = __builtin_amdgcn_make_buffer_rsrc(a.codes + m0 * a.ld, 0, K::T * (int)a.ld, 0x00027000);
  const __amdgpu_buffer_rsrc_t bbuf = __builtin_amdgcn_make_buffer_rsrc(b.codes + n0 * b.ld, 0, K::T * (int)b.ld, 0x00027000);
  lds_bytes* const lds0 = (lds_bytes*)smem + 8 * wave * CB;
  const int whole = a.cols / CB;  // steps that fill their columns
  // Scales: a thread's row of a and of b, or of a for half of the threads and of b for the others.
  const ScaleWords aw(a), bw(b);
  constexpr bool BOTH = 64 * NW == K::T;
  const bool half = !BOTH && wave >= NW / 2;
  const uint32_t srow = half ? bw.place(b, n0 + (t & (K::T - 1))) : aw.place(a, m0 + (t & (K::T - 1)));
  const uint32_t srow2 = BOTH ? bw.place(b, n0 + t) : 0u;
  lds_bytes* const slds = (lds_bytes*)smem + K::SCALES + wave * 64 * 4;
  // (past the last step: that step again, which nothing reads)
  auto fetch = [&](int kb) {
    const int stage = (kb & 1) * K::STAGE;
    kb = min(kb, whole - 1);
    K::copy(abuf, (int)a.ld, aoff, kb * CB, lds0 + stage);
    K::copy(bbuf, (int)b.ld, boff, kb * CB, lds0 + stage + K::STEP);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(half ? bw.words : aw.words, slds + stage, 4, (srow + kb) & ~3u, 0, 0, 0);
    if constexpr (BOTH)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(bw.words, slds + stage + K::T * 4, 4, (srow2 + kb) & ~3u, 0, 0, 0);
  };

  // Reading: a lane holds row l % 32 of a block, columns 32 (l / 32) + 64 s on of half s.
  const int r = lane & 31, h = lane >> 5, wm = (wave & 1) * 32 * K::FA, wn = (wave >> 1) * 32 * K::FB;
  const int sw = (r >> 1) & 7;
  const uint8_t* ap = smem + (wm + r) * CB;
  const uint8_t* bp = smem + K::STEP + (wn + r) * CB;
  const int at[2][2] = {{((2 * h) ^ sw) * 16, ((2 * h + 1) ^ sw) * 16}, {((2 * h + 4) ^ sw) * 16, ((2 * h + 5) ^ sw) * 16}};
  uint32_t ac[K::FA], bc[K::FB];  // places of the lane's rows' scales
#pragma unroll
  for (int i = 0; i < K::FA; i++) ac[i] = aw.place(a, m0 + wm + 32 * i + r);
#pragma unroll
  for (int j = 0; j < K::FB; j++) bc[j] = bw.place(b, n0 + wn + 32 * j + r);
  uint32_t sa[K::FA], sb[K::FB], na[K::FA], nb[K::FB];
  auto scales = [&](uint32_t (&pa)[K::FA], uint32_t (&pb)[K::FB], int kb) {
    const uint8_t* from = smem + (kb & 1) * K::STAGE + K::SCALES + r * 4;
#pragma unroll
    for (int i = 0; i < K::FA; i++) pa[i] = from[(wm + 32 * i) * 4 + ((ac[i] + kb) & 3u)];
#pragma unroll
    for (int j = 0; j < K::FB; j++) pb[j] = from[(K::T + wn + 32 * j) * 4 + ((bc[j] + kb) & 3u)];
  };

  cm_f32x16 acc[K::FA][K::FB];
#pragma unroll
  for (int i = 0; i < K::FA; i++)
#pragma unroll
    for (int j = 0; j < K::FB; j++) acc[i][j] = cm_f32x16{};
  typename K::Frag f0, f1;
  if (whole > 0) {
    fetch(0);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    fetch(1);
    scales(sa, sb, 0);
    K::read(f0, ap + at[0][0], ap + at[0][1], bp + at[0][0], bp + at[0][1]);
  }
  for (int kb = 0; kb < whole; kb++) {
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
    scales(na, nb, kb + 1);
    fetch(kb + 2);
    K::multiply(acc, f1, sa, sb);
    K::interleave();
#pragma unroll
    for (int i = 0; i < K::FA; i++) sa[i] = na[i];
#pragma unroll
    for (int j = 0; j < K::FB; j++) sb[j] = nb[j];
  }
  __builtin_amdgcn_s_waitcnt(0);  // no copy into LDS is under way when the workgroup ends
  if (whole < a.nb) {  // the columns that do not fill a step, straight from memory
#pragma unroll
    for (int i = 0; i < K::FA; i++) sa[i] = a.scales[ac[i] - aw.skip + whole];
#pragma unroll
    for (int j = 0; j < K::FB; j++) sb[j] = b.scales[bc[j] - bw.skip + whole];
#pragma unroll
    for (int s = 0; s < 2; s++) {
#pragma unroll
      for (int i = 0; i < K::FA; i++) f0.a[i] = row_fragment(a.codes + (m0 + wm + 32 * i + r) * a.ld, whole * CB + 64 * s + 32 * h, a.cols);
#pragma unroll
      for (int j = 0; j < K::FB; j++) f0.b[j] = row_fragment(b.codes + (n0 + wn + 32 * j + r) * b.ld, whole * CB + 64 * s + 32 * h, a.cols);
      K::multiply(acc, f0, sa, sb);
    }
  }
  // Results leave through LDS, so that whole rows of the tile are written: a lane's four neighbours
  // would be 16 bytes of each of 32 rows.  Chunks are exchanged by the row, as above.
  constexpr int ES = F32 ? 4 : 2, OROW = K::T * ES;
  constexpr int PASSES = 2 * K::STAGE >= K::T * OROW ? 1 : 2;  // fp32: half of each wave's rows at a time
  constexpr int PF = K::FA / PASSES, PROWS = K::T / PASSES;
#pragma unroll
  for (int p = 0; p < PASSES; p++) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < K::FB; j++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int n = wn + 32 * j + 8 * q + 4 * h;
        cm_f32x4 add = {0, 0, 0, 0};
        if (bias) __builtin_memcpy(&add, bias + n0 + n, 16);
#pragma unroll
        for (int i = 0; i < PF; i++) {
          const int row = (wave & 1) * 32 * PF + 32 * i + r;
          cm_f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; e++) v[e] = acc[PF * p + i][j][4 * q + e] + add[e];
          if constexpr (F32) {
            *reinterpret_cast<cm_f32x4*>(smem + row * OROW + (((n >> 2) ^ r) * 16)) = v;
          } else {
            const cm_i32x2 w = {(int)((uint32_t)bf16_of(v[0]) | ((uint32_t)bf16_of(v[1]) << 16)),
                                (int)((uint32_t)bf16_of(v[2]) | ((uint32_t)bf16_of(v[3]) << 16))};
            *reinterpret_cast<cm_i32x2*>(smem + row * OROW + (((n >> 3) ^ (r & (OROW / 16 - 1))) * 16) + (n & 4) * 2) = w;
          }
        }
      }
    __syncthreads();
    constexpr int RC = OROW / 16;  // chunks of a row
#pragma unroll 8
    for (int c = t; c < PROWS * RC; c += 64 * NW) {
      const int row = c / RC, in = c % RC;
      const cm_i32x4 v = *reinterpret_cast<const cm_i32x4*>(smem + row * OROW + ((in ^ (row & 31 & (RC - 1))) * 16));
      // rows of the two halves of the waves lie FA blocks apart
      const int m = m0 + row / (32 * PF) * (32 * K::FA) + p * 32 * PF + row % (32 * PF);
      __builtin_memcpy((uint8_t*)out + ((int64_t)m * ldo + n0) * ES + in * 16, &v, 16);
    }
  }
}

template <int FM, int FN, int NW, bool F32>
void launch_direct(const CodeView& a, const CodeView& b, const float* bias, void* out, int64_t ldo, hipStream_t s) {
  const dim3 g((b.rows + 16 * FN - 1) / (16 * FN), (a.rows + 16 * FM - 1) / (16 * FM));
  hipLaunchKernelGGL((az_matmul_direct<FM, FN, NW, F32>), g, dim3(NW * 64), 0, s, a, b, bias, out, ldo);
}

template <int W, int NW, bool F32>
void launch_tiled(const CodeView& a, const CodeView& b, const float* bias, void* out, int64_t ldo, hipStream_t s) {
  using K = Tiled<W, NW, F32>;
  static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void*>(az_matmul_tiled<W, NW, F32>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, 2 * K::STAGE);
  (void)once;
  const int mt = (a.rows + K::T - 1) / K::T, nt = (b.rows + K::T - 1) / K::T;
  hipLaunchKernelGGL((az_matmul_tiled<W, NW, F32>), dim3((unsigned)mt * (unsigned)nt), dim3(64 * NW), 2 * K::STAGE, s, a, b, bias, out, ldo, mt, nt);
}

template <bool F32>
void launch(const CodeView& a, const CodeView& b, const float* bias, void* out, int64_t ldo, hipStream_t s) {
  const bool fits = a.ld < (1 << 22) && b.ld < (1 << 22);  // a tile's offsets stay below 2^30
  if (fits && a.rows >= 1024 && b.rows >= 256) { launch_tiled<4, 4, F32>(a, b, bias, out, ldo, s); return; }
  if (fits && a.rows >= 128 && b.rows >= 128) { launch_tiled<2, 4, F32>(a, b, bias, out, ldo, s); return; }
  if (a.rows <= 16) launch_direct<1, 1, 8, F32>(a, b, bias, out, ldo, s);
  else if (a.rows <= 64) launch_direct<4, 1, 8, F32>(a, b, bias, out, ldo, s);
  else launch_direct<4, 4, 4, F32>(a, b, bias, out, ldo, s);
}

}  // namespace

extern "C" int az_codes_matmul(const az_code_matrix* a, const az_code_matrix* b, const float* bias, void* out,
                               int32_t dtype, int64_t ld_out, void* stream) {
  static const char who[] = "az_codes_matmul";
  int st = code_check(a, who);
  if (st == AZ_OK) st = code_check(b, who);
  if (st != AZ_OK) return st;
  if (a->cols != b->cols) return code_fail(AZ_ERR_INVALID_ARG, who, "a and b differ in cols");
  if (dtype != AZ_F32 && dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (a->rows == 0 || b->rows == 0) return AZ_OK;
  if ((st = dense_check(out, dtype, ld_out, b->rows, who)) != AZ_OK) return st;
  if ((uintptr_t)bias & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "bias must be 4-byte aligned");
  // 64 rows of a per workgroup row, and at most 65,535 of those in a grid
  if (a->rows > (int64_t)65535 * 64) return code_fail(AZ_ERR_UNSUPPORTED, who, "more than 4,194,240 rows of a");
  const CodeView va = code_view(*a), vb = code_view(*b);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (dtype == AZ_F32) launch<true>(va, vb, bias, out, ld_out, s);
  else launch<false>(va, vb, bias, out, ld_out, s);
  return launch_status(who);
}
