// Matrices in 4 bits (az_fp4_matrix): quantising, with the transposed matrix, and restoring.
//
// One pass over memory and bound by it.  As with e4m3 codes the scale is a power of two, x * 2^-e
// is exact and the rounding to the code is the only one.
#include "az_nibbles_common.h"

namespace {

constexpr int NT = 256;

// Scale byte of a block whose largest |x| has these bits: 6 = 1.5 * 2^2.
__device__ __forceinline__ int nibble_scale(uint32_t a) {
  if (a == 0) return 127;
  const int e = (int)(a >> 23) - 127 - 2 + ((a & 0x7fffffu) > 0x400000u ? 1 : 0);
  return min(max(e, -125), 125) + 127;
}

// Eight codes of eight values over the scale: the instruction divides, rounds to the nearest, ties to even, and saturates at 6.
__device__ __forceinline__ uint32_t nibbles8(const float* x, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

// Largest |x| of 16 values by its bits, 0x7f800000 and more if one is not finite: the largest number among the bits as
// whole numbers is the largest positive value's, or, unsigned, the largest negative one's.
__device__ __forceinline__ uint32_t largest16(const float (&v)[16]) {
  int32_t a = 0;
  uint32_t b = 0;
#pragma unroll
  for (int i = 0; i < 16; i++) {
    a = max(a, __float_as_int(v[i]));
    b = max(b, __float_as_uint(v[i]));
  }
  return max((uint32_t)a, b >> 31 ? b & 0x7fffffffu : 0u);
}

// 16 codes of a half block; of a block that is not finite, zeros.
__device__ __forceinline__ uint64_t nibbles16(const float (&v)[16], int s) {
  if (s == 255) return 0;
  const float scale = __uint_as_float((uint32_t)s << 23);
  return nibbles8(v, scale) | (uint64_t)nibbles8(v + 8, scale) << 32;
}

// Writes the codes of 16 columns from c on (a multiple of 16), whole bytes and none past cols.
__device__ __forceinline__ void store_nibbles(uint8_t* row, int c, int cols, uint64_t u) {
  uint8_t* to = row + (c >> 1);
  const int left = (cols - c + 1) >> 1;
  if (left >= 8) {
    *reinterpret_cast<uint64_t*>(to) = u;
  } else if (left > 0) {
    if (left & 4) {
      *reinterpret_cast<uint32_t*>(to) = (uint32_t)u;
      u >>= 32;
      to += 4;
    }
    if (left & 2) {
      *reinterpret_cast<uint16_t*>(to) = (uint16_t)u;
      u >>= 16;
      to += 2;
    }
    if (left & 1) *to = (uint8_t)u;
  }
}

// Two lanes take a block, 16 columns each, eight lanes 128 columns.  64 x 10240 bf16: 2.8 us; 16384 x 4096 bf16 31.1, 4672 x 8192
// fp32 32.1 (5.4 TB/s, a copy's rate).
template <bool BF16>
__global__ __launch_bounds__(NT) void az_nibble_rows(const void* __restrict__ x, int64_t ldx, NibbleView q) {
  const uint32_t nb = ((uint32_t)q.cols + 127) / 128, total = (uint32_t)q.rows * nb, lane8 = threadIdx.x & 7;
  for (uint64_t id = blockIdx.x * (uint64_t)(NT / 8) + (threadIdx.x >> 3); id < total; id += (uint64_t)gridDim.x * (NT / 8)) {
    const uint32_t r = (uint32_t)id / nb, kb = (uint32_t)id - r * nb;
    const int c = (int)(kb * 128 + lane8 * 16);
    float v[16];
    load16<BF16>(x, (int64_t)r * ldx, c, q.cols, v);
    uint32_t a = largest16(v);
    a = max(a, (uint32_t)__shfl_xor((int)a, 1));
    const int s = a >= INF_BITS ? 255 : nibble_scale(a);
    store_nibbles(q.codes + (int64_t)r * q.ld, c, q.cols, nibbles16(v, s));
    if (!(lane8 & 1) && c < q.cols) q.scales[(int64_t)r * q.ld_scales + c / NB] = (uint8_t)s;
  }
}

// Tiles of 64 x 128 through LDS: a wave reads whole lines of the rows, and a thread then takes a block of 32
// columns of a row, and one of 32 rows of a column.  LDS rows' 16-byte chunks are exchanged (place_of), so that
// none of the three meets a bank twice.  4672 x 8192 fp32: 51 us (3.8 TB/s), of which reading alone takes 40; an order of
// tiles that keeps neighbours on one XCD took 54.
constexpr int TROWS = 64;
__device__ __forceinline__ int place_of(int row, int chunk) {
  return row * 32 + (chunk ^ ((chunk >> 4) & 1) ^ ((row & 3) << 1) ^ ((row >> 5) << 3));
}

// The codes of 32 values and their scale byte.
__device__ __forceinline__ int nibbles32(const float (&lo)[16], const float (&hi)[16], cm_i32x4& w) {
  const uint32_t a = max(largest16(lo), largest16(hi));
  const int s = a >= INF_BITS ? 255 : nibble_scale(a);
  const uint64_t u = nibbles16(lo, s), v = nibbles16(hi, s);
  w = cm_i32x4{(int)u, (int)(u >> 32), (int)v, (int)(v >> 32)};
  return s;
}

// Writes a block's codes from column c on (a multiple of 32), whole bytes and none past cols.
__device__ __forceinline__ void store_block(uint8_t* row, int c, int cols, const cm_i32x4& w) {
  if (c + NB <= cols) {
    *reinterpret_cast<cm_i32x4*>(row + c / 2) = w;
  } else {
    store_nibbles(row, c, cols, (uint32_t)w[0] | (uint64_t)(uint32_t)w[1] << 32);
    if (c + 16 < cols) store_nibbles(row, c + 16, cols, (uint32_t)w[2] | (uint64_t)(uint32_t)w[3] << 32);
  }
}

// EDGE: of the loads.
template <bool BF16, int EDGE>
__global__ __launch_bounds__(NT) void az_nibble_tiles(const void* __restrict__ x, int64_t ldx, NibbleView q, NibbleView qt, int nt) {
  __shared__ cm_f32x4 tile[TROWS * 32];
  constexpr int N = BF16 ? 8 : 4, LANES = 128 / N, LOADS = TROWS * LANES / NT;  // columns of a load, and loads of a thread
  const int rb = (int)(blockIdx.x / (uint32_t)nt), kb = (int)(blockIdx.x % (uint32_t)nt);
  const int t = threadIdx.x, r0 = rb * TROWS, c0 = kb * 128, rows = min(q.rows - r0, TROWS), cl = t % LANES * N;
  Raw<BF16, N, EDGE> raw[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; i++) {
    const int r = min(i * (NT / LANES) + t / LANES, rows - 1);
    raw[i].load(x, (int64_t)(r0 + r) * ldx, c0 + cl, q.cols);
  }
#pragma unroll
  for (int i = 0; i < LOADS; i++) {
    const int r = i * (NT / LANES) + t / LANES;
    float v[N];
    raw[i].settle(v);
    const bool live = r < rows && (EDGE != EVEN || c0 + cl < q.cols);
#pragma unroll
    for (int k = 0; k < N / 4; k++)
      tile[place_of(r, cl / 4 + k)] = live ? cm_f32x4{v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]} : cm_f32x4{0, 0, 0, 0};
  }
  __syncthreads();
  float lo[16], hi[16];
  cm_i32x4 w;
  {
    const int r = t >> 2, c = c0 + (t & 3) * NB;
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const cm_f32x4 v = tile[place_of(r, (t & 3) * 8 + k)];
#pragma unroll
      for (int e = 0; e < 4; e++) (k < 4 ? lo : hi)[4 * (k & 3) + e] = v[e];
    }
    if (r < rows && c < q.cols) {
      const int s = nibbles32(lo, hi, w);
      store_block(q.codes + (int64_t)(r0 + r) * q.ld, c, q.cols, w);
      q.scales[(int64_t)(r0 + r) * q.ld_scales + c / NB] = (uint8_t)s;
    }
  }
  {
    const int j = t >> 1, i0 = (t & 1) * NB, rt = c0 + j, ct = r0 + i0;
    const float* column = reinterpret_cast<const float*>(tile) + (j & 3);
#pragma unroll
    for (int i = 0; i < 32; i++) (i < 16 ? lo : hi)[i & 15] = column[4 * place_of(i0 + i, j >> 2)];
    if (rt < qt.rows && ct < qt.cols) {
      const int s = nibbles32(lo, hi, w);
      store_block(qt.codes + (int64_t)rt * qt.ld, ct, qt.cols, w);
      qt.scales[(int64_t)rt * qt.ld_scales + ct / NB] = (uint8_t)s;
    }
  }
}

// A thread restores 16 bytes of a row at a time, so that a wave writes whole lines, AHEAD of them on their way together.
// 2^shift threads have one of the `parts` of a row.  4672 x 8192 to fp32: 32-42 us (16 columns a thread, 64 bytes apart: 69).
template <bool BF16, int AHEAD>
__global__ __launch_bounds__(NT) void az_nibble_values(NibbleView q, void* __restrict__ x, int64_t ldx, int shift, uint32_t parts) {
  constexpr int N = BF16 ? 8 : 4;
  const int t = threadIdx.x & ((1 << shift) - 1), step = N << shift, items = NT >> shift;
  const int64_t total = (int64_t)q.rows * parts;
  for (int64_t id = blockIdx.x * (int64_t)items + (threadIdx.x >> shift); id < total; id += (int64_t)gridDim.x * items) {
    const int64_t r = parts == 1 ? id : id / parts, first = (id - r * parts) * AHEAD * step + t * N;
    const uint8_t* from = q.codes + r * q.ld;
    const uint8_t* scales = q.scales + r * q.ld_scales;
    uint32_t w[AHEAD], sb[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      const int c = (int)min(first + (int64_t)a * step, (int64_t)(q.cols - 1) / N * N);  // (past the row: its last ones again)
      if constexpr (BF16) w[a] = *reinterpret_cast<const uint32_t*>(from + c / 2);
      else w[a] = *reinterpret_cast<const uint16_t*>(from + c / 2);
      sb[a] = scales[c / NB];
    }
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      const int64_t c = first + (int64_t)a * step;
      if (c >= q.cols) break;
      const float s = scale_value(sb[a]);
      float v[N];
      const auto f0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[a], 1.0f, 0), f1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[a], 1.0f, 1);
      v[0] = f0[0] * s, v[1] = f0[1] * s, v[2] = f1[0] * s, v[3] = f1[1] * s;
      if constexpr (BF16) {
        const auto f2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[a], 1.0f, 2), f3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[a], 1.0f, 3);
        v[4] = f2[0] * s, v[5] = f2[1] * s, v[6] = f3[0] * s, v[7] = f3[1] * s;
      }
      put<BF16, N>(x, r * ldx, (int)c, q.cols, v);
    }
  }
}

// Workgroups of a pass in which each takes NT / 8 parts of 128 columns at a time.
dim3 pass_grid(const NibbleView& q) {
  const int64_t groups = ((int64_t)q.rows * ((q.cols + 127) / 128) + NT / 8 - 1) / (NT / 8);
  return dim3((unsigned)(groups < 65536 ? groups : 65536));
}

// Threads of a part: as many as a row has use for.  Four loads a thread where that leaves every compute unit four workgroups
// (64 x 10240 bf16: 4.0 us with four, 2.7 with one).
template <bool BF16, int AHEAD>
void launch_values(const NibbleView& q, void* x, int64_t ldx, hipStream_t s) {
  constexpr int64_t N = BF16 ? 8 : 4;
  int shift = 3;
  while (shift < 8 && (N * AHEAD) << shift < q.cols) shift++;
  const int64_t parts = (q.cols + ((N * AHEAD) << shift) - 1) / ((N * AHEAD) << shift);
  const int64_t groups = ((int64_t)q.rows * parts + (NT >> shift) - 1) / (NT >> shift);
  hipLaunchKernelGGL((az_nibble_values<BF16, AHEAD>), dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20)), dim3(NT), 0, s, q, x, ldx, shift, (uint32_t)parts);
}

template <bool BF16>
void launch_values(const NibbleView& q, void* x, int64_t ldx, hipStream_t s) {
  if ((int64_t)q.rows * q.cols >= (int64_t)1024 * NT * 4 * (BF16 ? 8 : 4)) launch_values<BF16, 4>(q, x, ldx, s);
  else launch_values<BF16, 1>(q, x, ldx, s);
}

template <bool BF16>
int launch_quantize(const void* x, int64_t ldx, const NibbleView& q, const NibbleView* qt, hipStream_t s) {
  if (!qt) {
    hipLaunchKernelGGL((az_nibble_rows<BF16>), pass_grid(q), dim3(NT), 0, s, x, ldx, q);
    return AZ_OK;
  }
  const int64_t mt = ((int64_t)q.rows + TROWS - 1) / TROWS, nt = (q.cols + 127) / 128;
  if (!grid_fits(mt * nt, NT)) return AZ_ERR_UNSUPPORTED;
  const dim3 g((unsigned)(mt * nt));
  if (q.cols % (BF16 ? 8 : 4) == 0) hipLaunchKernelGGL((az_nibble_tiles<BF16, EVEN>), g, dim3(NT), 0, s, x, ldx, q, *qt, (int)nt);
  else if (q.cols >= 8) hipLaunchKernelGGL((az_nibble_tiles<BF16, PARTLY>), g, dim3(NT), 0, s, x, ldx, q, *qt, (int)nt);
  else hipLaunchKernelGGL((az_nibble_tiles<BF16, ANY>), g, dim3(NT), 0, s, x, ldx, q, *qt, (int)nt);
  return AZ_OK;
}

}  // namespace

extern "C" int az_nibbles_quantize(const void* x, int32_t dtype, int64_t ldx, const az_fp4_matrix* q, const az_fp4_matrix* qt,
                                   void* stream) {
  static const char who[] = "az_nibbles_quantize";
  int st = nibble_check(q, who);
  if (st != AZ_OK) return st;
  if (q->rows == 0) return AZ_OK;  // (its transposed form, of no columns, is no matrix to check)
  if (qt) {
    if (qt->rows != q->cols || qt->cols != q->rows) return code_fail(AZ_ERR_INVALID_ARG, who, "the transposed matrix has other sizes");
    if ((st = nibble_check(qt, who)) != AZ_OK) return st;
  }
  if ((st = dense_check(x, dtype, ldx, q->cols, who)) != AZ_OK) return st;
  const NibbleView v = nibble_view(*q), vt = qt ? nibble_view(*qt) : v;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const NibbleView* t = qt ? &vt : nullptr;
  st = dtype == AZ_BF16 ? launch_quantize<true>(x, ldx, v, t, s) : launch_quantize<false>(x, ldx, v, t, s);
  return launched(who, st);
}

extern "C" int az_nibbles_dequantize(const az_fp4_matrix* q, void* x, int32_t dtype, int64_t ldx, void* stream) {
  static const char who[] = "az_nibbles_dequantize";
  int st = nibble_check(q, who);
  if (st != AZ_OK) return st;
  if (q->rows == 0) return AZ_OK;
  if ((st = dense_check(x, dtype, ldx, q->cols, who)) != AZ_OK) return st;
  const NibbleView v = nibble_view(*q);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (dtype == AZ_BF16) launch_values<true>(v, x, ldx, s);
  else launch_values<false>(v, x, ldx, s);
  return launch_status(who);
}
