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

// Eight codes of eight values, scaled by inv: the instruction rounds to the nearest, ties to even, and is given
// nothing past 6.
__device__ __forceinline__ uint32_t nibbles8(const float* x, float inv) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; i++) y[i] = __builtin_amdgcn_fmed3f(x[i] * inv, -6.0f, 6.0f);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], 1.0f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.0f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.0f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.0f, 3);
}

// The factor of a block with this scale byte, 2^-e; 0 for 255, whose codes are zeros.
__device__ __forceinline__ float nibble_inverse(int s) { return s == 255 ? 0.0f : __uint_as_float((uint32_t)(254 - s) << 23); }

// Largest |x| of 16 values by its bits, 0x7f800000 and more if one is not finite.
__device__ __forceinline__ uint32_t largest16(const float (&v)[16]) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 16; i++) a = max(a, __float_as_uint(v[i]) & 0x7fffffffu);
  return a;
}

// 16 codes of a half block; of a block that is not finite, zeros.
__device__ __forceinline__ uint64_t nibbles16(const float (&v)[16], int s) {
  if (s == 255) return 0;
  const float inv = nibble_inverse(s);
  return nibbles8(v, inv) | (uint64_t)nibbles8(v + 8, inv) << 32;
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

// Two lanes take a block, 16 columns each, eight lanes 128 columns.
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

// Tiles of 128 x 128, their rows from registers and their columns through LDS.
template <bool BF16>
__global__ __launch_bounds__(NT) void az_nibble_tiles(const void* __restrict__ x, int64_t ldx, NibbleView q, NibbleView qt) {
  extern __shared__ __attribute__((aligned(16))) float tile[];  // [128][128]
  const uint32_t nb = ((uint32_t)q.cols + 127) / 128;
  const uint32_t rb = blockIdx.x / nb, kb = blockIdx.x - rb * nb;
  const int t = threadIdx.x, c = (int)kb * 128 + (t & 7) * 16;
  const int64_t r0 = (int64_t)rb * 128 + (t >> 3);
  float v[4][16];
#pragma unroll
  for (int p = 0; p < 4; p++) load16<BF16>(x, min(r0 + 32 * p, (int64_t)q.rows - 1) * ldx, c, q.cols, v[p]);
#pragma unroll
  for (int p = 0; p < 4; p++) {
    const int64_t r = r0 + 32 * p;
    uint32_t a = largest16(v[p]);
    a = max(a, (uint32_t)__shfl_xor((int)a, 1));
    const int s = a >= INF_BITS ? 255 : nibble_scale(a);
    if (r < q.rows && c < q.cols) {
      store_nibbles(q.codes + r * q.ld, c, q.cols, nibbles16(v[p], s));
      if (!(t & 1)) q.scales[r * q.ld_scales + c / NB] = (uint8_t)s;
    }
    cm_f32x4* to = reinterpret_cast<cm_f32x4*>(tile + ((t >> 3) + 32 * p) * 128 + (t & 7) * 16);
#pragma unroll
    for (int i = 0; i < 4; i++)
      to[i] = r < q.rows ? cm_f32x4{v[p][4 * i], v[p][4 * i + 1], v[p][4 * i + 2], v[p][4 * i + 3]} : cm_f32x4{0, 0, 0, 0};
  }
  __syncthreads();
  // A thread takes a column's rows, two blocks of 32.
  const int j = t & 127;
  const int64_t rt = (int64_t)kb * 128 + j;
#pragma unroll
  for (int p = 0; p < 2; p++) {
    const int i0 = (t >> 7) * 64 + 32 * p, ct = (int)rb * 128 + i0;
    if (rt >= qt.rows || ct >= qt.cols) continue;
    float lo[16], hi[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
      lo[i] = tile[(i0 + i) * 128 + j];
      hi[i] = tile[(i0 + 16 + i) * 128 + j];
    }
    const uint32_t a = max(largest16(lo), largest16(hi));
    const int s = a >= INF_BITS ? 255 : nibble_scale(a);
    uint8_t* row = qt.codes + rt * qt.ld;
    store_nibbles(row, ct, qt.cols, nibbles16(lo, s));
    if (ct + 16 < qt.cols) store_nibbles(row, ct + 16, qt.cols, nibbles16(hi, s));
    qt.scales[rt * qt.ld_scales + ct / NB] = (uint8_t)s;
  }
}

template <bool BF16>
__global__ __launch_bounds__(NT) void az_nibble_values(NibbleView q, void* __restrict__ x, int64_t ldx) {
  const uint32_t nb = ((uint32_t)q.cols + 127) / 128, total = (uint32_t)q.rows * nb, lane8 = threadIdx.x & 7;
  for (uint64_t id = blockIdx.x * (uint64_t)(NT / 8) + (threadIdx.x >> 3); id < total; id += (uint64_t)gridDim.x * (NT / 8)) {
    const uint32_t r = (uint32_t)id / nb, kb = (uint32_t)id - r * nb;
    const int c = (int)(kb * 128 + lane8 * 16);
    if (c >= q.cols) continue;
    const float s = scale_value(q.scales[(int64_t)r * q.ld_scales + c / NB]);
    const uint64_t u = *reinterpret_cast<const uint64_t*>(q.codes + (int64_t)r * q.ld + (c >> 1));
    float v[16];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const uint32_t w = (uint32_t)(u >> (32 * i));
      const auto f0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0), f1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
      const auto f2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2), f3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
      v[8 * i] = f0[0] * s, v[8 * i + 1] = f0[1] * s, v[8 * i + 2] = f1[0] * s, v[8 * i + 3] = f1[1] * s;
      v[8 * i + 4] = f2[0] * s, v[8 * i + 5] = f2[1] * s, v[8 * i + 6] = f3[0] * s, v[8 * i + 7] = f3[1] * s;
    }
    put16<BF16>(x, (int64_t)r * ldx, c, q.cols, v);
  }
}

int64_t parts_of(const NibbleView& q) { return (int64_t)q.rows * ((q.cols + 127) / 128); }

dim3 pass_grid(const NibbleView& q) {
  const int64_t groups = (parts_of(q) + NT / 8 - 1) / (NT / 8);
  return dim3((unsigned)(groups < 65536 ? groups : 65536));
}

template <bool BF16>
int launch_quantize(const void* x, int64_t ldx, const NibbleView& q, const NibbleView* qt, hipStream_t s) {
  if (!qt) {
    hipLaunchKernelGGL((az_nibble_rows<BF16>), pass_grid(q), dim3(NT), 0, s, x, ldx, q);
    return AZ_OK;
  }
  const int64_t tiles = ((int64_t)q.rows + 127) / 128 * ((q.cols + 127) / 128);
  if (!grid_fits(tiles, NT)) return AZ_ERR_UNSUPPORTED;
  const int lds = 128 * 128 * (int)sizeof(float);
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(az_nibble_tiles<BF16>), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return AZ_ERR_DEVICE;
  hipLaunchKernelGGL((az_nibble_tiles<BF16>), dim3((unsigned)tiles), dim3(NT), lds, s, x, ldx, q, *qt);
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
  if (dtype == AZ_BF16) hipLaunchKernelGGL((az_nibble_values<true>), pass_grid(v), dim3(NT), 0, s, v, x, ldx);
  else hipLaunchKernelGGL((az_nibble_values<false>), pass_grid(v), dim3(NT), 0, s, v, x, ldx);
  return launch_status(who);
}
