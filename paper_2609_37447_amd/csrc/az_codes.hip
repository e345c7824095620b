// Coded matrices (az_code_matrix): quantising and restoring.
//
// Both are one pass over memory and bound by it.  A block's scale is a power of
// two, so that x * 2^-e is exact and the only rounding is the one to the code: every
// code is the definition's, whatever the order of the block's maximum.
#include "az_codes_common.h"

namespace {

constexpr int NT = 256;
// Rows with a scale of their own: eight lanes take a block of 128, 16 columns each.
// 16384 x 4096 bf16: 42-46 us, 4.4-4.8 TB/s.
template <bool BF16>
__global__ __launch_bounds__(NT) void az_quantize_rows(const void* __restrict__ x, int64_t ldx, CodeView q) {
  const uint32_t total = (uint32_t)q.rows * (uint32_t)q.nb;
  const uint32_t lane8 = threadIdx.x & 7;
  for (uint32_t id = blockIdx.x * (NT / 8) + (threadIdx.x >> 3); id < total; id += gridDim.x * (NT / 8)) {
    const uint32_t r = id / (uint32_t)q.nb, kb = id - r * (uint32_t)q.nb;
    const int c = (int)(kb * CB + lane8 * 16);
    float v[16];
    load16<BF16>(x, (int64_t)r * ldx, c, q.cols, v);
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) a = max(a, finite_size(v[i]));
    for (int o = 4; o > 0; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 8));
    const int s = scale_byte(a);
    const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
    cm_i32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = (int)codes4(v + 4 * i, inv);
    store16(q.codes + (int64_t)r * q.ld, c, q.cols, w);
    if (lane8 == 0) q.scales[id] = (uint8_t)s;
  }
}

// Tiles of 128 x 128 with one scale, and their transposed copy through LDS.  4672 x 8192 fp32 and
// both copies: 48 us, 4.8 TB/s.
template <bool BF16, bool TRANSPOSED>
__global__ __launch_bounds__(NT) void az_quantize_tiles(const void* __restrict__ x, int64_t ldx, CodeView q, CodeView qt) {
  __shared__ uint32_t most[NT / 64];
  __shared__ __attribute__((aligned(16))) uint8_t tile[TRANSPOSED ? CB * (CB + 4) : 4];  // (written by words)
  const uint32_t rb = blockIdx.x / (uint32_t)q.nb, kb = blockIdx.x - rb * (uint32_t)q.nb;
  const int t = threadIdx.x, c = (int)kb * CB + (t & 7) * 16;
  const int64_t r0 = (int64_t)rb * CB + (t >> 3);
  float v[4][16];
  uint32_t a = 0;
#pragma unroll
  for (int p = 0; p < 4; p++) {
    const int64_t r = r0 + 32 * p;
    load16<BF16>(x, min(r, (int64_t)q.rows - 1) * ldx, c, q.cols, v[p]);
  }
#pragma unroll
  for (int p = 0; p < 4; p++)
#pragma unroll
    for (int i = 0; i < 16; i++) {
      if (r0 + 32 * p >= q.rows) v[p][i] = 0.0f;
      a = max(a, finite_size(v[p][i]));
    }
  for (int o = 32; o > 0; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o));
  if ((t & 63) == 0) most[t >> 6] = a;
  __syncthreads();
  a = max(max(most[0], most[1]), max(most[2], most[3]));
  const int s = scale_byte(a);
  const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
  if (t == 0) {
    q.scales[(int64_t)rb * q.nb + kb] = (uint8_t)s;
    if constexpr (TRANSPOSED) qt.scales[(int64_t)kb * qt.nb + rb] = (uint8_t)s;
  }
#pragma unroll
  for (int p = 0; p < 4; p++) {
    const int64_t r = r0 + 32 * p;
    cm_i32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = (int)codes4(v[p] + 4 * i, inv);
    if (r < q.rows && c < q.cols) store16(q.codes + r * q.ld, c, q.cols, w);
    if constexpr (TRANSPOSED) {
      uint32_t* to = reinterpret_cast<uint32_t*>(tile + ((t >> 3) + 32 * p) * (CB + 4) + (t & 7) * 16);
#pragma unroll
      for (int i = 0; i < 4; i++) to[i] = (uint32_t)w[i];
    }
  }
  if constexpr (TRANSPOSED) {
    __syncthreads();
    // Row j of the transposed tile is column j of the tile.
#pragma unroll
    for (int p = 0; p < 4; p++) {
      const int j = (t >> 3) + 32 * p, i0 = (t & 7) * 16;
      cm_i32x4 w;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        uint32_t u = 0;
#pragma unroll
        for (int b = 0; b < 4; b++) u |= (uint32_t)tile[(i0 + 4 * i + b) * (CB + 4) + j] << (8 * b);
        w[i] = (int)u;
      }
      const int64_t r = (int64_t)kb * CB + j;
      const int ct = (int)rb * CB + i0;
      if (r < qt.rows && ct < qt.cols) store16(qt.codes + r * qt.ld, ct, qt.cols, w);
    }
  }
}

// 16384 x 4096 to bf16: 31 us, two thirds of the traffic written.
template <bool BF16>
__global__ __launch_bounds__(NT) void az_dequantize(CodeView q, void* __restrict__ x, int64_t ldx) {
  const uint32_t total = (uint32_t)q.rows * (uint32_t)q.nb;
  const uint32_t lane8 = threadIdx.x & 7;
  for (uint32_t id = blockIdx.x * (NT / 8) + (threadIdx.x >> 3); id < total; id += gridDim.x * (NT / 8)) {
    const uint32_t r = id / (uint32_t)q.nb, kb = id - r * (uint32_t)q.nb;
    const int c = (int)(kb * CB + lane8 * 16);
    if (c >= q.cols) continue;
    const float s = scale_value(q.scales[(int64_t)(r >> q.shift) * q.nb + kb]);
    const cm_i32x4 w = code_chunk(q.codes + (int64_t)r * q.ld, c, q.cols);
    float v[16];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[4 * i] = __builtin_amdgcn_cvt_f32_fp8(w[i], 0) * s;
      v[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8(w[i], 1) * s;
      v[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8(w[i], 2) * s;
      v[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8(w[i], 3) * s;
    }
    const int64_t at = (int64_t)r * ldx + c;
    if constexpr (BF16) {
      uint16_t* o = (uint16_t*)x + at;
      if (c + 16 <= q.cols) {
        cm_i32x4 u[2];
#pragma unroll
        for (int i = 0; i < 8; i++)
          u[i >> 2][i & 3] = (int)((uint32_t)bf16_of(v[2 * i]) | ((uint32_t)bf16_of(v[2 * i + 1]) << 16));
        __builtin_memcpy(o, u, 32);
      } else {
#pragma unroll
        for (int i = 0; i < 16; i++)
          if (c + i < q.cols) o[i] = bf16_of(v[i]);
      }
    } else {
      float* o = (float*)x + at;
      if (c + 16 <= q.cols) {
        __builtin_memcpy(o, v, 64);
      } else {
#pragma unroll
        for (int i = 0; i < 16; i++)
          if (c + i < q.cols) o[i] = v[i];
      }
    }
  }
}

// Workgroups of a pass in which each takes NT / 8 blocks at a time.
int pass_grid(const CodeView& q) {
  const int64_t groups = ((int64_t)q.rows * q.nb + NT / 8 - 1) / (NT / 8);
  return (int)(groups < 65536 ? groups : 65536);
}

template <bool BF16>
int launch_quantize(const void* x, int64_t ldx, const CodeView& q, const CodeView* qt, hipStream_t s) {
  if (q.shift == 0) {
    hipLaunchKernelGGL((az_quantize_rows<BF16>), dim3(pass_grid(q)), dim3(NT), 0, s, x, ldx, q);
    return AZ_OK;
  }
  const int64_t tiles = ((int64_t)q.rows + CB - 1) / CB * q.nb;
  if (!grid_fits(tiles, NT)) return AZ_ERR_UNSUPPORTED;
  if (qt) hipLaunchKernelGGL((az_quantize_tiles<BF16, true>), dim3((unsigned)tiles), dim3(NT), 0, s, x, ldx, q, *qt);
  else hipLaunchKernelGGL((az_quantize_tiles<BF16, false>), dim3((unsigned)tiles), dim3(NT), 0, s, x, ldx, q, q);
  return AZ_OK;
}

}  // namespace

extern "C" int az_codes_quantize(const void* x, int32_t dtype, int64_t ldx, const az_code_matrix* q,
                                 const az_code_matrix* qt, void* stream) {
  static const char who[] = "az_codes_quantize";
  int st = code_check(q, who);
  if (st != AZ_OK) return st;
  if (qt && (q->scale_rows != CB || qt->scale_rows != CB))
    return code_fail(AZ_ERR_INVALID_ARG, who, "the transposed matrix needs scale_rows 128 in both");
  if (q->rows == 0) return AZ_OK;  // (its transposed form, of no columns, is no matrix to check)
  if (qt) {
    if (qt->rows != q->cols || qt->cols != q->rows)
      return code_fail(AZ_ERR_INVALID_ARG, who, "the transposed matrix has other sizes");
    if ((st = code_check(qt, who)) != AZ_OK) return st;
  }
  if ((st = dense_check(x, dtype, ldx, q->cols, who)) != AZ_OK) return st;
  const CodeView v = code_view(*q);
  const CodeView vt = qt ? code_view(*qt) : v;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const CodeView* t = qt ? &vt : nullptr;
  st = dtype == AZ_BF16 ? launch_quantize<true>(x, ldx, v, t, s) : launch_quantize<false>(x, ldx, v, t, s);
  return launched(who, st);
}

extern "C" int az_codes_dequantize(const az_code_matrix* q, void* x, int32_t dtype, int64_t ldx, void* stream) {
  static const char who[] = "az_codes_dequantize";
  int st = code_check(q, who);
  if (st != AZ_OK) return st;
  if (q->rows == 0) return AZ_OK;
  if ((st = dense_check(x, dtype, ldx, q->cols, who)) != AZ_OK) return st;
  const CodeView v = code_view(*q);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 g(pass_grid(v)), b(NT);
  (void)hipGetLastError();
  if (dtype == AZ_BF16) hipLaunchKernelGGL((az_dequantize<true>), g, b, 0, s, v, x, ldx);
  else hipLaunchKernelGGL((az_dequantize<false>), g, b, 0, s, v, x, ldx);
  return launch_status(who);
}
