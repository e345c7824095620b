// The weight's and bias's gradients of a dense layer whose input was saved as
// codes: dw[n][k] = sum_m dy[m][n] x[m][k], db[n] = sum_m dy[m][n].
//
// The summed dimension runs down the rows of both operands.  A saved value is a bf16
// number exactly, and dy is bf16, so the product runs on the bf16 matrix
// instruction with exact terms.
#include "az_codes_common.h"

namespace {

constexpr int NT = 256, TN = 64, TK = 64, BM = 64;
constexpr int LROW = BM + 8;  // LDS row of one n or k: BM bf16 and a pad that spreads the banks

template <bool F32>
__device__ __forceinline__ void put(void* p, int64_t at, float v, bool add) {
  if constexpr (F32) {
    float* o = (float*)p + at;
    *o = add ? *o + v : v;
  } else {
    uint16_t* o = (uint16_t*)p + at;
    *o = bf16_of(add ? f32_of_bf16(*o) + v : v);
  }
}

// 64 columns of dy summed by one workgroup: four groups of rows, joined in order.
__device__ void bias_columns(const uint16_t* __restrict__ dy, int64_t ldy, int n, int m, int n0, float* db, bool add) {
  __shared__ float sums[4][64];
  const int c = n0 + (threadIdx.x & 63), q = threadIdx.x >> 6;
  float s = 0.0f;
  if (c < n)
    for (int i = q; i < m; i += 4) s += f32_of_bf16(dy[i * ldy + c]);
  sums[q][threadIdx.x & 63] = s;
  __syncthreads();
  if (q == 0 && c < n) {
    const float v = (sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]);
    db[c] = add ? db[c] + v : v;
  }
}

template <bool F32>
__global__ __launch_bounds__(NT) void az_weight_grad(const uint16_t* __restrict__ dy, int64_t ldy, int n, CodeView x,
                                                     void* __restrict__ dw, int64_t ldw, float* __restrict__ db,
                                                     int tiles, int add) {
  if ((int)blockIdx.x >= tiles) {
    bias_columns(dy, ldy, n, x.rows, ((int)blockIdx.x - tiles) * 64, db, add);
    return;
  }
  __shared__ uint16_t ys[TN * LROW], xs[TK * LROW];
  const int kt = (x.cols + TK - 1) / TK;
  const int n0 = (int)(blockIdx.x / kt) * TN, k0 = (int)(blockIdx.x % kt) * TK;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int wn = (wave & 1) * 32, wk = (wave >> 1) * 32, r = lane & 31, h = lane >> 5;
  cm_f32x16 acc = {};
  for (int m0 = 0; m0 < x.rows; m0 += BM) {
    // A thread takes one row's 16 columns of both operands and writes them as columns.
    const int mr = t >> 2, c = (t & 3) * 16, m = m0 + mr;
    uint16_t yv[16], xv[16];
#pragma unroll
    for (int i = 0; i < 16; i++) yv[i] = m < x.rows && n0 + c + i < n ? dy[m * ldy + n0 + c + i] : (uint16_t)0;
    cm_i32x4 w = {0, 0, 0, 0};
    float s = 0.0f;
    if (m < x.rows && k0 + c < x.cols) {
      w = code_chunk(x.codes + m * x.ld, k0 + c, x.cols);
      s = scale_value(x.scales[(int64_t)(m >> x.shift) * x.nb + (k0 + c) / CB]);
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t lo = code_pair_bf16<false>((uint32_t)w[i], s), hi = code_pair_bf16<true>((uint32_t)w[i], s);
      xv[4 * i] = (uint16_t)lo;
      xv[4 * i + 1] = (uint16_t)(lo >> 16);
      xv[4 * i + 2] = (uint16_t)hi;
      xv[4 * i + 3] = (uint16_t)(hi >> 16);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; i++) {
      ys[(c + i) * LROW + mr] = yv[i];
      xs[(c + i) * LROW + mr] = xv[i];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < BM / 16; q++) {
      const cm_bf16x8 fx = *reinterpret_cast<const cm_bf16x8*>(xs + (wk + r) * LROW + 16 * q + 8 * h);
      const cm_bf16x8 fy = *reinterpret_cast<const cm_bf16x8*>(ys + (wn + r) * LROW + 16 * q + 8 * h);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx, fy, acc, 0, 0, 0);
    }
  }
  // D: rows are k, columns are n
  const int nn = n0 + wn + r;
  if (nn >= n) return;
#pragma unroll
  for (int i = 0; i < 16; i++) {
    const int k = k0 + wk + 8 * (i >> 2) + 4 * h + (i & 3);
    if (k < x.cols) put<F32>(dw, nn * ldw + k, acc[i], add);
  }
}

}  // namespace

extern "C" size_t az_codes_weight_grad_workspace(int64_t rows, int32_t n, int64_t cols) {
  (void)rows, (void)n, (void)cols;
  return 0;
}

extern "C" int az_codes_weight_grad(const void* dy, int64_t ld_dy, int32_t n, const az_code_matrix* x, void* dw,
                                    int32_t dtype, int64_t ld_dw, float* db, int32_t accumulate, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  static const char who[] = "az_codes_weight_grad";
  int st = code_check(x, who);
  if (st != AZ_OK) return st;
  if (x->scale_rows != 1) return code_fail(AZ_ERR_INVALID_ARG, who, "x needs scale_rows 1");
  if (n < 0) return code_fail(AZ_ERR_INVALID_ARG, who, "n < 0");
  if (n == 0) return AZ_OK;
  if ((st = dense_check(dw, dtype, ld_dw, x->cols, who)) != AZ_OK) return st;
  if (x->rows > 0 && (st = dense_check(dy, AZ_BF16, ld_dy, n, who)) != AZ_OK) return st;
  if ((uintptr_t)db & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "db must be 4-byte aligned");
  const size_t need = az_codes_weight_grad_workspace(x->rows, n, x->cols);
  if (workspace_bytes < need || (need && !workspace)) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace is too small");
  if ((uintptr_t)workspace & 15u) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace must be 16-byte aligned");
  const CodeView v = code_view(*x);
  const int64_t tiles = ((int64_t)n + TN - 1) / TN * ((x->cols + TK - 1) / TK);
  const int64_t blocks = tiles + (db ? ((int64_t)n + 63) / 64 : 0);
  if (blocks > (1 << 30)) return code_fail(AZ_ERR_UNSUPPORTED, who, "a gradient past the size limits");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const uint16_t* y = static_cast<const uint16_t*>(dy);
  (void)hipGetLastError();
  if (dtype == AZ_F32)
    hipLaunchKernelGGL((az_weight_grad<true>), dim3((unsigned)blocks), dim3(NT), 0, s, y, ld_dy, n, v, dw, ld_dw, db, (int)tiles, accumulate != 0);
  else
    hipLaunchKernelGGL((az_weight_grad<false>), dim3((unsigned)blocks), dim3(NT), 0, s, y, ld_dy, n, v, dw, ld_dw, db, (int)tiles, accumulate != 0);
  return launch_status(who);
}
