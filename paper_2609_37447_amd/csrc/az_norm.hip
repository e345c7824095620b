// Root-mean-square norm of rows with a residual's addition, into e4m3 codes or a dense matrix, and its gradients.
//
// Both are one pass over memory and bound by it: a row stays in registers, 16 columns a thread, between
// its sums and its results.  Sums over a row are fp64 (its rate is fp32's on this chip, and no finite row
// overflows); everything after them is fp32, rounded once.  A block of 128 columns is eight neighbouring
// lanes, which find its scale by lane exchanges.
#include <math.h>

#include "az_codes_common.h"

namespace {

constexpr int PER = 16;             // columns of a thread
constexpr int MOST = 1024 * PER;    // columns of a row that stays in registers
constexpr int MAX_COLS = 1 << 24;

struct NormView {
  const void* x;
  const void* residual;
  const float* weight;
  void* sum;
  void* y;
  uint8_t* codes;
  uint8_t* scales;
  int64_t ld_x, ld_residual, ld_sum, ld_y, ld_codes;
  int64_t rows;
  int cols, nb;
  float eps;
};

// Sum over the T threads of a row (T a power of two), in every thread.  `red`: a place for each wave of the workgroup.
template <int T, int N>
__device__ __forceinline__ void row_sums(double (&v)[N], double (*red)[N]) {
  for (int o = (T < 64 ? T : 64) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; i++) v[i] += __shfl_xor(v[i], o);
  if constexpr (T > 64) {
    const int wave = threadIdx.x >> 6, first = wave & ~(T / 64 - 1);
    __syncthreads();  // the last row's sums have been read
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; i++) red[wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) {
      v[i] = 0.0;
      for (int w = 0; w < T / 64; w++) v[i] += red[first + w][i];
    }
  }
}

__device__ __forceinline__ float inverse_root(double squares, int cols, float eps) {
  return (float)(1.0 / sqrt(squares / cols + (double)eps));
}

// h of 16 columns from c on.
template <bool BF16>
__device__ __forceinline__ void stream16(const NormView& p, int64_t r, int c, float (&v)[16]) {
  load16<BF16>(p.x, r * p.ld_x, c, p.cols, v);
  if (p.residual) {
    float add[16];
    load16<BF16>(p.residual, r * p.ld_residual, c, p.cols, add);
#pragma unroll
    for (int i = 0; i < 16; i++) {
      v[i] += add[i];
      if constexpr (BF16) v[i] = f32_of_bf16(bf16_of(v[i]));
    }
  }
}

// The results of 16 columns; the eight lanes of a block of 128 columns call it together.
template <bool BF16>
__device__ __forceinline__ void results16(const NormView& p, int64_t r, int c, float inv, const float (&w)[16], float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 16; i++) v[i] = v[i] * inv * w[i];
  if (p.y && c < p.cols) put16<BF16>(p.y, r * p.ld_y, c, p.cols, v);
  if (p.codes) {
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) {
      if (c + i >= p.cols) v[i] = 0.0f;  // (NaN of a NaN row)
      a = max(a, finite_size(v[i]));
    }
    for (int o = 4; o > 0; o >>= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o));
    const int s = scale_byte(a);
    const float scale = __uint_as_float((uint32_t)(254 - s) << 23);
    cm_i32x4 u;
#pragma unroll
    for (int i = 0; i < 4; i++) u[i] = (int)codes4(v + 4 * i, scale);
    if (c < p.cols) {
      store16(p.codes + r * p.ld_codes, c, p.cols, u);
      if ((threadIdx.x & 7) == 0) p.scales[r * p.nb + c / CB] = (uint8_t)s;
    }
  }
}

__device__ __forceinline__ void weights16(const float* weight, int c, int cols, float (&w)[16]) {
  if (weight) {
    load16<false>(weight, 0, c, cols, w);
  } else {
#pragma unroll
    for (int i = 0; i < 16; i++) w[i] = 1.0f;
  }
}

// T threads a row, 1,024 / T rows (T < 256: 256 / T) a workgroup at a time.
template <bool BF16, int T>
__global__ __launch_bounds__(T < 256 ? 256 : T) void az_norm_rows(NormView p) {
  constexpr int NT = T < 256 ? 256 : T, ROWS = NT / T;
  __shared__ double red[NT / 64][1];
  const int c = (int)(threadIdx.x % T) * PER;
  float w[16];
  weights16(p.weight, min(c, p.cols - 1), p.cols, w);
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < p.rows; r0 += (int64_t)gridDim.x * ROWS) {
    const int64_t r = r0 + threadIdx.x / T;
    const bool live = r < p.rows && c < p.cols;
    float v[16] = {};
    if (live) stream16<BF16>(p, r, c, v);
    if (live && p.sum) put16<BF16>(p.sum, r * p.ld_sum, c, p.cols, v);
    if (!p.y && !p.codes) continue;
    double s[1] = {0.0};
#pragma unroll
    for (int i = 0; i < 16; i++) s[0] = fma((double)v[i], (double)v[i], s[0]);
    row_sums<T, 1>(s, red);
    if (r < p.rows) results16<BF16>(p, r, c, inverse_root(s[0], p.cols, p.eps), w, v);
  }
}

// Longer rows are read twice; h comes from `sum` the second time where it was written there.
template <bool BF16>
__global__ __launch_bounds__(1024) void az_norm_long(NormView p) {
  __shared__ double red[16][1];
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    double s[1] = {0.0};
    for (int c0 = 0; c0 < p.cols; c0 += MOST) {
      const int c = c0 + (int)threadIdx.x * PER;
      if (c >= p.cols) continue;
      float v[16];
      stream16<BF16>(p, r, c, v);
      if (p.sum) put16<BF16>(p.sum, r * p.ld_sum, c, p.cols, v);
#pragma unroll
      for (int i = 0; i < 16; i++) s[0] = fma((double)v[i], (double)v[i], s[0]);
    }
    if (!p.y && !p.codes) continue;
    row_sums<1024, 1>(s, red);
    const float inv = inverse_root(s[0], p.cols, p.eps);
    NormView again = p;
    if (p.sum) {
      again.x = p.sum;
      again.ld_x = p.ld_sum;
      again.residual = nullptr;
    }
    for (int c0 = 0; c0 < p.cols; c0 += MOST) {
      const int c = c0 + (int)threadIdx.x * PER;
      float v[16] = {}, w[16];
      weights16(p.weight, min(c, p.cols - 1), p.cols, w);
      if (c < p.cols) stream16<BF16>(again, r, c, v);
      results16<BF16>(p, r, c, inv, w, v);
    }
  }
}

struct GradView {
  const void* dy;
  const void* h;
  const float* weight;
  const void* dsum;
  void* dx;
  float* parts;  // [slots][cols]: the weight's gradient over a slot's rows
  int64_t ld_dy, ld_h, ld_dsum, ld_dx;
  int64_t rows;
  int cols, slots;
  float eps;
};

// dx of 16 columns; d keeps dy.
template <bool BF16>
__device__ __forceinline__ void input_grad16(const GradView& p, int64_t r, int c, float inv, float mean, const float (&w)[16],
                                             const float (&h)[16], const float (&d)[16]) {
  float o[16];
  if (p.dsum) load16<BF16>(p.dsum, r * p.ld_dsum, c, p.cols, o);
#pragma unroll
  for (int i = 0; i < 16; i++) {
    const float g = inv * (d[i] * w[i] - h[i] * inv * mean);
    o[i] = p.dsum ? g + o[i] : g;
  }
  put16<BF16>(p.dx, r * p.ld_dx, c, p.cols, o);
}

// Slot i takes the rows i, i + slots, ...; T threads a slot.
template <bool BF16, int T>
__global__ __launch_bounds__(T < 256 ? 256 : T) void az_norm_grad_rows(GradView p) {
  constexpr int NT = T < 256 ? 256 : T;
  __shared__ double red[NT / 64][2];
  const int c = (int)(threadIdx.x % T) * PER, slot = (int)blockIdx.x * (NT / T) + (int)(threadIdx.x / T);
  float w[16], dw[16] = {};
  weights16(p.weight, min(c, p.cols - 1), p.cols, w);
  for (int64_t r0 = 0; r0 < p.rows; r0 += p.slots) {
    const int64_t r = r0 + slot;
    const bool live = r < p.rows && slot < p.slots && c < p.cols;
    float h[16] = {}, d[16] = {};
    if (live) {
      load16<BF16>(p.h, r * p.ld_h, c, p.cols, h);
      load16<BF16>(p.dy, r * p.ld_dy, c, p.cols, d);
    }
    double s[2] = {0.0, 0.0};
#pragma unroll
    for (int i = 0; i < 16; i++) {
      s[0] = fma((double)h[i], (double)h[i], s[0]);
      s[1] = fma((double)(d[i] * w[i]), (double)h[i], s[1]);
    }
    row_sums<T, 2>(s, red);
    const float inv = inverse_root(s[0], p.cols, p.eps), mean = (float)(s[1] * (double)inv / p.cols);
    if (live) {
#pragma unroll
      for (int i = 0; i < 16; i++) dw[i] = fmaf(d[i], h[i] * inv, dw[i]);
      if (p.dx) input_grad16<BF16>(p, r, c, inv, mean, w, h, d);
    }
  }
  if (p.parts && slot < p.slots && c < p.cols) put16<false>(p.parts, (int64_t)slot * p.cols, c, p.cols, dw);
}

// Rows past the registers: the sums first, then the results, and the weight's gradient through the slot's part.
template <bool BF16>
__global__ __launch_bounds__(1024) void az_norm_grad_long(GradView p) {
  __shared__ double red[16][2];
  float* const part = p.parts ? p.parts + (int64_t)blockIdx.x * p.cols : nullptr;
  for (int64_t r = blockIdx.x; r < p.rows; r += p.slots) {
    double s[2] = {0.0, 0.0};
    for (int c = (int)threadIdx.x * PER; c < p.cols; c += MOST) {
      float h[16], d[16], w[16];
      weights16(p.weight, c, p.cols, w);
      load16<BF16>(p.h, r * p.ld_h, c, p.cols, h);
      load16<BF16>(p.dy, r * p.ld_dy, c, p.cols, d);
#pragma unroll
      for (int i = 0; i < 16; i++) {
        s[0] = fma((double)h[i], (double)h[i], s[0]);
        s[1] = fma((double)(d[i] * w[i]), (double)h[i], s[1]);
      }
    }
    row_sums<1024, 2>(s, red);
    const float inv = inverse_root(s[0], p.cols, p.eps), mean = (float)(s[1] * (double)inv / p.cols);
    for (int c = (int)threadIdx.x * PER; c < p.cols; c += MOST) {
      float h[16], d[16], w[16];
      weights16(p.weight, c, p.cols, w);
      load16<BF16>(p.h, r * p.ld_h, c, p.cols, h);
      load16<BF16>(p.dy, r * p.ld_dy, c, p.cols, d);
      if (part) {
#pragma unroll
        for (int i = 0; i < 16; i++)
          if (c + i < p.cols) {
            const float u = d[i] * (h[i] * inv);
            part[c + i] = r == blockIdx.x ? u : part[c + i] + u;
          }
      }
      if (p.dx) input_grad16<BF16>(p, r, c, inv, mean, w, h, d);
    }
  }
}

// The weight's gradient from its parts, in their order: 32 columns a workgroup, 32 threads each, whose
// sums of every 32nd part meet in LDS.
__global__ __launch_bounds__(1024) void az_norm_join(const float* __restrict__ parts, int count, int cols, float* __restrict__ dw, int accumulate) {
  __shared__ float sums[32][33];
  const int j = threadIdx.x & 31, g = threadIdx.x >> 5, c = (int)blockIdx.x * 32 + j;
  float s = 0.0f;
  if (c < cols) {
#pragma unroll 8
    for (int i = g; i < count; i += 32) s += parts[(int64_t)i * cols + c];
  }
  sums[g][j] = s;
  __syncthreads();
  if (g == 0 && c < cols) {
    s = 0.0f;
    for (int i = 0; i < 32; i++) s += sums[i][j];
    dw[c] = accumulate ? dw[c] + s : s;
  }
}

// Threads of a row, 16 columns each; 0: the row is longer than a workgroup holds.
int row_threads(int64_t cols) {
  if (cols > MOST) return 0;
  int t = 8;
  while (t * PER < cols) t *= 2;
  return t;
}

// Slots that the weight's gradient is summed in: enough threads to fill the chip, and eight rows or more in
// each, so that the parts are little beside the rows.
int grad_slots(int64_t rows, int64_t cols) {
  const int t = row_threads(cols);
  const int64_t fill = t ? 262144 / t : 256, few = (rows + 7) / 8 > 256 ? (rows + 7) / 8 : 256;
  const int64_t slots = few < fill ? few : fill;
  return (int)(rows < slots ? rows : slots);
}

template <bool BF16>
void launch_norm(const NormView& p, hipStream_t s) {
  const int t = row_threads(p.cols), rows = t && t < 256 ? 256 / t : 1;
  const int64_t need = (p.rows + rows - 1) / rows;
  const dim3 g((unsigned)(need < (1 << 20) ? need : 1 << 20));
  switch (t) {
    case 8: hipLaunchKernelGGL((az_norm_rows<BF16, 8>), g, dim3(256), 0, s, p); break;
    case 16: hipLaunchKernelGGL((az_norm_rows<BF16, 16>), g, dim3(256), 0, s, p); break;
    case 32: hipLaunchKernelGGL((az_norm_rows<BF16, 32>), g, dim3(256), 0, s, p); break;
    case 64: hipLaunchKernelGGL((az_norm_rows<BF16, 64>), g, dim3(256), 0, s, p); break;
    case 128: hipLaunchKernelGGL((az_norm_rows<BF16, 128>), g, dim3(256), 0, s, p); break;
    case 256: hipLaunchKernelGGL((az_norm_rows<BF16, 256>), g, dim3(256), 0, s, p); break;
    case 512: hipLaunchKernelGGL((az_norm_rows<BF16, 512>), g, dim3(512), 0, s, p); break;
    case 1024: hipLaunchKernelGGL((az_norm_rows<BF16, 1024>), g, dim3(1024), 0, s, p); break;
    default: hipLaunchKernelGGL((az_norm_long<BF16>), g, dim3(1024), 0, s, p);
  }
}

template <bool BF16>
void launch_norm_grad(const GradView& p, hipStream_t s) {
  const int t = row_threads(p.cols), slots = t && t < 256 ? 256 / t : 1;
  const dim3 g((unsigned)((p.slots + slots - 1) / slots));
  switch (t) {
    case 8: hipLaunchKernelGGL((az_norm_grad_rows<BF16, 8>), g, dim3(256), 0, s, p); break;
    case 16: hipLaunchKernelGGL((az_norm_grad_rows<BF16, 16>), g, dim3(256), 0, s, p); break;
    case 32: hipLaunchKernelGGL((az_norm_grad_rows<BF16, 32>), g, dim3(256), 0, s, p); break;
    case 64: hipLaunchKernelGGL((az_norm_grad_rows<BF16, 64>), g, dim3(256), 0, s, p); break;
    case 128: hipLaunchKernelGGL((az_norm_grad_rows<BF16, 128>), g, dim3(256), 0, s, p); break;
    case 256: hipLaunchKernelGGL((az_norm_grad_rows<BF16, 256>), g, dim3(256), 0, s, p); break;
    case 512: hipLaunchKernelGGL((az_norm_grad_rows<BF16, 512>), g, dim3(512), 0, s, p); break;
    case 1024: hipLaunchKernelGGL((az_norm_grad_rows<BF16, 1024>), g, dim3(1024), 0, s, p); break;
    default: hipLaunchKernelGGL((az_norm_grad_long<BF16>), g, dim3(1024), 0, s, p);
  }
}

bool norm_sizes(int64_t rows, int64_t cols) { return rows <= INT32_MAX && cols <= MAX_COLS; }

int norm_sizes_check(int64_t rows, int64_t cols, int32_t dtype, float eps, const char* who) {
  if (rows < 0 || cols < 1) return code_fail(AZ_ERR_INVALID_ARG, who, "rows < 0 or cols < 1");
  if (dtype != AZ_F32 && dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (!(eps >= 0x1p-126f && eps < INFINITY)) return code_fail(AZ_ERR_INVALID_ARG, who, "eps is not a positive normal number");
  return norm_sizes(rows, cols) ? AZ_OK : code_fail(AZ_ERR_UNSUPPORTED, who, "rows > 2^31 - 1 or cols > 2^24");
}

}  // namespace

extern "C" int az_rms_norm(const az_norm* n, void* stream) {
  static const char who[] = "az_rms_norm";
  if (!n) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL norm");
  int st = norm_sizes_check(n->rows, n->cols, n->dtype, n->eps, who);
  if (st != AZ_OK) return st;
  if (n->q) {
    if ((st = code_check(n->q, who)) != AZ_OK) return st;
    if (n->q->scale_rows != 1) return code_fail(AZ_ERR_INVALID_ARG, who, "q needs scale_rows 1");
    if (n->q->rows != n->rows || n->q->cols != n->cols) return code_fail(AZ_ERR_INVALID_ARG, who, "q has other sizes");
  }
  if (n->rows == 0) return AZ_OK;
  if (!n->sum && !n->y && !n->q) return code_fail(AZ_ERR_INVALID_ARG, who, "neither sum, y nor q is given");
  if ((st = dense_check(n->x, n->dtype, n->ld_x, n->cols, who)) != AZ_OK) return st;
  if (n->residual && (st = dense_check(n->residual, n->dtype, n->ld_residual, n->cols, who)) != AZ_OK) return st;
  if (n->sum && (st = dense_check(n->sum, n->dtype, n->ld_sum, n->cols, who)) != AZ_OK) return st;
  if (n->y && (st = dense_check(n->y, n->dtype, n->ld_y, n->cols, who)) != AZ_OK) return st;
  if ((uintptr_t)n->weight & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "weight must be 4-byte aligned");
  const NormView p = {n->x, n->residual, n->weight, n->sum, n->y, n->q ? n->q->codes : nullptr, n->q ? n->q->scales : nullptr,
                      n->ld_x, n->ld_residual, n->ld_sum, n->ld_y, n->q ? n->q->ld : 0, n->rows, (int)n->cols,
                      (int)((n->cols + CB - 1) / CB), n->eps};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (n->dtype == AZ_BF16) launch_norm<true>(p, s);
  else launch_norm<false>(p, s);
  return launch_status(who);
}

extern "C" size_t az_rms_norm_grad_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || !norm_sizes(rows, cols)) return 0;
  return ((size_t)grad_slots(rows, cols) * (size_t)cols * sizeof(float) + 15) & ~(size_t)15;
}

extern "C" int az_rms_norm_grad(const az_norm_grad* n, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "az_rms_norm_grad";
  if (!n) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL gradient");
  int st = norm_sizes_check(n->rows, n->cols, n->dtype, n->eps, who);
  if (st != AZ_OK) return st;
  if (((uintptr_t)n->weight | (uintptr_t)n->dweight) & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "weight and dweight must be 4-byte aligned");
  if (n->rows > 0) {
    if (!n->dx && !n->dweight) return code_fail(AZ_ERR_INVALID_ARG, who, "neither dx nor dweight is given");
    if ((st = dense_check(n->dy, n->dtype, n->ld_dy, n->cols, who)) != AZ_OK) return st;
    if ((st = dense_check(n->h, n->dtype, n->ld_h, n->cols, who)) != AZ_OK) return st;
    if (n->dsum && (st = dense_check(n->dsum, n->dtype, n->ld_dsum, n->cols, who)) != AZ_OK) return st;
    if (n->dx && (st = dense_check(n->dx, n->dtype, n->ld_dx, n->cols, who)) != AZ_OK) return st;
  }
  const size_t need = n->dweight ? az_rms_norm_grad_workspace(n->rows, n->cols) : 0;
  if (workspace_bytes < need || (need && !workspace)) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace is too small");
  if (need && ((uintptr_t)workspace & 15u)) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace must be 16-byte aligned");
  const hipStream_t s = static_cast<hipStream_t>(stream);
  float* const parts = n->dweight ? static_cast<float*>(workspace) : nullptr;
  const int slots = grad_slots(n->rows, n->cols);
  (void)hipGetLastError();
  if (n->rows > 0) {
    const GradView p = {n->dy, n->h, n->weight, n->dsum, n->dx, parts, n->ld_dy, n->ld_h, n->ld_dsum, n->ld_dx,
                        n->rows, (int)n->cols, slots, n->eps};
    if (n->dtype == AZ_BF16) launch_norm_grad<true>(p, s);
    else launch_norm_grad<false>(p, s);
    if ((st = launch_status(who)) != AZ_OK) return st;
  }
  if (n->dweight) {
    hipLaunchKernelGGL(az_norm_join, dim3((unsigned)((n->cols + 31) / 32)), dim3(1024), 0, s, parts, slots, (int)n->cols,
                       n->dweight, n->accumulate != 0);
    st = launch_status(who);
  }
  return st;
}
