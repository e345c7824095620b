// Root-mean-square norm of rows with a residual's addition, into e4m3 codes or a dense matrix, and its gradients.
//
// Both are one pass over memory and bound by it: a row stays in registers between its sums and its results.  Rows of the norm
// overlap as workgroups of one row each (a persistent grid with the next row on its way: 127 us for 87 at 16384 x 4096);
// the gradient's workgroups keep sums over many rows, and fetch the next one meanwhile.  Sums over a row are fp64 (its
// rate is fp32's on this chip, and no finite row overflows); everything after them is fp32, rounded once.  A block of
// 128 columns is 16 neighbouring lanes, which find its scale by lane exchanges.
#include <math.h>

#include "az_codes_common.h"

namespace {

constexpr int PER = 8;                    // neighbouring columns of a thread: a group
constexpr int MOST = 1024 * PER;          // columns of a group of every thread of the largest workgroup
constexpr int MAX_COLS = 1 << 24;
constexpr int FILL = 256 * 1024;          // threads that fill half of the chip

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

// T: threads of a row, 16 or 64 with several rows a workgroup of 256, or WHOLE: the workgroup.
constexpr int WHOLE = 0;
template <int T>
__device__ __forceinline__ int threads_of_row() { return T == WHOLE ? (int)blockDim.x : T; }

template <int CTRL>
__device__ __forceinline__ double lane_move(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xf, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, false);
  return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double lane_value(double x, int lane) {
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}

// Sums over the threads of a row, in every one of them.  `red`: a place for each wave of the workgroup, another one each
// time that this is called (turn), so that one barrier does.
template <int T, int N>
__device__ __forceinline__ void row_sums(double (&v)[N], double (*red)[16][N], int turn) {
#pragma unroll
  for (int i = 0; i < N; i++) {
    v[i] += lane_move<0xb1>(v[i]);   // lane ^ 1
    v[i] += lane_move<0x4e>(v[i]);   // lane ^ 2
    v[i] += lane_move<0x141>(v[i]);  // the other four of eight
    v[i] += lane_move<0x140>(v[i]);  // the other eight of sixteen
    if constexpr (T != 16) v[i] = (lane_value(v[i], 0) + lane_value(v[i], 16)) + (lane_value(v[i], 32) + lane_value(v[i], 48));
  }
  if constexpr (T == WHOLE) {
    const int wave = threadIdx.x >> 6, waves = (int)blockDim.x / 64;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; i++) red[turn & 1][wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = 0.0;
    for (int w = 0; w < waves; w++)
#pragma unroll
      for (int i = 0; i < N; i++) v[i] += red[turn & 1][w][i];
  }
}

__device__ __forceinline__ float inverse_root(double squares, int cols, float eps) {
  return (float)(1.0 / sqrt(squares / cols + (double)eps));
}

// What h comes from, a group from c on: on its way, and added up.  EDGE, here and below: of its groups.
template <bool BF16, int EDGE>
struct Stream {
  Raw<BF16, PER, EDGE> x, residual;
  __device__ __forceinline__ void load(const NormView& p, int64_t r, int c) {
    x.load(p.x, r * p.ld_x, c, p.cols);
    if (p.residual) residual.load(p.residual, r * p.ld_residual, c, p.cols);
  }
  __device__ __forceinline__ void sum(const NormView& p, float (&v)[PER]) const {
    x.settle(v);
    if (p.residual) {
      float add[PER];
      residual.settle(add);
#pragma unroll
      for (int i = 0; i < PER; i++) {
        v[i] += add[i];
        if constexpr (BF16) v[i] = f32_of_bf16(bf16_of(v[i]));
      }
    }
  }
};

// The results of a group; the 16 lanes of a block of 128 columns call it together.
template <bool BF16, int EDGE>
__device__ __forceinline__ void results8(const NormView& p, int64_t r, int c, float inv, const float (&w)[PER], float (&v)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; i++) v[i] = v[i] * inv * w[i];
  if (p.y && c < p.cols) put<BF16, PER, EDGE>(p.y, r * p.ld_y, c, p.cols, v);
  if (p.codes) {
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < PER; i++) {
      if (EDGE != EVEN && c + i >= p.cols) v[i] = 0.0f;  // (NaN of a NaN row)
      a = max(a, finite_size(v[i]));
    }
    if (EDGE == EVEN && c >= p.cols) a = 0;
    a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0xb1, 0xf, 0xf, false));
    a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x4e, 0xf, 0xf, false));
    a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x141, 0xf, 0xf, false));
    a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x140, 0xf, 0xf, false));
    const int s = scale_byte(a);
    const float scale = __uint_as_float((uint32_t)(254 - s) << 23);
    if (c < p.cols) {
      uint64_t u = codes4(v, scale) | (uint64_t)codes4(v + 4, scale) << 32;
      uint8_t* to = p.codes + r * p.ld_codes + c;
      if (EDGE == EVEN || c + PER <= p.cols) {
        *reinterpret_cast<uint64_t*>(to) = u;
      } else {
        for (int i = c; i < p.cols; i++, u >>= 8) *to++ = (uint8_t)u;
      }
      if ((threadIdx.x & 15) == 0) p.scales[r * p.nb + c / CB] = (uint8_t)s;
    }
  }
}

// A group's weights.
template <int EDGE>
__device__ __forceinline__ void weights8(const float* weight, int c, int cols, float (&w)[PER]) {
  if (weight) {
    Raw<false, PER, EDGE> raw;
    raw.load(weight, 0, min(c, cols - 1), cols);
    raw.settle(w);
  } else {
#pragma unroll
    for (int i = 0; i < PER; i++) w[i] = 1.0f;
  }
}

// A thread has G groups, a row's threads' groups side by side.  Threads without a row or a column read one that there is.
// 16384 x 4096 bf16 with a residual into codes: 85-89 us, 5.3-5.5 TB/s (16384 x 4095, whose rows begin anywhere: 124); 333 x 10240 fp32: 9.5; one row of 8,192: 4.3.
template <bool BF16, int EDGE, int T, int G>
__global__ __launch_bounds__(T == WHOLE ? 1024 : 256) void az_norm_rows(NormView p) {
  constexpr int ROWS = T == WHOLE ? 1 : 256 / (T ? T : 1);
  __shared__ double red[2][16][1];
  const int threads = threads_of_row<T>(), t = T == WHOLE ? (int)threadIdx.x : (int)threadIdx.x % threads;
  int turn = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < p.rows; r0 += (int64_t)gridDim.x * ROWS, turn++) {
    const int64_t r = r0 + (T == WHOLE ? 0 : threadIdx.x / threads), at = min(r, p.rows - 1);
    Stream<BF16, EDGE> x[G];
    float v[G][PER], w[G][PER];
    double s[1] = {0.0};
#pragma unroll
    for (int g = 0; g < G; g++) x[g].load(p, at, min((g * threads + t) * PER, p.cols - 1));
#pragma unroll
    for (int g = 0; g < G; g++) weights8<EDGE>(p.weight, (g * threads + t) * PER, p.cols, w[g]);
#pragma unroll
    for (int g = 0; g < G; g++) {
      const int c = (g * threads + t) * PER;
      x[g].sum(p, v[g]);
      if (r < p.rows && c < p.cols && p.sum) put<BF16, PER, EDGE>(p.sum, r * p.ld_sum, c, p.cols, v[g]);
      double sum = 0.0;
#pragma unroll
      for (int i = 0; i < PER; i++) sum = fma((double)v[g][i], (double)v[g][i], sum);
      s[0] += c < p.cols ? sum : 0.0;
    }
    if (!p.y && !p.codes) continue;
    row_sums<T, 1>(s, red, turn);
    const float inv = inverse_root(s[0], p.cols, p.eps);
    if (r < p.rows) {
#pragma unroll
      for (int g = 0; g < G; g++) results8<BF16, EDGE>(p, r, (g * threads + t) * PER, inv, w[g], v[g]);
    }
  }
}

// Longer rows are read twice; h comes from `sum` the second time where it was written there.
template <bool BF16>
__global__ __launch_bounds__(1024) void az_norm_long(NormView p) {
  __shared__ double red[2][16][1];
  int turn = 0;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x, turn++) {
    double s[1] = {0.0};
    for (int c = (int)threadIdx.x * PER; c < p.cols; c += MOST) {
      Stream<BF16, PARTLY> x;
      float v[PER];
      x.load(p, r, c);
      x.sum(p, v);
      if (p.sum) put<BF16, PER>(p.sum, r * p.ld_sum, c, p.cols, v);
#pragma unroll
      for (int i = 0; i < PER; i++) s[0] = fma((double)v[i], (double)v[i], s[0]);
    }
    if (!p.y && !p.codes) continue;
    row_sums<WHOLE, 1>(s, red, turn);
    const float inv = inverse_root(s[0], p.cols, p.eps);
    NormView again = p;
    if (p.sum) {
      again.x = p.sum;
      again.ld_x = p.ld_sum;
      again.residual = nullptr;
    }
    for (int c0 = 0; c0 < p.cols; c0 += MOST) {
      const int c = c0 + (int)threadIdx.x * PER;
      float v[PER] = {}, w[PER];
      weights8<PARTLY>(p.weight, c, p.cols, w);
      if (c < p.cols) {
        Stream<BF16, PARTLY> x;
        x.load(again, r, c);
        x.sum(again, v);
      }
      results8<BF16, PARTLY>(p, r, c, inv, w, v);
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

// What the gradients of a group come from.
template <bool BF16, int EDGE>
struct GradStream {
  Raw<BF16, PER, EDGE> h, dy, dsum;
  __device__ __forceinline__ void load(const GradView& p, int64_t r, int c) {
    h.load(p.h, r * p.ld_h, c, p.cols);
    dy.load(p.dy, r * p.ld_dy, c, p.cols);
    if (p.dsum) dsum.load(p.dsum, r * p.ld_dsum, c, p.cols);
  }
};

__device__ __forceinline__ void grad_sums(double (&s)[2], const float (&w)[PER], const float (&h)[PER], const float (&d)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; i++) {
    s[0] = fma((double)h[i], (double)h[i], s[0]);
    s[1] = fma((double)(d[i] * w[i]), (double)h[i], s[1]);
  }
}

// dx of a group; o holds dsum.
template <bool BF16, int EDGE>
__device__ __forceinline__ void input_grad8(const GradView& p, int64_t r, int c, float inv, float mean, const float (&w)[PER],
                                            const float (&h)[PER], const float (&d)[PER], float (&o)[PER]) {
#pragma unroll
  for (int i = 0; i < PER; i++) {
    const float g = inv * (d[i] * w[i] - h[i] * inv * mean);
    o[i] = p.dsum ? g + o[i] : g;
  }
  put<BF16, PER, EDGE>(p.dx, r * p.ld_dx, c, p.cols, o);
}

// Keeps the compiler from holding what it makes of these words over this point: they are unpacked again.
template <bool BF16, int EDGE>
__device__ __forceinline__ void unpack_again(Raw<BF16, PER, EDGE>& x) {
#pragma unroll
  for (int i = 0; i < x.WORDS; i++) asm volatile("" : "+v"(x.w[i]));
}

// Slot i takes the rows i, i + slots, ...  A row stays as it lies in memory, and is unpacked for its sums and for its results;
// the next one is on its way meanwhile.  16384 x 4096 bf16 with dsum: 110 us with the join (4), 4.8 TB/s; 16384 x 4095: 142;
// 64 x 10240: 6.3 and the join.
template <bool BF16, int EDGE, int T, int G>
__global__ __launch_bounds__(T == WHOLE ? 1024 : 256) void az_norm_grad_rows(GradView p) {
  constexpr bool AHEAD = G == 1;  // (two groups' next row would not fit the registers)
  __shared__ double red[2][16][2];
  const int threads = threads_of_row<T>(), t = T == WHOLE ? (int)threadIdx.x : (int)threadIdx.x % threads;
  const int slot = T == WHOLE ? (int)blockIdx.x : (int)blockIdx.x * (256 / (T ? T : 1)) + (int)(threadIdx.x / threads);
  GradStream<BF16, EDGE> next[G];
  float w[G][PER], dw[G][PER] = {};
  auto fetch = [&](int64_t r) {
#pragma unroll
    for (int g = 0; g < G; g++) next[g].load(p, min(r, p.rows - 1), min((g * threads + t) * PER, p.cols - 1));
  };
  fetch(slot);
#pragma unroll
  for (int g = 0; g < G; g++) weights8<EDGE>(p.weight, (g * threads + t) * PER, p.cols, w[g]);
  int turn = 0;
  for (int64_t r0 = 0; r0 < p.rows; r0 += p.slots, turn++) {
    const int64_t r = r0 + slot;
    GradStream<BF16, EDGE> x[G];
    double s[2] = {0.0, 0.0};
    if constexpr (!AHEAD) {
      if (r0 > 0) fetch(r);
    }
#pragma unroll
    for (int g = 0; g < G; g++) x[g] = next[g];
    if constexpr (AHEAD) {
      if (r0 + p.slots < p.rows) fetch(r + p.slots);
    }
#pragma unroll
    for (int g = 0; g < G; g++) {
      float h[PER], d[PER];
      double sum[2] = {0.0, 0.0};
      x[g].h.settle(h);
      x[g].dy.settle(d);
      grad_sums(sum, w[g], h, d);
#pragma unroll
      for (int i = 0; i < 2; i++) s[i] += (g * threads + t) * PER < p.cols ? sum[i] : 0.0;
    }
    row_sums<T, 2>(s, red, turn);
    const float inv = inverse_root(s[0], p.cols, p.eps), mean = (float)(s[1] * (double)inv / p.cols);
    if (r < p.rows && slot < p.slots) {
#pragma unroll
      for (int g = 0; g < G; g++) {
        const int c = (g * threads + t) * PER;
        unpack_again(x[g].h);
        unpack_again(x[g].dy);
        float h[PER], d[PER], o[PER];
        x[g].h.settle(h);
        x[g].dy.settle(d);
        if (p.dsum) x[g].dsum.settle(o);
#pragma unroll
        for (int i = 0; i < PER; i++) dw[g][i] = fmaf(d[i], h[i] * inv, dw[g][i]);
        if (p.dx && c < p.cols) input_grad8<BF16, EDGE>(p, r, c, inv, mean, w[g], h, d, o);
      }
    }
  }
  if (p.parts && slot < p.slots) {
#pragma unroll
    for (int g = 0; g < G; g++) {
      const int c = (g * threads + t) * PER;
      if (c < p.cols) put<false, PER, EDGE>(p.parts, (int64_t)slot * p.cols, c, p.cols, dw[g]);
    }
  }
}

// Rows past the registers: the sums first, then the results, and the weight's gradient through the slot's part.
template <bool BF16>
__global__ __launch_bounds__(1024) void az_norm_grad_long(GradView p) {
  __shared__ double red[2][16][2];
  int turn = 0;
  float* const part = p.parts ? p.parts + (int64_t)blockIdx.x * p.cols : nullptr;
  for (int64_t r = blockIdx.x; r < p.rows; r += p.slots, turn++) {
    double s[2] = {0.0, 0.0};
    for (int c = (int)threadIdx.x * PER; c < p.cols; c += MOST) {
      GradStream<BF16, PARTLY> x;
      float h[PER], d[PER], w[PER];
      x.h.load(p.h, r * p.ld_h, c, p.cols);
      x.dy.load(p.dy, r * p.ld_dy, c, p.cols);
      weights8<PARTLY>(p.weight, c, p.cols, w);
      x.h.settle(h);
      x.dy.settle(d);
      grad_sums(s, w, h, d);
    }
    row_sums<WHOLE, 2>(s, red, turn);
    const float inv = inverse_root(s[0], p.cols, p.eps), mean = (float)(s[1] * (double)inv / p.cols);
    for (int c = (int)threadIdx.x * PER; c < p.cols; c += MOST) {
      GradStream<BF16, PARTLY> x;
      float h[PER], d[PER], w[PER], o[PER];
      x.load(p, r, c);
      weights8<PARTLY>(p.weight, c, p.cols, w);
      x.h.settle(h);
      x.dy.settle(d);
      if (p.dsum) x.dsum.settle(o);
      if (part) {
#pragma unroll
        for (int i = 0; i < PER; i++)
          if (c + i < p.cols) {
            const float u = d[i] * (h[i] * inv);
            part[c + i] = r == blockIdx.x ? u : part[c + i] + u;
          }
      }
      if (p.dx) input_grad8<BF16, PARTLY>(p, r, c, inv, mean, w, h, d, o);
    }
  }
}

// The weight's gradient from its parts, in their order (512 parts of 4,096: 4 us): 32 columns a workgroup, 32 threads each, whose
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

// Threads of a row of `groups` groups each: 16, 64 or whole waves; 0: the row is longer than a workgroup holds, two groups
// a thread.
struct Shape {
  int threads, groups;
};
Shape row_shape(int64_t cols) {
  if (cols > 2 * MOST) return {0, 0};
  if (cols <= 64 * PER) return {cols <= 16 * PER ? 16 : 64, 1};
  const int groups = cols > MOST ? 2 : 1, wave = 64 * PER * groups;
  return {(int)((cols + wave - 1) / wave) * 64, groups};
}

// Slots that the weight's gradient is summed in: enough threads to fill half of the chip, and from 2,048 rows on eight rows or
// more in each, so that the parts are little beside the rows.  Fewer rows have 256 slots, of a row each up to 256 rows: the
// parts are then as many fp32 numbers as the matrix has entries, written and read once (64 x 10240 bf16: 2.6 MB each way beside 5.2).
int grad_slots(int64_t rows, int64_t cols) {
  const int t = row_shape(cols).threads;
  const int64_t fill = t ? FILL / t : 256, few = (rows + 7) / 8 > 256 ? (rows + 7) / 8 : 256;
  const int64_t slots = few < fill ? few : fill;
  return (int)(rows < slots ? rows : slots);
}

template <bool BF16, int EDGE>
void launch_norm(const NormView& p, hipStream_t s) {
  const Shape f = row_shape(p.cols);
  const int rows = f.threads == 16 ? 16 : f.threads == 64 ? 4 : 1;
  const int64_t need = (p.rows + rows - 1) / rows;
  const dim3 g((unsigned)(need < (1 << 20) ? need : 1 << 20));
  if (f.threads == 0) hipLaunchKernelGGL((az_norm_long<BF16>), g, dim3(1024), 0, s, p);
  else if (f.threads == 16 && p.cols < PER) hipLaunchKernelGGL((az_norm_rows<BF16, ANY, 16, 1>), g, dim3(256), 0, s, p);
  else if (f.threads == 16) hipLaunchKernelGGL((az_norm_rows<BF16, EDGE, 16, 1>), g, dim3(256), 0, s, p);
  else if (f.threads == 64) hipLaunchKernelGGL((az_norm_rows<BF16, EDGE, 64, 1>), g, dim3(256), 0, s, p);
  else if (f.groups == 1) hipLaunchKernelGGL((az_norm_rows<BF16, EDGE, WHOLE, 1>), g, dim3(f.threads), 0, s, p);
  else hipLaunchKernelGGL((az_norm_rows<BF16, EDGE, WHOLE, 2>), g, dim3(f.threads), 0, s, p);
}

template <bool BF16, int EDGE>
void launch_norm_grad(const GradView& p, hipStream_t s) {
  const Shape f = row_shape(p.cols);
  const int slots = f.threads == 16 ? 16 : f.threads == 64 ? 4 : 1;
  const dim3 g((unsigned)((p.slots + slots - 1) / slots));
  if (f.threads == 0) hipLaunchKernelGGL((az_norm_grad_long<BF16>), g, dim3(1024), 0, s, p);
  else if (f.threads == 16 && p.cols < PER) hipLaunchKernelGGL((az_norm_grad_rows<BF16, ANY, 16, 1>), g, dim3(256), 0, s, p);
  else if (f.threads == 16) hipLaunchKernelGGL((az_norm_grad_rows<BF16, EDGE, 16, 1>), g, dim3(256), 0, s, p);
  else if (f.threads == 64) hipLaunchKernelGGL((az_norm_grad_rows<BF16, EDGE, 64, 1>), g, dim3(256), 0, s, p);
  else if (f.groups == 1) hipLaunchKernelGGL((az_norm_grad_rows<BF16, EDGE, WHOLE, 1>), g, dim3(f.threads), 0, s, p);
  else hipLaunchKernelGGL((az_norm_grad_rows<BF16, EDGE, WHOLE, 2>), g, dim3(f.threads), 0, s, p);
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
  const bool even = n->cols % PER == 0;
  if (n->dtype == AZ_BF16) even ? launch_norm<true, EVEN>(p, s) : launch_norm<true, PARTLY>(p, s);
  else even ? launch_norm<false, EVEN>(p, s) : launch_norm<false, PARTLY>(p, s);
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
    const bool even = n->cols % PER == 0;
    if (n->dtype == AZ_BF16) even ? launch_norm_grad<true, EVEN>(p, s) : launch_norm_grad<true, PARTLY>(p, s);
    else even ? launch_norm_grad<false, EVEN>(p, s) : launch_norm_grad<false, PARTLY>(p, s);
    if ((st = launch_status(who)) != AZ_OK) return st;
  }
  if (n->dweight) {
    hipLaunchKernelGGL(az_norm_join, dim3((unsigned)((n->cols + 31) / 32)), dim3(1024), 0, s, parts, slots, (int)n->cols,
                       n->dweight, n->accumulate != 0);
    st = launch_status(who);
  }
  return st;
}
