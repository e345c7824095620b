// Shared by the tiled products: how a tile's results leave, and how parts of the summed dimension are joined.  Private to
// the library.
#pragma once

#include "az_codes_common.h"

namespace {

typedef __attribute__((address_space(3))) uint8_t lds_bytes;

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

// Results leave through LDS, so that whole rows of the tile are written: a lane's four neighbours
// would be 16 bytes of each of 32 rows.  Chunks are exchanged by the row, as the kernels' operands are.
// K: FA x FB blocks of 32 x 32 a wave, ACROSS waves along the tile's TM rows, LDS bytes at smem.  `to`: the tile's first
// result, n0: its column, ms and ns: the rows and columns that there are, r and h: the lane's.
template <class K, bool F32>
__device__ __forceinline__ void write_tile(const cm_f32x16 (&acc)[K::FA][K::FB], uint8_t* smem, const float* __restrict__ bias, uint8_t* to,
                                           int64_t ldo, int n0, int ms, int ns, int wave, int r, int h) {
  const int t = threadIdx.x;
  const int wn = (wave / K::ACROSS) * 32 * K::FB;
  constexpr int ES = F32 ? 4 : 2, OROW = K::TN * ES, RC = OROW / 16;  // bytes and chunks of a row
  constexpr int PASSES = K::LDS >= K::TM * OROW ? 1 : 2;  // fp32 of the largest tile: half of each wave's rows at a time
  constexpr int PF = K::FA / PASSES, PROWS = K::TM / PASSES;
#pragma unroll
  for (int p = 0; p < PASSES; p++) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < K::FB; j++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const int n = wn + 32 * j + 8 * q + 4 * h;
        float add[4] = {};
        if (bias) {
#pragma unroll
          for (int e = 0; e < 4; e++) add[e] = bias[n0 + min(n + e, ns - 1)];
        }
#pragma unroll
        for (int i = 0; i < PF; i++) {
          const int row = (wave % K::ACROSS) * 32 * PF + 32 * i + r;
          cm_f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; e++) v[e] = acc[PF * p + i][j][4 * q + e] + add[e];
          if constexpr (F32) {
            *reinterpret_cast<cm_f32x4*>(smem + row * OROW + (((n >> 2) ^ r) * 16)) = v;
          } else {
            const cm_i32x2 w = {(int)((uint32_t)bf16_of(v[0]) | ((uint32_t)bf16_of(v[1]) << 16)),
                                (int)((uint32_t)bf16_of(v[2]) | ((uint32_t)bf16_of(v[3]) << 16))};
            *reinterpret_cast<cm_i32x2*>(smem + row * OROW + (((n >> 3) ^ (r & (RC - 1))) * 16) + (n & 4) * 2) = w;
          }
        }
      }
    __syncthreads();
#pragma unroll 8
    for (int c = t; c < PROWS * RC; c += 256) {
      const int row = c / RC, in = c % RC;
      const cm_i32x4 v = *reinterpret_cast<const cm_i32x4*>(smem + row * OROW + ((in ^ (row & 31 & (RC - 1))) * 16));
      // rows of the waves lie FA blocks apart
      const int m = row / (32 * PF) * (32 * K::FA) + p * 32 * PF + row % (32 * PF);
      const int left = ns * ES - in * 16;  // bytes of the row from here on
      uint8_t* o = to + (int64_t)m * ldo * ES + in * 16;
      if (m < ms && left >= 16) {
        __builtin_memcpy(o, &v, 16);
      } else if (m < ms && left > 0) {
#pragma unroll
        for (int e = 0; e < 16 / ES; e++)
          if (e * ES < left) {
            if constexpr (F32) reinterpret_cast<int*>(o)[e] = v[e];
            else reinterpret_cast<uint16_t*>(o)[e] = (uint16_t)((uint32_t)v[e >> 1] >> (16 * (e & 1)));
          }
      }
    }
  }
}

// Whether rows of n results are joined four neighbouring columns a thread.
__host__ __device__ inline bool join_by_four(int64_t n) { return n % 4 == 0 && n >= 256; }

// out from the sums over parts of the columns, in the order of the parts.  Wide rows by four neighbouring columns of a
// row a thread, blockIdx.y over the rows: four parts of 333 x 1880 2.6-2.7 us, each result for itself with its division 3.3-3.4.  Rows
// that are narrow or end inside a group of four each result for itself: eight parts of 3431 x 17 2.6 (by four columns 5.7, five of
// 256 threads at work), of 100 x 130 2.5 (4.0); four parts of 200 x 3001 3.3-3.4 (3.3-3.6).
template <bool F32>
__global__ __launch_bounds__(256) void az_join_products(const float* __restrict__ parts, int count, int m, int n,
                                                        const float* __restrict__ bias, void* __restrict__ out, int64_t ldo) {
  const int64_t total = (int64_t)m * n;
  if (join_by_four(n)) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (c >= n) return;
    float add[4] = {};
    if (bias) __builtin_memcpy(add, bias + c, 16);
    for (int64_t r = blockIdx.y; r < m; r += gridDim.y) {
      const float* from = parts + r * n + c;
      float v[4] = {};
#pragma unroll 4
      for (int p = 0; p < count; p++) {
        float x[4];
        __builtin_memcpy(x, from + p * total, 16);
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] += x[e];
      }
      put<!F32, 4, EVEN>(out, r * ldo, (int)c, n, {v[0] + add[0], v[1] + add[1], v[2] + add[2], v[3] + add[3]});
    }
  } else {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
      float v = 0.0f;
      for (int p = 0; p < count; p++) v += parts[p * total + i];
      const int64_t r = i / n, c = i - r * n;
      if (bias) v += bias[c];
      if constexpr (F32) ((float*)out)[r * ldo + c] = v;
      else ((uint16_t*)out)[r * ldo + c] = bf16_of(v);
    }
  }
}

// The workgroups that join results of m x n.
inline dim3 join_grid(int64_t m, int64_t n) {
  if (join_by_four(n)) return dim3((unsigned)((n + 1023) / 1024), (unsigned)(m < 65535 ? m : 65535));
  const int64_t groups = (m * n + 255) / 256;
  return dim3((unsigned)(groups < 8192 ? groups : 8192));
}

}  // namespace
