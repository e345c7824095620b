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

// out from the sums over parts of the columns, in the order of the parts.  A thread takes four neighbouring columns of a
// row at a time; blockIdx.y goes over the rows.  Four parts of 333 x 1880: 4.2 us (4.7 with a
// division for each result).
template <bool F32>
__global__ __launch_bounds__(256) void az_join_products(const float* __restrict__ parts, int count, int m, int n,
                                                        const float* __restrict__ bias, void* __restrict__ out, int64_t ldo) {
  const int64_t total = (int64_t)m * n, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= n) return;
  const int left = (int)min((int64_t)n - c, (int64_t)4);
  float add[4] = {};
  if (bias) {
#pragma unroll
    for (int e = 0; e < 4; e++) add[e] = bias[c + min(e, left - 1)];
  }
  for (int64_t r = blockIdx.y; r < m; r += gridDim.y) {
    const float* from = parts + r * n + c;
    float v[4] = {};
    if (left == 4) {
#pragma unroll 4
      for (int p = 0; p < count; p++) {
        float x[4];
        __builtin_memcpy(x, from + p * total, 16);
#pragma unroll
        for (int e = 0; e < 4; e++) v[e] += x[e];
      }
    } else {
      for (int p = 0; p < count; p++)
        for (int e = 0; e < left; e++) v[e] += from[p * total + e];
    }
    put<!F32, 4>(out, r * ldo, (int)c, n, {v[0] + add[0], v[1] + add[1], v[2] + add[2], v[3] + add[3]});
  }
}

// The workgroups that join results of m x n.
inline dim3 join_grid(int64_t m, int64_t n) { return dim3((unsigned)((n + 1023) / 1024), (unsigned)(m < 65535 ? m : 65535)); }

}  // namespace
