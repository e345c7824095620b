// Shared by the operators on matrices in 4 bits (az_fp4_matrix: e2m1 codes, two to a byte, one
// power-of-two scale for each block of 32 columns).  Private to the library.
#pragma once

#include "az_codes_common.h"

namespace {

constexpr int NB = AZ_FP4_BLOCK;  // a block's codes are 16 bytes: one chunk

struct NibbleView {
  uint8_t* codes;
  uint8_t* scales;
  int64_t ld, ld_scales;
  int rows, cols;
};

inline NibbleView nibble_view(const az_fp4_matrix& m) {
  return NibbleView{m.codes, m.scales, m.ld, m.ld_scales, (int)m.rows, (int)m.cols};
}

inline int nibble_check(const az_fp4_matrix* m, const char* who) {
  if (!m) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL matrix");
  if (m->rows < 0 || m->cols < 1) return code_fail(AZ_ERR_INVALID_ARG, who, "rows < 0 or cols < 1");
  if (!code_sizes(m->rows, m->cols)) return code_fail(AZ_ERR_UNSUPPORTED, who, "a matrix past the size limits");
  if (m->ld < (m->cols + 1) / 2 || m->ld % 16) return code_fail(AZ_ERR_INVALID_ARG, who, "ld is below half of cols or not a multiple of 16");
  if (m->ld_scales < (m->cols + NB - 1) / NB || m->ld_scales % 4)
    return code_fail(AZ_ERR_INVALID_ARG, who, "ld_scales is below a row's blocks or not a multiple of 4");
  if (m->rows == 0) return AZ_OK;
  if (!m->codes || !m->scales) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL codes or scales");
  if ((uintptr_t)m->codes & 15u) return code_fail(AZ_ERR_INVALID_ARG, who, "codes must be 16-byte aligned");
  if ((uintptr_t)m->scales & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "scales must be 4-byte aligned");
  return AZ_OK;
}

// The chunk of block `kb` of a row; codes at and past `cols` read as zeros.  A row holds whole chunks, so that
// every one that begins before cols can be read; one that does not reads the last such chunk and keeps nothing of it.
__device__ __forceinline__ cm_i32x4 nibble_chunk(const uint8_t* row, int kb, int cols) {
  cm_i32x4 v = *reinterpret_cast<const cm_i32x4*>(row + (int64_t)min(kb, (cols - 1) / NB) * 16);
  const int left = cols - kb * NB;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int n = max(left - 8 * i, 0);  // codes of this word that count
    v[i] &= n >= 8 ? -1 : (int)((1u << (4 * n)) - 1u);
  }
  return v;
}

}  // namespace
