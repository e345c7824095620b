// Shared by the operators on coded matrices (az_code_matrix: e4m3 codes, one
// power-of-two scale for each block of 128 columns of a row or of 128 x 128
// entries): host checks, the view that kernels take, and the format's
// arithmetic.  Private to the library: everything has internal linkage.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "az.h"
#include "az_internal.h"

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 cm_bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 cm_bf16x8;
typedef __attribute__((ext_vector_type(4))) float cm_f32x4;
typedef __attribute__((ext_vector_type(16))) float cm_f32x16;
typedef __attribute__((ext_vector_type(2))) int cm_i32x2;
typedef __attribute__((ext_vector_type(4))) int cm_i32x4;
typedef __attribute__((ext_vector_type(8))) int cm_i32x8;

constexpr int CB = AZ_CODE_BLOCK;

// A coded matrix as kernels take it.
struct CodeView {
  uint8_t* codes;
  uint8_t* scales;
  int64_t ld;
  int rows, cols;
  int nb;     // blocks of a row
  int shift;  // row r's scales are row r >> shift
};

inline CodeView code_view(const az_code_matrix& m) {
  return CodeView{m.codes, m.scales, m.ld, (int)m.rows, (int)m.cols, (int)((m.cols + CB - 1) / CB),
                  m.scale_rows == 1 ? 0 : 7};
}

inline int code_fail(int status, const char* who, const char* what) {
  char text[160];
  snprintf(text, sizeof text, "%s: %s", who, what);
  return az_fail(status, text);
}

// Whether sizes of at least one row and column are within the limits.
inline bool code_sizes(int64_t rows, int64_t cols) {
  return rows <= INT32_MAX && cols <= (1 << 30) && rows * ((cols + CB - 1) / CB) <= INT32_MAX;
}

// Checks of a matrix that every operator makes.  Pointers are checked where the
// matrix has entries.
inline int code_check(const az_code_matrix* m, const char* who) {
  if (!m) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL matrix");
  if (m->rows < 0 || m->cols < 1) return code_fail(AZ_ERR_INVALID_ARG, who, "rows < 0 or cols < 1");
  if (m->scale_rows != 1 && m->scale_rows != CB) return code_fail(AZ_ERR_INVALID_ARG, who, "scale_rows is neither 1 nor 128");
  if (m->ld < m->cols || m->ld % 16) return code_fail(AZ_ERR_INVALID_ARG, who, "ld is below cols or not a multiple of 16");
  if (!code_sizes(m->rows, m->cols)) return code_fail(AZ_ERR_UNSUPPORTED, who, "a matrix past the size limits");
  if (m->rows == 0) return AZ_OK;
  if (!m->codes || !m->scales) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL codes or scales");
  if ((uintptr_t)m->codes & 15u) return code_fail(AZ_ERR_INVALID_ARG, who, "codes must be 16-byte aligned");
  return AZ_OK;
}

// A dense fp32 or bf16 buffer of rows of `cols` elements.
inline int dense_check(const void* p, int32_t dtype, int64_t ld, int64_t cols, const char* who) {
  if (dtype != AZ_F32 && dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (ld < cols) return code_fail(AZ_ERR_INVALID_ARG, who, "a row stride below the row");
  if (!p) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL buffer");
  if ((uintptr_t)p & (dtype == AZ_F32 ? 3u : 1u)) return code_fail(AZ_ERR_INVALID_ARG, who, "a buffer that is not aligned to its element");
  return AZ_OK;
}

// Whether rows of `esz`-byte elements can be read and written 16 bytes at a time.
inline bool rows_aligned16(const void* p, int64_t ld, int esz) { return ((uintptr_t)p & 15u) == 0 && (ld * esz) % 16 == 0; }

inline int launch_status(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? AZ_OK : code_fail(AZ_ERR_DEVICE, who, hipGetErrorString(e));
}

// Whether a grid of this many workgroups can be launched (its threads are counted in 32 bits).
inline bool grid_fits(int64_t groups, int threads) { return groups * threads <= (int64_t)UINT32_MAX; }

// The status of a launch: one that was refused before it, or the runtime's.
inline int launched(const char* who, int status) {
  if (status == AZ_ERR_UNSUPPORTED) return code_fail(status, who, "more results than a launch can cover");
  if (status != AZ_OK) return code_fail(status, who, "the kernel's LDS size was refused");
  return launch_status(who);
}

// 2^(s - 127) of a scale byte in 10..246; NaN for 255.
__device__ __forceinline__ float scale_value(uint32_t s) {
  return __uint_as_float(s == 255u ? 0x7fc00000u : s << 23);
}

// Two codes of a word (the low or the high half) times a power of two, as bf16:
// exact while the values are normal bf16 numbers, which the format's scales assure.
template <bool HI>
__device__ __forceinline__ uint32_t code_pair_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, HI));
}

// 16 bytes of codes of a row from column c on; bytes at and past `cols` read as
// zero codes.  c is a multiple of 16, and a row holds a multiple of 16 bytes, so
// that every chunk that begins before cols can be read; one that does not reads the last
// such chunk and keeps nothing of it.
__device__ __forceinline__ cm_i32x4 code_chunk(const uint8_t* row, int c, int cols) {
  cm_i32x4 v = *reinterpret_cast<const cm_i32x4*>(row + min(c, (cols - 1) & ~15));
  const int left = cols - c;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int n = max(left - 4 * i, 0);  // bytes of this word that count
    v[i] &= n >= 4 ? -1 : (int)((1u << (8 * n)) - 1u);
  }
  return v;
}

__device__ __forceinline__ uint16_t bf16_of(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ float f32_of_bf16(uint32_t bits) { return __uint_as_float(bits << 16); }

}  // namespace
