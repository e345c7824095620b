// out = a b^T + bias, b in 4 bits and a in 4 bits or e4m3 codes, the summed dimension along the rows of both.
//
// The scaled f8f6f4 matrix instruction takes both formats, each operand with a scale byte for each row and 32 columns:
// a block of the 4-bit format exactly.  Two 4-bit operands run at twice the rate of e4m3, and
// their products (multiples of 1/4 up to 36) are summed exactly.  With an e4m3 operand small products are
// cut (see the products of two e4m3 matrices), so that fp32 results of a coded a run on the bf16 instruction,
// for which codes times their scale are exact operands.
#include "az_nibbles_common.h"

namespace {

enum { E4M3 = 0, E2M1 = 4 };  // the instruction's format numbers

// Either kind of the left operand.
struct LeftView {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t ld, ld_scales;
  int rows, cols, shift;
};

// A lane's 32 columns of step k (128 columns), zeros past cols.  The 16 x 16 x 128 instruction has lane group g's
// 4-bit columns at 32 g on, but 8-bit ones in two halves at 16 g and 64 + 16 g on.  (SPLIT; the bf16
// instruction takes any columns, if a and b agree.)
template <int FORMAT, bool SPLIT>
__device__ __forceinline__ cm_i32x8 fragment(const uint8_t* row, int k, int g, int cols) {
  if constexpr (FORMAT == E2M1) {
    const cm_i32x4 v = nibble_chunk(row, 4 * k + g, cols);
    return cm_i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0};
  } else {
    const int c = k * CB + g * (SPLIT ? 16 : 32);
    const cm_i32x4 lo = code_chunk(row, c, cols), hi = code_chunk(row, c + (SPLIT ? 64 : 16), cols);
    return cm_i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  }
}

// Eight codes (the i-th eight of a fragment) as exact bf16 values.
template <int FORMAT>
__device__ __forceinline__ cm_bf16x8 values8(const cm_i32x8& w, int i, float s) {
  cm_i32x4 u;
  if constexpr (FORMAT == E2M1) {
    const uint32_t c = (uint32_t)w[i];
    u = cm_i32x4{__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0)), __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1)),
                 __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2)), __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3))};
  } else {
    u = cm_i32x4{(int)code_pair_bf16<false>((uint32_t)w[2 * i], s), (int)code_pair_bf16<true>((uint32_t)w[2 * i], s),
                 (int)code_pair_bf16<false>((uint32_t)w[2 * i + 1], s), (int)code_pair_bf16<true>((uint32_t)w[2 * i + 1], s)};
  }
  return __builtin_bit_cast(cm_bf16x8, u);
}

// Few rows of a.  A workgroup of eight waves owns 16 rows of a times 16 rows of b; each wave takes every eighth
// step of 128 columns, a lane a block of 32, and the waves' sums meet in LDS in the order of the waves.
constexpr int DW = 8;

template <int A, bool EXACT, bool F32>
__global__ __launch_bounds__(DW * 64) void az_nibble_direct(LeftView a, NibbleView b, const float* __restrict__ bias,
                                                            void* __restrict__ out, int64_t ldo, int nt) {
  __shared__ cm_f32x4 part[DW - 1][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int m0 = (int)(blockIdx.x / (uint32_t)nt) * 16, n0 = (int)(blockIdx.x % (uint32_t)nt) * 16;
  const int64_t am = min((int64_t)m0 + r, (int64_t)a.rows - 1), bn = min((int64_t)n0 + r, (int64_t)b.rows - 1);
  const uint8_t *ar = a.codes + am * a.ld, *br = b.codes + bn * b.ld;
  const uint8_t *as = a.scales + (am >> a.shift) * a.ld_scales, *bs = b.scales + bn * b.ld_scales;
  const int blocks = (a.cols + NB - 1) / NB, steps = (blocks + 3) / 4;
  cm_f32x4 acc = {0, 0, 0, 0};
  for (int k = wave; k < steps; k += DW) {
    const int kb = 4 * k + g, last = min(kb, blocks - 1);
    const cm_i32x8 fa = fragment<A, !EXACT>(ar, k, g, a.cols), fb = fragment<E2M1, !EXACT>(br, k, g, a.cols);
    // (past cols: the last block's scale, which counts a NaN that is in the result already)
    const uint32_t sa = as[A == E2M1 ? last : last / 4], sb = bs[last];
    if constexpr (!EXACT) {
      acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, fa, acc, E2M1, A, 0, (int)sb, 0, (int)sa);
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8<E2M1>(fb, q, scale_value(sb)), values8<A>(fa, q, scale_value(sa)), acc, 0, 0, 0);
    }
  }
  if (wave > 0) part[wave - 1][lane] = acc;
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < DW - 1; w++) acc += part[w][lane];
  const int64_t m = (int64_t)m0 + r;
  if (m >= a.rows) return;
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const int64_t n = (int64_t)n0 + 4 * g + e;
    if (n >= b.rows) continue;
    const float v = acc[e] + (bias ? bias[n] : 0.0f);
    if constexpr (F32) ((float*)out)[m * ldo + n] = v;
    else ((uint16_t*)out)[m * ldo + n] = bf16_of(v);
  }
}

struct Operands {
  LeftView a;
  NibbleView b;
  const float* bias;
  void* out;
  int64_t ldo;
  hipStream_t stream;
};

template <int A, bool EXACT, bool F32>
int launch_direct(const Operands& o) {
  const int64_t nt = ((int64_t)o.b.rows + 15) / 16, groups = nt * (((int64_t)o.a.rows + 15) / 16);
  if (!grid_fits(groups, DW * 64)) return AZ_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((az_nibble_direct<A, EXACT, F32>), dim3((unsigned)groups), dim3(DW * 64), 0, o.stream, o.a, o.b, o.bias, o.out, o.ldo, (int)nt);
  return AZ_OK;
}

int matmul(const LeftView& a, int format, const az_fp4_matrix& b, const float* bias, void* out, int32_t dtype, int64_t ld_out,
           void* workspace, size_t workspace_bytes, void* stream, const char* who) {
  if (dtype != AZ_F32 && dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (a.rows == 0 || b.rows == 0) return AZ_OK;
  const int st = dense_check(out, dtype, ld_out, b.rows, who);
  if (st != AZ_OK) return st;
  if ((uintptr_t)bias & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "bias must be 4-byte aligned");
  if (a.ld >= (1 << 27) || b.ld >= (1 << 27) || b.ld_scales >= (1 << 26)) return code_fail(AZ_ERR_UNSUPPORTED, who, "rows of 2^27 bytes or scales of 2^26 or more");
  const Operands o = {a, nibble_view(b), bias, out, ld_out, static_cast<hipStream_t>(stream)};
  (void)hipGetLastError();
  if (format == E2M1) return launched(who, dtype == AZ_F32 ? launch_direct<E2M1, false, true>(o) : launch_direct<E2M1, false, false>(o));
  return launched(who, dtype == AZ_F32 ? launch_direct<E4M3, true, true>(o) : launch_direct<E4M3, false, false>(o));
}

}  // namespace

extern "C" size_t az_nibbles_matmul_workspace(const az_fp4_matrix*, const az_fp4_matrix*, int32_t) { return 0; }
extern "C" size_t az_codes_nibbles_matmul_workspace(const az_code_matrix*, const az_fp4_matrix*, int32_t) { return 0; }

extern "C" int az_nibbles_matmul(const az_fp4_matrix* a, const az_fp4_matrix* b, const float* bias, void* out, int32_t dtype,
                                 int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "az_nibbles_matmul";
  int st = nibble_check(a, who);
  if (st == AZ_OK) st = nibble_check(b, who);
  if (st != AZ_OK) return st;
  if (a->cols != b->cols) return code_fail(AZ_ERR_INVALID_ARG, who, "a and b differ in cols");
  if (a->ld_scales >= (1 << 26)) return code_fail(AZ_ERR_UNSUPPORTED, who, "scales of 2^26 bytes or more a row");
  const LeftView v = {a->codes, a->scales, a->ld, a->ld_scales, (int)a->rows, (int)a->cols, 0};
  return matmul(v, E2M1, *b, bias, out, dtype, ld_out, workspace, workspace_bytes, stream, who);
}

extern "C" int az_codes_nibbles_matmul(const az_code_matrix* a, const az_fp4_matrix* b, const float* bias, void* out, int32_t dtype,
                                       int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "az_codes_nibbles_matmul";
  int st = code_check(a, who);
  if (st == AZ_OK) st = nibble_check(b, who);
  if (st != AZ_OK) return st;
  if (a->cols != b->cols) return code_fail(AZ_ERR_INVALID_ARG, who, "a and b differ in cols");
  const CodeView c = code_view(*a);
  const LeftView v = {c.codes, c.scales, c.ld, c.nb, c.rows, c.cols, c.shift};
  return matmul(v, E4M3, *b, bias, out, dtype, ld_out, workspace, workspace_bytes, stream, who);
}
