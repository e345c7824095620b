// out = a b^T + bias of two coded matrices, both with the summed dimension along
// their rows.
//
// bf16 results run on the scaled f8f6f4 matrix instruction (K = 128, one scale byte
// per row and 128 columns: exactly a block, so that scales cost no arithmetic).  It
// aligns the products of a group to the largest and cuts what lies below, which costs
// about 1.5e-5 of the result's norm: nothing beside a bf16 rounding (2e-3), but
// visible in fp32.  fp32 results therefore run on the bf16 instruction, for which
// codes times their scale are exact operands and products exact fp32 terms.
//
// In both, D's rows are the n of b and its columns the m of a, so that a lane holds
// four neighbouring n of one m and stores them together.
#include "az_codes_common.h"

namespace {

// 32 consecutive codes of a row for K step kb, the operand of a lane (row l % 16,
// columns 32 (l / 16) on).
__device__ __forceinline__ cm_i32x8 row_fragment(const uint8_t* row, int k0, int cols) {
  const cm_i32x4 lo = code_chunk(row, k0, cols), hi = code_chunk(row, k0 + 16, cols);
  return cm_i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

// Eight codes (words 2i, 2i + 1 of a fragment) as exact bf16 values.
__device__ __forceinline__ cm_bf16x8 fragment_bf16(const cm_i32x8& w, int i, float s) {
  const cm_i32x4 u = {(int)code_pair_bf16<false>((uint32_t)w[2 * i], s), (int)code_pair_bf16<true>((uint32_t)w[2 * i], s),
                      (int)code_pair_bf16<false>((uint32_t)w[2 * i + 1], s), (int)code_pair_bf16<true>((uint32_t)w[2 * i + 1], s)};
  return __builtin_bit_cast(cm_bf16x8, u);
}

// A workgroup of NW waves owns 16 FM rows of a times 16 FN rows of b.  Each wave takes
// every NW-th K step straight from memory to registers; the partial sums meet in LDS in
// the order of the waves.
template <int FM, int FN, int NW, bool F32>
__global__ __launch_bounds__(NW * 64) void az_matmul_direct(CodeView a, CodeView b, const float* __restrict__ bias,
                                                            void* __restrict__ out, int64_t ldo) {
  __shared__ cm_f32x4 part[NW > 1 ? (NW - 1) * FM * FN * 64 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  const int m0 = blockIdx.y * 16 * FM, n0 = blockIdx.x * 16 * FN;
  cm_f32x4 acc[FM][FN];
  const uint8_t *ar[FM], *br[FN], *as[FM], *bs[FN];
#pragma unroll
  for (int i = 0; i < FM; i++) {
    const int row = min(m0 + 16 * i + r, a.rows - 1);
    ar[i] = a.codes + row * a.ld;
    as[i] = a.scales + (int64_t)(row >> a.shift) * a.nb;
  }
#pragma unroll
  for (int j = 0; j < FN; j++) {
    const int row = min(n0 + 16 * j + r, b.rows - 1);
    br[j] = b.codes + row * b.ld;
    bs[j] = b.scales + (int64_t)(row >> b.shift) * b.nb;
  }
#pragma unroll
  for (int i = 0; i < FM; i++)
#pragma unroll
    for (int j = 0; j < FN; j++) acc[i][j] = cm_f32x4{0, 0, 0, 0};
  for (int kb = wave; kb < a.nb; kb += NW) {
    const int k0 = kb * CB + g * 32;
    cm_i32x8 fa[FM], fb[FN];
    uint32_t sa[FM], sb[FN];
#pragma unroll
    for (int i = 0; i < FM; i++) { fa[i] = row_fragment(ar[i], k0, a.cols); sa[i] = as[i][kb]; }
#pragma unroll
    for (int j = 0; j < FN; j++) { fb[j] = row_fragment(br[j], k0, a.cols); sb[j] = bs[j][kb]; }
    if constexpr (!F32) {
#pragma unroll
      for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa[i], acc[i][j], 0, 0, 0, (int)sb[j], 0, (int)sa[i]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; q++) {
        cm_bf16x8 va[FM], vb[FN];
#pragma unroll
        for (int i = 0; i < FM; i++) va[i] = fragment_bf16(fa[i], q, scale_value(sa[i]));
#pragma unroll
        for (int j = 0; j < FN; j++) vb[j] = fragment_bf16(fb[j], q, scale_value(sb[j]));
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
          for (int j = 0; j < FN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb[j], va[i], acc[i][j], 0, 0, 0);
      }
    }
  }
  if constexpr (NW > 1) {
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) part[((wave - 1) * FM * FN + i * FN + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < NW - 1; w++)
#pragma unroll
      for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) acc[i][j] += part[(w * FM * FN + i * FN + j) * 64 + lane];
  }
#pragma unroll
  for (int i = 0; i < FM; i++) {
    const int m = m0 + 16 * i + r;
    if (m >= a.rows) continue;
#pragma unroll
    for (int j = 0; j < FN; j++) {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int n = n0 + 16 * j + 4 * g + e;
        if (n >= b.rows) continue;
        const float v = acc[i][j][e] + (bias ? bias[n] : 0.0f);
        if constexpr (F32) ((float*)out)[m * ldo + n] = v;
        else ((uint16_t*)out)[m * ldo + n] = bf16_of(v);
      }
    }
  }
}

template <int FM, int FN, int NW, bool F32>
void launch_direct(const CodeView& a, const CodeView& b, const float* bias, void* out, int64_t ldo, hipStream_t s) {
  const dim3 g((b.rows + 16 * FN - 1) / (16 * FN), (a.rows + 16 * FM - 1) / (16 * FM));
  hipLaunchKernelGGL((az_matmul_direct<FM, FN, NW, F32>), g, dim3(NW * 64), 0, s, a, b, bias, out, ldo);
}

template <bool F32>
void launch(const CodeView& a, const CodeView& b, const float* bias, void* out, int64_t ldo, hipStream_t s) {
  if (a.rows <= 16) launch_direct<1, 1, 8, F32>(a, b, bias, out, ldo, s);
  else if (a.rows <= 64) launch_direct<4, 1, 8, F32>(a, b, bias, out, ldo, s);
  else launch_direct<4, 4, 4, F32>(a, b, bias, out, ldo, s);
}

}  // namespace

extern "C" int az_codes_matmul(const az_code_matrix* a, const az_code_matrix* b, const float* bias, void* out,
                               int32_t dtype, int64_t ld_out, void* stream) {
  static const char who[] = "az_codes_matmul";
  int st = code_check(a, who);
  if (st == AZ_OK) st = code_check(b, who);
  if (st != AZ_OK) return st;
  if (a->cols != b->cols) return code_fail(AZ_ERR_INVALID_ARG, who, "a and b differ in cols");
  if (dtype != AZ_F32 && dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (a->rows == 0 || b->rows == 0) return AZ_OK;
  if ((st = dense_check(out, dtype, ld_out, b->rows, who)) != AZ_OK) return st;
  if ((uintptr_t)bias & 3u) return code_fail(AZ_ERR_INVALID_ARG, who, "bias must be 4-byte aligned");
  // 64 rows of a per workgroup row, and at most 65,535 of those in a grid
  if (a->rows > (int64_t)65535 * 64) return code_fail(AZ_ERR_UNSUPPORTED, who, "more than 4,194,240 rows of a");
  const CodeView va = code_view(*a), vb = code_view(*b);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (dtype == AZ_F32) launch<true>(va, vb, bias, out, ld_out, s);
  else launch<false>(va, vb, bias, out, ld_out, s);
  return launch_status(who);
}
