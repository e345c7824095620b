// Logits with penalties for what has been chosen before, a bias and a mask of what
// is allowed, and the policy over it: the legal-move softmax of the network kernels
// for logits that are in memory.
#include <math.h>

#include "az_codes_common.h"

namespace {

constexpr int NT = 256, CHUNK = 4096;

struct PolicyView {
  const void* logits;
  const void* mask;
  const float* bias;
  const int32_t* history;
  const int32_t* lengths;
  const float* penalties;
  float* out;
  int64_t ld, ld_mask, ld_bias, ld_history, ld_out;
  int vocab, max_history;
};

// (running maximum, sum of exp(l - maximum)) of two parts; a part without a finite
// entry has maximum -inf and sum 0, or NaN where it holds one.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  s = top == -INFINITY ? s + s2 : s * expf(m - top) + s2 * expf(m2 - top);
  m = top;
}

template <bool BF16, int MASK, bool HIST, bool PROBS>
__global__ __launch_bounds__(NT) void az_policy_kernel(PolicyView p) {
  __shared__ uint32_t count[HIST ? CHUNK : 1];
  __shared__ float red[2][NT / 64];
  const int64_t b = blockIdx.x;
  const int t = threadIdx.x;
  int n_hist = 0;
  float rep = 1.0f, freq = 0.0f, pres = 0.0f;
  if constexpr (HIST) {
    n_hist = p.lengths ? min(max(p.lengths[b], 0), p.max_history) : p.max_history;
    rep = p.penalties[3 * b];
    freq = p.penalties[3 * b + 1];
    pres = p.penalties[3 * b + 2];
  }
  float m = -INFINITY, s = 0.0f, inv = 0.0f;
  for (int pass = PROBS ? 0 : 1; pass < 2; pass++) {
    for (int v0 = 0; v0 < p.vocab; v0 += CHUNK) {
      if constexpr (HIST) {
        __syncthreads();
        for (int i = t; i < CHUNK; i += NT) count[i] = 0;
        __syncthreads();
        for (int i = t; i < n_hist; i += NT) {
          const int v = p.history[b * p.ld_history + i];
          if (v >= v0 && v < p.vocab && v - v0 < CHUNK) atomicAdd(&count[v - v0], 1u);
        }
        __syncthreads();
      }
      const int end = min(v0 + CHUNK, p.vocab);
      for (int v = v0 + t; v < end; v += NT) {
        float l;
        if constexpr (BF16) l = f32_of_bf16(((const uint16_t*)p.logits)[b * p.ld + v]);
        else l = ((const float*)p.logits)[b * p.ld + v];
        if constexpr (HIST) {
          const uint32_t c = count[v - v0];
          if (c) l = (l > 0.0f ? l / rep : l * rep) - (freq * (float)c + pres);
        }
        if (p.bias) l += p.bias[b * p.ld_bias + v];
        bool ok = true;
        if constexpr (MASK == AZ_MASK_BYTES) ok = ((const uint8_t*)p.mask)[b * p.ld_mask + v] != 0;
        if constexpr (MASK == AZ_MASK_BITS) ok = (((const uint32_t*)p.mask)[b * p.ld_mask + (v >> 5)] >> (v & 31)) & 1u;
        if (!ok) l = -INFINITY;
        if (pass == 0) {
          if (l != l) s = l;  // a NaN stays in the sum
          else if (l != -INFINITY) join(m, s, l, 1.0f);
        } else if constexpr (PROBS) {
          p.out[b * p.ld_out + v] = ok ? expf(l - m) * inv : 0.0f;
        } else {
          p.out[b * p.ld_out + v] = l;
        }
      }
    }
    if (pass == 0) {
      for (int o = 32; o > 0; o >>= 1) {
        const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o);
        join(m, s, m2, s2);
      }
      if ((t & 63) == 0) { red[0][t >> 6] = m; red[1][t >> 6] = s; }
      __syncthreads();
      m = red[0][0];
      s = red[1][0];
      for (int w = 1; w < NT / 64; w++) join(m, s, red[0][w], red[1][w]);
      if (m == -INFINITY && s == 0.0f) { m = 0.0f; inv = 0.0f; }
      else inv = 1.0f / s;
    }
  }
}

template <bool BF16, int MASK, bool HIST>
void launch(const PolicyView& p, int rows, bool probs, hipStream_t s) {
  if (probs) hipLaunchKernelGGL((az_policy_kernel<BF16, MASK, HIST, true>), dim3(rows), dim3(NT), 0, s, p);
  else hipLaunchKernelGGL((az_policy_kernel<BF16, MASK, HIST, false>), dim3(rows), dim3(NT), 0, s, p);
}

template <bool BF16, int MASK>
void launch_mask(const PolicyView& p, int rows, bool probs, hipStream_t s) {
  if (p.history) launch<BF16, MASK, true>(p, rows, probs, s);
  else launch<BF16, MASK, false>(p, rows, probs, s);
}

template <bool BF16>
void launch_type(const PolicyView& p, int mask, int rows, bool probs, hipStream_t s) {
  if (mask == AZ_MASK_BYTES) launch_mask<BF16, AZ_MASK_BYTES>(p, rows, probs, s);
  else if (mask == AZ_MASK_BITS) launch_mask<BF16, AZ_MASK_BITS>(p, rows, probs, s);
  else launch_mask<BF16, AZ_MASK_NONE>(p, rows, probs, s);
}

}  // namespace

extern "C" size_t az_logits_policy_workspace(int32_t rows, int32_t vocab) {
  (void)rows, (void)vocab;
  return 0;
}

extern "C" int az_logits_policy(const az_logits* in, int32_t probabilities, float* out, int64_t ld_out, void* workspace,
                                size_t workspace_bytes, void* stream) {
  static const char who[] = "az_logits_policy";
  if (!in) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL logits");
  if (in->rows < 0 || in->vocab < 1) return code_fail(AZ_ERR_INVALID_ARG, who, "rows < 0 or vocab < 1");
  if (in->rows > (1 << 20) || in->vocab > (1 << 24)) return code_fail(AZ_ERR_UNSUPPORTED, who, "rows > 2^20 or vocab > 2^24");
  if (in->dtype != AZ_F32 && in->dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (in->mask_kind < AZ_MASK_NONE || in->mask_kind > AZ_MASK_BITS) return code_fail(AZ_ERR_INVALID_ARG, who, "unknown mask kind");
  if (in->max_history < 0) return code_fail(AZ_ERR_INVALID_ARG, who, "max_history < 0");
  if (in->rows == 0) return AZ_OK;
  int st = dense_check(in->logits, in->dtype, in->ld, in->vocab, who);
  if (st == AZ_OK) st = dense_check(out, AZ_F32, ld_out, in->vocab, who);
  if (st != AZ_OK) return st;
  const bool hist = in->history && in->max_history > 0;
  if (in->mask_kind != AZ_MASK_NONE) {
    if (!in->mask) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL mask");
    const int64_t row = in->mask_kind == AZ_MASK_BYTES ? in->vocab : (in->vocab + 31) / 32;
    if (in->ld_mask < row) return code_fail(AZ_ERR_INVALID_ARG, who, "a row stride below the row");
    if (in->mask_kind == AZ_MASK_BITS && ((uintptr_t)in->mask & 3u)) return code_fail(AZ_ERR_INVALID_ARG, who, "mask words must be 4-byte aligned");
  }
  if (in->bias && in->ld_bias != 0 && in->ld_bias < in->vocab) return code_fail(AZ_ERR_INVALID_ARG, who, "a row stride below the row");
  if (hist) {
    if (!in->penalties) return code_fail(AZ_ERR_INVALID_ARG, who, "a history needs penalties");
    if (in->ld_history < in->max_history) return code_fail(AZ_ERR_INVALID_ARG, who, "a row stride below the row");
  }
  if (((uintptr_t)in->bias | (uintptr_t)in->history | (uintptr_t)in->lengths | (uintptr_t)in->penalties) & 3u)
    return code_fail(AZ_ERR_INVALID_ARG, who, "a buffer that is not aligned to its element");
  const size_t need = az_logits_policy_workspace(in->rows, in->vocab);
  if (workspace_bytes < need || (need && !workspace)) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace is too small");
  if ((uintptr_t)workspace & 15u) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace must be 16-byte aligned");
  const PolicyView p = {in->logits, in->mask, in->bias, hist ? in->history : nullptr, in->lengths, in->penalties, out,
                        in->ld, in->ld_mask, in->ld_bias, in->ld_history, ld_out, in->vocab, in->max_history};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (in->dtype == AZ_BF16) launch_type<true>(p, in->mask_kind, in->rows, probabilities != 0, s);
  else launch_type<false>(p, in->mask_kind, in->rows, probabilities != 0, s);
  return launch_status(who);
}
