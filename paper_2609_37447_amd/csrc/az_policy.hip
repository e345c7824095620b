// Logits with penalties for what has been chosen before, a bias and a mask of what
// is allowed, and the policy over it: the legal-move softmax of the network kernels
// for logits that are in memory.
//
// Bound by memory: a row's logits, mask and bias are read and its results written.  A thread
// keeps 16 entries in registers, so that a row of up to 16,384 entries is read once by one
// workgroup.  Longer rows are cut into chunks: a first kernel leaves each chunk's maximum
// and sum in the workspace, a second one joins them and reads the logits again, which the
// caches still hold, to write the result.  What has been chosen before is counted in LDS, a
// counter for each entry of the chunk, so that penalties cost no search.
#include <math.h>

#include "az_codes_common.h"

namespace {

constexpr int PER = 16;           // entries of a thread, in two groups of eight
constexpr int MOST = 1024 * PER;  // entries of a workgroup
constexpr float LOG2E = 1.44269504088896340736f;

struct PolicyView {
  const void* logits;
  const void* mask;
  const float* bias;
  const int32_t* history;
  const int32_t* lengths;
  const float* penalties;
  float* out;
  float2* stats;  // [rows][chunks]: maximum, sum of exp(l - maximum)
  int64_t ld, ld_mask, ld_bias, ld_history, ld_out;
  int vocab, max_history, bf16, mask_kind;
};

// exp(l - m); 0 for l = -inf where m is finite.
__device__ __forceinline__ float exp_below(float l, float m) { return __builtin_amdgcn_exp2f((l - m) * LOG2E); }

// (maximum, sum of exp(l - maximum)) of two parts; a part without an entry above -inf
// has maximum -inf and sum 0, or NaN where it holds one.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  s = top == -INFINITY ? s + s2 : s * exp_below(m, top) + s2 * exp_below(m2, top);
  m = top;
}

// Eight entries from v on, adjusted; -inf where they are not allowed and past the vocabulary.
template <bool HIST>
__device__ __forceinline__ void load8(const PolicyView& p, int64_t b, int v, const uint32_t* count, float rep, float freq, float pres,
                                      float (&l)[8]) {
  if (v + 8 <= p.vocab) {
    if (p.bf16) {
      cm_i32x4 w;
      __builtin_memcpy(&w, (const uint16_t*)p.logits + b * p.ld + v, 16);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        l[2 * i] = __uint_as_float((uint32_t)w[i] << 16);
        l[2 * i + 1] = __uint_as_float((uint32_t)w[i] & 0xffff0000u);
      }
    } else {
      __builtin_memcpy(l, (const float*)p.logits + b * p.ld + v, 32);
    }
    float add[8] = {};
    if (p.bias) __builtin_memcpy(add, p.bias + b * p.ld_bias + v, 32);
    uint32_t ok = 0xffu;
    if (p.mask_kind == AZ_MASK_BYTES) {
      uint64_t w;
      __builtin_memcpy(&w, (const uint8_t*)p.mask + b * p.ld_mask + v, 8);
      ok = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) ok |= ((w >> (8 * i)) & 0xffu) != 0 ? 1u << i : 0u;
    } else if (p.mask_kind == AZ_MASK_BITS) {
      ok = ((const uint8_t*)p.mask)[4 * b * p.ld_mask + (v >> 3)];
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
      if constexpr (HIST) {
        const uint32_t c = count[i];
        if (c) l[i] = (l[i] > 0.0f ? l[i] / rep : l[i] * rep) - (freq * (float)c + pres);
      }
      l[i] = ok & (1u << i) ? l[i] + add[i] : -INFINITY;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      l[i] = -INFINITY;
      const int64_t u = v + i;
      if (u < p.vocab) {
        float x = p.bf16 ? f32_of_bf16(((const uint16_t*)p.logits)[b * p.ld + u]) : ((const float*)p.logits)[b * p.ld + u];
        if constexpr (HIST) {
          const uint32_t c = count[i];
          if (c) x = (x > 0.0f ? x / rep : x * rep) - (freq * (float)c + pres);
        }
        if (p.bias) x += p.bias[b * p.ld_bias + u];
        bool ok = true;
        if (p.mask_kind == AZ_MASK_BYTES) ok = ((const uint8_t*)p.mask)[b * p.ld_mask + u] != 0;
        else if (p.mask_kind == AZ_MASK_BITS) ok = (((const uint8_t*)p.mask)[4 * b * p.ld_mask + (u >> 3)] >> (u & 7)) & 1;
        if (ok) l[i] = x;
      }
    }
  }
}

__device__ __forceinline__ void store8(const PolicyView& p, int64_t b, int v, const float (&l)[8]) {
  float* o = p.out + b * p.ld_out + v;
  if (v + 8 <= p.vocab) {
    __builtin_memcpy(o, l, 32);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (v + i < p.vocab) o[i] = l[i];
  }
}

// ADJUST: the adjusted logits.  WHOLE: the policy of rows that one workgroup holds.  STATS and
// WRITE: the two kernels of longer rows.
enum { ADJUST = 0, WHOLE = 1, STATS = 2, WRITE = 3 };

// blockIdx.x: a chunk of 16 entries a thread; blockIdx.y + 65535 blockIdx.z: the row.
template <int MODE, bool HIST>
__global__ __launch_bounds__(1024) void az_policy_kernel(PolicyView p, int rows) {
  extern __shared__ uint32_t count[];  // HIST: one for each entry of the chunk
  __shared__ float red[2][16];
  const int64_t b = (int64_t)blockIdx.z * 65535 + blockIdx.y;
  if (b >= rows) return;
  const int nt = blockDim.x, t = threadIdx.x, v0 = (int)blockIdx.x * nt * PER;
  float rep = 1.0f, freq = 0.0f, pres = 0.0f;
  if constexpr (HIST) {
    const int n = p.lengths ? min(max(p.lengths[b], 0), p.max_history) : p.max_history;
    rep = p.penalties[3 * b];
    freq = p.penalties[3 * b + 1];
    pres = p.penalties[3 * b + 2];
#pragma unroll
    for (int i = 0; i < PER / 4; i++) reinterpret_cast<cm_i32x4*>(count)[i * nt + t] = cm_i32x4{0, 0, 0, 0};
    __syncthreads();
    for (int i = t; i < n; i += nt) {
      const int v = p.history[b * p.ld_history + i];
      if (v >= v0 && v < p.vocab && v - v0 < nt * PER) atomicAdd(&count[v - v0], 1u);
    }
    __syncthreads();
  }
  float l[2][8];
#pragma unroll
  for (int g = 0; g < 2; g++) load8<HIST>(p, b, v0 + (g * nt + t) * 8, count + (g * nt + t) * 8, rep, freq, pres, l[g]);

  float m = 0.0f, inv = 1.0f;
  if constexpr (MODE == WHOLE || MODE == STATS) {
    m = -INFINITY;
#pragma unroll
    for (int g = 0; g < 2; g++)
#pragma unroll
      for (int i = 0; i < 8; i++) m = fmaxf(m, l[g][i]);
    const float base = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int g = 0; g < 2; g++)
#pragma unroll
      for (int i = 0; i < 8; i++) s += exp_below(l[g][i], base);
    for (int o = 32; o > 0; o >>= 1) {
      const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o);
      join(m, s, m2, s2);
    }
    if ((t & 63) == 0) {
      red[0][t >> 6] = m;
      red[1][t >> 6] = s;
    }
    __syncthreads();
    m = red[0][0];
    s = red[1][0];
    for (int w = 1; w < nt / 64; w++) join(m, s, red[0][w], red[1][w]);
    if constexpr (MODE == STATS) {
      if (t == 0) p.stats[b * gridDim.x + blockIdx.x] = make_float2(m, s);
      return;
    }
    inv = 1.0f / s;
    if (m == -INFINITY && s == 0.0f) m = inv = 0.0f;
  }
  if constexpr (MODE == WRITE) {
    // Every wave joins the row's chunks: lane i those of i, i + 64, ..., then the lanes.
    float s = 0.0f;
    m = -INFINITY;
    for (int i = t & 63; i < (int)gridDim.x; i += 64) {
      const float2 x = p.stats[b * gridDim.x + i];
      join(m, s, x.x, x.y);
    }
    for (int o = 32; o > 0; o >>= 1) {
      const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o);
      join(m, s, m2, s2);
    }
    inv = 1.0f / s;
    if (m == -INFINITY && s == 0.0f) m = inv = 0.0f;
  }
#pragma unroll
  for (int g = 0; g < 2; g++) {
    if constexpr (MODE != ADJUST) {
#pragma unroll
      for (int i = 0; i < 8; i++) l[g][i] = l[g][i] == -INFINITY ? 0.0f : exp_below(l[g][i], m) * inv;
    }
    store8(p, b, v0 + (g * nt + t) * 8, l[g]);
  }
}

// Threads of a workgroup: enough for the row, up to 1,024.  Rows that need several
// workgroups get smaller ones where there are few of them, so that the chip is used.
int policy_threads(int64_t rows, int64_t vocab) {
  if (vocab <= MOST) return vocab <= 256 * PER ? 256 : vocab <= 512 * PER ? 512 : 1024;
  for (int nt = 1024; nt > 256; nt /= 2)
    if (rows * ((vocab + nt * PER - 1) / (nt * PER)) >= 512) return nt;
  return 256;
}

template <int MODE>
void launch(const PolicyView& p, int rows, int nt, hipStream_t s) {
  const dim3 g((unsigned)((p.vocab + nt * PER - 1) / (nt * PER)), (unsigned)(rows < 65535 ? rows : 65535), (unsigned)((rows + 65534) / 65535));
  if (p.history) hipLaunchKernelGGL((az_policy_kernel<MODE, true>), g, dim3(nt), nt * PER * sizeof(uint32_t), s, p, rows);
  else hipLaunchKernelGGL((az_policy_kernel<MODE, false>), g, dim3(nt), 0, s, p, rows);
}

}  // namespace

extern "C" size_t az_logits_policy_workspace(int32_t rows, int32_t vocab) {
  if (rows <= 0 || vocab <= MOST) return 0;
  const int chunk = policy_threads(rows, vocab) * PER;
  return (size_t)rows * (size_t)((vocab + chunk - 1) / chunk) * sizeof(float2);
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
  const int nt = policy_threads(in->rows, in->vocab);
  const PolicyView p = {in->logits, in->mask, in->bias, hist ? in->history : nullptr, in->lengths, in->penalties, out,
                        static_cast<float2*>(workspace), in->ld, in->ld_mask, in->ld_bias, in->ld_history, ld_out,
                        in->vocab, in->max_history, in->dtype == AZ_BF16, in->mask_kind};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (!probabilities) {
    launch<ADJUST>(p, in->rows, nt, s);
  } else if (in->vocab <= MOST) {
    launch<WHOLE>(p, in->rows, nt, s);
  } else {
    launch<STATS>(p, in->rows, nt, s);
    if ((st = launch_status(who)) != AZ_OK) return st;
    launch<WRITE>(p, in->rows, nt, s);
  }
  return launch_status(who);
}
