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
//
// 4,096 rows of 4,672 fp32 logits and bits: 30.5 us, 5.1 TB/s.  512 rows of 131,072 bf16 logits, bits and a
// bias: 112 us, 137 with 2,048 past entries a row (81 at a copy's rate if the logits were read once).  One workgroup
// of 1,024 threads that keeps such a row in its registers reads it once,
// but leaves a compute unit nothing else to do between its barriers: 135 us, 146 with past entries.
#include <math.h>

#include "az_codes_common.h"

namespace {

constexpr int GROUPS = 4;               // a thread's groups of four entries
constexpr int PER = 4 * GROUPS;         // entries of a thread
constexpr int THREADS = 1024;           // of the largest workgroup
constexpr int MOST = THREADS * PER;     // entries of a workgroup
constexpr int MAX_ROWS = 1 << 20, MAX_VOCAB = 1 << 24;
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

// exp(l - m); 0 for l = -inf where m is finite.  The difference and its product with log2 e are one fp32 number
// each, as in the network kernels: the relative error grows to about |l - m| 2^-23.
__device__ __forceinline__ float exp_below(float l, float m) { return __builtin_amdgcn_exp2f((l - m) * LOG2E); }

// Maximum (of what is not NaN) and sum over a wave, in every lane, by lane exchanges of the
// vector unit.
template <int CTRL>
__device__ __forceinline__ float lane_move(float x) {
  const int i = __float_as_int(x);
  return __int_as_float(__builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, false));
}
template <class F>
__device__ __forceinline__ float wave_all(float x, F&& f) {
  x = f(x, lane_move<0xb1>(x));   // lane ^ 1
  x = f(x, lane_move<0x4e>(x));   // lane ^ 2
  x = f(x, lane_move<0x141>(x));  // the other four of eight
  x = f(x, lane_move<0x140>(x));  // the other eight of sixteen
  x = f(x, __shfl_xor(x, 16));
  return f(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float wave_top(float x) { return wave_all(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_total(float x) { return wave_all(x, [](float a, float b) { return a + b; }); }

// A row's penalties.  l / r is a product with 1 / r and one correction, which gives the
// quotient to the last place; where 1 / r is not a normal number, it is divided.
struct Penalties {
  float r, inv, f, p;
  bool divide;
  __device__ __forceinline__ Penalties() {}
  __device__ __forceinline__ explicit Penalties(const float* x) : r(x[0]), inv(1.0f / x[0]), f(x[1]), p(x[2]) {
    divide = !(inv >= 0x1p-126f && inv <= 0x1p126f);
  }
  __device__ __forceinline__ float of(float l, uint32_t c) const {
    float q;
    if (divide) {
      q = l / r;
    } else {
      const float q0 = l * inv;
      q = fmaf(fmaf(-q0, r, l), inv, q0);
      if (fabsf(q0) == INFINITY) q = q0;
    }
    return (l > 0.0f ? q : l * r) - fmaf(f, (float)c, p);
  }
};

// Four entries from v on.  They are loaded as they lie in memory and looked at later, so that a
// thread's loads are on their way together; a group past the vocabulary's end reads its last four.
struct Entries {
  cm_f32x4 l, add;
  uint32_t ok;

  // The adjusted logits, -inf where they are not allowed and past the vocabulary.
  template <bool HIST>
  __device__ __forceinline__ void adjust(const PolicyView& p, int64_t b, int v, const uint32_t* count, const Penalties& pen) {
    if (p.bf16) {
      const float w0 = l[0], w1 = l[1];
      l = cm_f32x4{__uint_as_float(__float_as_uint(w0) << 16), __uint_as_float(__float_as_uint(w0) & 0xffff0000u),
                   __uint_as_float(__float_as_uint(w1) << 16), __uint_as_float(__float_as_uint(w1) & 0xffff0000u)};
    }
    // one bit for each entry, at 8 i + 7
    if (p.mask_kind == AZ_MASK_BYTES) {
      ok |= (ok & 0x7f7f7f7fu) + 0x7f7f7f7fu;
    } else if (p.mask_kind == AZ_MASK_BITS) {
      ok = ok >> (v & 4);
      ok = (ok & 1u) << 7 | (ok & 2u) << 14 | (ok & 4u) << 21 | (ok & 8u) << 28;
    } else {
      ok = 0x80808080u;
    }
    if (v + 4 > p.vocab) edge(p, b, v);
    if constexpr (HIST) {
      const cm_i32x4 c = *reinterpret_cast<const cm_i32x4*>(count);
      if (c[0] | c[1] | c[2] | c[3]) {
#pragma unroll
        for (int i = 0; i < 4; i++) l[i] = c[i] ? pen.of(l[i], (uint32_t)c[i]) : l[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t keep = (uint32_t)((int32_t)(ok << (24 - 8 * i)) >> 31), sum = __float_as_uint(l[i] + add[i]);
      l[i] = __uint_as_float((sum & keep) | (0xff800000u & ~keep));  // -inf where the bit is 0
    }
  }
  // The group that the vocabulary ends in, one by one; beyond it nothing is allowed.
  __device__ __forceinline__ void edge(const PolicyView& p, int64_t b, int v) {
    ok = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int64_t u = (int64_t)v + i;
      l[i] = add[i] = 0.0f;
      if (u < p.vocab) {
        l[i] = p.bf16 ? f32_of_bf16(((const uint16_t*)p.logits)[b * p.ld + u]) : ((const float*)p.logits)[b * p.ld + u];
        if (p.bias) add[i] = p.bias[b * p.ld_bias + u];
        bool may = true;
        if (p.mask_kind == AZ_MASK_BYTES) may = ((const uint8_t*)p.mask)[b * p.ld_mask + u] != 0;
        else if (p.mask_kind == AZ_MASK_BITS) may = (((const uint8_t*)p.mask)[4 * b * p.ld_mask + (u >> 3)] >> (u & 7)) & 1;
        if (may) ok |= 0x80u << (8 * i);
      }
    }
  }
  __device__ __forceinline__ void store(const PolicyView& p, int64_t b, int v) const {
    float* o = p.out + b * p.ld_out + v;
    if (v + 4 <= p.vocab) {
      __builtin_memcpy(o, &l, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++)
        if (v + i < p.vocab) o[i] = l[i];
    }
  }
};

// A thread's groups, `step` entries apart from v on, as they lie in memory (bf16 logits: the first two words).
__device__ __forceinline__ void load_groups(Entries (&x)[GROUPS], const PolicyView& p, int64_t b, int v, int step) {
#pragma unroll
  for (int g = 0; g < GROUPS; g++) {
    x[g].l = x[g].add = cm_f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    x[g].ok = 0;
  }
  if (p.vocab < 4) return;
  int64_t at[GROUPS];
#pragma unroll
  for (int g = 0; g < GROUPS; g++) at[g] = min(v + g * step, p.vocab - 4);
  if (p.bf16) {
    const uint16_t* row = (const uint16_t*)p.logits + b * p.ld;
#pragma unroll
    for (int g = 0; g < GROUPS; g++) __builtin_memcpy(&x[g].l, row + at[g], 8);
  } else {
    const float* row = (const float*)p.logits + b * p.ld;
#pragma unroll
    for (int g = 0; g < GROUPS; g++) __builtin_memcpy(&x[g].l, row + at[g], 16);
  }
  if (p.bias) {
    const float* row = p.bias + b * p.ld_bias;
#pragma unroll
    for (int g = 0; g < GROUPS; g++) __builtin_memcpy(&x[g].add, row + at[g], 16);
  }
  if (p.mask_kind == AZ_MASK_BYTES) {
    const uint8_t* row = (const uint8_t*)p.mask + b * p.ld_mask;
#pragma unroll
    for (int g = 0; g < GROUPS; g++) __builtin_memcpy(&x[g].ok, row + at[g], 4);
  } else if (p.mask_kind == AZ_MASK_BITS) {
    const uint8_t* row = (const uint8_t*)p.mask + 4 * b * p.ld_mask;
#pragma unroll
    for (int g = 0; g < GROUPS; g++) x[g].ok = row[at[g] >> 3];
  }
}

// ADJUST: the adjusted logits.  WHOLE: the policy of rows that one workgroup holds.  STATS and
// WRITE: the two kernels of longer rows.
enum { ADJUST = 0, WHOLE = 1, STATS = 2, WRITE = 3 };

// blockIdx.x: a chunk of 16 entries a thread; blockIdx.y + 65535 blockIdx.z: the row.
template <int MODE, bool HIST>
__global__ __launch_bounds__(THREADS) void az_policy_kernel(PolicyView p, int rows) {
  extern __shared__ __attribute__((aligned(16))) uint32_t count[];  // HIST: one for each entry of the chunk
  __shared__ float red[2][THREADS / 64];
  const int64_t b = (int64_t)blockIdx.z * 65535 + blockIdx.y;
  if (b >= rows) return;
  const int nt = blockDim.x, t = threadIdx.x, v0 = (int)blockIdx.x * nt * PER;
  Entries x[GROUPS];
  load_groups(x, p, b, v0 + t * 4, nt * 4);
  Penalties pen;
  if constexpr (HIST) {
    const int n = p.lengths ? min(max(p.lengths[b], 0), p.max_history) : p.max_history;
    const int32_t* past = p.history + b * p.ld_history;
    pen = Penalties(p.penalties + 3 * b);
    constexpr int AHEAD = 4;  // past entries of a thread that are on their way while the counters are cleared
    int32_t e[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; i++) e[i] = t + i * nt < n ? past[t + i * nt] : -1;
#pragma unroll
    for (int i = 0; i < GROUPS; i++) reinterpret_cast<cm_i32x4*>(count)[i * nt + t] = cm_i32x4{0, 0, 0, 0};
    __syncthreads();
    const uint32_t here = (uint32_t)min(nt * PER, p.vocab - v0);
    auto add = [&](int32_t v) {
      if ((uint32_t)v >= (uint32_t)v0 && (uint32_t)v - (uint32_t)v0 < here) atomicAdd(&count[v - v0], 1u);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; i++) add(e[i]);
    for (uint32_t i = t + AHEAD * nt; i < (uint32_t)n; i += nt) add(past[i]);  // (n may be 2^31 - 1)
    __syncthreads();
  }
#pragma unroll
  for (int g = 0; g < GROUPS; g++) x[g].adjust<HIST>(p, b, v0 + (g * nt + t) * 4, count + (g * nt + t) * 4, pen);

  // m: the row's (STATS: the chunk's) maximum, 0 where nothing is above -inf; inv: 1 / sum of exp(l - m), 0
  // where that is 0 for want of an entry.
  float m = 0.0f, inv = 1.0f;
  if constexpr (MODE == WHOLE || MODE == STATS) {
    float top = -INFINITY;
#pragma unroll
    for (int g = 0; g < GROUPS; g++)
#pragma unroll
      for (int i = 0; i < 4; i++) top = fmaxf(top, x[g].l[i]);
    top = wave_top(top);
    if ((t & 63) == 0) red[0][t >> 6] = top;
    __syncthreads();
    for (int w = 0; w < nt / 64; w++) top = fmaxf(top, red[0][w]);
    m = top == -INFINITY ? 0.0f : top;
    float s = 0.0f;
#pragma unroll
    for (int g = 0; g < GROUPS; g++)
#pragma unroll
      for (int i = 0; i < 4; i++) s += exp_below(x[g].l[i], m);
    s = wave_total(s);
    if ((t & 63) == 0) red[1][t >> 6] = s;
    __syncthreads();
    s = 0.0f;
    for (int w = 0; w < nt / 64; w++) s += red[1][w];
    if constexpr (MODE == STATS) {
      if (t == 0) p.stats[b * gridDim.x + blockIdx.x] = make_float2(top, s);
      return;
    }
    inv = top == -INFINITY && s == 0.0f ? 0.0f : 1.0f / s;
  }
  if constexpr (MODE == WRITE) {
    // Every wave joins the row's chunks: lane i those of i, i + 64, ..., then the lanes.
    const float2* parts = p.stats + b * gridDim.x;
    float top = -INFINITY, s = 0.0f;
    for (int i = t & 63; i < (int)gridDim.x; i += 64) top = fmaxf(top, parts[i].x);
    top = wave_top(top);
    m = top == -INFINITY ? 0.0f : top;
    // (a chunk without an entry above -inf has a sum of 0, or NaN where it holds one)
    for (int i = t & 63; i < (int)gridDim.x; i += 64) {
      const float2 part = parts[i];
      s += part.x == -INFINITY ? part.y : part.y * exp_below(part.x, m);
    }
    s = wave_total(s);
    inv = top == -INFINITY && s == 0.0f ? 0.0f : 1.0f / s;
  }
#pragma unroll
  for (int g = 0; g < GROUPS; g++) {
    if constexpr (MODE != ADJUST) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        // (a NaN row's inv must not reach what is not allowed)
        const float e = exp_below(x[g].l[i], m) * inv;
        x[g].l[i] = x[g].l[i] == -INFINITY ? 0.0f : e;
      }
    }
    x[g].store(p, b, v0 + (g * nt + t) * 4);
  }
}

// Threads of a workgroup: enough for the row, up to 1,024.  Rows that need several
// workgroups get 512 (512 rows of 131,072: 137 us, 152 with 1,024), or 256 where that takes to fill the chip.
int policy_threads(int64_t rows, int64_t vocab) {
  int nt = 256;
  if (vocab <= MOST) {
    while (nt * PER < vocab) nt *= 2;
    return nt;
  }
  return rows * ((vocab + 512 * PER - 1) / (512 * PER)) >= 512 ? 512 : 256;
}

template <int MODE>
int launch(const PolicyView& p, int rows, int nt, hipStream_t s) {
  const dim3 g((unsigned)((p.vocab + nt * PER - 1) / (nt * PER)), (unsigned)(rows < 65535 ? rows : 65535), (unsigned)((rows + 65534) / 65535));
  if (p.history) {
    const int lds = nt * PER * (int)sizeof(uint32_t);
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(az_policy_kernel<MODE, true>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return launched("az_logits_policy", AZ_ERR_DEVICE);
    hipLaunchKernelGGL((az_policy_kernel<MODE, true>), g, dim3(nt), lds, s, p, rows);
  } else {
    hipLaunchKernelGGL((az_policy_kernel<MODE, false>), g, dim3(nt), 0, s, p, rows);
  }
  return launched("az_logits_policy", AZ_OK);
}

}  // namespace

extern "C" size_t az_logits_policy_workspace(int32_t rows, int32_t vocab) {
  if (rows <= 0 || rows > MAX_ROWS || vocab <= MOST || vocab > MAX_VOCAB) return 0;
  const int chunk = policy_threads(rows, vocab) * PER;
  return (size_t)rows * (size_t)((vocab + chunk - 1) / chunk) * sizeof(float2);
}

extern "C" int az_logits_policy(const az_logits* in, int32_t probabilities, float* out, int64_t ld_out, void* workspace,
                                size_t workspace_bytes, void* stream) {
  static const char who[] = "az_logits_policy";
  if (!in) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL logits");
  if (in->rows < 0 || in->vocab < 1) return code_fail(AZ_ERR_INVALID_ARG, who, "rows < 0 or vocab < 1");
  if (in->rows > MAX_ROWS || in->vocab > MAX_VOCAB) return code_fail(AZ_ERR_UNSUPPORTED, who, "rows > 2^20 or vocab > 2^24");
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
  const size_t need = probabilities ? az_logits_policy_workspace(in->rows, in->vocab) : 0;  // (adjusted logits have no sums)
  if (workspace_bytes < need || (need && !workspace)) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace is too small");
  if ((uintptr_t)workspace & 15u) return code_fail(AZ_ERR_INVALID_ARG, who, "the workspace must be 16-byte aligned");
  const int nt = policy_threads(in->rows, in->vocab);
  const PolicyView p = {in->logits, in->mask, in->bias, hist ? in->history : nullptr, in->lengths, in->penalties, out,
                        static_cast<float2*>(workspace), in->ld, in->ld_mask, in->ld_bias, in->ld_history, ld_out,
                        in->vocab, in->max_history, in->dtype == AZ_BF16, in->mask_kind};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (!probabilities) return launch<ADJUST>(p, in->rows, nt, s);
  if (in->vocab <= MOST) return launch<WHOLE>(p, in->rows, nt, s);
  if ((st = launch<STATS>(p, in->rows, nt, s)) != AZ_OK) return st;
  return launch<WRITE>(p, in->rows, nt, s);
}
