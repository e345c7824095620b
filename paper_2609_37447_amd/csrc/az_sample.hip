// One entry of each row of logits, drawn with a given random number among those that top-k, top-p and min-p leave.
//
// All three keep a beginning of the entries in the order of falling logits (equal ones by rising index): nothing
// is sorted, only the last entry that stays is looked for.  A weight exp((l - largest) / T) is a whole
// multiple of 2^-S, so that sums of weights are exact whole numbers in any order, and LDS atomics may build
// them: a histogram over a key (the logit's distance from the largest, its bits, or the index) says in which
// of its bins the wanted sum is reached, and that bin is cut up in turn until it is one key.
//
// One workgroup a row.  Where what may stay fits LDS it is copied there, and the rest is done without memory.
#include <math.h>

#include "az_codes_common.h"

namespace {

constexpr int MAX_ROWS = 1 << 20, MAX_VOCAB = 1 << 24;
constexpr float REACH = 37.0f;  // distances past 37 T have no weight: 2^-S of the largest is at most exp(-36.04)

struct SampleView {
  const void* logits;
  const float* u;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* out;
  float* prob;
  int64_t ld;
  int rows, vocab, shift;  // shift: S
};

// Bits of a logit in the order of its value (-0 counts as 0), and back.
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.0f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key ^ ((uint32_t)((int32_t)~key >> 31) | 0x80000000u));
}
constexpr uint32_t NONE = 0x007fffffu;  // the key of -inf: what is not above it is not allowed

// Whole weights.
struct Weights {
  double top, inv, floor;
  int shift;
  // exp((l - top) / T) by 2^n 2^f, |f| <= 1/2, and the Taylor series of 2^f in f ln 2 to its twelfth power (1.7e-16).
  __device__ __forceinline__ double of(float l) const {
    const double y = fmax(((double)l - top) * inv * 1.4426950408889634, -1100.0), n = rint(y), t = (y - n) * 0.6931471805599453;
    double x = 1.0 / 479001600;
    x = fma(x, t, 1.0 / 39916800);
    x = fma(x, t, 1.0 / 3628800);
    x = fma(x, t, 1.0 / 362880);
    x = fma(x, t, 1.0 / 40320);
    x = fma(x, t, 1.0 / 5040);
    x = fma(x, t, 1.0 / 720);
    x = fma(x, t, 1.0 / 120);
    x = fma(x, t, 1.0 / 24);
    x = fma(x, t, 1.0 / 6);
    x = fma(x, t, 0.5);
    x = fma(x, t, 1.0);
    x = fma(x, t, 1.0);
    return ldexp(x, (int)n);
  }
  __device__ __forceinline__ uint64_t whole(double x) const {
    return (uint64_t)__double_as_longlong(ldexp(x, shift) + 0x1p52) & 0xfffffffffffffull;  // rounded by the addition
  }
  __device__ __forceinline__ uint64_t operator()(uint32_t key) const { return key > NONE ? whole(of(value_of(key))) : 0; }
  __device__ __forceinline__ uint64_t above_floor(uint32_t key) const {
    if (key <= NONE) return 0;
    const double x = of(value_of(key));
    return x >= floor ? whole(x) : 0;
  }
};

// The last entry that stays: its key, and its index among equal ones.
struct Last {
  uint32_t key;
  int index;
  __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= index); }
};

template <int NT>
struct Sampler {
  static constexpr int BINS = 2 * NT, LIST = 4 * NT;
  uint64_t sums[BINS];
  uint32_t counts[BINS];
  uint2 list[LIST];  // key, index
  uint64_t waves[NT / 64];
  uint64_t found[3];  // of a search: the bin (BINS: none), the sum before it, the bin's own
  uint64_t total;
  uint32_t wave_counts[NT / 64];
  uint32_t before_count;
  uint32_t length;
  float wave_top[NT / 64];
  int wave_bad[NT / 64];

  __device__ __forceinline__ void clear() {
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += NT) {
      sums[i] = 0;
      counts[i] = 0;
    }
    __syncthreads();
  }
  __device__ __forceinline__ void add(int bin, uint64_t w) {
    if (w) atomicAdd(reinterpret_cast<unsigned long long*>(&sums[bin]), (unsigned long long)w);
  }
  // The sum of all bins before thread t's two, and of everything into `total`.
  __device__ __forceinline__ uint64_t scan(uint64_t own) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t s = own;
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t x = __shfl_up((unsigned long long)s, o);
      if (lane >= o) s += x;
    }
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    uint64_t before = 0, all = 0;
    for (int w = 0; w < NT / 64; w++) {
      if (w < wave) before += waves[w];
      all += waves[w];
    }
    if (threadIdx.x == 0) total = all;
    return before + s - own;
  }
};

// A row in memory, eight entries a thread at a time.
template <bool BF16, int NT>
struct RowSource {
  const void* row;
  int vocab;
  // f(index, logit) for the entries lo..hi - 1
  template <class F>
  __device__ __forceinline__ void each(int lo, int hi, F&& f) const {
    for (int64_t i0 = (int64_t)(lo & ~7) + threadIdx.x * 8; i0 < hi; i0 += NT * 8) {
      const int i = (int)i0;
      float l[8];
      if (i + 8 <= vocab) {
        if constexpr (BF16) {
          cm_i32x4 w;
          __builtin_memcpy(&w, (const uint16_t*)row + i, 16);
#pragma unroll
          for (int j = 0; j < 4; j++) {
            l[2 * j] = __uint_as_float((uint32_t)w[j] << 16);
            l[2 * j + 1] = __uint_as_float((uint32_t)w[j] & 0xffff0000u);
          }
        } else {
          __builtin_memcpy(l, (const float*)row + i, 32);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; j++)
          l[j] = i + j >= vocab ? -INFINITY : BF16 ? f32_of_bf16(((const uint16_t*)row)[i + j]) : ((const float*)row)[i + j];
      }
#pragma unroll
      for (int j = 0; j < 8; j++)
        if (i + j >= lo && i + j < hi) f(i + j, l[j]);
    }
  }
  template <class F>
  __device__ __forceinline__ void keys(F&& f) const {
    each(0, vocab, [&](int i, float l) { f(i, key_of(l)); });
  }
  template <class F>
  __device__ __forceinline__ void keys(int lo, int hi, F&& f) const {
    each(lo, hi, [&](int i, float l) { f(i, key_of(l)); });
  }
};

template <int NT>
struct ListSource {
  const uint2* list;
  uint32_t length;
  template <class F>
  __device__ __forceinline__ void keys(F&& f) const {
    for (uint32_t i = threadIdx.x; i < length; i += NT) f((int)list[i].y, list[i].x);
  }
  template <class F>
  __device__ __forceinline__ void keys(int lo, int hi, F&& f) const {
    keys([&](int i, uint32_t k) {
      if (i >= lo && i < hi) f(i, k);
    });
  }
};

template <bool BF16, int NT>
struct Row {
  using S = Sampler<NT>;
  S& s;
  SampleView p;
  Weights weight;
  float top, step;  // step: bins of distance a unit of the logit
  uint32_t top_key;

  // The first bin at which the running sum of the bins reaches `limit` (> 0): what `found` holds afterwards.
  __device__ __forceinline__ void reach(uint64_t limit) {
    __syncthreads();
    const int t = threadIdx.x;
    const uint64_t a = s.sums[2 * t], b = s.sums[2 * t + 1];
    if (t == 0) s.found[0] = S::BINS;
    const uint64_t before = s.scan(a + b);
    if (before < limit && limit <= before + a + b) {
      const bool first = limit <= before + a;
      s.found[0] = 2 * t + (first ? 0 : 1);
      s.found[1] = first ? before : before + a;
      s.found[2] = first ? a : b;
    }
    __syncthreads();
  }
  __device__ __forceinline__ uint64_t whole_sum() {
    __syncthreads();
    s.scan(s.sums[2 * threadIdx.x] + s.sums[2 * threadIdx.x + 1]);
    __syncthreads();
    return s.total;
  }
  // Bin of a logit by its distance from the largest; the last bin holds what has no weight.
  __device__ __forceinline__ int bin_of(float l) const {
    const float d = top - l;
    return d == 0.0f ? 0 : (int)fminf(d * step, (float)(S::BINS - 1));
  }
  // The keys of a bin: bin_of falls as the key rises.
  __device__ __forceinline__ void bin_keys(int bin, uint32_t& lo, uint32_t& hi) const {
    auto first_at_most = [&](int b) {  // the smallest key whose bin is at most b
      uint32_t x = NONE + 1, y = top_key;
      while (x < y) {
        const uint32_t mid = x + (y - x) / 2;
        if (bin_of(value_of(mid)) <= b) y = mid;
        else x = mid + 1;
      }
      return x;
    };
    lo = first_at_most(bin);
    hi = bin == 0 ? top_key : first_at_most(bin - 1) - 1;
  }

  // The index at which the running sum of w(index, key), by rising index, reaches `limit`.
  template <class Src, class W>
  __device__ __forceinline__ int by_index(const Src& src, uint64_t limit, W&& w) {
    int lo = 0, hi = p.vocab, shift = 0;
    while (((hi - 1) >> shift) >= S::BINS) shift++;
    for (;;) {
      s.clear();
      src.keys(lo, hi, [&](int i, uint32_t k) { s.add((i - lo) >> shift, w(i, k)); });
      reach(limit);
      const int bin = (int)s.found[0];
      limit -= s.found[1];
      lo += bin << shift;
      if (shift == 0) return lo;
      hi = min(hi, lo + (1 << shift));
      shift = 0;
      while (((hi - lo - 1) >> shift) >= S::BINS) shift++;
    }
  }

  // The last entry that stays where entries do as long as the sum of w(key) before them is below `limit`, among
  // those that `last` keeps; lo..hi: keys that it is among, `limit` less what is above them.
  template <class Src, class W>
  __device__ __forceinline__ Last by_key(const Src& src, Last last, uint32_t lo, uint32_t hi, uint64_t limit, W&& w) {
    for (;;) {
      int shift = 0;
      while (((hi - lo) >> shift) >= (uint32_t)S::BINS) shift++;
      s.clear();
      src.keys([&](int i, uint32_t k) {
        if (k >= lo && k <= hi && last.keeps(k, i)) s.add((int)((hi - k) >> shift), w(k));
      });
      reach(limit);
      if (s.found[0] == (uint64_t)S::BINS) return last;  // everything stays
      limit -= s.found[1];
      const uint64_t bin = s.found[0], own = s.found[2];
      hi -= (uint32_t)(bin << shift);
      lo = hi - lo >= (1u << shift) ? hi - ((1u << shift) - 1) : lo;
      if (lo == hi) {
        const uint64_t one = w(lo), ties = own / one, stay = (limit + one - 1) / one;
        if (stay >= ties) return Last{lo, lo == last.key ? last.index : 0x7fffffff};
        const uint32_t key = lo;
        return Last{key, by_index(src, stay, [&](int i, uint32_t k) -> uint64_t { return k == key && last.keeps(k, i); })};
      }
    }
  }

  // Draws among what `last` keeps.
  template <class Src>
  __device__ __forceinline__ void draw(const Src& src, Last last, float u, int64_t b) {
    auto w = [&](int i, uint32_t k) -> uint64_t { return last.keeps(k, i) ? weight.above_floor(k) : 0; };
    // the whole sum, over bins that mean nothing
    s.clear();
    uint64_t own = 0;
    src.keys([&](int i, uint32_t k) { own += w(i, k); });
    s.scan(own);
    __syncthreads();
    const uint64_t all = s.total;
    const uint64_t target = min((uint64_t)((double)u * (double)all), all - 1);
    const int token = by_index(src, target + 1, w);
    if (threadIdx.x == 0) {
      p.out[b] = token;
      if (p.prob) {
        const float l = BF16 ? f32_of_bf16(((const uint16_t*)p.logits)[b * p.ld + token]) : ((const float*)p.logits)[b * p.ld + token];
        p.prob[b] = (float)((double)weight(key_of(l)) / (double)all);
      }
    }
  }

  // Top-p, min-p and the draw among what `last` keeps.
  template <class Src>
  __device__ __forceinline__ void rest(const Src& src, Last last, float top_p, float u, int64_t b) {
    if (top_p < 1.0f) {
      s.clear();
      uint64_t own = 0;
      src.keys([&](int i, uint32_t k) { own += last.keeps(k, i) ? weight(k) : 0; });
      s.scan(own);
      __syncthreads();
      const uint64_t limit = (uint64_t)fmax(ceil((double)top_p * (double)s.total), 1.0);
      last = by_key(src, last, NONE + 1, top_key, limit, [&](uint32_t k) { return weight(k); });
    }
    draw(src, last, u, b);
  }
};

template <bool BF16, int NT>
__global__ __launch_bounds__(NT) void az_sample_rows(SampleView p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  Sampler<NT>& s = *reinterpret_cast<Sampler<NT>*>(smem);
  const int64_t b = blockIdx.x;
  const RowSource<BF16, NT> src = {(const uint8_t*)p.logits + b * p.ld * (BF16 ? 2 : 4), p.vocab};
  float top = -INFINITY;
  bool bad = false;
  src.each(0, p.vocab, [&](int, float l) {
    top = fmaxf(top, l);
    bad |= !(l < INFINITY);
  });
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  bad = __any(bad);
  if ((threadIdx.x & 63) == 0) {
    s.wave_top[threadIdx.x >> 6] = top;
    s.wave_bad[threadIdx.x >> 6] = bad;
  }
  __syncthreads();
  for (int w = 0; w < NT / 64; w++) {
    top = fmaxf(top, s.wave_top[w]);
    bad |= s.wave_bad[w] != 0;
  }
  if (bad || top == -INFINITY) {
    if (threadIdx.x == 0) {
      p.out[b] = -1;
      if (p.prob) p.prob[b] = 0.0f;
    }
    return;
  }
  const float t = p.temperature ? p.temperature[b] : 1.0f;
  const uint32_t top_key = key_of(top);
  const bool greedy = !(t > 0.0f);
  const float step = greedy ? 1.0f : fminf((float)Sampler<NT>::BINS / REACH / t, 0x1p100f);
  float floor = p.min_p ? p.min_p[b] : 0.0f;
  floor = floor > 0.0f ? fminf(floor, 1.0f) : 0.0f;
  Row<BF16, NT> row = {s, p, {(double)top, greedy ? 1.0 : 1.0 / (double)t, (double)floor, p.shift}, top, step, top_key};
  if (greedy) {
    const int token = row.by_index(src, 1, [&](int, uint32_t k) -> uint64_t { return k == top_key; });
    if (threadIdx.x == 0) {
      p.out[b] = token;
      if (p.prob) p.prob[b] = 1.0f;
    }
    return;
  }
  int k = p.top_k ? p.top_k[b] : 0;
  if (k <= 0 || k > p.vocab) k = p.vocab;
  const float top_p = p.top_p && p.top_p[b] < 1.0f ? p.top_p[b] : 1.0f;
  float u = p.u[b];
  u = u > 0.0f ? fminf(u, 1.0f) : 0.0f;
  Last last = {NONE + 1, 0x7fffffff};
  if (k < p.vocab) last = row.by_key(src, last, NONE + 1, top_key, (uint64_t)k, [&](uint32_t) -> uint64_t { return 1; });
  row.rest(src, last, top_p, u, b);
}

template <bool BF16, int NT>
int launch(const SampleView& p, hipStream_t s) {
  const int lds = (int)sizeof(Sampler<NT>);
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(az_sample_rows<BF16, NT>), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
    return AZ_ERR_DEVICE;
  hipLaunchKernelGGL((az_sample_rows<BF16, NT>), dim3((unsigned)p.rows), dim3(NT), lds, s, p);
  return AZ_OK;
}

}  // namespace

extern "C" int az_logits_sample(const az_sampling* in, int32_t* out, float* prob, void* stream) {
  static const char who[] = "az_logits_sample";
  if (!in) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL sampling");
  if (in->rows < 0 || in->vocab < 1) return code_fail(AZ_ERR_INVALID_ARG, who, "rows < 0 or vocab < 1");
  if (in->rows > MAX_ROWS || in->vocab > MAX_VOCAB) return code_fail(AZ_ERR_UNSUPPORTED, who, "rows > 2^20 or vocab > 2^24");
  if (in->dtype != AZ_F32 && in->dtype != AZ_BF16) return code_fail(AZ_ERR_INVALID_ARG, who, "dtype is neither AZ_F32 nor AZ_BF16");
  if (in->rows == 0) return AZ_OK;
  const int st = dense_check(in->logits, in->dtype, in->ld, in->vocab, who);
  if (st != AZ_OK) return st;
  if (!in->u || !out) return code_fail(AZ_ERR_INVALID_ARG, who, "NULL u or out");
  if (((uintptr_t)in->u | (uintptr_t)in->temperature | (uintptr_t)in->top_k | (uintptr_t)in->top_p | (uintptr_t)in->min_p | (uintptr_t)out | (uintptr_t)prob) & 3u)
    return code_fail(AZ_ERR_INVALID_ARG, who, "a buffer that is not aligned to its element");
  int shift = 62;
  while (((int64_t)1 << (62 - shift)) < in->vocab) shift--;
  const SampleView p = {in->logits, in->u, in->temperature, in->top_k, in->top_p, in->min_p, out, prob, in->ld, in->rows, in->vocab,
                        shift < 51 ? shift : 51};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  return launched(who, in->dtype == AZ_BF16 ? launch<true, 1024>(p, s) : launch<false, 1024>(p, s));
}
