// One entry of each row of logits, drawn with a given random number among those that top-k, top-p and min-p leave.
//
// All three keep a beginning of the entries in the order of falling logits (equal ones by rising index): nothing
// is sorted, only the last entry that stays is looked for.  A weight exp((l - largest) / T) is a whole
// multiple of 2^-S, so that sums of weights are exact whole numbers in any order, and LDS atomics may build
// them.  A histogram over the distance from the largest says in which bin the wanted count or sum is reached; if
// few entries are in it, their order among each other is found by comparing all with all, otherwise the bin
// is cut up by the logits' bits until it is few, or one value.  The draw is the same over the index.
//
// One workgroup a row.  The row is read for its largest logits, and once more for what may stay, which is copied to LDS where it
// fits; the rest is done without memory.  Where it does not fit, each step reads the row again.
//
// 512 x 131072 bf16 with all filters: 64 us with all rows full (134 MB are read at 5.6 TB/s in 24 us the first time, in 28 the
// second; 13 are the steps in LDS), 66 where half of the rows allow some 30 entries.  Without filters 121 and with top-p alone 258,
// the exponentials in fp64 of every entry once and three times.  One row of 131,072, by one workgroup: 24 us with all filters, 56
// without, 80 with top-p alone.  1 x 4672: 9.6 us, a chain of some twenty barriers and lane exchanges of one workgroup.
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

// 2^f in f ln 2 by the Taylor series to the twelfth power, |f| <= 1/2: 1.7e-16.
__device__ __forceinline__ double power_of_two(double f) {
  const double t = f * 0.6931471805599453;
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
  return fma(x, t, 1.0);
}

// Whole weights: exp((l - top) / T) 2^S by 2^(e + S) 2^(j / 32) 2^f, 0 <= j < 32, |f| <= 1/64, with a table of 2^(j / 32) and the
// Taylor series of 2^f to its fifth power (2.3e-15).
constexpr int PARTS = 32;
struct Weights {
  double top, scale, floor;  // scale: 32 log2(e) / T; floor: min-p times 2^S
  const double* table;
  int shift;
  // exp((l - top) / T) 2^S; what is below 2^-64 (-inf too) counts as that
  __device__ __forceinline__ double scaled(float l) const {
    constexpr double ROUND = 0x1.8p52, LN = 0.6931471805599453 / PARTS;
    const double y = fmax(((double)l - top) * scale, -64.0 * PARTS), m = y + ROUND, f = y - (m - ROUND);
    const int n = (int)__double_as_longlong(m);  // the nearest whole number to y
    double x = LN * LN * LN * LN * LN / 120;
    x = fma(x, f, LN * LN * LN * LN / 24);
    x = fma(x, f, LN * LN * LN / 6);
    x = fma(x, f, LN * LN / 2);
    x = fma(x, f, LN);
    x = fma(x, f, 1.0) * table[n & (PARTS - 1)];
    return __longlong_as_double(__double_as_longlong(x) + ((int64_t)((n >> 5) + shift) << 52));
  }
  static __device__ __forceinline__ uint64_t whole(double x) {
    return (uint64_t)__double_as_longlong(x + 0x1p52) & 0xfffffffffffffull;  // rounded by the addition
  }
  __device__ __forceinline__ uint64_t operator()(float l) const { return whole(scaled(l)); }
  __device__ __forceinline__ uint64_t above_floor(float l) const {
    const double x = scaled(l);
    return x >= floor ? whole(x) : 0;
  }
};

// The last entry that stays: its key, and its index among equal ones.
struct Last {
  uint32_t key;
  int index;
  __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= index); }
};

// The sums of a wave's values up to each lane, by lane moves: within rows of 16, then from row to row.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t move_add(uint64_t x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, false);
  return x + ((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
  x = move_add<0x111, 0xf>(x);     // from the lane before
  x = move_add<0x112, 0xf>(x);     // two before
  x = move_add<0x114, 0xf>(x);     // four
  x = move_add<0x118, 0xf>(x);     // eight
  x = move_add<0x142, 0xa>(x);     // the last lane of rows 0 and 2 to rows 1 and 3
  return move_add<0x143, 0xc>(x);  // lane 31 to the upper half
}

template <int NT>
struct Sampler {
  static constexpr int BINS = 2 * NT, LIST = NT < 1024 ? 8 * NT : 4 * NT, FEW = 256, SLOTS = 64;
  uint64_t sums[BINS];
  uint64_t few_order[FEW];   // of the entries that are compared with each other: what orders them,
  uint64_t few_weight[FEW];  // and their weights
  uint64_t slots[SLOTS];
  uint64_t waves[NT / 64];
  uint64_t found[3];  // of a search: the bin (BINS: none), the sum before it, the bin's own
  uint64_t total;
  uint64_t token_weight;
  double table[PARTS];
  uint32_t counts[BINS];
  uint2 list[LIST];  // logit, index
  uint32_t length, few;
  float wave_top[NT / 64];
  uint32_t wave_groups[NT / 64];
  int wave_bad[NT / 64];
  int token;

  // The sum of all threads' values before thread t's, and of all of them into `total` (after the next barrier).
  __device__ __forceinline__ uint64_t scan(uint64_t own) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t s = wave_scan(own);
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

// What a thread has seen of a row: bits of the largest entries as signed numbers (of positive ones, and NaN and +inf above them), the
// smallest and the largest as unsigned ones (of negative ones the largest, and NaN past -inf), in halves for bf16.
template <bool BF16>
struct Seen {
  typedef short i16x2 __attribute__((ext_vector_type(2)));
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  static constexpr uint32_t NOTHING = BF16 ? 0xff80ff80u : 0xff800000u;  // -inf
  uint32_t high = BF16 ? 0x80008000u : 0x80000000u, low = NOTHING;
  __device__ __forceinline__ void add(uint32_t w) {
    if constexpr (BF16) {
      high = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, high), __builtin_bit_cast(i16x2, w)));
      low = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(u16x2, low), __builtin_bit_cast(u16x2, w)));
    } else {
      high = (uint32_t)max((int32_t)high, (int32_t)w);
      low = min(low, w);
    }
  }
  static __device__ __forceinline__ uint32_t highest(uint32_t a, uint32_t b) {
    if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    return max(a, b);
  }
  // The largest entry's bits in the upper half (bf16), and whether a NaN or +inf is among the entries.
  __device__ __forceinline__ float largest() const {
    if constexpr (!BF16) return __uint_as_float((int32_t)high >= 0 ? high : low);
    const int32_t hi = max((int32_t)high >> 16, (int32_t)(high << 16) >> 16);
    return __uint_as_float((hi >= 0 ? (uint32_t)hi : min(low >> 16, low & 0xffffu)) << 16);
  }
  __device__ __forceinline__ bool bad(uint32_t top) const {  // top: the largest as unsigned numbers
    if constexpr (!BF16) return (int32_t)high >= 0x7f800000 || top > NOTHING;
    return max((int32_t)high >> 16, (int32_t)(high << 16) >> 16) >= 0x7f80 || max(top >> 16, top & 0xffffu) > 0xff80u;
  }
};

// A row in memory.  A thread takes eight entries at a time, AHEAD of which are on their way together.
template <bool BF16, int NT>
struct RowSource {
  static constexpr int AHEAD = 4, WORDS = BF16 ? 4 : 8;
  const void* row;
  int vocab;
  __device__ __forceinline__ void load(int i, uint32_t (&w)[WORDS]) const {
    __builtin_memcpy(w, (const uint8_t*)row + (int64_t)i * (BF16 ? 2 : 4), WORDS * 4);
  }
  static __device__ __forceinline__ float entry(const uint32_t (&w)[WORDS], int j) {
    return __uint_as_float(!BF16 ? w[j & (WORDS - 1)] : j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
  }
  // The largest entry of each of the thread's AHEAD parts, whether a NaN or +inf is among them, and how many of its groups of
  // eight hold anything above -inf (or not a number).
  __device__ __forceinline__ void look(float (&top)[AHEAD], bool& bad, uint32_t& groups) const {
    Seen<BF16> seen[AHEAD];
    uint32_t high = 0;
    groups = 0;
    auto eight = [&](const uint32_t (&w)[WORDS], int a) {
      uint32_t all = ~0u;
#pragma unroll
      for (int j = 0; j < WORDS; j++) {
        seen[a].add(w[j]);
        high = Seen<BF16>::highest(high, w[j]);
        all &= w[j];
      }
      groups += all != Seen<BF16>::NOTHING;
    };
    int64_t i0 = threadIdx.x * 8;
    for (; i0 + (AHEAD - 1) * NT * 8 + 8 <= vocab; i0 += AHEAD * NT * 8) {
      uint32_t w[AHEAD][WORDS];
#pragma unroll
      for (int a = 0; a < AHEAD; a++) load((int)i0 + a * NT * 8, w[a]);
#pragma unroll
      for (int a = 0; a < AHEAD; a++) eight(w[a], a);
    }
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      if (i0 < vocab) {
        uint32_t w[WORDS];
        if (i0 + 8 <= vocab) {
          load((int)i0, w);
        } else {
#pragma unroll
          for (int j = 0; j < WORDS; j++) w[j] = Seen<BF16>::NOTHING;
#pragma unroll
          for (int j = 0; j < 8; j++)
            if (i0 + j < vocab) {
              const uint32_t l = __float_as_uint(single((int)i0 + j));
              if constexpr (!BF16) w[j] = l;
              else w[j >> 1] = j & 1 ? (w[j >> 1] & 0xffffu) | l : (w[j >> 1] & 0xffff0000u) | l >> 16;
            }
        }
        eight(w, a);
        i0 += NT * 8;
      }
    }
    bad = false;
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      top[a] = seen[a].largest();
      bad |= seen[a].bad(high);
    }
  }
  __device__ __forceinline__ float single(int i) const {
    return BF16 ? f32_of_bf16(((const uint16_t*)row)[i]) : ((const float*)row)[i];
  }
  // f(index, logit) for the entries lo..hi - 1
  template <class F>
  __device__ __forceinline__ void each(int lo, int hi, F&& f) const {
    int64_t i0 = (int64_t)(lo & ~7) + threadIdx.x * 8;
    for (; i0 + (AHEAD - 1) * NT * 8 + 8 <= hi; i0 += AHEAD * NT * 8) {
      uint32_t w[AHEAD][WORDS];
#pragma unroll
      for (int a = 0; a < AHEAD; a++) load((int)i0 + a * NT * 8, w[a]);
#pragma unroll
      for (int a = 0; a < AHEAD; a++)
#pragma unroll
        for (int j = 0; j < 8; j++)
          if ((int)i0 + a * NT * 8 + j >= lo) f((int)i0 + a * NT * 8 + j, entry(w[a], j));
    }
    if (i0 >= hi) return;
    uint32_t w[AHEAD][WORDS];
#pragma unroll
    for (int a = 0; a < AHEAD; a++)
      if (i0 + a * NT * 8 + 8 <= vocab) load((int)i0 + a * NT * 8, w[a]);
#pragma unroll
    for (int a = 0; a < AHEAD; a++) {
      const int64_t i = i0 + a * NT * 8;
      if (i + 8 <= vocab) {
#pragma unroll
        for (int j = 0; j < 8; j++)
          if (i + j >= lo && i + j < hi) f((int)i + j, entry(w[a], j));
      } else {
        for (int64_t j = i < lo ? lo : i; j < hi; j++) f((int)j, single((int)j));
      }
    }
  }
};

template <int NT>
struct ListSource {
  const uint2* list;
  uint32_t length;
  template <class F>
  __device__ __forceinline__ void each(int lo, int hi, F&& f) const {
    for (uint32_t n = threadIdx.x; n < length; n += NT) {
      const int i = (int)list[n].y;
      if (i >= lo && i < hi) f(i, __uint_as_float(list[n].x));
    }
  }
};

// Where a limit is reached: a bin of the distance from the largest, what is left of the limit in it, and the entries in it
// and up to its end.
struct Reached {
  int bin;
  uint64_t limit;
  uint32_t entries, upto;
};

template <bool BF16, int NT>
struct Row {
  using S = Sampler<NT>;
  S& s;
  SampleView p;
  Weights weight;
  float top, step;  // step: bins of distance a unit of the logit
  uint32_t top_key;

  __device__ __forceinline__ void clear(bool count) {
    __syncthreads();
    for (int i = threadIdx.x; i < S::BINS; i += NT) {
      s.sums[i] = 0;
      if (count) s.counts[i] = 0;
    }
    __syncthreads();
  }
  __device__ __forceinline__ void add(int bin, uint64_t w) {
    atomicAdd(reinterpret_cast<unsigned long long*>(&s.sums[bin]), (unsigned long long)w);
  }
  // The first bin at which the running sum of the bins reaches limit(their whole sum) (> 0), into `found`.
  template <class L>
  __device__ __forceinline__ void reach(L&& limit_of) {
    __syncthreads();
    const int t = threadIdx.x;
    const uint64_t a = s.sums[2 * t], b = s.sums[2 * t + 1];
    if (t == 0) s.found[0] = S::BINS;
    const uint64_t before = s.scan(a + b);
    __syncthreads();
    const uint64_t limit = limit_of(s.total);
    if (before < limit && limit <= before + a + b) {
      const bool first = limit <= before + a;
      s.found[0] = 2 * t + (first ? 0 : 1);
      s.found[1] = limit - (first ? before : before + a);
      s.found[2] = first ? a : b;
    }
    __syncthreads();
  }
  // Bin of a logit by its distance from the largest; the last bin holds what has no weight.  (Of half the distance, which
  // no two finite logits have past fp32.)
  __device__ __forceinline__ int bin_of(float l) const { return (int)fminf(fmaf(-0.5f, l, 0.5f * top) * (2.0f * step), (float)(S::BINS - 1)); }
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

  // The index at which the running sum of w(index, logit), by rising index, reaches limit(their whole sum), and that sum.
  template <class Src, class W, class L>
  __device__ __forceinline__ int by_index(const Src& src, W&& w, L&& limit_of, uint64_t& all) {
    int lo = 0, hi = p.vocab;
    uint64_t limit = 0;
    bool known = false;  // the limit
    auto limit_now = [&](uint64_t sum) { return known ? limit : limit_of(sum); };
    while (hi - lo > S::SLOTS) {
      int shift = 0;
      while (((hi - lo - 1) >> shift) >= S::BINS) shift++;
      clear(false);
      int bin = 0;  // neighbours go to the same bin together
      uint64_t sum = 0;
      src.each(lo, hi, [&](int i, float l) {
        const uint64_t x = w(i, l);
        const int to = (i - lo) >> shift;
        if (to != bin) {
          if (sum) add(bin, sum);
          bin = to;
          sum = 0;
        }
        sum += x;
      });
      if (sum) add(bin, sum);
      reach(limit_now);
      if (!known) all = s.total;
      known = true;
      limit = s.found[1];
      lo += (int)s.found[0] << shift;
      hi = min(hi, lo + (1 << shift));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < S::SLOTS; i += NT) s.slots[i] = 0;
    __syncthreads();
    src.each(lo, hi, [&](int i, float l) { s.slots[i - lo] = w(i, l); });
    __syncthreads();
    if (threadIdx.x < 64) {
      const uint64_t own = s.slots[threadIdx.x], sum = wave_scan(own);
      const uint64_t whole = __shfl((unsigned long long)sum, 63), want = limit_now(whole);
      if (sum - own < want && want <= sum) {
        s.token = lo + (int)threadIdx.x;
        s.token_weight = own;
      }
      if (threadIdx.x == 0) s.total = whole;
    }
    __syncthreads();
    if (!known) all = s.total;
    return s.token;
  }

  // The last entry that stays where entries do as long as the sum of the weights (COUNT: the number) of those before it is below
  // the limit, in two steps: the bin that it is in, among what `last` keeps,
  template <bool COUNT, class Src, class L>
  __device__ __forceinline__ Reached find_bin(const Src& src, Last last, L&& limit_of) {
    clear(!COUNT);
    src.each(0, p.vocab, [&](int i, float l) {
      const int bin = bin_of(l);
      if (bin < S::BINS - 1 && last.keeps(key_of(l), i)) {
        add(bin, COUNT ? 1 : weight(l));
        if (!COUNT) atomicAdd(&s.counts[bin], 1u);
      }
    });
    reach(limit_of);
    Reached r;
    r.bin = (int)s.found[0];
    r.limit = s.found[1];
    if (r.bin == S::BINS) return r;
    if constexpr (COUNT) {
      r.entries = (uint32_t)s.found[2];
      r.upto = (uint32_t)(limit_of(0) - r.limit) + r.entries;
    } else {
      r.entries = s.counts[r.bin];
      const int t = threadIdx.x;
      s.scan((2 * t <= r.bin ? s.counts[2 * t] : 0) + (2 * t + 1 <= r.bin ? s.counts[2 * t + 1] : 0));
      __syncthreads();
      r.upto = (uint32_t)s.total;
    }
    return r;
  }
  // and the entry in it.
  template <bool COUNT, class Src>
  __device__ __forceinline__ Last find_last(const Src& src, Last last, const Reached& r) {
    auto w = [&](float l) -> uint64_t { return COUNT ? 1 : weight(l); };
    if (r.entries <= S::FEW)
      return find_among(src, r.limit, [&](int i, float l) { return bin_of(l) == r.bin && last.keeps(key_of(l), i); }, w);
    uint32_t lo, hi;
    bin_keys(r.bin, lo, hi);
    uint64_t limit = r.limit;
    for (;;) {
      int shift = 0;
      while (((hi - lo) >> shift) >= (uint32_t)S::BINS) shift++;
      clear(true);
      src.each(0, p.vocab, [&](int i, float l) {
        const uint32_t k = key_of(l);
        if (k >= lo && k <= hi && last.keeps(k, i)) {
          add((int)((hi - k) >> shift), w(l));
          atomicAdd(&s.counts[(hi - k) >> shift], 1u);
        }
      });
      reach([&](uint64_t) { return limit; });
      const uint32_t bin = (uint32_t)s.found[0], entries = s.counts[bin];
      limit = s.found[1];
      hi -= bin << shift;
      lo = hi - lo >= (1u << shift) ? hi - ((1u << shift) - 1) : lo;
      if (entries <= S::FEW)
        return find_among(src, limit, [&](int i, float l) { const uint32_t k = key_of(l); return k >= lo && k <= hi && last.keeps(k, i); }, w);
      if (lo == hi) {  // equal logits: the number of them that stay, by rising index
        const uint64_t one = s.found[2] / entries, stay = (limit + one - 1) / one;
        uint64_t all;
        const uint32_t key = lo;
        return Last{key, by_index(src, [&](int i, float l) -> uint64_t { return key_of(l) == key && last.keeps(key, i); },
                                  [&](uint64_t) { return stay; }, all)};
      }
    }
  }
  // Of at most FEW entries in(index, logit), by comparing all with all.
  template <class Src, class In, class W>
  __device__ __forceinline__ Last find_among(const Src& src, uint64_t limit, In&& in, W&& w) {
    __syncthreads();
    if (threadIdx.x == 0) s.few = 0;
    __syncthreads();
    src.each(0, p.vocab, [&](int i, float l) {
      if (in(i, l)) {
        const uint32_t at = atomicAdd(&s.few, 1u);
        s.few_order[at] = (uint64_t)key_of(l) << 32 | (uint32_t)~i;
        s.few_weight[at] = w(l);
      }
    });
    __syncthreads();
    const int n = (int)s.few;
    if ((int)threadIdx.x < n) {
      const uint64_t me = s.few_order[threadIdx.x];
      uint64_t before = 0;
      for (int i = 0; i < n; i++) before += s.few_order[i] > me ? s.few_weight[i] : 0;
      if (before < limit && limit <= before + s.few_weight[threadIdx.x]) s.found[0] = me;
    }
    __syncthreads();
    const uint64_t got = s.found[0];
    return Last{(uint32_t)(got >> 32), (int)~(uint32_t)got};
  }

  // Copies in(index, logit) to LDS; the list's length is past LIST where they do not fit.
  template <class Src, class In>
  __device__ __forceinline__ ListSource<NT> gather(const Src& src, In&& in) {
    __syncthreads();
    if (threadIdx.x == 0) s.length = 0;
    __syncthreads();
    src.each(0, p.vocab, [&](int i, float l) {
      if (in(i, l)) {
        const uint32_t at = atomicAdd(&s.length, 1u);
        if (at < (uint32_t)S::LIST) s.list[at] = make_uint2(__float_as_uint(l), (uint32_t)i);
      }
    });
    __syncthreads();
    return ListSource<NT>{s.list, s.length};
  }

  // The entry that u falls on, among what `last` keeps.
  template <class Src>
  __device__ __forceinline__ void draw(const Src& src, Last last, float u, int64_t b) {
    uint64_t all = 0;
    const int token = by_index(
        src, [&](int i, float l) -> uint64_t { return last.keeps(key_of(l), i) ? weight.above_floor(l) : 0; },
        [&](uint64_t sum) { return min((uint64_t)((double)u * (double)sum), sum - 1) + 1; }, all);
    if (threadIdx.x == 0) {
      p.out[b] = token;
      if (p.prob) p.prob[b] = (float)((double)s.token_weight / (double)all);
    }
  }

  __device__ __forceinline__ auto number(int k) const {
    return [k](uint64_t) { return (uint64_t)k; };
  }
  __device__ __forceinline__ auto share(float top_p) const {
    return [top_p](uint64_t sum) { return (uint64_t)fmax(ceil((double)top_p * (double)sum), 1.0); };
  }

  // Filters and draw over what is in LDS.
  __device__ __forceinline__ void run_list(const ListSource<NT>& list, int k, float top_p, float u, int64_t b) {
    Last last = {NONE + 1, 0x7fffffff};
    if (k < p.vocab) {
      const Reached r = find_bin<true>(list, last, number(k));
      if (r.bin < S::BINS) last = find_last<true>(list, last, r);
    }
    if (top_p < 1.0f) {
      const Reached r = find_bin<false>(list, last, share(top_p));
      last = find_last<false>(list, last, r);
    }
    draw(list, last, u, b);
  }

  // Filters and draw.  `part`: the largest entries of the thread's parts of the row; at most `allowed` are above -inf.
  template <int PARTS_OF>
  __device__ __forceinline__ void run(const RowSource<BF16, NT>& row, const float (&part)[PARTS_OF], uint32_t allowed, int k, float top_p, float u, int64_t b) {
    Last last = {NONE + 1, 0x7fffffff};
    if (allowed <= S::LIST) return run_list(gather(row, [&](int, float l) { return l > -INFINITY; }), k, top_p, u, b);
    if (k <= PARTS_OF * NT / 2) {
      // Of the k largest parts' largest entries the smallest is no larger than the k-th entry: what lies below it need not be
      // looked at.  (Of normal logits some k to 1.4 k are left.)  Its bin's lower end, rounded down, is taken for it.
      clear(false);
#pragma unroll
      for (int a = 0; a < PARTS_OF; a++) {
        const int bin = bin_of(part[a]);
        if (bin < S::BINS - 1) add(bin, 1);
      }
      reach(number(k));
      if (s.found[0] < (uint64_t)S::BINS) {
        const float least = top - (float)(s.found[0] + 1) / step * 1.00001f - fabsf(top) * 1e-6f;
        const auto list = gather(row, [&](int, float l) { return l >= least && l > -INFINITY; });
        if (list.length <= (uint32_t)S::LIST) return run_list(list, k, top_p, u, b);
      }
    }
    if (k < p.vocab) {
      const Reached r = find_bin<true>(row, last, number(k));
      if (r.bin < S::BINS && r.upto <= S::LIST) {
        return run_list(gather(row, [&](int, float l) { return bin_of(l) <= r.bin; }), k, top_p, u, b);
      }
      if (r.bin < S::BINS) last = find_last<true>(row, last, r);
    }
    if (top_p < 1.0f) {
      const Reached r = find_bin<false>(row, last, share(top_p));
      if (r.upto <= S::LIST) {
        const auto list = gather(row, [&](int i, float l) { return bin_of(l) <= r.bin && last.keeps(key_of(l), i); });
        draw(list, find_last<false>(list, last, r), u, b);
        return;
      }
      last = find_last<false>(row, last, r);
    }
    draw(row, last, u, b);
  }
};

template <bool BF16, int NT>
__global__ __launch_bounds__(NT, 4) void az_sample_rows(SampleView p) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  Sampler<NT>& s = *reinterpret_cast<Sampler<NT>*>(smem);
  const int64_t b = blockIdx.x;
  const RowSource<BF16, NT> src = {(const uint8_t*)p.logits + b * p.ld * (BF16 ? 2 : 4), p.vocab};
  // (the row's parameters are on their way while the row is looked at)
  const float t = p.temperature ? p.temperature[b] : 1.0f, min_p = p.min_p ? p.min_p[b] : 0.0f, given_p = p.top_p ? p.top_p[b] : 1.0f, given_u = p.u[b];
  const int given_k = p.top_k ? p.top_k[b] : 0;
  float part[RowSource<BF16, NT>::AHEAD], top = -INFINITY;
  bool bad;
  uint32_t groups;
  src.look(part, bad, groups);
#pragma unroll
  for (int a = 0; a < src.AHEAD; a++) top = fmaxf(top, part[a]);
  for (int o = 32; o > 0; o >>= 1) {
    top = fmaxf(top, __shfl_xor(top, o));
    groups += __shfl_xor(groups, o);
  }
  bad = __any(bad);
  if ((threadIdx.x & 63) == 0) {
    s.wave_top[threadIdx.x >> 6] = top;
    s.wave_groups[threadIdx.x >> 6] = groups;
    s.wave_bad[threadIdx.x >> 6] = bad;
  }
  if (threadIdx.x < PARTS) {
    const double f = (double)threadIdx.x / PARTS;
    s.table[threadIdx.x] = f < 0.5 ? power_of_two(f) : 2.0 * power_of_two(f - 1.0);
  }
  __syncthreads();
  groups = 0;
  for (int w = 0; w < NT / 64; w++) {
    top = fmaxf(top, s.wave_top[w]);
    groups += s.wave_groups[w];
    bad |= s.wave_bad[w] != 0;
  }
  if (bad || top == -INFINITY) {
    if (threadIdx.x == 0) {
      p.out[b] = -1;
      if (p.prob) p.prob[b] = 0.0f;
    }
    return;
  }
  const bool greedy = !(t > 0.0f);
  const float step = greedy ? 1.0f : fminf((float)Sampler<NT>::BINS / REACH / t, 0x1p100f);
  const float floor = min_p > 0.0f ? fminf(min_p, 1.0f) : 0.0f;
  Row<BF16, NT> row = {s, p, {(double)top, greedy ? 1.0 : 46.166241308446828 / (double)t, ldexp((double)floor, p.shift), s.table, p.shift},
                       top, step, key_of(top)};
  if (greedy) {
    uint64_t all;
    const int token = row.by_index(src, [&](int, float l) -> uint64_t { return l == top; }, row.number(1), all);
    if (threadIdx.x == 0) {
      p.out[b] = token;
      if (p.prob) p.prob[b] = 1.0f;
    }
    return;
  }
  const int k = given_k <= 0 || given_k > p.vocab ? p.vocab : given_k;
  row.run(src, part, groups < 0x10000000u ? groups * 8 : ~0u, k, given_p < 1.0f ? given_p : 1.0f, given_u > 0.0f ? fminf(given_u, 1.0f) : 0.0f, b);
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
  // Few rows: as many threads as take the row eight entries each (64 x 4672 with top-p: 15.4 us, 22.2 with 256).  Rows for every
  // compute unit: smaller workgroups, of which two overlap (512 x 131072, an earlier form: 85 us, 94 with 1,024).
  const int nt = in->rows > 256 ? (in->vocab <= 8192 ? 256 : 512) : in->vocab <= 2048 ? 256 : in->vocab <= 4096 ? 512 : 1024;
  if (nt == 256) return launched(who, in->dtype == AZ_BF16 ? launch<true, 256>(p, s) : launch<false, 256>(p, s));
  if (nt == 512) return launched(who, in->dtype == AZ_BF16 ? launch<true, 512>(p, s) : launch<false, 512>(p, s));
  return launched(who, in->dtype == AZ_BF16 ? launch<true, 1024>(p, s) : launch<false, 1024>(p, s));
}
