// tq_sample: the next token of each row of logits, by temperature, top-k, top-p and
// min-p, from given exponential random numbers.
//
//   w_v = e^((x_v - max x) / T);   kept: a prefix of the order (x descending, then v
//   ascending): the first k; of those the ones with less than p of their weight in front
//   of them; of those the ones with w >= min-p;   token = argmax of w_v / noise_v
//
// A setting ends the prefix at a cut (value, token).  It is found without sorting the
// row: a histogram over 2,048 equal steps of x (counts and weights as integers, so that
// no order of additions changes them) says in which step the cut lies; the step's
// tokens, if they are at most 2,048, are sorted in shared memory; if they are more, the
// step is cut into 2,048 again; if they all have one value, the tokens in front of the
// cut are counted in their own order.  For small k the largest values of the block's
// threads bound the k-th value from below, and what lies above that bound is sorted at
// once, cut, and raced.
//
// Quotients are taken in float32; those within 2^-18 of the largest are compared again
// in 64 bits, so that the token is that of exact arithmetic.
#include <algorithm>

#include "tq_kv.cuh"
#include "tq_sample.h"
#include "tq_topk.cuh"

namespace tq {
namespace {

constexpr int BINS = 2048, LIST = 2048;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float FIXED = 549755813888.0f;  // 2^39: weights as integers; 2^24 of them fit 63 bits

struct SampleArgs {
  const void* logits;
  int64_t logits_stride;
  const float* noise;
  int64_t noise_stride;
  int vocab;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int32_t* tokens;
  float* logprobs;
};

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A logit: NaN counts as -inf, +inf as the largest float; -0 as 0.
__device__ __forceinline__ float logit(float x) { return fminf(fmaxf(x, -INFINITY), 3.402823466e38f) + 0.0f; }

// Floats as unsigned integers in their order.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
// A token's place in the order: larger comes first.
__device__ __forceinline__ uint64_t place_of(float x, int v) { return (uint64_t)ordered(x) << 32 | (uint32_t)~v; }
__device__ __forceinline__ int token_of(uint64_t place) { return (int)~(uint32_t)place; }
__device__ __forceinline__ float value_of(uint64_t place) { return unordered((uint32_t)(place >> 32)); }

// Weight of a value: 2^((x - top) * (c_hi + c_lo)), about 2^-22 off; 0 below 2^-126 (and
// for masked values, whatever the temperature).
struct Weigh {
  float top, hi, lo;
  __device__ __forceinline__ float operator()(float x) const {
    const float t = x - top, h = t * hi;
    const float l = fmaf(t, lo, fmaf(t, hi, -h));
    return h > -126.0f ? ex2f(h) * fmaf(l, LN2, 1.0f) : 0.0f;
  }
};
__device__ __forceinline__ Weigh weigh_of(float top, float temperature) {
  constexpr float LOG2E_LO = (float)(1.4426950408889634 - (double)LOG2E);
  Weigh w;
  w.top = top;
  w.hi = LOG2E / temperature;
  w.lo = (fmaf(-w.hi, temperature, LOG2E) + LOG2E_LO) / temperature;
  if (!(w.hi < 1e30f)) w.hi = 1e30f, w.lo = 0.0f;  // (only equals of the largest weigh anything)
  if (!(fabsf(w.lo) < 1e30f)) w.lo = 0.0f;
  return w;
}
__device__ __forceinline__ uint64_t fixed(float w) { return __float2ull_rn(w * FIXED); }

// The least integer that is not below p * x, for p in (0, 1) and x below 2^63 (p to 2^-32):
// 1 at least.
__device__ __forceinline__ uint64_t part_of(float p, uint64_t x) {
  const uint64_t m = (uint64_t)(uint32_t)__float2uint_rn(p * 4294967296.0f) << 32;
  return max(1ull, (unsigned long long)(__umul64hi(x, m) + (x * m != 0)));
}
// Logarithm of x / 2^39, x > 0: about 2^-25 off.
__device__ __forceinline__ double log_fixed(uint64_t x) {
  const int e = 63 - __clzll((long long)x);
  const float m = (float)(x << (63 - e)) * 0x1p-63f;  // in [1, 2]
  return (double)(e - 39) * 0.6931471805599453 + (double)logf(m);
}

// A row's elements by 16-byte pieces of memory, E of them at a time; the row may begin
// and end within a piece.
template <typename T>
struct Row {
  static constexpr int E = 16 / (int)sizeof(T);
  static constexpr bool ANY_ORDER = false;
  const T* p;
  int n, lead;  // elements of the first piece that lie in front of the row
  __device__ __forceinline__ Row(const void* base, int64_t stride, int64_t row, int vocab) {
    p = static_cast<const T*>(base) + row * stride;
    n = vocab;
    lead = (int)(((uintptr_t)p & 15) / sizeof(T));
  }
  __device__ __forceinline__ int pieces() const { return (n + lead + E - 1) / E; }
  // Elements of piece g; returns the token of the first (which may be below 0).
  __device__ __forceinline__ int load(int g, float (&x)[E]) const {
    const int v = g * E - lead;
    if (v >= 0 && v + E <= n) {
      union {
        uint4 u;
        T e[E];
      } in;
      in.u = *reinterpret_cast<const uint4*>(p + v);
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = logit(to_float(in.e[i]));
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = v + i >= 0 && v + i < n ? logit(to_float(p[v + i])) : -INFINITY;
    }
    return v;
  }
};

// Places in memory, one at a time, in any order.
struct Places {
  static constexpr int E = 1;
  static constexpr bool ANY_ORDER = true;
  const uint64_t* p;
  int n;
  __device__ __forceinline__ int pieces() const { return n; }
  __device__ __forceinline__ int load(int g, float (&x)[1]) const {
    const uint64_t place = __ldcg(p + g);
    x[0] = value_of(place);
    return token_of(place);
  }
};

// Sums and extremes over the block; every thread gets the result.
struct Scratch {
  uint64_t words[32];
};
template <int N, typename F>
__device__ __forceinline__ uint64_t block_reduce(uint64_t x, Scratch& s, F join) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = join(x, __shfl_xor_sync(FULL, x, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.words[threadIdx.x >> 5] = x;
  __syncthreads();
  x = s.words[threadIdx.x & (N / 32 - 1)];
#pragma unroll
  for (int o = N / 64; o; o >>= 1) x = join(x, __shfl_xor_sync(FULL, x, o));
  return x;
}
template <int N>
__device__ __forceinline__ uint64_t block_max(uint64_t x, Scratch& s) {
  return block_reduce<N>(x, s, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}
template <int N>
__device__ __forceinline__ uint64_t block_sum(uint64_t x, Scratch& s) {
  return block_reduce<N>(x, s, [](uint64_t a, uint64_t b) { return a + b; });
}
// Sum of the threads in front (exclusive), and of all.
template <int N>
__device__ __forceinline__ uint64_t block_scan(uint64_t x, Scratch& s, uint64_t& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t upto = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(FULL, upto, o);
    if (lane >= o) upto += y;
  }
  __syncthreads();
  if (lane == 31) s.words[warp] = upto;
  __syncthreads();
  const uint64_t w = lane < N / 32 ? s.words[lane] : 0;
  uint64_t wup = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(FULL, wup, o);
    if (lane >= o) wup += y;
  }
  all = __shfl_sync(FULL, wup, 31);
  return upto - x + __shfl_sync(FULL, wup - w, warp);
}

struct Shared {
  uint64_t list[LIST];          // places
  uint32_t bins[BINS];
  Scratch scratch;
  int listed, bin;
  uint32_t low, high;           // extremes of a step's values, ordered
  uint64_t cut, taken;          // results of a search
  int candidates;
};

// Sorts the first n (at most LIST) places of the list, largest first; n is padded to a
// power of two with zeros.
template <int N>
__device__ void sort_list(Shared& sh, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += N) sh.list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j; j >>= 1) {
      for (int t = threadIdx.x; t < size / 2; t += N) {
        const int a = 2 * t - (t & (j - 1)), b = a + j;
        const uint64_t x = sh.list[a], y = sh.list[b];
        if ((x < y) == ((a & k) == 0)) {
          sh.list[a] = y;
          sh.list[b] = x;
        }
      }
      __syncthreads();
    }
}

// The cut of a prefix of the kept tokens: the first `want` of them (by count), or those with
// less than `want` of the weight (in fixed point) in front of them.  The prefix has one
// token at least; `want` is less than what all of them have.
// front: what of them lies above `high`.  0 where more than LIST tokens of a list have one value.
template <int N, bool BY_COUNT, typename Source>
__device__ uint64_t find_cut(const Source& row, const Weigh& weigh, uint64_t kept, uint64_t front, uint64_t want,
                             float scale, float low, float high, Shared& sh) {
  constexpr int E = Source::E;
  for (int level = 0;; ++level) {
    // a histogram of the tokens with low <= x <= high: equal steps of x, then of x as an
    // ordered integer, so that every further level parts the smallest from the largest
    const float step = high > low ? (BINS - 1) / (high - low) : 0.0f;
    const uint32_t low_u = ordered(low), high_u = ordered(high);
    const int shift = max(0, 32 - __clz(high_u - low_u) - 11);  // (2^11 bins)
    auto bin_of = [&](float x) {
      return level ? (int)((high_u - ordered(x)) >> shift) : (int)fminf((high - x) * step, (float)(BINS - 1));
    };
    for (int i = threadIdx.x; i < BINS; i += N) sh.bins[i] = 0;
    __syncthreads();
    for (int g = threadIdx.x; g < row.pieces(); g += N) {
      float x[E];
      const int v = row.load(g, x);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] >= low && x[i] <= high && place_of(x[i], v + i) >= kept) {
          if (BY_COUNT)
            atomicAdd(&sh.bins[bin_of(x[i])], 1u);
          else
            atomicAdd(&sh.bins[bin_of(x[i])], __float2uint_rn(weigh(x[i]) * scale));
        }
    }
    __syncthreads();
    // the first bin that reaches what is wanted
    const uint64_t rest = want > front ? want - front : 0;
    const uint64_t need = BY_COUNT ? rest : (uint64_t)((float)rest * (scale / FIXED));
    uint64_t mine = 0, all;
#pragma unroll
    for (int i = 0; i < BINS / N; ++i) {
      const int b = threadIdx.x * (BINS / N) + i;
      mine += sh.bins[b];
    }
    if (threadIdx.x == 0) sh.bin = -1;
    uint64_t upto = block_scan<N>(mine, sh.scratch, all);
#pragma unroll
    for (int i = 0; i < BINS / N; ++i) {
      const int b = threadIdx.x * (BINS / N) + i;
      const uint64_t here = sh.bins[b];
      if (here && upto < need && upto + here >= need) sh.bin = b;
      upto += here;
    }
    __syncthreads();
    int bin = sh.bin;
    if (bin < 0) {  // (rounded weights fall short, or nothing is needed): the last bin that has any, or the first
      int last = -1, first = BINS;
      for (int i = threadIdx.x; i < BINS; i += N)
        if (sh.bins[i]) last = max(last, i), first = min(first, i);
      last = (int)block_max<N>((uint64_t)(last + 1), sh.scratch) - 1;
      first = BINS - (int)block_max<N>((uint64_t)(BINS - first), sh.scratch);
      bin = need ? max(last, 0) : first < BINS ? first : 0;
    }
    // its tokens to the list, their extremes; exactly what lies in front of them
    if (threadIdx.x == 0) {
      sh.listed = 0;
      sh.low = 0xffffffffu;
      sh.high = 0;
    }
    __syncthreads();
    uint64_t above = 0;
    uint32_t lo = 0xffffffffu, hi = 0;
    for (int g = threadIdx.x; g < row.pieces(); g += N) {
      float x[E];
      const int v = row.load(g, x);
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] >= low && x[i] <= high && place_of(x[i], v + i) >= kept) {
          const int b = bin_of(x[i]);
          if (b < bin) {
            if (BY_COUNT)
              ++above;
            else
              sum += weigh(x[i]);
          } else if (b == bin) {
            const int at = atomicAdd(&sh.listed, 1);
            if (at < LIST) sh.list[at] = place_of(x[i], v + i);
            lo = min(lo, ordered(x[i]));
            hi = max(hi, ordered(x[i]));
          }
        }
      if (!BY_COUNT) above += fixed(sum);
    }
    if (lo <= hi) {
      atomicMin(&sh.low, lo);
      atomicMax(&sh.high, hi);
    }
    front += block_sum<N>(above, sh.scratch);
    const int listed = sh.listed;
    if (listed == 0) return kept;  // (nothing is kept at all)
    low = unordered(sh.low);
    high = unordered(sh.high);
    if (listed <= LIST) {
      // sorted: the last of them with too little in front of it
      sort_list<N>(sh, listed);
      if (threadIdx.x == 0) sh.cut = sh.list[0];
      uint64_t here[LIST / N], sum = 0;
#pragma unroll
      for (int i = 0; i < LIST / N; ++i) {
        const int at = threadIdx.x * (LIST / N) + i;
        here[i] = at < listed ? (BY_COUNT ? 1 : fixed(weigh(value_of(sh.list[at])))) : 0;
        sum += here[i];
      }
      uint64_t before = front + block_scan<N>(sum, sh.scratch, all);
#pragma unroll
      for (int i = 0; i < LIST / N; ++i) {
        const int at = threadIdx.x * (LIST / N) + i;
        if (at < listed && before < want && (before + here[i] >= want || at == listed - 1)) sh.cut = sh.list[at];
        before += here[i];
      }
      __syncthreads();
      const uint64_t cut = sh.cut;
      __syncthreads();
      return cut;
    }
    if (low == high && Source::ANY_ORDER) return 0;
    if (low == high) {
      // one value: all weigh the same; the first of them in their own order.  A warp takes
      // a run of pieces.
      const uint64_t each = BY_COUNT ? 1 : max((unsigned long long)fixed(weigh(low)), 1ull);
      uint64_t take = want > front ? (want - front + each - 1) / each : 1;
      if (take > (uint64_t)listed) take = listed;
      const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
      const int run = (row.pieces() + (N / 32) - 1) / (N / 32), begin = warp * run, end = min(row.pieces(), begin + run);
      auto equal = [&](int g, int& v) {  // bits of the piece's tokens with that value
        float x[E];
        unsigned bits = 0;
        if (g >= end) return bits;
        v = row.load(g, x);
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (x[i] == low && v + i >= 0 && v + i < row.n && place_of(x[i], v + i) >= kept) bits |= 1u << i;
        return bits;
      };
      int v = 0, some = 0;
      for (int g = begin + lane; g < end; g += 32) some += __popc(equal(g, v));
#pragma unroll
      for (int o = 16; o; o >>= 1) some += __shfl_xor_sync(FULL, some, o);
      uint64_t before = block_scan<N>(lane == 0 ? some : 0, sh.scratch, all);
      before = __shfl_sync(FULL, before, 0);
      if (before < take && before + some >= take) {
        int left = (int)(take - before);
        for (int g0 = begin; g0 < end && left > 0; g0 += 32) {
          unsigned bits = equal(g0 + lane, v);
          int upto = __popc(bits);
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(FULL, upto, o);
            if (lane >= o) upto += y;
          }
          const int front_of = upto - __popc(bits);
          if (left > front_of && left <= upto) {
            for (int skip = left - front_of - 1; skip; --skip) bits &= bits - 1;
            sh.cut = place_of(low, v + __ffs(bits) - 1);
          }
          left -= __shfl_sync(FULL, upto, 31);
        }
      }
      __syncthreads();
      const uint64_t cut = sh.cut;
      __syncthreads();
      return cut;
    }
  }
}

// The race among kept tokens: quotients in float32, those next to the best in 64 bits.
constexpr float NEAR = 1.0f - 0x1p-18f;

struct Setting {
  float temperature, top_p, min_p;
  int k;        // vocab: all
  bool hot;     // else the first token alone
};
__device__ __forceinline__ Setting setting_of(const SampleArgs& a, int64_t r) {
  Setting s;
  s.temperature = a.temperature ? a.temperature[r] : 1.0f;
  s.top_p = a.top_p ? a.top_p[r] : 1.0f;
  s.min_p = a.min_p ? a.min_p[r] : 0.0f;
  const int k = a.top_k ? a.top_k[r] : 0;
  s.k = k > 0 && k < a.vocab ? k : a.vocab;
  s.hot = s.temperature > 0.0f && s.min_p <= 1.0f && s.top_p > 0.0f;
  return s;
}

struct Race {
  const Setting& s;
  const Weigh& weigh;
  const float* noise;
  uint64_t first;        // the place that is always kept
  float best = 0.0f;
  uint64_t winner = 0;   // 0: none yet

  // (no quotient is negative, NaN or infinite, whatever the noise)
  static __device__ __forceinline__ float number(float e) { return fmaxf(e, 0x1p-126f); }
  __device__ __forceinline__ double weight(float x) const {
    return exp(((double)x - (double)weigh.top) / (double)s.temperature);
  }
  __device__ __forceinline__ double quotient(uint64_t place) const {
    return weight(value_of(place)) / (double)number(noise[token_of(place)]);
  }
  // The better of two in 64 bits.
  __device__ __noinline__ uint64_t better(uint64_t a, uint64_t b) const {
    const double x = quotient(a), y = quotient(b);
    return x > y || (x == y && token_of(a) < token_of(b)) ? a : b;
  }
  __device__ __forceinline__ void enter(float x, int v) { enter(x, v, weigh(x)); }
  __device__ __forceinline__ void enter(float x, int v, float w) { enter(x, v, w, noise[v]); }
  __device__ __forceinline__ void enter(float x, int v, float w, float e) {
    const uint64_t place = place_of(x, v);
    if (w < s.min_p * (1.0f + 0x1p-18f) || w == 0.0f) {  // (next to the border: in 64 bits)
      if (place != first && (w < s.min_p * (1.0f - 0x1p-18f) || w == 0.0f || weight(x) < (double)s.min_p)) return;
    }
    const float q = w / number(e);
    if (winner) {
      if (!(q >= best * NEAR)) return;
      if (q * NEAR <= best && better(place, winner) == winner) return;
    }
    best = q;
    winner = place;
  }
};

// The best of a block's racers, in every thread; by the whole block.
template <int N>
__device__ uint64_t block_winner(const Race& race, Shared& sh, float& best) {
  const uint64_t key = race.winner ? (uint64_t)__float_as_uint(race.best) + 1 : 0;
  const uint64_t most = block_max<N>(key, sh.scratch);
  best = 0.0f;
  if (most == 0) return 0;
  best = __uint_as_float((uint32_t)(most - 1));
  if (threadIdx.x == 0) sh.candidates = 0;
  __syncthreads();
  if (race.winner && !(race.best < best * NEAR)) sh.list[atomicAdd(&sh.candidates, 1)] = race.winner;  // (at most N)
  __syncthreads();
  if (threadIdx.x == 0) {
    uint64_t w = sh.list[0];
    for (int i = 1; i < sh.candidates; ++i) w = race.better(w, sh.list[i]);
    sh.cut = w;
  }
  __syncthreads();
  return sh.cut;
}

__device__ __forceinline__ void finish(const SampleArgs& a, int64_t r, uint64_t place, float top, uint64_t sum1) {
  a.tokens[r] = place ? token_of(place) : 0;
  if (a.logprobs) a.logprobs[r] = place ? (float)((double)value_of(place) - (double)top - log_fixed(sum1)) : -INFINITY;
}

// The n places of the list, sorted: how many of them the settings keep.
template <int N>
__device__ int cut_list(const Setting& s, const Weigh& weigh, int n, Shared& sh) {
  n = min(n, s.k);
  if (!(s.top_p < 1.0f)) return n;
  uint64_t here[LIST / N], part = 0, sum;
#pragma unroll
  for (int i = 0; i < LIST / N; ++i) {
    const int e = threadIdx.x * (LIST / N) + i;
    here[i] = e < n ? fixed(weigh(value_of(sh.list[e]))) : 0;
    part += here[i];
  }
  uint64_t before = block_scan<N>(part, sh.scratch, sum);
  const uint64_t want = part_of(s.top_p, sum);
  int count = 0;
#pragma unroll
  for (int i = 0; i < LIST / N; ++i) {
    const int e = threadIdx.x * (LIST / N) + i;
    if (e < n && (e == 0 || before < want)) ++count;
    before += here[i];
  }
  return (int)block_sum<N>((uint64_t)count, sh.scratch);
}

// What tokens below are too light: together less than the part that top-p leaves out.
__device__ __forceinline__ float least_value(const Setting& s, float top, uint64_t sum, int vocab) {
  const float least = (1.0f - s.top_p) * ((float)sum / FIXED) / (float)vocab;
  return fmaxf(top + logf(least) * s.temperature * 1.0001f - 1e-3f, -3.0e38f);
}

// A row by one block of N threads, whatever its settings.
template <int N, typename T>
__device__ __noinline__ void whole_row(const SampleArgs& a, int64_t r, Shared& sh) {
  constexpr int E = Row<T>::E;
  const Row<T> row(a.logits, a.logits_stride, r, a.vocab);
  const Setting s = setting_of(a, r);

  // ---- the largest value and its lowest token, the sums of e^(x - max) at both temperatures
  float top = -INFINITY;
  int at = a.vocab;
  for (int g = threadIdx.x; g < row.pieces(); g += N) {
    float x[E];
    const int v = row.load(g, x);
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (x[i] > top) {
        top = x[i];
        at = v + i;
      }
  }
  const uint32_t mine = ordered(top);  // (of this thread's tokens)
  const uint64_t first = block_max<N>(at < a.vocab ? place_of(top, at) : 0, sh.scratch);
  if (first == 0) {  // nothing but -inf
    if (threadIdx.x == 0) finish(a, r, 0, 0.0f, 0);
    return;
  }
  top = value_of(first);
  const Weigh plain = weigh_of(top, 1.0f), weigh = weigh_of(top, s.hot ? s.temperature : 1.0f);
  uint64_t sum1 = 0, sum = 0;
  for (int g = threadIdx.x; g < row.pieces(); g += N) {
    float x[E], y1 = 0.0f, y = 0.0f;
    row.load(g, x);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      y1 += plain(x[i]);
      y += weigh(x[i]);
    }
    sum1 += fixed(y1);
    sum += fixed(y);
  }
  sum1 = block_sum<N>(sum1, sh.scratch);
  sum = block_sum<N>(sum, sh.scratch);
  if (!s.hot) {
    if (threadIdx.x == 0) finish(a, r, first, top, sum1);
    return;
  }

  // ---- what is kept
  uint64_t kept = place_of(-INFINITY, a.vocab);  // every token that is not masked
  bool listed = false;  // the kept tokens lie in the list
  int n = 0;
  if (s.k < a.vocab) {
    if (s.k <= N / 2) {
      // the k-th largest of the threads' own largest values: at least k tokens reach it
      if (threadIdx.x == 0) sh.listed = 0;
      sh.list[threadIdx.x] = (uint64_t)mine << 32 | threadIdx.x;
      sort_list<N>(sh, N);
      const float bound = unordered((uint32_t)(sh.list[s.k - 1] >> 32));
      __syncthreads();
      if (bound > -INFINITY) {
        for (int g = threadIdx.x; g < row.pieces(); g += N) {
          float x[E];
          const int v = row.load(g, x);
#pragma unroll
          for (int i = 0; i < E; ++i)
            if (x[i] >= bound) {
              const int to = atomicAdd(&sh.listed, 1);
              if (to < LIST) sh.list[to] = place_of(x[i], v + i);
            }
        }
        __syncthreads();
        n = sh.listed;
        listed = n <= LIST;
      }
      __syncthreads();
    }
    if (listed) {
      sort_list<N>(sh, n);
      n = cut_list<N>(s, weigh, n, sh);
    } else {
      // more of them: by counts, from the smallest value that is not masked
      uint64_t count = 0;
      uint32_t lo = 0xffffffffu;
      for (int g = threadIdx.x; g < row.pieces(); g += N) {
        float x[E];
        row.load(g, x);
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (x[i] > -INFINITY) {
            ++count;
            lo = min(lo, ordered(x[i]));
          }
      }
      count = block_sum<N>(count, sh.scratch);
      lo = ~(uint32_t)block_max<N>((uint64_t)~lo, sh.scratch);
      if (count > (uint64_t)s.k) {
        kept = find_cut<N, true>(row, weigh, kept, 0, s.k, 0.0f, unordered(lo), top, sh);
        uint64_t part = 0;
        for (int g = threadIdx.x; g < row.pieces(); g += N) {
          float x[E], y = 0.0f;
          const int v = row.load(g, x);
#pragma unroll
          for (int i = 0; i < E; ++i) y += place_of(x[i], v + i) >= kept ? weigh(x[i]) : 0.0f;
          part += fixed(y);
        }
        sum = block_sum<N>(part, sh.scratch);
      }
    }
  }
  if (!listed && s.top_p < 1.0f) {
    const uint64_t want = part_of(s.top_p, sum);
    if (want < sum) {
      const uint64_t cut = find_cut<N, false>(row, weigh, kept, 0, want, 0x1p31f / ((float)sum / FIXED),
                                              least_value(s, top, sum, a.vocab), top, sh);
      kept = cut > kept ? cut : kept;
    }
  }

  // ---- the race
  Race race = {s, weigh, a.noise + r * a.noise_stride, first};
  if (listed) {
    for (int i = threadIdx.x; i < n; i += N) race.enter(value_of(sh.list[i]), token_of(sh.list[i]));
  } else {
    for (int g = threadIdx.x; g < row.pieces(); g += N) {
      float x[E];
      const int v = row.load(g, x);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] > -INFINITY && place_of(x[i], v + i) >= kept) race.enter(x[i], v + i);
    }
  }
  float best;
  const uint64_t winner = block_winner<N>(race, sh, best);
  if (threadIdx.x == 0) finish(a, r, winner, top, sum1);
}

template <int N, typename T>
__global__ __launch_bounds__(N) void k_sample_row(SampleArgs a) {
  __shared__ Shared sh;
  whole_row<N, T>(a, blockIdx.x, sh);
}

// ---- a row by several blocks ------------------------------------------------
//
// k_sample_parts: a block per PART tokens, read once: its largest, its sums, and what
// tells where the row's cut lies: the largest of every 64 tokens (small k), or the
// weights of 1,024 steps of 1/32 of x / T (top-p; steps at fixed places, so that parts
// which do not know of one another's largest add up).  The row's last block says which
// step or bound that is.
// k_sample_race: the same blocks again: what lies above the step races at once and is
// summed, what lies in it (or above the bound) goes to the row's list, which its last
// block cuts and races, and joins with the parts' winners.  A list that is too long, and
// what fits neither form (large k), is left to whole_row there.
constexpr int SPLIT = 256, EACH = 16, PART = SPLIT * EACH;
constexpr int GROUP = 64, GROUPS = PART / GROUP;
constexpr int STEPS = 1024;            // of 1/32: weights down to e^-32 of a part's largest
constexpr float STEP_ONE = 524288.0f;  // weight at a step's upper end, as an integer: PART of them fit
constexpr int MOST_K = 512, MOST_LISTED = 4096, MOST_PARTS = 128;
constexpr int MOST_ROWS = 512, MOST_BLOCKS = 16384;  // of a launch: what the workspace is for

enum class Mode : int { DONE, ALONE, BOUND, CUT };

struct RowRecord {
  // zero at the start
  unsigned arrived, raced, listed;
  unsigned unused;
  uint64_t above;       // weight above the step
  // from the first kernel's last block
  uint64_t first, sum1, sum;
  Mode mode;
  float bound;          // BOUND
  int step;             // CUT: the list's step; what lies above it is kept, what lies below is not
  int unused2;
};
struct PartRecord {
  uint64_t first;
  float sum1, sum;
};
struct PartWinner {
  uint64_t place;
  float best;
};

struct SplitArgs {
  SampleArgs a;
  int64_t row0;
  int parts;
  RowRecord* rows;
  PartRecord* part;
  PartWinner* winner;
  float* groups;     // [blocks][GROUPS]
  uint32_t* steps;   // [blocks][STEPS]
  uint64_t* list;    // [rows][MOST_LISTED]
};

// Step of x: floor(32 x / T), which grows with x.
__device__ __forceinline__ float steps_per(float temperature) { return fminf(32.0f / temperature, 1e30f); }
__device__ __forceinline__ int step_of(float x, float per) { return (int)floorf(fminf(fmaxf(x * per, -1e9f), 1e9f)); }
// Steps of b below a (no less than -1: they may be 2^31 apart).
__device__ __forceinline__ int steps_below(int a, int b) { return (int)max(-1ll, min((long long)STEPS, (long long)a - b)); }

template <typename T>
__device__ __forceinline__ void load_part(const Row<T>& row, int part, float (&x)[EACH], int (&v)[EACH / Row<T>::E]) {
  constexpr int E = Row<T>::E;
#pragma unroll
  for (int j = 0; j < EACH / E; ++j) {
    float y[E];
    const int g = part * (PART / E) + j * SPLIT + threadIdx.x;
    v[j] = g * E - row.lead;
    if (g < row.pieces()) {
      row.load(g, y);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) x[j * E + i] = y[i];
  }
}

__device__ __forceinline__ float block_sum(float x, Scratch& s) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.words[threadIdx.x >> 5] = __float_as_uint(x);
  __syncthreads();
  x = __uint_as_float((uint32_t)s.words[threadIdx.x & (SPLIT / 32 - 1)]);
#pragma unroll
  for (int o = SPLIT / 64; o; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
  return x;
}

// True in every thread of the block that arrives last of `parts`; what the others wrote
// in front of it is then visible.
__device__ __forceinline__ bool last_of(unsigned* counter, int parts, Shared& sh) {
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    sh.bin = (int)atomicAdd(counter, 1u) == parts - 1;
    __threadfence();
  }
  __syncthreads();
  return sh.bin;
}

// The row's record, by the last block of k_sample_parts.
template <typename T>
__device__ void settle_row(const SplitArgs& q, int64_t r, RowRecord& rec, Shared& sh) {
  const SampleArgs& a = q.a;
  const Setting s = setting_of(a, r);
  const PartRecord* part = q.part + blockIdx.y * (int64_t)q.parts;
  const int t = threadIdx.x;
  PartRecord mine = {0, 0.0f, 0.0f};  // (parts <= threads)
  if (t < q.parts) {
    mine.first = __ldcg(&part[t].first);
    mine.sum1 = __ldcg(&part[t].sum1);
    mine.sum = __ldcg(&part[t].sum);
  }
  const uint64_t first = block_max<SPLIT>(mine.first, sh.scratch);
  if (first == 0) {
    if (t == 0) {
      finish(a, r, 0, 0.0f, 0);
      rec.mode = Mode::DONE;
    }
    return;
  }
  const float top = value_of(first), m = value_of(mine.first);
  const Weigh plain = weigh_of(top, 1.0f), weigh = weigh_of(top, s.hot ? s.temperature : 1.0f);
  const uint64_t sum1 = block_sum<SPLIT>(mine.first ? fixed(mine.sum1 * plain(m)) : 0, sh.scratch);
  const uint64_t sum = block_sum<SPLIT>(mine.first ? fixed(mine.sum * weigh(m)) : 0, sh.scratch);
  Mode mode = Mode::DONE;
  float bound = -INFINITY;
  int step = -2000000000;
  if (!s.hot) {
    if (t == 0) finish(a, r, first, top, sum1);
  } else if (s.k < a.vocab) {
    mode = Mode::ALONE;
    if (s.k <= MOST_K) {
      // the least value that k groups reach, by a histogram of their largest
      const float* groups = q.groups + blockIdx.y * (int64_t)q.parts * GROUPS;
      const int n = q.parts * GROUPS;
      uint32_t lo = 0xffffffffu;
      for (int i = t; i < n; i += SPLIT) {
        const float x = __ldcg(groups + i);
        if (x > -INFINITY) lo = min(lo, ordered(x));
      }
      const float low = unordered(~(uint32_t)block_max<SPLIT>((uint64_t)~lo, sh.scratch));
      const float per = top > low ? (BINS - 1) / (top - low) : 0.0f;
      for (int i = t; i < BINS; i += SPLIT) sh.bins[i] = 0;
      if (t == 0) sh.listed = -1;
      __syncthreads();
      auto bin_of = [&](float x) { return (int)fminf((top - x) * per, (float)(BINS - 1)); };
      for (int i = t; i < n; i += SPLIT) {
        const float x = __ldcg(groups + i);
        if (x > -INFINITY) atomicAdd(&sh.bins[bin_of(x)], 1u);
      }
      __syncthreads();
      uint64_t some = 0, all;
#pragma unroll
      for (int i = 0; i < BINS / SPLIT; ++i) some += sh.bins[t * (BINS / SPLIT) + i];
      uint64_t upto = block_scan<SPLIT>(some, sh.scratch, all);
#pragma unroll
      for (int i = 0; i < BINS / SPLIT; ++i) {
        const unsigned here = sh.bins[t * (BINS / SPLIT) + i];
        if (upto < (uint64_t)s.k && upto + here >= (uint64_t)s.k) sh.listed = t * (BINS / SPLIT) + i;
        upto += here;
      }
      __syncthreads();
      const int bin = sh.listed;
      if (bin >= 0) {  // (else fewer groups than k)
        uint32_t least = 0xffffffffu;
        for (int i = t; i < n; i += SPLIT) {
          const float x = __ldcg(groups + i);
          if (x > -INFINITY && bin_of(x) <= bin) least = min(least, ordered(x));
        }
        bound = unordered(~(uint32_t)block_max<SPLIT>((uint64_t)~least, sh.scratch));
        mode = Mode::BOUND;
      }
    }
  } else if (s.top_p < 1.0f && !(fabsf(top) * steps_per(s.temperature) < 1e6f)) {
    mode = Mode::ALONE;  // (float32 holds too few bits behind a step's number)
  } else {
    mode = Mode::CUT;
    if (s.top_p < 1.0f) {
      // the steps' weights from the row's largest down, 4 of them a thread, relative to that
      const float per = steps_per(s.temperature);
      const int highest = step_of(top, per), at = t * (STEPS / SPLIT);
      uint64_t w[STEPS / SPLIT] = {0, 0, 0, 0};
      static_assert(STEPS / SPLIT == 4, "steps of a thread");
      if (t < q.parts) sh.bins[t] = mine.first ? steps_below(highest, step_of(m, per)) : STEPS;
      __syncthreads();
      const uint32_t* steps = q.steps + blockIdx.y * (int64_t)q.parts * STEPS;
#pragma unroll 4
      for (int p = 0; p < q.parts; ++p) {
        const int from = at - (int)sh.bins[p];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (from + i >= 0) w[i] += __ldcg(steps + (int64_t)p * STEPS + from + i);
      }
      uint64_t some = 0, all;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // weight at the step's upper end; at most 1 in the largest's own step, up to rounding
        const float up = ((float)(highest - at - i + 1) - top * per) * (1.0f / 32.0f);
        w[i] = (uint64_t)((float)w[i] * (FIXED / STEP_ONE) * ex2f(fminf(up * LOG2E, 1.0f)));
        some += w[i];
      }
      const uint64_t want = part_of(s.top_p, sum);
      if (t == 0) sh.listed = -1;
      uint64_t upto = block_scan<SPLIT>(some, sh.scratch, all);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (w[i] && upto < want && upto + w[i] >= want) sh.listed = at + i;
        upto += w[i];
      }
      __syncthreads();
      // (none: all but what is e^-32 of the largest, or the parts' sums rounded apart)
      step = highest - (sh.listed < 0 ? STEPS : sh.listed);
    }
  }
  if (t == 0) {
    rec.first = first;
    rec.sum1 = sum1;
    rec.sum = sum;
    rec.mode = mode;
    rec.bound = bound;
    rec.step = step;
  }
}

template <typename T>
__global__ __launch_bounds__(SPLIT, 4) void k_sample_parts(SplitArgs q) {
  constexpr int E = Row<T>::E;
  __shared__ Shared sh;
  const SampleArgs& a = q.a;
  const int64_t r = q.row0 + blockIdx.y, block = blockIdx.y * (int64_t)q.parts + blockIdx.x;
  const Row<T> row(a.logits, a.logits_stride, r, a.vocab);
  const int t = threadIdx.x;
  griddep_launch_dependents();
  float x[EACH];
  int v[EACH / E];
  load_part(row, blockIdx.x, x, v);
  const Setting s = setting_of(a, r);
  const bool cut = s.hot && s.k == a.vocab && s.top_p < 1.0f, few = s.hot && s.k < a.vocab && s.k <= MOST_K;

  float m = x[0];
#pragma unroll
  for (int i = 1; i < EACH; ++i) m = fmaxf(m, x[i]);
  if (few) {
    float y = fmaxf(m, __shfl_xor_sync(FULL, m, 1));
    y = fmaxf(y, __shfl_xor_sync(FULL, y, 2));
    if ((t & 3) == 0) q.groups[block * GROUPS + t / 4] = y;
  }
  if (cut)
    for (int i = t; i < STEPS; i += SPLIT) sh.bins[i] = 0;
  int at = a.vocab;
#pragma unroll
  for (int i = EACH - 1; i >= 0; --i)
    if (x[i] == m) at = v[i / E] + i % E;
  const uint64_t first = block_max<SPLIT>(m > -INFINITY ? place_of(m, at) : 0, sh.scratch);
  m = first ? value_of(first) : 0.0f;
  float sum1 = 0.0f, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < EACH; ++i) sum1 += ex2f((x[i] - m) * LOG2E);
  sum1 = block_sum(sum1, sh.scratch);
  if (cut) {
    const Weigh weigh = weigh_of(m, s.temperature);
    const float per = steps_per(s.temperature);
    const int highest = step_of(m, per);
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (x[i] > -INFINITY) {
        sum += weigh(x[i]);
        const int step = step_of(x[i], per), slot = steps_below(highest, step);
        // (a product that rounds up to the step's end, or past it where x is huge, is held at 1)
        const float up = fminf((x[i] * per - (float)(step + 1)) * (LOG2E / 32.0f), 0.0f);
        if (slot >= 0 && slot < STEPS) atomicAdd(&sh.bins[slot], __float2uint_rn(STEP_ONE * ex2f(up)));
      }
    sum = block_sum(sum, sh.scratch);  // (a barrier behind the steps too)
    for (int i = t; i < STEPS / 4; i += SPLIT)
      reinterpret_cast<uint4*>(q.steps + block * STEPS)[i] = reinterpret_cast<const uint4*>(sh.bins)[i];
  }
  if (t == 0) q.part[block] = {first, sum1, sum};
  RowRecord& rec = q.rows[blockIdx.y];
  __threadfence();
  if (last_of(&rec.arrived, q.parts, sh)) settle_row<T>(q, r, rec, sh);
}

// The rest of a row, by the last block of k_sample_race.
template <typename T>
__device__ void settle_race(const SplitArgs& q, int64_t r, const RowRecord& rec, const Setting& s, const Weigh& weigh,
                            Shared& sh) {
  const SampleArgs& a = q.a;
  const int t = threadIdx.x, listed = (int)__ldcg(&rec.listed);
  const uint64_t* list = q.list + blockIdx.y * (int64_t)MOST_LISTED;
  Race race = {s, weigh, a.noise + r * a.noise_stride, rec.first};
  bool alone = listed > MOST_LISTED || (rec.mode == Mode::BOUND && listed > LIST);
  if (!alone && rec.mode == Mode::BOUND) {
    for (int i = t; i < listed; i += SPLIT) sh.list[i] = __ldcg(list + i);
    sort_list<SPLIT>(sh, listed);
    const int n = cut_list<SPLIT>(s, weigh, listed, sh);
    for (int i = t; i < n; i += SPLIT) race.enter(value_of(sh.list[i]), token_of(sh.list[i]));
  } else if (!alone && rec.mode == Mode::CUT) {
    if (listed) {
      const uint64_t want = part_of(s.top_p, rec.sum), front = __ldcg(&rec.above);
      uint64_t lo = ~0ull, hi = 0;
      for (int i = t; i < listed; i += SPLIT) {
        const uint64_t x = __ldcg(list + i);
        lo = min((unsigned long long)lo, (unsigned long long)x);
        hi = max((unsigned long long)hi, (unsigned long long)x);
      }
      lo = ~block_max<SPLIT>(~lo, sh.scratch);
      hi = block_max<SPLIT>(hi, sh.scratch);
      const Places places = {list, listed};
      const uint64_t cut = find_cut<SPLIT, false>(places, weigh, 0, front, want, 0x1p31f / ((float)rec.sum / FIXED),
                                                  value_of(lo), value_of(hi), sh);
      alone = cut == 0;
      if (!alone)
        for (int i = t; i < listed; i += SPLIT) {
          const uint64_t x = __ldcg(list + i);
          if (x >= cut) race.enter(value_of(x), token_of(x));
        }
    }
    if (!alone && t < q.parts) {
      const PartWinner* w = q.winner + blockIdx.y * (int64_t)q.parts + t;
      const uint64_t place = __ldcg(&w->place);
      const float best = __ldcg(&w->best);
      if (place && (!race.winner || !(best < race.best * NEAR))) {
        if (!race.winner || best * NEAR > race.best || race.better(place, race.winner) == place) {
          race.best = best;
          race.winner = place;
        }
      }
    }
  }
  if (alone) {  // (uniform)
    whole_row<SPLIT, T>(a, r, sh);
    return;
  }
  float best;
  const uint64_t winner = block_winner<SPLIT>(race, sh, best);
  if (t == 0) finish(a, r, winner, weigh.top, rec.sum1);
}

template <typename T>
__global__ __launch_bounds__(SPLIT, 3) void k_sample_race(SplitArgs q) {
  constexpr int E = Row<T>::E;
  __shared__ Shared sh;
  const SampleArgs& a = q.a;
  const int64_t r = q.row0 + blockIdx.y, block = blockIdx.y * (int64_t)q.parts + blockIdx.x;
  const Row<T> row(a.logits, a.logits_stride, r, a.vocab);
  const int t = threadIdx.x;
  float x[EACH];
  int v[EACH / E];
  load_part(row, blockIdx.x, x, v);
  const Setting s = setting_of(a, r);
  griddep_wait();
  RowRecord& rec = q.rows[blockIdx.y];
  const Mode mode = rec.mode;
  if (mode == Mode::DONE) return;
  if (mode == Mode::ALONE) {
    if (blockIdx.x == 0) whole_row<SPLIT, T>(a, r, sh);
    return;
  }
  const Weigh weigh = weigh_of(value_of(rec.first), s.temperature);
  uint64_t* list = q.list + blockIdx.y * (int64_t)MOST_LISTED;
  auto append = [&](float y, int token) {
    const unsigned to = atomicAdd(&rec.listed, 1u);
    if (to < MOST_LISTED) list[to] = place_of(y, token);
  };
  if (mode == Mode::BOUND) {
    const float bound = rec.bound;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (x[i] >= bound) append(x[i], v[i / E] + i % E);
  } else {
    const float per = steps_per(s.temperature);
    const int step = rec.step;
    Race race = {s, weigh, a.noise + r * a.noise_stride, rec.first};
    float above = 0.0f;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (x[i] > -INFINITY) {
        const int mine = step_of(x[i], per);
        if (mine > step) {
          const float w = weigh(x[i]);
          above += w;
          race.enter(x[i], v[i / E] + i % E, w);
        } else if (mine == step) {
          append(x[i], v[i / E] + i % E);
        }
      }
    above = block_sum(above, sh.scratch);
    float best;
    const uint64_t winner = block_winner<SPLIT>(race, sh, best);
    if (t == 0) {
      q.winner[block] = {winner, best};
      if (above > 0.0f) atomicAdd((unsigned long long*)&rec.above, (unsigned long long)fixed(above));
    }
  }
  __threadfence();
  if (last_of(&rec.raced, q.parts, sh)) settle_race<T>(q, r, rec, s, weigh, sh);
}

// Parts of a row (one more piece than it has, where it begins within one).
int64_t parts_of(int64_t vocab) { return (vocab + 7 + PART - 1) / PART; }

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

struct Sizes {
  size_t rows, part, winner, groups, steps, list, total;
};
Sizes sizes_of(int64_t rows, int64_t blocks) {
  Sizes z;
  z.rows = round_up(rows * sizeof(RowRecord));
  z.part = round_up(blocks * sizeof(PartRecord));
  z.winner = round_up(blocks * sizeof(PartWinner));
  z.groups = round_up(blocks * GROUPS * sizeof(float));
  z.steps = round_up(blocks * STEPS * sizeof(uint32_t));
  z.list = round_up(rows * MOST_LISTED * sizeof(uint64_t));
  z.total = z.rows + z.part + z.winner + z.groups + z.steps + z.list;
  return z;
}

template <typename T>
cudaError_t sample(const SampleArgs& a, int64_t n, void* workspace, cudaStream_t s) {
  const int64_t parts = parts_of(a.vocab);
  if (parts == 1 || parts > MOST_PARTS) {
    if (parts == 1)
      k_sample_row<256, T><<<(unsigned)n, 256, 0, s>>>(a);
    else
      k_sample_row<1024, T><<<(unsigned)n, 1024, 0, s>>>(a);
    return cudaGetLastError();
  }
  const int64_t rows = std::min<int64_t>({n, MOST_ROWS, MOST_BLOCKS / parts});
  const Sizes z = sizes_of(rows, rows * parts);
  char* p = static_cast<char*>(workspace);
  SplitArgs q;
  q.a = a;
  q.parts = (int)parts;
  q.rows = reinterpret_cast<RowRecord*>(p), p += z.rows;
  q.part = reinterpret_cast<PartRecord*>(p), p += z.part;
  q.winner = reinterpret_cast<PartWinner*>(p), p += z.winner;
  q.groups = reinterpret_cast<float*>(p), p += z.groups;
  q.steps = reinterpret_cast<uint32_t*>(p), p += z.steps;
  q.list = reinterpret_cast<uint64_t*>(p);
  for (q.row0 = 0; q.row0 < n; q.row0 += rows) {
    const dim3 grid((unsigned)parts, (unsigned)std::min(rows, n - q.row0));
    cudaError_t e = cudaMemsetAsync(q.rows, 0, grid.y * sizeof(RowRecord), s);
    if (e != cudaSuccess) return e;
    k_sample_parts<T><<<grid, SPLIT, 0, s>>>(q);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    if ((e = launch_maybe_pdl(true, k_sample_race<T>, grid, dim3(SPLIT), 0, s, q)) != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

// Enough for every smaller call too: of as many rows as a launch takes, or as many blocks.
size_t sample_workspace(int64_t n, int64_t vocab) {
  const int64_t parts = std::min<int64_t>(parts_of(vocab), MOST_PARTS);
  if (n == 0 || parts == 1) return 0;
  const int64_t rows = std::min<int64_t>(n, MOST_ROWS);
  return sizes_of(rows, std::min<int64_t>(rows * parts, MOST_BLOCKS)).total;
}

cudaError_t launch_sample(const void* logits, int type, int64_t logits_stride, const float* noise, int64_t noise_stride,
                          int64_t n, int vocab, const float* temperature, const int32_t* top_k, const float* top_p,
                          const float* min_p, int32_t* tokens, float* logprobs, void* workspace, cudaStream_t s) {
  const SampleArgs a = {logits, logits_stride, noise, noise_stride, vocab, temperature, top_k, top_p, min_p, tokens, logprobs};
  return type == TQ_BF16 ? sample<__nv_bfloat16>(a, n, workspace, s)
         : type == TQ_FP16 ? sample<__half>(a, n, workspace, s)
                           : sample<float>(a, n, workspace, s);
}

}  // namespace tq
