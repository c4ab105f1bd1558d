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
//
// A block per row.
#include <algorithm>

#include "tq_kv.cuh"
#include "tq_sample.h"
#include "tq_topk.cuh"

namespace tq {
namespace {

constexpr int THREADS = 1024, WARPS = THREADS / 32;
constexpr int BINS = 2048, LIST = 2048;
constexpr int SMALL_K = 512;      // up to here the threads' largest values bound the k-th
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

// The least integer that is not below p * x, for p in (0, 1) and x below 2^63 (p to 2^-32).
__device__ __forceinline__ uint64_t part_of(float p, uint64_t x) {
  const uint64_t m = (uint64_t)(uint32_t)__float2uint_rn(p * 4294967296.0f) << 32;
  return __umul64hi(x, m) + (x * m != 0);
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

// Sums and extremes over the block; every thread gets the result.
struct Scratch {
  uint64_t words[WARPS];
};
template <typename F>
__device__ __forceinline__ uint64_t block_reduce(uint64_t x, Scratch& s, F join) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = join(x, __shfl_xor_sync(FULL, x, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.words[threadIdx.x >> 5] = x;
  __syncthreads();
  x = s.words[threadIdx.x & 31];
#pragma unroll
  for (int o = 16; o; o >>= 1) x = join(x, __shfl_xor_sync(FULL, x, o));
  return x;
}
__device__ __forceinline__ uint64_t block_max(uint64_t x, Scratch& s) {
  return block_reduce(x, s, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint64_t block_sum(uint64_t x, Scratch& s) {
  return block_reduce(x, s, [](uint64_t a, uint64_t b) { return a + b; });
}
// Sum of the threads in front (exclusive), and of all.
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
  uint64_t w = s.words[lane], wup = w;
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
  uint32_t count[BINS], weight[BINS];
  Scratch scratch;
  int listed, bin;
  uint32_t low, high;           // extremes of a step's values, ordered
  uint64_t cut, taken;          // results of a search
  int candidates;
};

// Sorts the first n (at most LIST) places of the list, largest first; n is padded to a
// power of two with zeros.
__device__ void sort_list(Shared& sh, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += THREADS) sh.list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j; j >>= 1) {
      for (int t = threadIdx.x; t < size / 2; t += THREADS) {
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
template <typename T, bool BY_COUNT>
__device__ uint64_t find_cut(const Row<T>& row, const Weigh& weigh, uint64_t kept, uint64_t want, float scale, float low,
                             float high, Shared& sh) {
  constexpr int E = Row<T>::E;
  uint64_t front = 0;  // what lies above `high`
  for (int level = 0;; ++level) {
    // a histogram of the tokens with low <= x <= high: equal steps of x, then of x as an
    // ordered integer, so that every further level parts the smallest from the largest
    const float step = high > low ? (BINS - 1) / (high - low) : 0.0f;
    const uint32_t low_u = ordered(low), high_u = ordered(high);
    const int shift = max(0, 32 - __clz(high_u - low_u) - 11);  // (2^11 bins)
    auto bin_of = [&](float x) {
      return level ? (int)((high_u - ordered(x)) >> shift) : (int)fminf((high - x) * step, (float)(BINS - 1));
    };
    for (int i = threadIdx.x; i < BINS; i += THREADS) sh.count[i] = sh.weight[i] = 0;
    __syncthreads();
    for (int g = threadIdx.x; g < row.pieces(); g += THREADS) {
      float x[E];
      const int v = row.load(g, x);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] >= low && x[i] <= high && place_of(x[i], v + i) >= kept) {
          if (BY_COUNT)
            atomicAdd(&sh.count[bin_of(x[i])], 1u);
          else
            atomicAdd(&sh.weight[bin_of(x[i])], __float2uint_rn(weigh(x[i]) * scale));
        }
    }
    __syncthreads();
    // the first bin that reaches what is wanted
    const uint64_t rest = want > front ? want - front : 0;
    const uint64_t need = BY_COUNT ? rest : (uint64_t)((float)rest * (scale / FIXED));
    uint64_t mine = 0, all;
#pragma unroll
    for (int i = 0; i < BINS / THREADS; ++i) {
      const int b = threadIdx.x * (BINS / THREADS) + i;
      mine += BY_COUNT ? sh.count[b] : sh.weight[b];
    }
    if (threadIdx.x == 0) sh.bin = -1;
    uint64_t upto = block_scan(mine, sh.scratch, all);
#pragma unroll
    for (int i = 0; i < BINS / THREADS; ++i) {
      const int b = threadIdx.x * (BINS / THREADS) + i;
      const uint64_t here = BY_COUNT ? sh.count[b] : sh.weight[b];
      if (here && upto < need && upto + here >= need) sh.bin = b;
      upto += here;
    }
    __syncthreads();
    int bin = sh.bin;
    if (bin < 0) {  // (rounded weights fall short, or nothing is needed): the last bin that has any, or the first
      int last = -1, first = BINS;
      for (int i = threadIdx.x; i < BINS; i += THREADS)
        if (BY_COUNT ? sh.count[i] : sh.weight[i]) last = max(last, i), first = min(first, i);
      last = (int)block_max((uint64_t)(last + 1), sh.scratch) - 1;
      first = BINS - (int)block_max((uint64_t)(BINS - first), sh.scratch);
      bin = need ? max(last, 0) : min(first, BINS - 1);
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
    for (int g = threadIdx.x; g < row.pieces(); g += THREADS) {
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
    front += block_sum(above, sh.scratch);
    const int listed = sh.listed;
    if (listed == 0) return kept;  // (nothing is kept at all)
    low = unordered(sh.low);
    high = unordered(sh.high);
    if (listed <= LIST) {
      // sorted: the last of them with too little in front of it
      sort_list(sh, listed);
      if (threadIdx.x == 0) sh.cut = sh.list[0];
      uint64_t here[LIST / THREADS], sum = 0;
#pragma unroll
      for (int i = 0; i < LIST / THREADS; ++i) {
        const int at = threadIdx.x * (LIST / THREADS) + i;
        here[i] = at < listed ? (BY_COUNT ? 1 : fixed(weigh(value_of(sh.list[at])))) : 0;
        sum += here[i];
      }
      uint64_t before = front + block_scan(sum, sh.scratch, all);
#pragma unroll
      for (int i = 0; i < LIST / THREADS; ++i) {
        const int at = threadIdx.x * (LIST / THREADS) + i;
        if (at < listed && before < want && (before + here[i] >= want || at == listed - 1)) sh.cut = sh.list[at];
        before += here[i];
      }
      __syncthreads();
      const uint64_t cut = sh.cut;
      __syncthreads();
      return cut;
    }
    if (low == high) {
      // one value: all weigh the same; the first of them in their own order.  A warp takes
      // a run of pieces.
      const uint64_t each = BY_COUNT ? 1 : max((unsigned long long)fixed(weigh(low)), 1ull);
      uint64_t take = want > front ? (want - front + each - 1) / each : 1;
      if (take > (uint64_t)listed) take = listed;
      const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
      const int run = (row.pieces() + WARPS - 1) / WARPS, begin = warp * run, end = min(row.pieces(), begin + run);
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
      uint64_t before = block_scan(lane == 0 ? some : 0, sh.scratch, all);
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

// The race: candidates are weighed in float32, and those next to the best in 64 bits.
struct Racer {
  float best;
  uint64_t place;  // 0: none yet
};
__device__ __forceinline__ double exact_weight(float x, float top, float temperature) {
  return exp(((double)x - (double)top) / (double)temperature);
}
constexpr float NEAR = 1.0f - 0x1p-18f;

template <typename T>
__global__ __launch_bounds__(THREADS) void k_sample(SampleArgs a) {
  constexpr int E = Row<T>::E;
  __shared__ Shared sh;
  const int64_t r = blockIdx.x;
  const Row<T> row(a.logits, a.logits_stride, r, a.vocab);
  const float* noise = a.noise + r * a.noise_stride;
  const float temperature = a.temperature ? a.temperature[r] : 1.0f, top_p = a.top_p ? a.top_p[r] : 1.0f;
  const float min_p = a.min_p ? a.min_p[r] : 0.0f;
  const int want_k = a.top_k ? a.top_k[r] : 0, k = want_k > 0 && want_k < a.vocab ? want_k : a.vocab;

  // ---- the largest value and its lowest token, the sums of e^(x - max) at both temperatures
  float top = -INFINITY;
  int at = a.vocab;
  for (int g = threadIdx.x; g < row.pieces(); g += THREADS) {
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
  const uint64_t first = block_max(at < a.vocab ? place_of(top, at) : 0, sh.scratch);
  if (first == 0) {  // nothing but -inf
    if (threadIdx.x == 0) {
      a.tokens[r] = 0;
      if (a.logprobs) a.logprobs[r] = -INFINITY;
    }
    return;
  }
  top = value_of(first);
  const bool hot = temperature > 0.0f;
  const Weigh plain = weigh_of(top, 1.0f), weigh = weigh_of(top, hot ? temperature : 1.0f);
  uint64_t sum1 = 0, sum = 0;
  for (int g = threadIdx.x; g < row.pieces(); g += THREADS) {
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
  sum1 = block_sum(sum1, sh.scratch);
  sum = block_sum(sum, sh.scratch);
  auto finish = [&](uint64_t place) {
    a.tokens[r] = token_of(place);
    if (a.logprobs) a.logprobs[r] = (float)((double)value_of(place) - (double)top - log_fixed(sum1));
  };
  if (!hot) {
    if (threadIdx.x == 0) finish(first);
    return;
  }

  // ---- what is kept
  uint64_t kept = place_of(-INFINITY, a.vocab);  // every token that is not masked
  if (!(min_p <= 1.0f) || !(top_p > 0.0f)) kept = first;
  bool listed = false;  // the kept tokens lie in the list
  int n = 0;
  if (kept != first && k < a.vocab) {
    if (k <= SMALL_K) {
      // the k-th largest of the threads' own largest values: at least k tokens reach it
      if (threadIdx.x == 0) sh.listed = 0;
      sh.list[threadIdx.x] = (uint64_t)mine << 32 | threadIdx.x;
      sort_list(sh, THREADS);
      const float bound = unordered((uint32_t)(sh.list[k - 1] >> 32));
      __syncthreads();
      if (bound > -INFINITY) {
        for (int g = threadIdx.x; g < row.pieces(); g += THREADS) {
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
      sort_list(sh, n);
      n = min(n, k);
      kept = sh.list[n - 1];
      uint64_t here[LIST / THREADS], part = 0;
#pragma unroll
      for (int i = 0; i < LIST / THREADS; ++i) {
        const int e = threadIdx.x * (LIST / THREADS) + i;
        here[i] = e < n ? fixed(weigh(value_of(sh.list[e]))) : 0;
        part += here[i];
      }
      uint64_t before = block_scan(part, sh.scratch, sum);
      if (top_p < 1.0f) {
        const uint64_t want = part_of(top_p, sum);
        int count = 0;
#pragma unroll
        for (int i = 0; i < LIST / THREADS; ++i) {
          const int e = threadIdx.x * (LIST / THREADS) + i;
          if (e < n && (e == 0 || before < want)) ++count;
          before += here[i];
        }
        n = (int)block_sum((uint64_t)count, sh.scratch);
        kept = sh.list[n - 1];
      }
    } else {
      // more of them: by counts, from the smallest value that is not masked
      uint64_t count = 0;
      uint32_t lo = 0xffffffffu;
      for (int g = threadIdx.x; g < row.pieces(); g += THREADS) {
        float x[E];
        row.load(g, x);
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (x[i] > -INFINITY) {
            ++count;
            lo = min(lo, ordered(x[i]));
          }
      }
      count = block_sum(count, sh.scratch);
      lo = ~(uint32_t)block_max((uint64_t)~lo, sh.scratch);
      if (count > (uint64_t)k) {
        kept = find_cut<T, true>(row, weigh, kept, k, 0.0f, unordered(lo), top, sh);
        uint64_t part = 0;
        for (int g = threadIdx.x; g < row.pieces(); g += THREADS) {
          float x[E], y = 0.0f;
          const int v = row.load(g, x);
#pragma unroll
          for (int i = 0; i < E; ++i) y += place_of(x[i], v + i) >= kept ? weigh(x[i]) : 0.0f;
          part += fixed(y);
        }
        sum = block_sum(part, sh.scratch);
      }
    }
  }
  if (kept != first && !listed && top_p < 1.0f) {
    const uint64_t want = part_of(top_p, sum);
    // tokens below (1 - p) of the mean weight are together too light to be reached
    const float least = (1.0f - top_p) * ((float)sum / FIXED) / (float)a.vocab;
    const float low = fmaxf(top + logf(least) * temperature * 1.0001f - 1e-3f, -3.0e38f);
    if (want < sum)
      kept = max((unsigned long long)kept,
                 (unsigned long long)find_cut<T, false>(row, weigh, kept, want,
                                                        0x1p31f / ((float)sum / FIXED), low, top, sh));
  }

  // ---- the race
  const float min_hi = min_p * (1.0f + 0x1p-18f), min_lo = min_p * (1.0f - 0x1p-18f);
  auto races = [&](uint64_t place, float w) {
    return place == first || (w > 0.0f && (w >= min_hi || (w >= min_lo && exact_weight(value_of(place), top, temperature) >= (double)min_p)));
  };
  float best = 0.0f;
  uint64_t winner = 0;
  auto enter = [&](uint64_t place) {
    const float w = weigh(value_of(place));
    if (!races(place, w)) return;
    const float e = noise[token_of(place)], q = w / e;
    if (!(q >= best * NEAR) || winner == 0) {
      if (winner == 0) {
        best = q;
        winner = place;
      }
      return;
    }
    if (q * NEAR <= best) {  // too close for float32
      const double x = exact_weight(value_of(place), top, temperature) / (double)e;
      const double y = exact_weight(value_of(winner), top, temperature) / (double)noise[token_of(winner)];
      if (!(x > y || (x == y && token_of(place) < token_of(winner)))) return;
    }
    best = q;
    winner = place;
  };
  if (listed) {
    for (int i = threadIdx.x; i < n; i += THREADS) enter(sh.list[i]);
  } else {
    for (int g = threadIdx.x; g < row.pieces(); g += THREADS) {
      float x[E];
      const int v = row.load(g, x);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] > -INFINITY && place_of(x[i], v + i) >= kept) enter(place_of(x[i], v + i));
    }
  }
  // the block's best, and those that float32 does not tell from it
  const float most = __uint_as_float((uint32_t)block_max(winner ? (uint64_t)__float_as_uint(best) : 0, sh.scratch));
  const bool close = winner && !(best < most * NEAR);
  if (threadIdx.x == 0) sh.candidates = 0;
  __syncthreads();
  if (close) {
    const int to = atomicAdd(&sh.candidates, 1);
    sh.list[to] = winner;  // (THREADS of them fit)
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    uint64_t w = sh.list[0];
    if (sh.candidates > 1) {
      double q = exact_weight(value_of(w), top, temperature) / (double)noise[token_of(w)];
      for (int i = 1; i < sh.candidates; ++i) {
        const uint64_t p = sh.list[i];
        const double x = exact_weight(value_of(p), top, temperature) / (double)noise[token_of(p)];
        if (x > q || (x == q && token_of(p) < token_of(w))) {
          q = x;
          w = p;
        }
      }
    }
    finish(w);
  }
}

}  // namespace

size_t sample_workspace(int64_t, int64_t) { return 0; }

cudaError_t launch_sample(const void* logits, int type, int64_t logits_stride, const float* noise, int64_t noise_stride,
                          int64_t n, int vocab, const float* temperature, const int32_t* top_k, const float* top_p,
                          const float* min_p, int32_t* tokens, float* logprobs, void*, cudaStream_t s) {
  const SampleArgs a = {logits, logits_stride, noise, noise_stride, vocab, temperature, top_k, top_p, min_p, tokens, logprobs};
  (type == TQ_BF16 ? k_sample<__nv_bfloat16> : type == TQ_FP16 ? k_sample<__half> : k_sample<float>)<<<(unsigned)n, THREADS, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace tq
