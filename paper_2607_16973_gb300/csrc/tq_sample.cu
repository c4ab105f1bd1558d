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
// Quotients are taken in float32; those within 2^-16 of the largest are compared again
// in 64 bits, so that the token is that of exact arithmetic.
//
// Three forms.  Rows of up to 256 pieces of 16 bytes, and rows beyond 256 parts, by a block
// that reads them again for every step (whole_row).  Rows of up to 8 pieces for each of
// 1,024 threads by a block that holds them in registers (k_sample_one; with 8 pieces 100
// to 116 bytes a thread spill).  Longer ones in parts, by four kernels.
//
// Bound: HBM for the parts' first reading; the rest is the chain of a row's steps and, for
// code that runs once a launch, its fetching.  256 rows of 128,000 bf16 logits with settings
// of all kinds (65.5 MB, and 16 to 20 MB of noise): 106 us on a GB300, of which the first
// reading 32, the cuts 12, the race 53, the lists 21.  48 rows of 100,003 float32, flat, top-p
// 0.9: 55 us (14, 12, 26, 14 one by one).  One row of 32,000: 18 us, 20 to 24 a call.  (A block per row
// throughout: 236, 138 and 25 us; the settling steps in the last block of each kernel
// instead of kernels of their own: 225 and 81.)
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

// A logit: NaN counts as -inf, +inf as the largest float.
__device__ __forceinline__ float logit(float x) { return fminf(fmaxf(x, -INFINITY), 3.402823466e38f); }

// Floats as unsigned integers in their order.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);  // (-0 is 0)
  return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
// A token's place in the order: larger comes first.
__device__ __forceinline__ uint64_t place_of(float x, int v) { return (uint64_t)ordered(x) << 32 | (uint32_t)~v; }
__device__ __forceinline__ int token_of(uint64_t place) { return (int)~(uint32_t)place; }
__device__ __forceinline__ float value_of(uint64_t place) { return unordered((uint32_t)(place >> 32)); }

// Weight of a value: 2^((x - top) * (c_hi + c_lo)), about 2^-22 off, and for float32 values by
// the rounding of x - top, which is 2^-24 of an exponent of up to 88: 2^-17.5.  0 below 2^-126
// (and for masked values, whatever the temperature).
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

// The least integer that is not below p * x, for p in (0, 1) and x of up to 2^63: 1 at least.
__device__ __forceinline__ uint64_t part_of(float p, uint64_t x) {
  // p = m / 2^shift, the product hi * 2^64 + lo
  const uint32_t u = __float_as_uint(p);
  const uint64_t m = (u & 0x7fffffu) | (u >> 23 ? 0x800000u : 0u);
  const int shift = 150 - max((int)(u >> 23), 1);  // 24 to 149
  const uint64_t hi = __umul64hi(x, m), lo = x * m;
  uint64_t whole, rest;
  if (shift < 64) {
    whole = hi << (64 - shift) | lo >> shift;
    rest = lo << (64 - shift);
  } else {
    whole = shift == 64 ? hi : hi >> (shift - 64 < 63 ? shift - 64 : 63);  // (hi is below 2^24)
    rest = 1;
  }
  return max(1ull, (unsigned long long)(whole + (rest != 0)));
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
    const uint64_t place = p[g];
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

// Sorts the first n (at most LIST) places of the list, largest first: few of them by
// counting those in front of each, more by a bitonic network, n padded to a power of
// two with zeros.  (100 places in a block of 1,024 threads: 28 steps of the network with
// their barriers, or 100 reads of shared memory by four warps.)
template <int N>
__device__ void sort_list(Shared& sh, int n) {
  if (n <= 256) {
    static_assert(N >= 256, "a thread for each");
    __syncthreads();
    const uint64_t mine = threadIdx.x < n ? sh.list[threadIdx.x] : 0;
    int front = 0;
    if ((int)(threadIdx.x & ~31u) < n)
#pragma unroll 4
      for (int i = 0; i < n; ++i) front += sh.list[i] > mine;
    __syncthreads();
    if (threadIdx.x < n) sh.list[front] = mine;
    __syncthreads();
    return;
  }
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
// Weights are added up as what `want` counts, to the last bit: with bins of 2^-31 of all weight,
// 128,000 equal tokens came out 2^-16 too light, and tokens of 2^-33 as nothing.
template <int N, bool BY_COUNT, typename Source>
__device__ uint64_t find_cut(const Source& row, const Weigh& weigh, uint64_t kept, uint64_t front, uint64_t want,
                             float low, float high, Shared& sh) {
  constexpr int E = Source::E;
  uint32_t* more = reinterpret_cast<uint32_t*>(sh.list);  // the upper halves of the bins' weights, until the list is made
  static_assert(BINS * sizeof(uint32_t) <= sizeof(sh.list), "room for them");
  for (int level = 0;; ++level) {
    // a histogram of the tokens with low <= x <= high: equal steps of x, then of x as an
    // ordered integer, so that every further level parts the smallest from the largest
    const float step = high > low ? (BINS - 1) / (high - low) : 0.0f;
    const uint32_t low_u = ordered(low), high_u = ordered(high);
    const int shift = max(0, 32 - __clz(high_u - low_u) - 11);  // (2^11 bins)
    auto bin_of = [&](float x) {
      return level ? (int)((high_u - ordered(x)) >> shift) : (int)fminf((high - x) * step, (float)(BINS - 1));
    };
    for (int i = threadIdx.x; i < BINS; i += N) {
      sh.bins[i] = 0;
      if (!BY_COUNT) more[i] = 0;
    }
    __syncthreads();
    int held = 0;  // weights of a thread's tokens in a row that share a bin go there together
    uint64_t some = 0;
    auto put = [&] {
      if (some == 0) return;
      const uint32_t part = (uint32_t)some, old = atomicAdd(&sh.bins[held], part);
      const uint32_t up = (uint32_t)(some >> 32) + (old + part < old);
      if (up) atomicAdd(&more[held], up);
      some = 0;
    };
    for (int g = threadIdx.x; g < row.pieces(); g += N) {
      float x[E];
      const int v = row.load(g, x);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] >= low && x[i] <= high && place_of(x[i], v + i) >= kept) {
          const int b = bin_of(x[i]);
          if (BY_COUNT) {
            atomicAdd(&sh.bins[b], 1u);
            continue;
          }
          if (b != held) put();
          held = b;
          some += fixed(weigh(x[i]));
        }
    }
    put();
    __syncthreads();
    // the first bin that reaches what is wanted
    const uint64_t need = want > front ? want - front : 0;
    auto bin_sum = [&](int b) { return (BY_COUNT ? 0 : (uint64_t)more[b] << 32) | sh.bins[b]; };
    uint64_t mine = 0, all;
#pragma unroll 1
    for (int i = 0; i < BINS / N; ++i) mine += bin_sum(threadIdx.x * (BINS / N) + i);
    if (threadIdx.x == 0) {
      sh.bin = -1;
      sh.taken = 0;
    }
    uint64_t upto = block_scan<N>(mine, sh.scratch, all);
#pragma unroll 1
    for (int i = 0; i < BINS / N; ++i) {
      const int b = threadIdx.x * (BINS / N) + i;
      const uint64_t here = bin_sum(b);
      if (here && upto < need && upto + here >= need) {
        sh.bin = b;
        sh.taken = upto;
      }
      upto += here;
    }
    __syncthreads();
    int bin = sh.bin;
    uint64_t before_bin = sh.taken;
    if (bin < 0) {  // (sums of several weights are rounded apart, or nothing is needed): the last bin that has any, or the first
      int last = -1, first = BINS;
      for (int i = threadIdx.x; i < BINS; i += N)
        if (bin_sum(i)) last = max(last, i), first = min(first, i);
      last = (int)block_max<N>((uint64_t)(last + 1), sh.scratch) - 1;
      first = BINS - (int)block_max<N>((uint64_t)(BINS - first), sh.scratch);
      bin = need ? max(last, 0) : first < BINS ? first : 0;
      if (need) before_bin = all - bin_sum(bin);
    }
    front += before_bin;
    // its tokens to the list, their extremes
    if (threadIdx.x == 0) {
      sh.listed = 0;
      sh.low = 0xffffffffu;
      sh.high = 0;
    }
    __syncthreads();
    uint32_t lo = 0xffffffffu, hi = 0;
    for (int g = threadIdx.x; g < row.pieces(); g += N) {
      float x[E];
      const int v = row.load(g, x);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] >= low && x[i] <= high && place_of(x[i], v + i) >= kept && bin_of(x[i]) == bin) {
          const int at = atomicAdd(&sh.listed, 1);
          if (at < LIST) sh.list[at] = place_of(x[i], v + i);
          lo = min(lo, ordered(x[i]));
          hi = max(hi, ordered(x[i]));
        }
    }
    if (lo <= hi) {
      atomicMin(&sh.low, lo);
      atomicMax(&sh.high, hi);
    }
    __syncthreads();
    const int listed = sh.listed;
    if (listed == 0) return kept;  // (nothing is kept at all)
    low = unordered(sh.low);
    high = unordered(sh.high);
    if (listed <= LIST) {
      // sorted: the last of them with too little in front of it
      sort_list<N>(sh, listed);
      if (threadIdx.x == 0) sh.cut = sh.list[0];
      const int each = (listed + N - 1) / N, from = threadIdx.x * each, to = min(listed, from + each);
      auto here = [&](int at) { return BY_COUNT ? (uint64_t)1 : fixed(weigh(value_of(sh.list[at]))); };
      uint64_t sum = 0;
#pragma unroll 1
      for (int at = from; at < to; ++at) sum += here(at);
      uint64_t before = front + block_scan<N>(sum, sh.scratch, all);
#pragma unroll 1
      for (int at = from; at < to; ++at) {
        const uint64_t x = here(at);
        if (before < want && (before + x >= want || at == listed - 1)) sh.cut = sh.list[at];
        before += x;
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

// The race among kept tokens: quotients in float32, those next to the best in 64 bits.  NEAR
// holds two quotients' errors, each 2^-17.4 at most (the weight's, and the division's).
constexpr float NEAR = 1.0f - 0x1p-16f;
// The same for weights of one product, ex2f((x - top) * c): the difference, c and the product
// are each 2^-24 off, of an exponent of up to 88, so the weight is by 2^-15.9 at most.
constexpr float ABOUT = 0x1p-15f, NEAR_ABOUT = 1.0f - 0x1p-14f;

struct Setting {
  float temperature, top_p, min_p;
  int k;        // vocab: all
  bool hot;     // else the first token alone
};
__device__ __forceinline__ Setting setting_of(const SampleArgs& a, int64_t r) {
  Setting s;
  s.temperature = a.temperature ? a.temperature[r] : 1.0f;
  if (s.temperature > 1e30f) s.temperature = 1e30f;  // (infinite: products with masked values would be NaN)
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

  // (no quotient is negative, NaN, infinite or, for a weight above 2^-100, zero, whatever the noise)
  static __device__ __forceinline__ float number(float e) { return fminf(fmaxf(e, 0x1p-126f), 0x1p20f); }
  // (rarely asked, and long: not inlined where a row's tokens go by)
  static __device__ __noinline__ double exact(float x, float top, float temperature) {
    return exp(((double)x - (double)top) / (double)temperature);
  }
  __device__ __forceinline__ double weight(float x) const { return exact(x, weigh.top, s.temperature); }
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
  // Whether min-p lets a token of about weight w race: in 64 bits next to its border.
  __device__ __forceinline__ bool keeps(float x, float w) const {
    if (w > s.min_p * (1.0f + ABOUT)) return true;
    return w > 0.0f && w >= s.min_p * (1.0f - ABOUT) && weight(x) >= (double)s.min_p;
  }
  __device__ __forceinline__ void enter(float x, int v, float w, float e) {
    const uint64_t place = place_of(x, v);
    if (place != first && !keeps(x, w)) return;
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
  // a thread takes some neighbours.  (Rolled: code that runs once costs more to fetch than to run.)
  const int each = (n + N - 1) / N, from = threadIdx.x * each, to = min(n, from + each);
  uint64_t part = 0, sum;
#pragma unroll 1
  for (int e = from; e < to; ++e) part += fixed(weigh(value_of(sh.list[e])));
  uint64_t before = block_scan<N>(part, sh.scratch, sum);
  const uint64_t want = part_of(s.top_p, sum);
  int count = 0;
#pragma unroll 1
  for (int e = from; e < to; ++e) {
    count += e == 0 || before < want;
    before += fixed(weigh(value_of(sh.list[e])));
  }
  return (int)block_sum<N>((uint64_t)count, sh.scratch);
}

// What tokens below are too light: together less than the part that top-p leaves out.
__device__ __forceinline__ float least_value(const Setting& s, float top, uint64_t sum, int vocab) {
  const float least = (1.0f - s.top_p) * ((float)sum / FIXED) / (float)vocab;
  return fmaxf(top + logf(least) * s.temperature * 1.0001f - 1e-3f, -3.402823466e38f);  // (not a masked one's, nor above top)
}

// What tokens below are ruled out by min-p (> 0).
__device__ __forceinline__ float least_kept(const Setting& s, float top) {
  float x = top + (logf(s.min_p) - 1e-3f) * s.temperature;
  x -= fabsf(x) * 0x1p-21f;
  return x < top ? x : -INFINITY;
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
        kept = find_cut<N, true>(row, weigh, kept, 0, s.k, unordered(lo), top, sh);
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
      const uint64_t cut = find_cut<N, false>(row, weigh, kept, 0, want, least_value(s, top, sum, a.vocab), top, sh);
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
// k_sample_parts: a block per part of 256 x JP pieces of 16 bytes, read once and held as
// they are: its largest, its sums, and what tells where the row's cut lies: the largest of
// every 64 tokens (small k), or the weights of 1,024 steps of 1/32 of x / T (top-p; steps at
// fixed places, so that parts which do not know of one another's largest add up).
// k_sample_cut: a block per row joins the parts and finds that step, or a bound of k values.
// k_sample_race: the parts again, from L2: what lies above the step races at once and is
// summed, what lies in it (or above the bound) goes to the row's list.
// k_sample_finish: a block per row cuts the list, races it, and joins the parts' winners.
// A list that is too long, and what fits neither form (large k, infinities), is left to
// whole_row there.
constexpr int SPLIT = 256;
constexpr int GROUP = 64;              // tokens
constexpr int STEPS = 1024;            // of 1/32: weights down to e^-32 of a part's largest
// The weight at a step's upper end as an integer: a part of `tokens` brings 2^31 at most, even
// where all of them lie at one step's end, so no step wraps; and 2^22 at most, what ROUND holds.
constexpr float unit_of(int tokens) { return (float)((1u << 31) / tokens); }
constexpr float ROUND = 12582912.0f;   // 1.5 * 2^23: what is added to it is rounded to an integer, in its low bits
constexpr float MOST_STEP = 1e6f;      // steps' numbers up to which that holds, and leaves bits behind the point
constexpr int MOST_K = 512, MOST_LISTED = 4096, MOST_PARTS = SPLIT;
constexpr int MOST_ROWS = 512, MOST_BLOCKS = 16384;  // of a launch: what the workspace is for
constexpr int FEW_BLOCKS = 304;        // with less of 8 pieces a thread, 2 a thread

enum class Mode : int { DONE, ALONE, BOUND, CUT };

struct RowRecord {
  uint64_t first, sum1, sum;
  Mode mode;
  float bound;          // BOUND: the list's least value.  CUT: nothing below it is kept or listed
  int step;             // CUT: the list's step; what lies above it is kept, what lies below is not.  INT_MIN: no cut
  unsigned listed;      // (0 until the race)
};
struct PartRecord {
  uint64_t first;
  float sum1, sum;
};
struct PartWinner {
  uint64_t place;
  float best, above;    // its quotient; the part's weight above the step
};

struct SplitArgs {
  SampleArgs a;
  int64_t row0;
  int parts;
  RowRecord* rows;
  PartRecord* part;
  PartWinner* winner;
  float* groups;     // [blocks][SPLIT]
  uint32_t* steps;   // [blocks][STEPS]
  uint64_t* list;    // [rows][MOST_LISTED]
};

// 16 bytes of a row as they lie in memory.
template <typename T> struct Packed;
template <> struct Packed<float> {
  static constexpr uint32_t MASKED = 0xff800000u;
  static __device__ __forceinline__ uint32_t largest(uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }
  static __device__ __forceinline__ float top(uint32_t a) { return __uint_as_float(a); }
  static __device__ __forceinline__ float at(const uint4& u, int i) {
    return __uint_as_float(i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w);
  }
};
template <typename T2, typename T, uint32_t MASK> struct Packed16 {
  static constexpr uint32_t MASKED = MASK;
  static __device__ __forceinline__ uint32_t largest(uint32_t a, uint32_t b) {
    T2 x, y;
    memcpy(&x, &a, 4);
    memcpy(&y, &b, 4);
    x = __hmax2(x, y);
    memcpy(&a, &x, 4);
    return a;
  }
  static __device__ __forceinline__ float at(uint32_t w, int i) {
    const uint16_t h = (uint16_t)(i ? w >> 16 : w);
    T x;
    memcpy(&x, &h, 2);
    return to_float(x);
  }
  static __device__ __forceinline__ float top(uint32_t a) { return fmaxf(at(a, 0), at(a, 1)); }
  static __device__ __forceinline__ float at(const uint4& u, int i) {
    return at(i < 2 ? u.x : i < 4 ? u.y : i < 6 ? u.z : u.w, i & 1);
  }
};
template <> struct Packed<__nv_bfloat16> : Packed16<__nv_bfloat162, __nv_bfloat16, 0xff80ff80u> {
  // (the upper half of the float)
  static __device__ __forceinline__ float at(uint32_t w, int i) { return __uint_as_float(i ? w & 0xffff0000u : w << 16); }
  static __device__ __forceinline__ float top(uint32_t a) { return fmaxf(at(a, 0), at(a, 1)); }
  static __device__ __forceinline__ float at(const uint4& u, int i) {
    return at(i < 2 ? u.x : i < 4 ? u.y : i < 6 ? u.z : u.w, i & 1);
  }
};
template <> struct Packed<__half> : Packed16<__half2, __half, 0xfc00fc00u> {};

// Piece g of a row, NaN and what is not the row's as -inf.
template <typename T>
__device__ __forceinline__ uint4 load_raw(const Row<T>& row, int g) {
  using P = Packed<T>;
  constexpr int E = Row<T>::E;
  uint4 u = make_uint4(P::MASKED, P::MASKED, P::MASKED, P::MASKED);
  const int v = g * E - row.lead;
  if (v >= 0 && v + E <= row.n) {
    u = *reinterpret_cast<const uint4*>(row.p + v);
  } else if (v < row.n) {
    union {
      uint4 u;
      T e[E];
    } x;
    x.u = u;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (v + i >= 0 && v + i < row.n) x.e[i] = row.p[v + i];
    u = x.u;
  }
  return u;
}
template <typename T>
__device__ __forceinline__ void mask_nan(uint4& u) {
  using P = Packed<T>;
  u.x = P::largest(u.x, P::MASKED), u.y = P::largest(u.y, P::MASKED);
  u.z = P::largest(u.z, P::MASKED), u.w = P::largest(u.w, P::MASKED);
}
// What follows converts the pieces again rather than keep 64 floats from before.
template <int JP>
__device__ __forceinline__ void hold(uint4 (&u)[JP]) {
#pragma unroll
  for (int j = 0; j < JP; ++j) asm volatile("" : "+r"(u[j].x), "+r"(u[j].y), "+r"(u[j].z), "+r"(u[j].w));
}
template <typename T>
__device__ __forceinline__ uint32_t piece_top(const uint4& u) {
  using P = Packed<T>;
  return P::largest(P::largest(u.x, u.y), P::largest(u.z, u.w));
}

// Number of the step that x is in, which grows with x: 32 x / T, rounded.  (Up to MOST_STEP.)
__device__ __forceinline__ float steps_per(float temperature) { return fminf(32.0f / temperature, 1e30f); }
__device__ __forceinline__ int step_of(float x, float per) {
  return __float_as_int(__fadd_rn(__fmul_rn(x, per), ROUND)) - __float_as_int(ROUND);
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
  return x;
}
// The block's largest x >= 0; y becomes its sum.
__device__ __forceinline__ float block_most(float x, float& y, Scratch& s) {
  x = __uint_as_float(__reduce_max_sync(FULL, __float_as_uint(x)));
  y = warp_sum(y);
  if ((threadIdx.x & 31) == 0) s.words[threadIdx.x >> 5] = (uint64_t)__float_as_uint(x) << 32 | __float_as_uint(y);
  __syncthreads();
  x = y = 0.0f;
#pragma unroll
  for (int w = 0; w < SPLIT / 32; ++w) {
    x = fmaxf(x, __uint_as_float((uint32_t)(s.words[w] >> 32)));
    y += __uint_as_float((uint32_t)s.words[w]);
  }
  return x;
}
__device__ __forceinline__ void block_sums(float& x, float& y, Scratch& s) {
  x = warp_sum(x);
  y = warp_sum(y);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s.words[threadIdx.x >> 5] = (uint64_t)__float_as_uint(x) << 32 | __float_as_uint(y);
  __syncthreads();
  x = y = 0.0f;
#pragma unroll
  for (int w = 0; w < SPLIT / 32; ++w) {
    x += __uint_as_float((uint32_t)(s.words[w] >> 32));
    y += __uint_as_float((uint32_t)s.words[w]);
  }
}

// The row's record; groups: of a part; unit: of its steps' weights.  A block per row.
__global__ __launch_bounds__(SPLIT) void k_sample_cut(SplitArgs q, int groups_of_part, float unit) {
  __shared__ Shared sh;
  const SampleArgs& a = q.a;
  const int64_t r = q.row0 + blockIdx.x, block0 = blockIdx.x * (int64_t)q.parts;
  RowRecord& rec = q.rows[blockIdx.x];
  griddep_launch_dependents();
  const Setting s = setting_of(a, r);
  griddep_wait();
  const PartRecord* part = q.part + block0;
  const int t = threadIdx.x;
  PartRecord mine = {0, 0.0f, 0.0f};  // (parts <= threads)
  if (t < q.parts) {
    mine.first = __ldcg(&part[t].first);
    mine.sum1 = __ldcg(&part[t].sum1);
    mine.sum = __ldcg(&part[t].sum);
  }
  const uint64_t first = block_max<SPLIT>(mine.first, sh.scratch);
  const float top = first ? value_of(first) : 0.0f, m = mine.first ? value_of(mine.first) : 0.0f;
  if (first == 0 || top == INFINITY) {
    if (t == 0) {
      if (first == 0) finish(a, r, 0, 0.0f, 0);
      rec.mode = first ? Mode::ALONE : Mode::DONE;
      rec.first = first;
    }
    return;
  }
  const Weigh plain = weigh_of(top, 1.0f), weigh = weigh_of(top, s.hot ? s.temperature : 1.0f);
  const uint64_t sum1 = block_sum<SPLIT>(mine.first ? fixed(mine.sum1 * plain(m)) : 0, sh.scratch);
  const uint64_t sum = block_sum<SPLIT>(mine.first ? fixed(mine.sum * weigh(m)) : 0, sh.scratch);
  const float per = steps_per(s.temperature);
  Mode mode = Mode::DONE;
  float bound = -INFINITY;
  int step = INT_MIN;
  if (!s.hot) {
    if (t == 0) finish(a, r, first, top, sum1);
  } else if (s.k < a.vocab) {
    mode = Mode::ALONE;
    if (s.k <= MOST_K) {
      // a value that k groups' largest reach, by a histogram of them
      const float* groups = q.groups + block0 * SPLIT;
      const int n = q.parts * groups_of_part;
      auto group = [&](int i) { return __ldcg(groups + (int64_t)(i / groups_of_part) * SPLIT + i % groups_of_part); };
      uint32_t lo = 0xffffffffu;
      for (int i = t; i < n; i += SPLIT) {
        const float x = group(i);
        if (x > -INFINITY) lo = min(lo, ordered(x));
      }
      const float low = unordered(~(uint32_t)block_max<SPLIT>((uint64_t)~lo, sh.scratch));
      const float bins_per = top > low ? (BINS - 1) / (top - low) : 0.0f;
      for (int i = t; i < BINS; i += SPLIT) sh.bins[i] = 0;
      if (t == 0) sh.listed = -1;
      __syncthreads();
      auto bin_of = [&](float x) { return (int)fminf((top - x) * bins_per, (float)(BINS - 1)); };
      for (int i = t; i < n; i += SPLIT) {
        const float x = group(i);
        if (x > -INFINITY) atomicAdd(&sh.bins[bin_of(x)], 1u);
      }
      __syncthreads();
      uint64_t some = 0, all;
#pragma unroll 1
      for (int i = 0; i < BINS / SPLIT; ++i) some += sh.bins[t * (BINS / SPLIT) + i];
      uint64_t upto = block_scan<SPLIT>(some, sh.scratch, all);
#pragma unroll 1
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
          const float x = group(i);
          if (x > -INFINITY && bin_of(x) <= bin) least = min(least, ordered(x));
        }
        bound = unordered(~(uint32_t)block_max<SPLIT>((uint64_t)~least, sh.scratch));
        mode = Mode::BOUND;
      }
    }
  } else if (!(s.top_p < 1.0f)) {
    mode = Mode::CUT;  // (of nothing: all race that min-p lets)
    if (s.min_p > 0.0f) bound = least_kept(s, top);
  } else if (!(fabsf(top) * per < MOST_STEP)) {
    mode = Mode::ALONE;  // (a step's number is too large)
  } else {
    mode = Mode::CUT;
    // the steps' weights from the row's largest down, 4 of them a thread, relative to that
    const int highest = step_of(top, per), at = t * (STEPS / SPLIT);
    uint64_t w[4] = {0, 0, 0, 0};
    static_assert(STEPS / SPLIT == 4, "steps of a thread");
    int shift = STEPS;  // of this part's steps; STEPS: it has none that count
    if (mine.first && (top - m) * per < (float)STEPS) shift = highest - step_of(m, per);
    sh.bins[t] = shift;
    __syncthreads();
    const uint32_t* steps = q.steps + block0 * STEPS;
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
      // the weight at the step's upper end: about 1 in the largest's own step
      const float up = ((float)(highest - at - i) + 0.5f - top * per) * (1.0f / 32.0f);
      w[i] = (uint64_t)((float)w[i] * (FIXED / unit) * ex2f(up * LOG2E));
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
    // (none: all but what is e^-32 of the largest, or the sums rounded apart, or a part without steps)
    step = highest - (sh.listed < 0 ? STEPS - 1 : sh.listed);
    bound = ((float)step - 0.51f) / per;
    bound -= fabsf(bound) * 0x1p-21f;
  }
  if (t == 0) {
    rec.first = first;
    rec.sum1 = sum1;
    rec.sum = sum;
    rec.mode = mode;
    rec.bound = bound;
    rec.step = step;
    rec.listed = 0;
  }
}

template <typename T, int JP>
__global__ __launch_bounds__(SPLIT, 4) void k_sample_parts(SplitArgs q) {
  using P = Packed<T>;
  constexpr int E = Row<T>::E, LANES = GROUP / (JP * E);  // of a group
  constexpr float UNIT = unit_of(SPLIT * JP * E);
  static_assert(UNIT >= 0x1p16f && UNIT <= 0x1p22f, "weights to 2^-17, sums to 2^31");
  __shared__ struct {
    uint32_t bins[STEPS];
    Scratch scratch;
    uint32_t low;
  } sh;
  const SampleArgs& a = q.a;
  const int64_t r = q.row0 + blockIdx.y, block = blockIdx.y * (int64_t)q.parts + blockIdx.x;
  const Row<T> row(a.logits, a.logits_stride, r, a.vocab);
  const int t = threadIdx.x, g0 = blockIdx.x * (SPLIT * JP) + t;
  griddep_launch_dependents();
  uint4 raw[JP];
#pragma unroll
  for (int j = 0; j < JP; ++j) raw[j] = load_raw(row, g0 + j * SPLIT);
  const Setting s = setting_of(a, r);
  const bool cut = s.hot && s.k == a.vocab && s.top_p < 1.0f, few = s.hot && s.k < a.vocab && s.k <= MOST_K;
  uint32_t most = P::MASKED;
#pragma unroll
  for (int j = 0; j < JP; ++j) {
    mask_nan<T>(raw[j]);
    most = P::largest(most, piece_top<T>(raw[j]));
  }
  const float mine = P::top(most);
  hold(raw);
  if (few) {
    float y = mine;
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) y = fmaxf(y, __shfl_xor_sync(FULL, y, o));
    if (t % LANES == 0) q.groups[block * SPLIT + t / LANES] = y;
  }
  if (cut)
    for (int i = t; i < STEPS; i += SPLIT) sh.bins[i] = 0;
  // the block's largest, then its lowest token
  const uint32_t high = __reduce_max_sync(FULL, ordered(mine));
  if ((t & 31) == 0) sh.scratch.words[t >> 5] = high;
  if (t == 0) sh.low = 0xffffffffu;
  __syncthreads();
  uint32_t high_u = 0;
#pragma unroll
  for (int w = 0; w < SPLIT / 32; ++w) high_u = max(high_u, (uint32_t)sh.scratch.words[w]);
  const float m = unordered(high_u);
  float sum1 = 0.0f, sum = 0.0f;
  if (m > -INFINITY) {  // (uniform)
    if (mine == m) {
      int at = INT_MAX;
#pragma unroll
      for (int j = 0; j < JP; ++j)
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (P::at(raw[j], i) == m) at = min(at, (g0 + j * SPLIT) * E - row.lead + i);
      atomicMin(&sh.low, (uint32_t)at);
    }
    hold(raw);
#pragma unroll
    for (int j = 0; j < JP; ++j) {
      float y[E];
#pragma unroll
      for (int i = 0; i < E; ++i) y[i] = ex2f((P::at(raw[j], i) - m) * LOG2E);
#pragma unroll
      for (int o = 1; o < E; o <<= 1)
#pragma unroll
        for (int i = 0; i < E; i += 2 * o) y[i] += y[i + o];
      sum1 += y[0];
    }
    if (cut) {
      const float per = steps_per(s.temperature), c = weigh_of(m, s.temperature).hi;
      const bool steps = fabsf(m) * per < MOST_STEP;  // (else the row is done by a block alone, or this part is far below it)
      const int highest = steps ? step_of(m, per) : 0;
      const float least = m - (STEPS + 8) / per;
      hold(raw);
#pragma unroll
      for (int j = 0; j < JP; ++j) {
        if (P::top(piece_top<T>(raw[j])) < least) continue;
        float y = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float x = P::at(raw[j], i);
          y += x > -INFINITY ? ex2f((x - m) * c) : 0.0f;
          if (x >= least && steps) {
            const int step = step_of(x, per), slot = highest - step;
            const float up = (__fmul_rn(x, per) - ((float)step + 0.5f)) * (LOG2E / 32.0f);
            const uint32_t w = __float_as_uint(fmaf(ex2f(up), UNIT, ROUND)) - __float_as_uint(ROUND);
            if (slot < STEPS) atomicAdd(&sh.bins[slot], w);
          }
        }
        sum += y;
      }
    }
  }
  block_sums(sum1, sum, sh.scratch);  // (a barrier behind the steps too)
  if (cut)
    for (int i = t; i < STEPS / 4; i += SPLIT)
      reinterpret_cast<uint4*>(q.steps + block * STEPS)[i] = reinterpret_cast<const uint4*>(sh.bins)[i];
  if (t == 0) q.part[block] = {m > -INFINITY ? place_of(m, (int)sh.low) : 0, sum1, sum};
}

// The noise of E tokens from v on, or 1 where there is none; wide: pieces begin at every 16
// bytes of the noise too, as they do where its rows lie as the logits' do.
template <int E>
__device__ __forceinline__ void noise_of(const float* noise, bool wide, int v, int n, float (&e)[E]) {
  if (wide && v >= 0 && v + E <= n) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>(noise + v + i));
      e[i] = f.x, e[i + 1] = f.y, e[i + 2] = f.z, e[i + 3] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) e[i] = v + i >= 0 && v + i < n ? noise[v + i] : 1.0f;
  }
}
// Races the tokens above the step whose quotient is about `high`: those of the pieces
// first + j * THREADS of each lane that has one (`mine`).  By a whole warp, a token a lane.
template <typename T, int JP, int THREADS>
__device__ __noinline__ void race_again(Race& race, const Row<T>& row, bool mine, int first, float bound, int step, float per,
                                        float c, float high) {
  constexpr int E = Row<T>::E;
  for (unsigned left = __ballot_sync(FULL, mine); left; left &= left - 1) {
    const int g0 = __shfl_sync(FULL, first, __ffs(left) - 1);
#pragma unroll 1
    for (int k = threadIdx.x & 31; k < JP * E; k += 32) {
      const int v = (g0 + k / E * THREADS) * E - row.lead + k % E;
      if (v < 0 || v >= row.n) continue;
      const float x = fmaxf(to_float(row.p[v]), -INFINITY);
      if (!(x >= bound) || x == -INFINITY || (step != INT_MIN && step_of(x, per) <= step)) continue;
      const float w = ex2f((x - race.weigh.top) * c), e = race.noise[v];
      if (__fdividef(w, Race::number(e)) >= high * NEAR_ABOUT) race.enter(x, v, race.weigh(x), e);
    }
  }
}

// The cut that lies among the listed places (there may be none); front: weight in front of
// them, want: what the cut is at.  The step was found with rounded weights, or none was, and
// in one row of some thousands the cut lies right beside it: up to 2^-20 away it is taken at
// the step's end.  0 where it is further off, or cannot be told: no step is trusted unseen.
template <int N>
__device__ uint64_t cut_places(const Places& places, const Weigh& weigh, uint64_t front, uint64_t want, Shared& sh) {
  uint64_t lo = ~0ull, hi = 0, sum = 0;
  for (int i = threadIdx.x; i < places.n; i += N) {
    const uint64_t x = places.p[i];
    lo = min((unsigned long long)lo, (unsigned long long)x);
    hi = max((unsigned long long)hi, (unsigned long long)x);
    sum += fixed(weigh(value_of(x)));
  }
  lo = ~block_max<N>(~lo, sh.scratch);
  hi = block_max<N>(hi, sh.scratch);
  sum = block_sum<N>(sum, sh.scratch);
  if (front >= want) return front - want <= want >> 20 ? ~0ull : 0;
  if (front + sum < want) return want - (front + sum) <= want >> 20 ? lo : 0;
  return find_cut<N, false>(places, weigh, 0, front, want, value_of(lo), value_of(hi), sh);
}

constexpr int STAGE = 1024;  // places that a block brings to the list at most

template <typename T, int JP>
__global__ __launch_bounds__(SPLIT, 4) void k_sample_race(SplitArgs q) {
  using P = Packed<T>;
  constexpr int E = Row<T>::E;
  __shared__ struct {
    uint64_t list[STAGE];
    Scratch scratch;
    int listed, candidates, to;
    uint64_t place[SPLIT];
  } sh;
  const SampleArgs& a = q.a;
  const int64_t r = q.row0 + blockIdx.y, block = blockIdx.y * (int64_t)q.parts + blockIdx.x;
  const Row<T> row(a.logits, a.logits_stride, r, a.vocab);
  const int t = threadIdx.x, g0 = blockIdx.x * (SPLIT * JP) + t;
  griddep_launch_dependents();
  const Setting s = setting_of(a, r);
  if (t == 0) sh.listed = sh.candidates = 0;
  uint4 raw[JP];
#pragma unroll
  for (int j = 0; j < JP; ++j) raw[j] = load_raw(row, g0 + j * SPLIT);
  griddep_wait();
  RowRecord& rec = q.rows[blockIdx.y];
  const Mode mode = rec.mode;
  if (mode == Mode::DONE || mode == Mode::ALONE) return;
  const float bound = rec.bound;
  __syncthreads();
  auto append = [&](float y, int token) {
    const int to = atomicAdd(&sh.listed, 1);
    if (to < STAGE) sh.list[to] = place_of(y, token);
  };
  if (mode == Mode::BOUND) {
    unsigned here = 0;  // pieces that have some
#pragma unroll
    for (int j = 0; j < JP; ++j) {
      mask_nan<T>(raw[j]);
      here |= (unsigned)(P::top(piece_top<T>(raw[j])) >= bound) << j;
    }
    for (; here; here &= here - 1) {  // (read again: few of them)
      const int j = __ffs(here) - 1;
      uint4 u = load_raw(row, g0 + j * SPLIT);
      mask_nan<T>(u);
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (P::at(u, i) >= bound) append(P::at(u, i), (g0 + j * SPLIT) * E - row.lead + i);
    }
    __syncthreads();
  } else {
    const Weigh weigh = weigh_of(value_of(rec.first), s.temperature);
    const float per = steps_per(s.temperature), c = weigh.hi, top = weigh.top;
    const int step = rec.step;
    const float* noise = a.noise + r * a.noise_stride;
    const bool wide = ((uintptr_t)(noise - row.lead) & 15) == 0;
    Race race = {s, weigh, noise, rec.first};
    // weights of one product first (ABOUT): their largest quotient over the block says whom to
    // race.  A piece is weighed while the noise of the next one, which is asked
    // for where some token of it matters, and the one behind are on their way.
    // (A piece at a time, read from L2 again: unrolled, the code is more than the SM's caches hold.)
    float above = 0.0f, most = 0.0f, e0[E], e1[E];
    uint4 u0 = raw[0], u1, next;
    bool need0, need1 = false;
    auto ask = [&](uint4& u, int j, float (&e)[E]) {
      mask_nan<T>(u);
      const float highest = P::top(piece_top<T>(u));
      const bool need = highest >= bound && highest > -INFINITY;
      if (need) noise_of<E>(noise, wide, (g0 + j * SPLIT) * E - row.lead, row.n, e);
      return need;
    };
    next = raw[1];
    need0 = ask(u0, 0, e0);
#pragma unroll 1
    for (int j = 0; j < JP; ++j) {
      u1 = next;
      if (j + 2 < JP) next = load_raw(row, g0 + (j + 2) * SPLIT);
      need1 = j + 1 < JP && ask(u1, j + 1, e1);
      if (need0) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float x = P::at(u0, i);
          const int mine = step == INT_MIN ? 0 : x >= bound ? step_of(x, per) : INT_MIN;
          if (mine > step) {
            const float w = ex2f((x - top) * c);
            above += w;
            if (race.keeps(x, w)) most = fmaxf(most, __fdividef(w, Race::number(e0[i])));
          } else if (mine == step) {
            append(x, (g0 + j * SPLIT) * E - row.lead + i);
          }
        }
      }
      u0 = u1;
      need0 = need1;
#pragma unroll
      for (int i = 0; i < E; ++i) e0[i] = e1[i];
    }
    const float high = block_most(most, above, sh.scratch);  // (and the sum of the weights)
    const bool mine = most > 0.0f && most >= high * NEAR_ABOUT;
    if (__any_sync(FULL, mine)) race_again<T, JP, SPLIT>(race, row, mine, g0, bound, step, per, c, high);
    if (race.winner) sh.place[atomicAdd(&sh.candidates, 1)] = race.winner;
    __syncthreads();
    if (t == 0) {
      uint64_t w = sh.candidates ? sh.place[0] : 0;
      for (int i = 1; i < sh.candidates; ++i) w = race.better(w, sh.place[i]);
      // (its quotient as k_sample_finish takes the list's: `high` is not near enough)
      q.winner[block] = {w, w ? race.weigh(value_of(w)) / Race::number(noise[token_of(w)]) : 0.0f, above};
    }
  }
  // the list, behind what other blocks bring
  const int n = sh.listed;
  if (n == 0) return;
  if (t == 0) sh.to = (int)min(atomicAdd(&rec.listed, (unsigned)(n > STAGE ? MOST_LISTED + 1 : n)), (unsigned)MOST_LISTED + 1);
  __syncthreads();
  uint64_t* list = q.list + blockIdx.y * (int64_t)MOST_LISTED;
  for (int i = t; i < min(n, STAGE); i += SPLIT)
    if (sh.to + i < MOST_LISTED) list[sh.to + i] = sh.list[i];
}

// The rest of a row: the list's cut and its race, the parts' winners.  A block per row.
template <typename T>
__global__ __launch_bounds__(SPLIT) void k_sample_finish(SplitArgs q) {
  __shared__ Shared sh;
  const SampleArgs& a = q.a;
  const int64_t r = q.row0 + blockIdx.x;
  const int t = threadIdx.x;
  const Setting s = setting_of(a, r);
  griddep_wait();
  const RowRecord rec = q.rows[blockIdx.x];
  if (rec.mode == Mode::DONE) return;
  const int listed = (int)rec.listed;
  if (rec.mode == Mode::ALONE || listed > (rec.mode == Mode::BOUND ? LIST : MOST_LISTED)) {
    whole_row<SPLIT, T>(a, r, sh);
    return;
  }
  const uint64_t* list = q.list + blockIdx.x * (int64_t)MOST_LISTED;
  const Weigh weigh = weigh_of(value_of(rec.first), s.temperature);
  Race race = {s, weigh, a.noise + r * a.noise_stride, rec.first};
  if (rec.mode == Mode::BOUND) {
    for (int i = t; i < listed; i += SPLIT) sh.list[i] = list[i];
    sort_list<SPLIT>(sh, listed);
    const int n = cut_list<SPLIT>(s, weigh, listed, sh);
    for (int i = t; i < n; i += SPLIT) race.enter(value_of(sh.list[i]), token_of(sh.list[i]));
  } else {
    PartWinner w = {0, 0.0f, 0.0f};
    if (t < q.parts) w = q.winner[blockIdx.x * (int64_t)q.parts + t];
    if (w.place) {
      race.best = w.best;
      race.winner = w.place;
    }
    if (rec.step != INT_MIN) {
      const uint64_t want = part_of(s.top_p, rec.sum), front = block_sum<SPLIT>(fixed(w.above), sh.scratch);
      const uint64_t cut = cut_places<SPLIT>({list, listed}, weigh, front, want, sh);
      if (cut == 0) {  // (uniform)
        whole_row<SPLIT, T>(a, r, sh);
        return;
      }
      for (int i = t; i < listed; i += SPLIT) {
        const uint64_t x = list[i];
        if (x >= cut) race.enter(value_of(x), token_of(x));
      }
    }
  }
  float best;
  const uint64_t winner = block_winner<SPLIT>(race, sh, best);
  if (t == 0) finish(a, r, winner ? winner : rec.first, weigh.top, rec.sum1);  // (none: every quotient is 0)
}

// ---- a row of up to 8 pieces a thread by one block, held in registers --------
//
// The four kernels' steps in one: no round trip over memory in between.
constexpr int ONE = 1024;
struct OneShared {
  Shared sh;
  uint64_t places[LIST];
  uint32_t steps[STEPS];
  float most[ONE / 32], sums[2][ONE / 32];
};

template <typename T, int JP>
__global__ __launch_bounds__(ONE) void k_sample_one(SampleArgs a) {
  using P = Packed<T>;
  constexpr int E = Row<T>::E;
  constexpr float UNIT = unit_of(ONE * JP * E);
  static_assert(UNIT >= 0x1p15f && UNIT <= 0x1p22f, "weights to 2^-16, sums to 2^31");
  extern __shared__ unsigned char raw_smem[];
  OneShared& one = *reinterpret_cast<OneShared*>(raw_smem);
  Shared& sh = one.sh;
  const int64_t r = blockIdx.x;
  const Row<T> row(a.logits, a.logits_stride, r, a.vocab);
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  uint4 raw[JP];
#pragma unroll
  for (int j = 0; j < JP; ++j) raw[j] = load_raw(row, t + j * ONE);
  const Setting s = setting_of(a, r);
  const bool cut = s.hot && s.k == a.vocab && s.top_p < 1.0f;
  const float* noise = a.noise + r * a.noise_stride;
  uint32_t packed = P::MASKED;
#pragma unroll
  for (int j = 0; j < JP; ++j) {
    mask_nan<T>(raw[j]);
    packed = P::largest(packed, piece_top<T>(raw[j]));
  }
  const float mine = P::top(packed);
  hold(raw);
  if (t < STEPS) one.steps[t] = 0;
  for (int i = t; i < BINS; i += ONE) sh.bins[i] = 0;
  // the row's largest and smallest thread's largest, then the lowest token
  const uint32_t high = __reduce_max_sync(FULL, ordered(mine));
  const uint32_t low = __reduce_max_sync(FULL, mine > -INFINITY ? ~ordered(mine) : 0u);
  if (lane == 0) sh.scratch.words[warp] = (uint64_t)high << 32 | low;
  if (t == 0) {
    sh.low = 0xffffffffu;
    sh.listed = sh.candidates = 0;
    sh.bin = -1;
  }
  __syncthreads();
  const uint64_t word = sh.scratch.words[lane];
  const float top = unordered(__reduce_max_sync(FULL, (uint32_t)(word >> 32)));
  const float least_top = unordered(~__reduce_max_sync(FULL, (uint32_t)word));
  if (top == -INFINITY) {
    if (t == 0) finish(a, r, 0, 0.0f, 0);
    return;
  }
  const float per = steps_per(s.temperature);
  const bool alone = top == INFINITY || (s.hot && (s.k < a.vocab ? s.k > MOST_K : s.top_p < 1.0f && !(fabsf(top) * per < MOST_STEP)));
  if (alone) {  // (uniform)
    __syncthreads();
    whole_row<ONE, T>(a, r, sh);
    return;
  }
  const Weigh weigh = weigh_of(top, s.hot ? s.temperature : 1.0f);
  const float c = weigh.hi;
  if (mine == top) {
    int at = INT_MAX;
#pragma unroll
    for (int j = 0; j < JP; ++j)
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (P::at(raw[j], i) == top) at = min(at, (t + j * ONE) * E - row.lead + i);
    atomicMin(&sh.low, (uint32_t)at);
  }
  hold(raw);
  const Weigh plain = weigh_of(top, 1.0f);  // (to 2^-22: a lone row's log-probability shows it)
  float sum1 = 0.0f, sum = 0.0f;
#pragma unroll
  for (int j = 0; j < JP; ++j) {
    float y[E];
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = plain(P::at(raw[j], i));
#pragma unroll
    for (int o = 1; o < E; o <<= 1)
#pragma unroll
      for (int i = 0; i < E; i += 2 * o) y[i] += y[i + o];
    sum1 += y[0];
  }
  hold(raw);
  const int highest = cut ? step_of(top, per) : 0;
  if (cut) {
    const float least = top - (STEPS + 8) / per;
#pragma unroll
    for (int j = 0; j < JP; ++j) {
      if (P::top(piece_top<T>(raw[j])) < least) continue;
      float y = 0.0f;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float x = P::at(raw[j], i);
        if (x >= least) {
          y += ex2f((x - top) * c);
          const int step = step_of(x, per), slot = highest - step;
          const float up = (__fmul_rn(x, per) - ((float)step + 0.5f)) * (LOG2E / 32.0f);
          const uint32_t w = __float_as_uint(fmaf(ex2f(up), UNIT, ROUND)) - __float_as_uint(ROUND);
          if (slot < STEPS) atomicAdd(&one.steps[slot], w);
        }
      }
      sum += y;
    }
  } else if (s.hot && s.k < a.vocab && mine > -INFINITY) {
    // how many threads' largest lie in each of equal steps
    const float bins_per = top > least_top ? (BINS - 1) / (top - least_top) : 0.0f;
    atomicAdd(&sh.bins[(int)fminf((top - mine) * bins_per, (float)(BINS - 1))], 1u);
  }
  sum1 = warp_sum(sum1);
  sum = warp_sum(sum);
  if (lane == 0) {
    one.sums[0][warp] = sum1;
    one.sums[1][warp] = sum;
  }
  __syncthreads();
  const uint64_t total1 = fixed(warp_sum(one.sums[0][lane])), total = fixed(warp_sum(one.sums[1][lane]));
  const uint64_t first = place_of(top, (int)sh.low);
  if (!s.hot) {
    if (t == 0) finish(a, r, first, top, total1);
    return;
  }
  Race race = {s, weigh, noise, first};
  auto append = [&](float y, int token) {
    const int to = atomicAdd(&sh.listed, 1);
    if (to < LIST) one.places[to] = place_of(y, token);
  };
  if (s.k < a.vocab) {
    // ---- the values that k threads' largest reach, sorted
    uint64_t all;
    const uint64_t some = sh.bins[2 * t] + sh.bins[2 * t + 1], upto = block_scan<ONE>(some, sh.scratch, all);
    if (upto < (uint64_t)s.k && upto + some >= (uint64_t)s.k) sh.bin = upto + sh.bins[2 * t] >= (uint64_t)s.k ? 2 * t : 2 * t + 1;
    __syncthreads();
    const int bin = sh.bin;
    if (bin < 0) {  // (fewer threads with tokens than k)
      whole_row<ONE, T>(a, r, sh);
      return;
    }
    const float bins_per = top > least_top ? (BINS - 1) / (top - least_top) : 0.0f;
    const float reach = bins_per > 0.0f ? top - (bin + 2) / bins_per : -INFINITY;  // (a little below the bin's end)
#pragma unroll
    for (int j = 0; j < JP; ++j)
      if (P::top(piece_top<T>(raw[j])) >= reach && P::top(piece_top<T>(raw[j])) > -INFINITY) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float x = P::at(raw[j], i);
          if (x > -INFINITY && (int)fminf((top - x) * bins_per, (float)(BINS - 1)) <= bin)
            append(x, (t + j * ONE) * E - row.lead + i);
        }
      }
    __syncthreads();
    const int n = sh.listed;
    __syncthreads();
    if (n > LIST) {
      whole_row<ONE, T>(a, r, sh);
      return;
    }
    for (int i = t; i < n; i += ONE) sh.list[i] = one.places[i];
    sort_list<ONE>(sh, n);
    const int kept = cut_list<ONE>(s, weigh, n, sh);
    for (int i = t; i < kept; i += ONE) race.enter(value_of(sh.list[i]), token_of(sh.list[i]));
  } else {
    // ---- what lies above the step that top-p's cut is in; what lies in it
    int step = INT_MIN;
    float bound = -INFINITY;
    const uint64_t want = cut ? part_of(s.top_p, total) : 0;
    if (cut) {
      const float up = ((float)(highest - t) + 0.5f - top * per) * (1.0f / 32.0f);
      const uint64_t w = (uint64_t)((float)one.steps[t] * (FIXED / UNIT) * ex2f(up * LOG2E));
      uint64_t all;
      const uint64_t upto = block_scan<ONE>(w, sh.scratch, all);
      if (w && upto < want && upto + w >= want) sh.bin = t;
      __syncthreads();
      step = highest - (sh.bin < 0 ? STEPS - 1 : sh.bin);
      bound = ((float)step - 0.51f) / per;
      bound -= fabsf(bound) * 0x1p-21f;
    } else if (s.min_p > 0.0f) {
      bound = least_kept(s, top);
    }
    const bool wide = ((uintptr_t)(noise - row.lead) & 15) == 0;
    float above = 0.0f, most = 0.0f;
#pragma unroll
    for (int j = 0; j < JP; ++j) {
      const float here = P::top(piece_top<T>(raw[j]));
      if (!(here >= bound) || here == -INFINITY) continue;
      const int v = (t + j * ONE) * E - row.lead;
      float e[E];
      noise_of<E>(noise, wide, v, row.n, e);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float x = P::at(raw[j], i);
        const int at = step == INT_MIN ? 0 : x >= bound ? step_of(x, per) : INT_MIN;
        if (at > step) {
          const float w = ex2f((x - top) * c);
          above += w;
          if (race.keeps(x, w)) most = fmaxf(most, __fdividef(w, Race::number(e[i])));
        } else if (at == step) {
          append(x, v + i);
        }
      }
    }
    const float warp_most = __uint_as_float(__reduce_max_sync(FULL, __float_as_uint(most)));
    above = warp_sum(above);
    if (lane == 0) {
      one.most[warp] = warp_most;
      one.sums[0][warp] = above;
    }
    __syncthreads();
    const float high_q = __uint_as_float(__reduce_max_sync(FULL, __float_as_uint(one.most[lane])));
    const bool ahead = most > 0.0f && most >= high_q * NEAR_ABOUT;
    if (__any_sync(FULL, ahead)) race_again<T, JP, ONE>(race, row, ahead, t, bound, step, per, c, high_q);
    const int listed = sh.listed;
    if (cut) {
      const uint64_t front = fixed(warp_sum(one.sums[0][lane]));
      const uint64_t at = listed <= LIST ? cut_places<ONE>({one.places, listed}, weigh, front, want, sh) : 0;
      if (at == 0) {  // (uniform)
        __syncthreads();
        whole_row<ONE, T>(a, r, sh);
        return;
      }
      for (int i = t; i < listed; i += ONE) {
        const uint64_t x = one.places[i];
        if (x >= at) race.enter(value_of(x), token_of(x));
      }
    }
  }
  float best;
  const uint64_t winner = block_winner<ONE>(race, sh, best);
  if (t == 0) finish(a, r, winner ? winner : first, top, total1);
}

// Parts of a row of pieces of E tokens, JP of them a thread (and one more piece than it
// has, where it begins within one).
int64_t parts_of(int64_t vocab, int each, int jp) {
  return (vocab + each - 1 + (int64_t)SPLIT * jp * each - 1) / ((int64_t)SPLIT * jp * each);
}

size_t round_up(size_t x) { return (x + 255) / 256 * 256; }

struct Sizes {
  size_t rows, part, winner, groups, steps, list, total;
};
Sizes sizes_of(int64_t rows, int64_t blocks) {
  Sizes z;
  z.rows = round_up(rows * sizeof(RowRecord));
  z.part = round_up(blocks * sizeof(PartRecord));
  z.winner = round_up(blocks * sizeof(PartWinner));
  z.groups = round_up(blocks * SPLIT * sizeof(float));
  z.steps = round_up(blocks * STEPS * sizeof(uint32_t));
  z.list = round_up(rows * MOST_LISTED * sizeof(uint64_t));
  z.total = z.rows + z.part + z.winner + z.groups + z.steps + z.list;
  return z;
}

template <typename T, int JP>
cudaError_t one_block(const SampleArgs& a, int64_t n, cudaStream_t s) {
  auto* kernel = k_sample_one<T, JP>;
  const cudaError_t e = set_max_dynamic_smem(reinterpret_cast<const void*>(kernel), sizeof(OneShared));
  if (e != cudaSuccess) return e;
  kernel<<<(unsigned)n, ONE, sizeof(OneShared), s>>>(a);
  return cudaGetLastError();
}

// Shared memory that k_sample_finish asks for and does not use: two of its blocks to an SM.  They
// start where k_sample_race's blocks end, three to an SM where they may, and then a row that is
// left to whole_row waits for its neighbours: 64 rows of 128,000 bf16 with top-k 1,000 took 348
// us, 286 this way, 48 flat float32 rows 55.8 and 54.8; one to an SM: 256 and 53.3, but 256 rows
// of all settings 106.2 instead of 104.6.
constexpr size_t SPREAD = 80 * 1024;

template <typename T>
cudaError_t sample(const SampleArgs& a, int64_t n, void* workspace, cudaStream_t s) {
  constexpr int E = Row<T>::E;
  const int64_t wide = parts_of(a.vocab, E, 8), narrow = parts_of(a.vocab, E, 2);
  const int64_t pieces = (a.vocab + 2 * E - 2) / E;  // (and one more, where a row begins within one)
  if (pieces <= 256) {
    k_sample_row<256, T><<<(unsigned)n, 256, 0, s>>>(a);
    return cudaGetLastError();
  }
  if (pieces <= 8 * ONE) return pieces <= 2 * ONE ? one_block<T, 2>(a, n, s) : pieces <= 4 * ONE ? one_block<T, 4>(a, n, s) : one_block<T, 8>(a, n, s);
  if (wide > MOST_PARTS) {
    k_sample_row<1024, T><<<(unsigned)n, 1024, 0, s>>>(a);
    return cudaGetLastError();
  }
  const bool few = n * wide < FEW_BLOCKS && narrow <= MOST_PARTS;
  const int64_t parts = few ? narrow : wide;
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
  const int jp = few ? 2 : 8;
  const cudaError_t spread = set_max_dynamic_smem(reinterpret_cast<const void*>(k_sample_finish<T>), SPREAD);
  if (spread != cudaSuccess) return spread;
  for (q.row0 = 0; q.row0 < n; q.row0 += rows) {
    const dim3 grid((unsigned)parts, (unsigned)std::min(rows, n - q.row0)), per_row(grid.y), block(SPLIT);
    (few ? k_sample_parts<T, 2> : k_sample_parts<T, 8>)<<<grid, block, 0, s>>>(q);
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess)
      e = launch_maybe_pdl(true, k_sample_cut, per_row, block, 0, s, q, SPLIT * jp * E / GROUP, unit_of(SPLIT * jp * E));
    if (e == cudaSuccess) e = launch_maybe_pdl(true, few ? k_sample_race<T, 2> : k_sample_race<T, 8>, grid, block, 0, s, q);
    if (e == cudaSuccess) e = launch_maybe_pdl(true, k_sample_finish<T>, per_row, block, SPREAD, s, q);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

// Enough for every smaller call too, whatever the type: rows of a launch, and the blocks
// that either form has of float32.
size_t sample_workspace(int64_t n, int64_t vocab) {
  if (n == 0 || parts_of(vocab, 4, 2) == 1) return 0;
  const int64_t wide = std::min<int64_t>(parts_of(vocab, 4, 8), MOST_PARTS), rows = std::min<int64_t>(n, MOST_ROWS);
  const int64_t few = std::min<int64_t>(n * parts_of(vocab, 4, 2), 4 * FEW_BLOCKS + rows);
  return sizes_of(rows, std::max(std::min<int64_t>(rows * wide, MOST_BLOCKS), few)).total;
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
