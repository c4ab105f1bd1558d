// tq_verify_drafts: drafted tokens accepted or rejected by the target's
// probabilities, and the token behind the accepted ones drawn from what is
// left of the target's row.
//
// A sequence accepts its first drafts with u_i q_i(x_i) < p_i(x_i).  Behind them
// one token is drawn from weights w (max(p - q, 0) after a rejection, p without
// one) by a race: with noise(v) exponentially distributed, argmax_v w(v) /
// noise(v) is distributed as w.  Unlike the inverse of a running sum, an argmax
// does not depend on the order in which it is taken, so the row can be split
// over many blocks.
//
// k_verify: several blocks per sequence settle the acceptance each for
// themselves (a few loads), then race over a part of one row; their winners
// go to the workspace as 64-bit keys (weight's bits, then the token
// inverted).  k_verify_finish: a block per sequence takes the largest key and
// writes the tokens.  It may start while k_verify still writes the keys, so they
// are not read-only to it.
//
// Bound: HBM, one row of the target's probabilities, the noise, and after a
// rejection the draft's row, read once per sequence; 256 sequences over 128,000
// bfloat16 entries (249 MB): 54 us, 4.6 TB/s, on inputs that change from call to call.
// (In a graph, on one set of inputs, part of them in L2: 46; with 8 blocks of a call
// per SM 52, with 32 54.)
#include <algorithm>

#include "tq_kv.cuh"
#include "tq_topk.cuh"

namespace tq {
namespace {

constexpr int VERIFY = 256;
constexpr int VERIFY_MIN = 2048;  // vocabulary entries that are worth a block
constexpr int PER_SM = 16;        // blocks of a call per SM, twice what fits: the shorter ones even out

struct Verdict {
  int accepted;   // drafts accepted
  int drafts;     // drafts the sequence had
  int rejected;   // token of the rejected draft, or -1
};

template <typename T>
__device__ Verdict judge(const T* __restrict__ target, const T* __restrict__ draft, const int32_t* __restrict__ drafts,
                         const int32_t* __restrict__ draft_lens, const float* __restrict__ uniforms, int64_t i, int t,
                         int vocab) {
  // every warp for itself: lane l judges drafts l and l + 32
  const int lane = threadIdx.x & 31;
  Verdict r;
  r.drafts = draft_lens ? min(max(draft_lens[i], 0), t) : t;
  unsigned long long good = 0;
  for (int base = 0; base < r.drafts; base += 32) {
    const int j = base + lane;
    bool ok = false;
    if (j < r.drafts) {
      const int x = drafts[i * t + j];
      if (x >= 0 && x < vocab) {
        const float p = to_float(target[(i * (t + 1) + j) * vocab + x]);
        const float q = draft ? to_float(draft[(i * t + j) * vocab + x]) : 1.0f;
        ok = __fmul_rn(uniforms[i * t + j], q) < p;
      }
    }
    good |= (unsigned long long)__ballot_sync(0xffffffffu, ok) << base;
  }
  r.accepted = ~good ? __ffsll((long long)~good) - 1 : 64;
  r.accepted = min(r.accepted, r.drafts);
  r.rejected = r.accepted < r.drafts ? drafts[i * t + r.accepted] : -1;
  return r;
}

// Key of a racer: larger weights first, then lower tokens.  Weights are >= 0,
// so their bits order as they do.
__device__ __forceinline__ uint64_t race_key(float w, int v) {
  return (uint64_t)__float_as_uint(w) << 32 | (uint32_t)~v;
}

// EACH neighbours of a row, from 16-byte loads where the row allows them.
constexpr int EACH = 8;

template <typename T>
__device__ __forceinline__ void load_each(const T* __restrict__ p, float (&x)[EACH]) {
  union {
    uint4 v[EACH * sizeof(T) / 16];
    T e[EACH];
  } u;
#pragma unroll
  for (int c = 0; c < (int)(EACH * sizeof(T) / 16); ++c) u.v[c] = __ldcs(reinterpret_cast<const uint4*>(p) + c);
#pragma unroll
  for (int j = 0; j < EACH; ++j) x[j] = to_float(u.e[j]);
}

// The race over tokens [begin, end); begin is a multiple of EACH.  A quotient that
// could win is a correctly rounded division; most are ruled out before, by
// w < 0.999999 best * noise (the margin is more than the products round; below
// float32's normal range both sides are multiples of one step, and the product's
// rounding is at most half of it).
template <typename T>
__device__ uint64_t race(const T* __restrict__ p, const T* __restrict__ q, int without, const float* __restrict__ noise,
                         int begin, int end) {
  float best = 0.0f, bar = 0.0f;
  int token = -1;
  const bool wide = (((uintptr_t)p | (uintptr_t)q | (uintptr_t)noise) & 15u) == 0;
  for (int base = begin; base < end; base += VERIFY * EACH) {
    // aligned rows: a thread's tokens lie side by side, else VERIFY apart
    const bool whole = base + VERIFY * EACH <= end && wide;
    const int first = base + (int)threadIdx.x * (whole ? EACH : 1), stride = whole ? 1 : VERIFY;
    float w[EACH], e[EACH];
    if (whole) {
      load_each(p + first, w);
      load_each(noise + first, e);
      if (q) {
        float x[EACH];
        load_each(q + first, x);
#pragma unroll
        for (int j = 0; j < EACH; ++j) w[j] -= x[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const int v = first + j * VERIFY;
        w[j] = v < end ? to_float(p[v]) : 0.0f;
        e[j] = v < end ? noise[v] : 1.0f;
        if (q && v < end) w[j] -= to_float(q[v]);
      }
    }
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const int v = first + j * stride;
      if (!(w[j] >= fmaxf(bar * e[j], 0x1p-149f)) || v == without) continue;  // (0x1p-149: weights that are 0 or less)
      const float x = __fdiv_rn(w[j], e[j]);
      if (x > best) {
        best = x;
        bar = best * 0.999999f;
        token = v;
      }
    }
  }
  return token < 0 ? 0 : race_key(best, token);
}

__device__ __forceinline__ uint64_t warp_max(uint64_t key) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const uint64_t other = __shfl_xor_sync(0xffffffffu, key, o);
    key = other > key ? other : key;
  }
  return key;
}

__device__ uint64_t block_max(uint64_t key, uint64_t* shared) {
  key = warp_max(key);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = key;
  __syncthreads();
  return warp_max((threadIdx.x & 31) < VERIFY / 32 ? shared[threadIdx.x & 31] : 0);
}

template <typename T>
__global__ __launch_bounds__(VERIFY) void k_verify(const T* __restrict__ target, const T* __restrict__ draft,
                                                   const int32_t* __restrict__ drafts,
                                                   const int32_t* __restrict__ draft_lens,
                                                   const float* __restrict__ uniforms, const float* __restrict__ noise,
                                                   int64_t n, int t, int vocab, uint64_t* __restrict__ keys) {
  __shared__ uint64_t shared[VERIFY / 32];
  const int64_t i = blockIdx.y;
  griddep_launch_dependents();
  const int each = ((vocab + gridDim.x - 1) / gridDim.x + EACH - 1) / EACH * EACH;
  const int begin = blockIdx.x * each, end = min(vocab, begin + each);
  // which row of the probabilities it is follows from the verdict; the noise is known before
  if (begin + (int)threadIdx.x * 32 < end)
    asm volatile("prefetch.global.L2 [%0];" ::"l"(noise + i * vocab + begin + threadIdx.x * 32));
  const Verdict r = judge(target, draft, drafts, draft_lens, uniforms, i, t, vocab);
  const bool rejected = r.accepted < r.drafts;
  const T* q = rejected && draft ? draft + (i * t + r.accepted) * vocab : nullptr;
  uint64_t key = race(target + (i * (t + 1) + r.accepted) * vocab, q, rejected && !draft ? r.rejected : -1,
                      noise + i * vocab, begin, end);
  key = block_max(key, shared);
  if (threadIdx.x == 0) keys[i * gridDim.x + blockIdx.x] = key;
}

template <typename T>
__global__ __launch_bounds__(VERIFY) void k_verify_finish(const T* __restrict__ target, const T* __restrict__ draft,
                                                          const int32_t* __restrict__ drafts,
                                                          const int32_t* __restrict__ draft_lens,
                                                          const float* __restrict__ uniforms,
                                                          const float* __restrict__ noise, int64_t n, int t, int vocab,
                                                          const uint64_t* keys, int parts,
                                                          int32_t* __restrict__ tokens, int32_t* __restrict__ accepted) {
  __shared__ uint64_t shared[2][VERIFY / 32];
  const int64_t i = blockIdx.x;
  const Verdict r = judge(target, draft, drafts, draft_lens, uniforms, i, t, vocab);
  griddep_wait();  // (the verdict needs the call's inputs alone)
  uint64_t key = 0;
  for (int j = threadIdx.x; j < parts; j += VERIFY) key = max(key, keys[i * parts + j]);
  key = block_max(key, shared[0]);
  if (key == 0 && r.accepted < r.drafts)  // nothing is left of the row: draw from the row itself
    key = block_max(race<T>(target + (i * (t + 1) + r.accepted) * vocab, nullptr, -1, noise + i * vocab, 0, vocab),
                    shared[1]);
  const int drawn = key ? (int)~(uint32_t)key : 0;
  for (int j = threadIdx.x; j <= t; j += VERIFY)
    tokens[i * (t + 1) + j] = j < r.accepted ? drafts[i * t + j] : j == r.accepted ? drawn : -1;
  if (threadIdx.x == 0) accepted[i] = r.accepted;
}

// Blocks per sequence: enough for every SM to have several, none with less
// than VERIFY_MIN entries.
int verify_parts(int64_t n, int64_t vocab) {
  const int64_t most = (vocab + VERIFY_MIN - 1) / VERIFY_MIN;
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, (int64_t)device_sm_count() * PER_SM / n));
}

template <typename T>
cudaError_t verify(const void* target, const void* draft, const int32_t* drafts, const int32_t* draft_lens,
                   const float* uniforms, const float* noise, int64_t n, int t, int vocab, int32_t* tokens,
                   int32_t* accepted, void* workspace, cudaStream_t s) {
  const int parts = verify_parts(n, vocab);
  uint64_t* keys = static_cast<uint64_t*>(workspace);
  k_verify<T><<<dim3(parts, (unsigned)n), VERIFY, 0, s>>>(static_cast<const T*>(target), static_cast<const T*>(draft),
                                                          drafts, draft_lens, uniforms, noise, n, t, vocab, keys);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_maybe_pdl(true, k_verify_finish<T>, dim3((unsigned)n), dim3(VERIFY), 0, s,
                          static_cast<const T*>(target), static_cast<const T*>(draft), drafts, draft_lens, uniforms,
                          noise, n, t, vocab, static_cast<const uint64_t*>(keys), parts, tokens, accepted);
}

}  // namespace

// Enough for every smaller batch too, which may be split further.
size_t verify_workspace(int64_t n, int64_t vocab) {
  return (size_t)std::max<int64_t>(n, (int64_t)device_sm_count() * PER_SM) * sizeof(uint64_t);
}

cudaError_t launch_verify(const void* target, const void* draft, int type, const int32_t* drafts,
                          const int32_t* draft_lens, const float* uniforms, const float* noise, int64_t n, int t,
                          int vocab, int32_t* tokens, int32_t* accepted, void* workspace, cudaStream_t s) {
  switch (type) {
    case TQ_BF16:
      return verify<__nv_bfloat16>(target, draft, drafts, draft_lens, uniforms, noise, n, t, vocab, tokens, accepted,
                                   workspace, s);
    case TQ_FP16:
      return verify<__half>(target, draft, drafts, draft_lens, uniforms, noise, n, t, vocab, tokens, accepted,
                            workspace, s);
    default:
      return verify<float>(target, draft, drafts, draft_lens, uniforms, noise, n, t, vocab, tokens, accepted,
                           workspace, s);
  }
}

}  // namespace tq
