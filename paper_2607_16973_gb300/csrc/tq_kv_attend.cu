// tq_kv_attend: causal attention of the last tokens of each sequence over the
// 8-bit cache.
//
// out = sum_j e^(s_j) v_j / sum_j e^(s_j), s_j = scale * q . k_j, with the running
// maximum m and sum l of the softmax: one pass over the tokens a query sees.
// A warp takes one query of one head; lane l holds D / 32 of its elements.
#include <algorithm>

#include "tq_kv.cuh"

namespace tq {
namespace {

constexpr int ATTEND_WARPS = 8;

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <typename T, int D, int CODES>
__global__ __launch_bounds__(ATTEND_WARPS * 32) void k_kv_attend(KvView kv, int layer,
                                                                 const int32_t* __restrict__ slots,
                                                                 const int32_t* __restrict__ starts, int64_t n,
                                                                 KvRows q, int64_t total, int heads, float scale,
                                                                 int window, T* __restrict__ out,
                                                                 float* __restrict__ lse) {
  constexpr int E = D / 32;  // elements of a lane
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * ATTEND_WARPS + (threadIdx.x >> 5);
  if (w >= total * heads) return;
  const int64_t token = w / heads;
  const int head = (int)(w % heads), kv_head = head / (heads / kv.c.kv_heads);
  const int64_t i = warp_last_not_above(n, token, [&](int64_t j) { return (int64_t)starts[j]; });
  KvSeq seq;
  const bool ok = kv_seq(kv, slots, starts, i, total, true, seq);
  if (!ok && lane == 0) kv_status(kv, kKvBadEntry);
  const int place = ok ? seq.len - seq.count + (int)(token - seq.token) : -1;
  const T* x = static_cast<const T*>(q.p) + token * q.token_stride + head * q.head_stride + lane * E;
  float qv[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    qv[e] = to_float(x[e]) * scale;
    o[e] = 0.0f;
  }
  for (int t = window ? max(0, place - window + 1) : 0; t <= place; ++t) {
    const int page = kv.c.table[seq.slot * kv.c.max_pages + (t >> kv.page_shift)];
    if (page < 0 || page >= kv.c.pages) {
      if (lane == 0) kv_status(kv, kKvBadEntry);
      break;
    }
    const int inside = t & (kv.c.page_tokens - 1);
    const int64_t at = kv.codes_at(layer, page, kv_head) + (int64_t)inside * D + lane * E;
    const int64_t sat = kv.scales_at(layer, page, kv_head) + inside / kKvBlock;
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += qv[e] * kv_value<CODES>(kv.c.k[at + e], 0);
#pragma unroll
    for (int b = 16; b; b >>= 1) s += __shfl_xor_sync(0xffffffffu, s, b);
    s *= kv.c.k_scale[sat];
    const float top = fmaxf(m, s), keep = expf(m - top), p = expf(s - top);
    const float pv = p * kv.c.v_scale[sat];
    l = l * keep + p;
    m = top;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * keep + pv * kv_value<CODES>(kv.c.v[at + e], 0);
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  T* y = out + (token * heads + head) * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = from_float<T>(o[e] * inv);
  if (lse && lane == 0) lse[token * heads + head] = l > 0.0f ? m + logf(l) : -INFINITY;
}

template <typename T, int D>
cudaError_t attend(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                   const KvRows& q, int64_t total, int heads, float scale, int window, void* out, float* lse,
                   cudaStream_t s) {
  const unsigned grid = (unsigned)((total * heads + ATTEND_WARPS - 1) / ATTEND_WARPS);
  (kv.c.codes == TQ_KV_INT8 ? k_kv_attend<T, D, TQ_KV_INT8> : k_kv_attend<T, D, TQ_KV_E4M3>)<<<grid, ATTEND_WARPS * 32, 0, s>>>(
      kv, layer, slots, starts, n, q, total, heads, scale, window, static_cast<T*>(out), lse);
  return cudaGetLastError();
}

template <typename T>
cudaError_t attend_for(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                       const KvRows& q, int64_t total, int heads, float scale, int window, void* out, float* lse,
                       cudaStream_t s) {
  return (kv.c.head_dim == 64    ? attend<T, 64>
          : kv.c.head_dim == 128 ? attend<T, 128>
                                 : attend<T, 256>)(kv, layer, slots, starts, n, q, total, heads, scale, window, out,
                                                   lse, s);
}

}  // namespace

size_t kv_attend_workspace(const KvView&, int64_t, int64_t, int) { return 16; }

cudaError_t launch_kv_attend(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                             const KvRows& q, int type, int64_t total, int heads, float scale, int window, void* out,
                             float* lse, void* workspace, cudaStream_t s) {
  return (type == TQ_BF16 ? attend_for<__nv_bfloat16> : attend_for<__half>)(kv, layer, slots, starts, n, q, total,
                                                                            heads, scale, window, out, lse, s);
}

}  // namespace tq
