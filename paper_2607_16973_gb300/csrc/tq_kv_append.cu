// tq_kv_append: new keys and values quantised into the cache's pages.
//
// A warp takes one block of 16 tokens of one head, of K or of V: it reads the
// block's new elements once into registers, takes their largest magnitude,
// settles the block's scale, brings the codes of older tokens of the block to
// it where it grew, and writes the new codes.  Nothing is shared between
// warps, so there is one launch and no scratch.
//
// Bound: HBM, 2 + 1 bytes per element (16-bit input); for single tokens
// (a decoding step) the latency of the chain starts -> lens -> table -> codes.
// 64 single tokens: 13 us a call, 4.1 on the GPU.  Prompts (154 MB) on inputs that
// change from call to call: 39 us, 4.0 TB/s.  In a graph, on one set of inputs (part
// of them in L2): 34 us; 72 with a division for every element, 53 with a test for
// each that a product may round otherwise.
#include <algorithm>
#include <cstdint>

#include "tq_kv.cuh"

namespace tq {
namespace {

constexpr int APPEND_WARPS = 8;

// Codes of a chunk by the definition: divided, NaN and everything at scale 0 to 0,
// infinities to the ends.  A call, because it is rare and eight of it would not
// stay in the instruction cache.
template <typename T, int CODES>
__device__ __noinline__ uint2 exact_codes(uint4 raw, float s) {
  union {
    uint4 u;
    T e[16 / sizeof(T)];
  } r;
  r.u = raw;
  float y[8] = {};
#pragma unroll
  for (int j = 0; j < (int)(16 / sizeof(T)); ++j) {
    const float a = to_float(r.e[j]);
    y[j] = s > 0.0f && a == a ? __fdiv_rn(a, s) : 0.0f;
    y[j] = fminf(fmaxf(y[j], -kv_qmax<CODES>()), kv_qmax<CODES>());
  }
  return make_uint2(kv_pack4<CODES>(y[0], y[1], y[2], y[3]), kv_pack4<CODES>(y[4], y[5], y[6], y[7]));
}

// The largest finite magnitude of a chunk.
template <typename T>
__device__ __noinline__ float finite_top(uint4 raw) {
  union {
    uint4 u;
    T e[16 / sizeof(T)];
  } r;
  r.u = raw;
  float top = 0.0f;
#pragma unroll
  for (int j = 0; j < (int)(16 / sizeof(T)); ++j) {
    const float a = fabsf(to_float(r.e[j]));
    if (a < INFINITY) top = fmaxf(top, a);  // (not for NaN)
  }
  return top;
}

// kv_pack4 of four products.
template <int CODES>
__device__ __forceinline__ uint32_t pack_products(const float* x, float f) {
  if (CODES == TQ_KV_INT8) {
    const float m = 12582912.0f;  // (as in kv_pack4; the sum rounds the exact product)
    const uint32_t ab = __byte_perm(__float_as_uint(fmaf(x[0], f, m)), __float_as_uint(fmaf(x[1], f, m)), 0x0040);
    const uint32_t cd = __byte_perm(__float_as_uint(fmaf(x[2], f, m)), __float_as_uint(fmaf(x[3], f, m)), 0x0040);
    return __byte_perm(ab, cd, 0x5410);
  }
  return kv_pack4<CODES>(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}

template <typename T, int D, int CODES, bool VEC>
__global__ __launch_bounds__(APPEND_WARPS * 32, kKvBlock * D * sizeof(T) <= 4096 ? 4 : 1) void k_kv_append(KvView kv, int layer,
                                                                 const int32_t* __restrict__ slots,
                                                                 const int32_t* __restrict__ starts, int64_t n,
                                                                 KvRows k, KvRows v, int64_t total, int64_t work) {
  constexpr int E = 16 / sizeof(T);           // elements of a 16-byte chunk
  constexpr int CHUNKS = kKvBlock * D / E / 32;  // chunks of the block per lane
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * APPEND_WARPS + (threadIdx.x >> 5);
  if (w >= work) return;
  int head;
  int64_t rest;
  if (work <= UINT32_MAX) {  // (a division of 32 bits; nearly always)
    rest = (uint32_t)w / (uint32_t)kv.c.kv_heads;
    head = (int)((uint32_t)w - (uint32_t)rest * (uint32_t)kv.c.kv_heads);
  } else {
    rest = w / kv.c.kv_heads;
    head = (int)(w - rest * kv.c.kv_heads);
  }
  const bool is_v = rest & 1;
  const int64_t unit = rest >> 1;
  // m tokens touch at most m / 16 + 2 blocks (rounded down), so units
  // starts[i] / 16 + 2 i on are enough for sequence i, whatever its length
  const int64_t i = warp_last_not_above(n, unit, [&](int64_t j) { return (int64_t)(starts[j] >> 4) + 2 * j; });
  KvSeq q;
  if (!kv_seq(kv, slots, starts, i, total, false, q)) {
    if (lane == 0) kv_status(kv, kKvBadEntry);
    return;
  }
  const int first = q.len - q.count;
  const int64_t block = (first >> 4) + unit - ((int64_t)(starts[i] >> 4) + 2 * i);
  const int64_t at = block * kKvBlock;
  if (unit < (int64_t)(starts[i] >> 4) + 2 * i || at >= q.len || q.count == 0) return;
  const int lo = max(first - (int)at, 0), hi = min(q.len - (int)at, kKvBlock);  // new tokens of the block
  const int page = kv.c.table[q.slot * kv.c.max_pages + (at >> kv.page_shift)];
  if (page < 0 || page >= kv.c.pages) {
    if (lane == 0) kv_status(kv, kKvBadEntry);
    return;
  }
  const int64_t inside = at & (kv.c.page_tokens - 1);
  uint8_t* codes = (is_v ? kv.c.v : kv.c.k) + kv.codes_at(layer, page, head) + inside * D;
  float* scale = (is_v ? kv.c.v_scale : kv.c.k_scale) + kv.scales_at(layer, page, head) + inside / kKvBlock;
  const KvRows& src = is_v ? v : k;
  const T* x = static_cast<const T*>(src.p) + (q.token + (at - first)) * src.token_stride + head * src.head_stride;

  union Chunk {
    uint4 u;
    T e[E];
  } r[CHUNKS];
  // a chunk's row: 32 lanes cover STEP rows, or a row takes several chunks
  constexpr int STEP = 32 * E >= D ? 32 * E / D : 1, PIECES = 32 * E >= D ? 1 : D / (32 * E);
  const T* p = x + (32 * E >= D ? lane * E / D : 0) * src.token_stride + lane * E % D;
  const int64_t down = STEP * src.token_stride;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int row = (c * 32 + lane) * E / D;
    r[c].u = make_uint4(0, 0, 0, 0);
    if (row >= lo && row < hi) {
      const T* y = p + c % PIECES * 32 * E;
      if (VEC) {
        r[c].u = __ldcs(reinterpret_cast<const uint4*>(y));
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) r[c].e[j] = y[j];
      }
    }
    if (c % PIECES == PIECES - 1) p += down;
  }
  // the largest magnitude, by the bits without their sign; an infinity or a NaN
  // shows in it, and only then are the finite values looked for one by one
  uint32_t bits = 0;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) bits = max_magnitude<T>(bits, r[c].u);
#pragma unroll
  for (int o = 16; o; o >>= 1) bits = max_magnitude<T>(bits, __shfl_xor_sync(0xffffffffu, bits, o));
  float top = magnitude<T>(bits);
  const bool finite = top < INFINITY;
  if (!finite) {
    top = 0.0f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) top = fmaxf(top, finite_top<T>(r[c].u));
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  }

  float s = __fdiv_rn(top, kv_qmax<CODES>());
  if (lo > 0) {
    const float old = *scale;
    if (s > old) {
      const float ratio = __fdiv_rn(old, s);
      uint32_t* words = reinterpret_cast<uint32_t*>(codes);
      for (int e = lane; e < lo * D / 4; e += 32) {
        const uint32_t u = words[e];
        words[e] = kv_pack4<CODES>(kv_value<CODES>(u, 0) * ratio, kv_value<CODES>(u, 1) * ratio,
                                   kv_value<CODES>(u, 2) * ratio, kv_value<CODES>(u, 3) * ratio);
      }
    } else {
      s = old;
    }
  }
  __syncwarp();
  if (lane == 0) *scale = s;
  // x / s as a product where that gives the same code: products with factors just
  // below and just above 1 / s (by 2^-21, more than what the reciprocal, the
  // product and the division round) enclose the quotient, and rounding to codes
  // keeps order, so where both give one code it is the quotient's.  Not for
  // values that are not finite or scales whose reciprocal leaves the normal range.
  const bool fast = finite && s > 0x1p-100f && s < 0x1p100f;
  const float inv = fast ? __frcp_rn(s) : 0.0f;
  const float below = inv * (1.0f - 0x1p-21f), above = inv * (1.0f + 0x1p-21f);
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int e = (c * 32 + lane) * E, row = e / D;
    if (row < lo || row >= hi) continue;
    float a[E];
#pragma unroll
    for (int j = 0; j < E; ++j) a[j] = to_float(r[c].e[j]);
    uint2 out = make_uint2(pack_products<CODES>(a, below), pack_products<CODES>(a + (E - 4), below));
    const uint2 up = make_uint2(pack_products<CODES>(a, above), pack_products<CODES>(a + (E - 4), above));
    if (!fast || out.x != up.x || out.y != up.y) out = exact_codes<T, CODES>(r[c].u, s);
    if (E == 8)
      *reinterpret_cast<uint2*>(codes + e) = out;
    else
      *reinterpret_cast<uint32_t*>(codes + e) = out.x;
  }
}

template <typename T, int D, int CODES>
cudaError_t append(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                   const KvRows& k, const KvRows& v, int64_t total, cudaStream_t s) {
  const int64_t units = total / kKvBlock + 2 * n;
  const int64_t work = units * 2 * kv.c.kv_heads;
  const unsigned grid = (unsigned)((work + APPEND_WARPS - 1) / APPEND_WARPS);
  bool vec = true;
  for (const KvRows* r : {&k, &v})
    vec = vec && aligned16(r->p) && (r->token_stride * sizeof(T)) % 16 == 0 && (r->head_stride * sizeof(T)) % 16 == 0;
  (vec ? k_kv_append<T, D, CODES, true> : k_kv_append<T, D, CODES, false>)<<<grid, APPEND_WARPS * 32, 0, s>>>(
      kv, layer, slots, starts, n, k, v, total, work);
  return cudaGetLastError();
}

template <typename T>
cudaError_t append_for(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                       const KvRows& k, const KvRows& v, int64_t total, cudaStream_t s) {
  const bool i8 = kv.c.codes == TQ_KV_INT8;
  switch (kv.c.head_dim) {
    case 64:
      return (i8 ? append<T, 64, TQ_KV_INT8> : append<T, 64, TQ_KV_E4M3>)(kv, layer, slots, starts, n, k, v, total, s);
    case 128:
      return (i8 ? append<T, 128, TQ_KV_INT8> : append<T, 128, TQ_KV_E4M3>)(kv, layer, slots, starts, n, k, v, total, s);
    default:
      return (i8 ? append<T, 256, TQ_KV_INT8> : append<T, 256, TQ_KV_E4M3>)(kv, layer, slots, starts, n, k, v, total, s);
  }
}

}  // namespace

cudaError_t launch_kv_append(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                             const KvRows& k, const KvRows& v, int type, int64_t total, cudaStream_t s) {
  switch (type) {
    case TQ_BF16:
      return append_for<__nv_bfloat16>(kv, layer, slots, starts, n, k, v, total, s);
    case TQ_FP16:
      return append_for<__half>(kv, layer, slots, starts, n, k, v, total, s);
    default:
      return append_for<float>(kv, layer, slots, starts, n, k, v, total, s);
  }
}

}  // namespace tq
