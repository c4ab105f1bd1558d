// Device helpers shared by the kernels of the 8-bit key-value cache.  Each
// translation unit gets its own copies (internal linkage).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

#include "tq_kv.h"

namespace tq {
namespace {

__device__ __forceinline__ void kv_status(const KvView& kv, int bits) { atomicOr(kv.c.status, bits); }

// Largest i in [0, n) with at(i) <= x, for a non-decreasing at() with at(0) <= x;
// called by a whole warp, 32 probes at a time.
template <typename F>
__device__ __forceinline__ int64_t warp_last_not_above(int64_t n, int64_t x, F at) {
  const int lane = threadIdx.x & 31;
  int64_t lo = 0, count = n;  // the answer lies in [lo, lo + count)
  while (count > 1) {
    const int64_t step = (count + 31) / 32;
    const int64_t i = lo + lane * step;
    const unsigned yes = __ballot_sync(0xffffffffu, lane * step < count && at(i) <= x);
    const int last = 31 - __clz(yes | 1u);
    lo += last * step;
    count = min(step, count - last * step);
  }
  return lo;
}

// Sequence i of a call that brings tokens starts[i] .. starts[i+1] - 1 (its last
// ones): false, with the status set, where the entry cannot be carried out.
struct KvSeq {
  int slot, token, len, count;
};
__device__ __forceinline__ bool kv_seq(const KvView& kv, const int32_t* __restrict__ slots,
                                       const int32_t* __restrict__ starts, int64_t i, int64_t total, bool clip,
                                       KvSeq& q) {
  const int a = starts[i], b = starts[i + 1];
  q.slot = slots[i];
  q.token = a;
  q.count = b - a;
  q.len = 0;
  if (a < 0 || b < a || b > total || q.slot < 0 || q.slot >= kv.c.slots) return false;
  q.len = kv.c.lens[q.slot];
  return q.len >= 0 && q.len <= kv.max_len && (clip || q.len >= q.count);
}

// Four int8 or e4m3 codes from four floats in the codes' range, rounded to
// nearest even.
template <int CODES>
__device__ __forceinline__ uint32_t kv_pack4(float a, float b, float c, float d) {
  if (CODES == TQ_KV_INT8) {
    // adding 1.5 * 2^23 leaves the rounded integer in the low bits
    const float m = 12582912.0f;
    const uint32_t ab = __byte_perm(__float_as_uint(a + m), __float_as_uint(b + m), 0x0040);
    const uint32_t cd = __byte_perm(__float_as_uint(c + m), __float_as_uint(d + m), 0x0040);
    return __byte_perm(ab, cd, 0x5410);
  }
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | hi << 16;
}

// The value of byte i of a word of codes.
template <int CODES>
__device__ __forceinline__ float kv_value(uint32_t word, int i) {
  const uint32_t b = (word >> (8 * i)) & 0xffu;
  if (CODES == TQ_KV_INT8) return (float)(int8_t)b;
  const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)b, __NV_E4M3);
  return __half2float(__half(h));
}

template <int CODES>
constexpr float kv_qmax() { return CODES == TQ_KV_INT8 ? 127.0f : 448.0f; }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// Largest magnitude of the elements of two words (one element of float32, two of
// the 16-bit types side by side), as bits without sign: they order as the values
// do, infinity above them and NaN above that.
template <typename T>
__device__ __forceinline__ uint32_t max_magnitude(uint32_t a, uint32_t b) {
  return sizeof(T) == 2 ? __vmaxu2(a, b & 0x7FFF7FFFu) : max(a, b & 0x7FFFFFFFu);
}
template <typename T>
__device__ __forceinline__ uint32_t max_magnitude(uint32_t a, const uint4& b) {
  return max_magnitude<T>(max_magnitude<T>(max_magnitude<T>(max_magnitude<T>(a, b.x), b.y), b.z), b.w);
}
template <typename T>
__device__ __forceinline__ float magnitude(uint32_t bits) {
  if (sizeof(T) == 4) return __uint_as_float(bits);
  const uint32_t top = max(bits & 0xFFFFu, bits >> 16);
  T x;
  memcpy(&x, &top, sizeof(T));
  return to_float(x);
}

}  // namespace
}  // namespace tq
