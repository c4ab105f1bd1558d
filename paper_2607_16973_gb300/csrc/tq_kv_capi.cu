// C ABI entry points of the 8-bit key-value cache and of draft verification:
// every argument is checked before any work is queued.
#include <cuda_runtime.h>

#include <cmath>

#include "tq_internal.h"
#include "tq_kv.h"

using tq::fail;

namespace {

tq_status cuda_fail(const char* where, cudaError_t e) {
  return fail(TQ_ECUDA, "%s: %s (%s)", where, cudaGetErrorString(e), cudaGetErrorName(e));
}

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// The caller's struct, checked.
tq_status view(const char* fn, const tq_kv_cache* c, tq::KvView& kv) {
  if (!c) return fail(TQ_EINVAL, "%s: NULL cache", fn);
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return fail(TQ_EINVAL, "%s: head_dim=%d must be 64, 128 or 256", fn, c->head_dim);
  if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1)))
    return fail(TQ_EINVAL, "%s: page_tokens=%d must be a power of two in [16, 256]", fn, c->page_tokens);
  if (c->codes != TQ_KV_INT8 && c->codes != TQ_KV_E4M3) return fail(TQ_EINVAL, "%s: unknown codes %d", fn, c->codes);
  if (c->layers < 1 || c->layers > 1024 || c->kv_heads < 1 || c->kv_heads > tq::kKvMaxHeads)
    return fail(TQ_EINVAL, "%s: layers=%d and kv_heads=%d must be in [1, 1024]", fn, c->layers, c->kv_heads);
  if (c->slots < 1 || c->slots > tq::kKvMaxSlots)
    return fail(TQ_EINVAL, "%s: slots=%lld outside [1, %d]", fn, (long long)c->slots, tq::kKvMaxSlots);
  if (c->pages < 1 || c->pages > INT32_MAX - 1)
    return fail(TQ_EINVAL, "%s: pages=%lld outside [1, 2^31-2]", fn, (long long)c->pages);
  if (c->max_pages < 1 || c->max_pages > INT32_MAX / c->page_tokens)
    return fail(TQ_EINVAL, "%s: max_pages=%lld: 1 <= max_pages and max_pages * page_tokens < 2^31", fn,
                (long long)c->max_pages);
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->table || !c->lens || !c->refs || !c->status)
    return fail(TQ_EINVAL, "%s: NULL device pointer in the cache", fn);
  if (!tq::aligned16(c->k) || !tq::aligned16(c->v))
    return fail(TQ_EINVAL, "%s: k and v must be 16-byte aligned", fn);
  for (const void* p : {(const void*)c->k_scale, (const void*)c->v_scale, (const void*)c->table, (const void*)c->lens,
                        (const void*)c->refs, (const void*)c->status})
    if (!aligned(p, 4)) return fail(TQ_EINVAL, "%s: the cache's arrays must be 4-byte aligned", fn);
  kv.c = *c;
  kv.page_shift = 0;
  while ((1 << kv.page_shift) < c->page_tokens) ++kv.page_shift;
  kv.max_len = c->max_pages * c->page_tokens;
  return TQ_OK;
}

tq_status check_layer(const char* fn, const tq::KvView& kv, int layer) {
  if (layer < 0 || layer >= kv.c.layers)
    return fail(TQ_EINVAL, "%s: layer=%d outside [0, %d)", fn, layer, kv.c.layers);
  return TQ_OK;
}

tq_status check_entries(const char* fn, const tq::KvView& kv, int64_t n) {
  if (n < 0 || n > kv.c.slots || n > 65535)
    return fail(TQ_EINVAL, "%s: n=%lld outside [0, min(slots, 65535)]", fn, (long long)n);
  return TQ_OK;
}

tq_status check_index(const char* fn, const void* a, const void* b) {
  if (!a || !b) return fail(TQ_EINVAL, "%s: NULL device pointer", fn);
  if (!aligned(a, 4) || !aligned(b, 4)) return fail(TQ_EINVAL, "%s: index arrays must be 4-byte aligned", fn);
  return TQ_OK;
}

tq_status check_rows(const char* fn, const char* name, const tq::KvRows& r, int type) {
  const size_t size = type == TQ_FP32 ? 4 : 2;
  if (!r.p) return fail(TQ_EINVAL, "%s: NULL %s", fn, name);
  if (!aligned(r.p, size)) return fail(TQ_EINVAL, "%s: %s must be aligned to its elements", fn, name);
  if (r.token_stride < 0 || r.head_stride < 0 || r.token_stride > INT32_MAX || r.head_stride > INT32_MAX)
    return fail(TQ_EINVAL, "%s: strides of %s outside [0, 2^31-1]", fn, name);
  return TQ_OK;
}

tq_status check_workspace(const char* fn, const void* ws, size_t have, size_t need) {
  if (!ws || !tq::aligned16(ws)) return fail(TQ_EINVAL, "%s: the workspace must be 16-byte aligned", fn);
  if (have < need) return fail(TQ_EINVAL, "%s: workspace of %zu bytes, %zu needed", fn, have, need);
  return TQ_OK;
}

#define TRY(call)                      \
  do {                                 \
    const tq_status try_st = (call);   \
    if (try_st != TQ_OK) return try_st; \
  } while (0)

}  // namespace

extern "C" tq_status tq_kv_append(const tq_kv_cache* cache, int layer, const int32_t* slots, const int32_t* starts,
                                  int64_t n, const void* k, const void* v, int type, int64_t total,
                                  int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                                  int64_t v_head_stride, void* stream) {
  const char* fn = "tq_kv_append";
  tq::KvView kv;
  TRY(view(fn, cache, kv));
  TRY(check_layer(fn, kv, layer));
  TRY(check_entries(fn, kv, n));
  if (type != TQ_BF16 && type != TQ_FP16 && type != TQ_FP32) return fail(TQ_EINVAL, "%s: unknown type %d", fn, type);
  if (total < 0 || total > INT32_MAX - 1)
    return fail(TQ_EINVAL, "%s: total=%lld outside [0, 2^31-2]", fn, (long long)total);
  if ((total / tq::kKvBlock + 2 * n) * 2 * kv.c.kv_heads / 8 >= INT32_MAX)
    return fail(TQ_EUNSUPPORTED, "%s: total=%lld tokens of %d heads: bring them in several calls", fn,
                (long long)total, kv.c.kv_heads);
  if (total == 0 || n == 0) return tq::ok();
  TRY(check_index(fn, slots, starts));
  const tq::KvRows kr = {k, k_token_stride, k_head_stride}, vr = {v, v_token_stride, v_head_stride};
  TRY(check_rows(fn, "k", kr, type));
  TRY(check_rows(fn, "v", vr, type));
  const cudaError_t e =
      tq::launch_kv_append(kv, layer, slots, starts, n, kr, vr, type, total, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? tq::ok() : cuda_fail(fn, e);
}

static tq_status check_attend(const char* fn, const tq::KvView& kv, int64_t n, int64_t total, int heads) {
  TRY(check_entries(fn, kv, n));
  if (heads < 1 || heads % kv.c.kv_heads)
    return fail(TQ_EINVAL, "%s: heads=%d is not a multiple of kv_heads=%d", fn, heads, kv.c.kv_heads);
  if (total < 0 || total > INT32_MAX - 1 || total * heads > INT32_MAX)
    return fail(TQ_EINVAL, "%s: total=%lld queries of %d heads are too many", fn, (long long)total, heads);
  return TQ_OK;
}

extern "C" tq_status tq_kv_attend_workspace(const tq_kv_cache* cache, int64_t n, int64_t total, int heads,
                                            size_t* bytes) {
  const char* fn = "tq_kv_attend_workspace";
  tq::KvView kv;
  if (!bytes) return fail(TQ_EINVAL, "%s: NULL bytes", fn);
  TRY(view(fn, cache, kv));
  TRY(check_attend(fn, kv, n, total, heads));
  *bytes = tq::kv_attend_workspace(kv, n, total, heads);
  return tq::ok();
}

extern "C" tq_status tq_kv_attend(const tq_kv_cache* cache, int layer, const int32_t* slots, const int32_t* starts,
                                  int64_t n, const void* q, int type, int64_t total, int heads,
                                  int64_t q_token_stride, int64_t q_head_stride, float scale, int window, void* out,
                                  float* lse, void* workspace, size_t ws_bytes, void* stream) {
  const char* fn = "tq_kv_attend";
  tq::KvView kv;
  TRY(view(fn, cache, kv));
  TRY(check_layer(fn, kv, layer));
  TRY(check_attend(fn, kv, n, total, heads));
  if (type != TQ_BF16 && type != TQ_FP16)
    return fail(TQ_EINVAL, "%s: type %d: queries are TQ_BF16 or TQ_FP16", fn, type);
  if (!std::isfinite(scale)) return fail(TQ_EINVAL, "%s: scale is not finite", fn);
  if (window < 0) return fail(TQ_EINVAL, "%s: window=%d is negative", fn, window);
  if (total == 0) return tq::ok();
  if (n == 0) return fail(TQ_EINVAL, "%s: total=%lld queries of no sequence", fn, (long long)total);
  TRY(check_index(fn, slots, starts));
  const tq::KvRows rows = {q, q_token_stride, q_head_stride};
  TRY(check_rows(fn, "q", rows, type));
  if (!out || !tq::aligned16(out)) return fail(TQ_EINVAL, "%s: out must be 16-byte aligned", fn);
  if (!aligned(lse, 4)) return fail(TQ_EINVAL, "%s: lse must be 4-byte aligned", fn);
  TRY(check_workspace(fn, workspace, ws_bytes, tq::kv_attend_needs(kv, n, total, heads)));
  const cudaError_t e = tq::launch_kv_attend(kv, layer, slots, starts, n, rows, type, total, heads, scale, window, out,
                                             lse, workspace, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? tq::ok() : cuda_fail(fn, e);
}

extern "C" tq_status tq_kv_fork(const tq_kv_cache* cache, const int32_t* dst, const int32_t* src, int64_t n,
                                void* stream) {
  const char* fn = "tq_kv_fork";
  tq::KvView kv;
  TRY(view(fn, cache, kv));
  TRY(check_entries(fn, kv, n));
  if (n == 0) return tq::ok();
  TRY(check_index(fn, dst, src));
  const cudaError_t e = tq::launch_kv_fork(kv, dst, src, n, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? tq::ok() : cuda_fail(fn, e);
}

extern "C" tq_status tq_kv_truncate(const tq_kv_cache* cache, const int32_t* slots, const int32_t* lens, int64_t n,
                                    void* stream) {
  const char* fn = "tq_kv_truncate";
  tq::KvView kv;
  TRY(view(fn, cache, kv));
  TRY(check_entries(fn, kv, n));
  if (n == 0) return tq::ok();
  TRY(check_index(fn, slots, lens));
  const cudaError_t e = tq::launch_kv_truncate(kv, slots, lens, n, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? tq::ok() : cuda_fail(fn, e);
}

extern "C" tq_status tq_kv_extend_workspace(const tq_kv_cache* cache, int64_t n, size_t* bytes) {
  const char* fn = "tq_kv_extend_workspace";
  tq::KvView kv;
  if (!bytes) return fail(TQ_EINVAL, "%s: NULL bytes", fn);
  TRY(view(fn, cache, kv));
  TRY(check_entries(fn, kv, n));
  *bytes = tq::kv_extend_workspace(kv, n);
  return tq::ok();
}

extern "C" tq_status tq_kv_extend(const tq_kv_cache* cache, const int32_t* slots, const int32_t* counts, int64_t n,
                                  void* workspace, size_t ws_bytes, void* stream) {
  const char* fn = "tq_kv_extend";
  tq::KvView kv;
  TRY(view(fn, cache, kv));
  TRY(check_entries(fn, kv, n));
  if (n == 0) return tq::ok();
  TRY(check_index(fn, slots, counts));
  TRY(check_workspace(fn, workspace, ws_bytes, tq::kv_extend_workspace(kv, n)));
  const cudaError_t e = tq::launch_kv_extend(kv, slots, counts, n, workspace, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? tq::ok() : cuda_fail(fn, e);
}

extern "C" tq_status tq_kv_compact_workspace(const tq_kv_cache* cache, size_t* bytes) {
  const char* fn = "tq_kv_compact_workspace";
  tq::KvView kv;
  if (!bytes) return fail(TQ_EINVAL, "%s: NULL bytes", fn);
  TRY(view(fn, cache, kv));
  *bytes = tq::kv_compact_workspace(kv);
  return tq::ok();
}

extern "C" tq_status tq_kv_compact(const tq_kv_cache* cache, int32_t* used, void* workspace, size_t ws_bytes,
                                   void* stream) {
  const char* fn = "tq_kv_compact";
  tq::KvView kv;
  TRY(view(fn, cache, kv));
  if (!aligned(used, 4)) return fail(TQ_EINVAL, "%s: used must be 4-byte aligned", fn);
  TRY(check_workspace(fn, workspace, ws_bytes, tq::kv_compact_workspace(kv)));
  const cudaError_t e = tq::launch_kv_compact(kv, used, workspace, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? tq::ok() : cuda_fail(fn, e);
}

extern "C" tq_status tq_kv_check(const tq_kv_cache* cache, void* stream) {
  const char* fn = "tq_kv_check";
  tq::KvView kv;
  TRY(view(fn, cache, kv));
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  int32_t word = 0;
  cudaError_t e = cudaMemcpyAsync(&word, kv.c.status, sizeof(word), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && word) e = cudaMemsetAsync(kv.c.status, 0, sizeof(word), s);
  if (e != cudaSuccess) return cuda_fail(fn, e);
  if (word & tq::kKvTimeout) return fail(TQ_ETIMEOUT, "%s: tq_kv_attend gave up on a bounded wait", fn);
  if (word & tq::kKvNoPages) return fail(TQ_ENOMEM, "%s: too few free pages", fn);
  if (word) return fail(TQ_EINVAL, "%s: entries were left out (slot, length, count or page not valid)", fn);
  return tq::ok();
}

static tq_status check_verify(const char* fn, int64_t n, int64_t vocab) {
  if (n < 0 || n > 65535) return fail(TQ_EINVAL, "%s: n=%lld outside [0, 65535]", fn, (long long)n);
  if (vocab < 1 || vocab > (1 << 24))
    return fail(TQ_EINVAL, "%s: vocab=%lld outside [1, 2^24]", fn, (long long)vocab);
  return TQ_OK;
}

extern "C" tq_status tq_verify_drafts_workspace(int64_t n, int64_t vocab, size_t* bytes) {
  const char* fn = "tq_verify_drafts_workspace";
  if (!bytes) return fail(TQ_EINVAL, "%s: NULL bytes", fn);
  TRY(check_verify(fn, n, vocab));
  *bytes = tq::verify_workspace(n, vocab);
  return tq::ok();
}

extern "C" tq_status tq_verify_drafts(const void* target, const void* draft, int type, const int32_t* drafts,
                                      const int32_t* draft_lens, const float* uniforms, const float* noise, int64_t n,
                                      int t, int vocab, int32_t* tokens, int32_t* accepted, void* workspace,
                                      size_t ws_bytes, void* stream) {
  const char* fn = "tq_verify_drafts";
  TRY(check_verify(fn, n, vocab));
  if (t < 0 || t > tq::kVerifyMaxDrafts) return fail(TQ_EINVAL, "%s: t=%d outside [0, %d]", fn, t, tq::kVerifyMaxDrafts);
  if (type != TQ_BF16 && type != TQ_FP16 && type != TQ_FP32) return fail(TQ_EINVAL, "%s: unknown type %d", fn, type);
  if (n == 0) return tq::ok();
  if (!target || !noise || !tokens || !accepted || (t > 0 && (!drafts || !uniforms)))
    return fail(TQ_EINVAL, "%s: NULL device pointer", fn);
  const size_t size = type == TQ_FP32 ? 4 : 2;
  if (!aligned(target, size) || !aligned(draft, size))
    return fail(TQ_EINVAL, "%s: the probabilities must be aligned to their elements", fn);
  for (const void* p : {(const void*)drafts, (const void*)draft_lens, (const void*)uniforms, (const void*)noise,
                        (const void*)tokens, (const void*)accepted})
    if (!aligned(p, 4)) return fail(TQ_EINVAL, "%s: arrays must be 4-byte aligned", fn);
  TRY(check_workspace(fn, workspace, ws_bytes, tq::verify_workspace(n, vocab)));
  const cudaError_t e = tq::launch_verify(target, draft, type, drafts, draft_lens, uniforms, noise, n, t, vocab,
                                          tokens, accepted, workspace, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? tq::ok() : cuda_fail(fn, e);
}
