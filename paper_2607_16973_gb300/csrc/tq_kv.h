// Internal declarations of the 8-bit key-value cache (tq_kv_* in tq.h) and of
// draft verification, shared by their translation units.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "tq_internal.h"
#include "tq_kernels.h"

namespace tq {

constexpr int kKvBlock = 16;          // tokens that share a scale
constexpr int kKvMaxSlots = 65536;    // slots of a cache (one bit each fits in shared memory)
constexpr int kKvMaxHeads = 1024;
constexpr int kVerifyMaxDrafts = 64;

// What a call leaves in a cache's status word (tq_kv_check).
constexpr int kKvBadEntry = 1;   // an entry was left out
constexpr int kKvNoPages = 2;    // too few free pages: the call changed nothing
constexpr int kKvTimeout = 4;    // a bounded wait gave up

// A cache as the kernels see it: the caller's struct and what follows from it.
struct KvView {
  tq_kv_cache c;
  int page_shift;       // log2(page_tokens)
  int64_t max_len;      // tokens that a table has room for

  // First code of a (layer, page, head), and its first scale.
  __host__ __device__ int64_t rows(int layer, int64_t page, int head) const {
    return (((int64_t)layer * c.pages + page) * c.kv_heads + head) << page_shift;
  }
  __host__ __device__ int64_t codes_at(int layer, int64_t page, int head) const {
    return rows(layer, page, head) * c.head_dim;
  }
  __host__ __device__ int64_t scales_at(int layer, int64_t page, int head) const {
    return rows(layer, page, head) / kKvBlock;
  }
  __host__ __device__ int64_t pages_of(int64_t tokens) const {
    return (tokens + c.page_tokens - 1) >> page_shift;
  }
};

struct KvRows {  // new keys or values, or queries: rows of head_dim elements
  const void* p;
  int64_t token_stride, head_stride;  // in elements
};

cudaError_t launch_kv_append(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                             const KvRows& k, const KvRows& v, int type, int64_t total, cudaStream_t s);

// What the rows of an attention call see of a sequence.
enum class KvSees : int {
  CAUSAL,  // the tokens up to their own place
  ALL,     // all of them
  SHARED,  // the tokens that a plan's requests share (sums only)
  OWN,     // the others, up to their own place; joined with the shared ones' sums
};

size_t kv_attend_needs(const KvView& kv, int64_t n, int64_t total, int heads);      // of this call
size_t kv_attend_workspace(const KvView& kv, int64_t n, int64_t total, int heads);  // of every one that is not larger
cudaError_t launch_kv_attend(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                             const KvRows& q, int type, int64_t total, int heads, float scale, int window, void* out,
                             float* lse, void* workspace, cudaStream_t s, bool all = false);

size_t kv_shared_workspace(const KvView& kv, int64_t n, int64_t total, int heads);
cudaError_t launch_kv_attend_shared(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts,
                                    const int32_t* plan, int64_t n, int64_t groups, const KvRows& q, int type,
                                    int64_t total, int heads, float scale, void* out, float* lse, void* workspace,
                                    cudaStream_t s);
cudaError_t launch_kv_share(const KvView& kv, const int32_t* slots, const int32_t* starts, int64_t n, int32_t* plan,
                            cudaStream_t s);
// What a plan's entry comes to: the tokens that its request shares (0: none), and the
// queries of its group if it is the group's first (else 0).
struct KvShared {
  int tokens, queries;
};
cudaError_t launch_kv_entries(const KvView& kv, const int32_t* slots, const int32_t* starts, const int32_t* plan,
                              int64_t n, int64_t total, KvShared* entries, cudaStream_t s);

cudaError_t launch_kv_fork(const KvView& kv, const int32_t* dst, const int32_t* src, int64_t n, cudaStream_t s);
size_t kv_extend_workspace(const KvView& kv, int64_t n);
cudaError_t launch_kv_extend(const KvView& kv, const int32_t* slots, const int32_t* counts, int64_t n,
                             void* workspace, cudaStream_t s);
cudaError_t launch_kv_truncate(const KvView& kv, const int32_t* slots, const int32_t* lens, int64_t n,
                               cudaStream_t s);
size_t kv_compact_workspace(const KvView& kv);
cudaError_t launch_kv_compact(const KvView& kv, int32_t* used, void* workspace, cudaStream_t s);

size_t verify_workspace(int64_t n, int64_t vocab);
cudaError_t launch_verify(const void* target, const void* draft, int type, const int32_t* drafts,
                          const int32_t* draft_lens, const float* uniforms, const float* noise, int64_t n, int t,
                          int vocab, int32_t* tokens, int32_t* accepted, void* workspace, cudaStream_t s);

}  // namespace tq
