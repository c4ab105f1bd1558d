// Pages of the 8-bit key-value cache: tq_kv_fork, tq_kv_extend,
// tq_kv_truncate, tq_kv_compact.
//
// The tables, lengths and counts live on the device and the calls decide
// there, so that a decoding step (and a graph of one) needs no answer on the
// host.  A free page is one whose count is 0; there is no free list beside
// the counts to keep in step with them.  Which pages a call takes follows from
// the counts alone (lowest first), not from the order in which blocks run.
//
// Bound: for the tables, latency (one block settles an extend or a compact:
// scans over the counts, 16,384 pages a step); for pages that move, HBM, read
// and written once with 16-byte accesses.  1.94 GB of moves: 334 to 340 us with all
// around them, 5.8 TB/s; 256 requests forked and extended by 40 tokens: 35 us (28 in a
// graph).
#include <algorithm>

#include "tq_kv.cuh"
#include "tq_topk.cuh"

namespace tq {
namespace {

constexpr int ONE = 1024;        // threads of the kernels that settle a call in one block
constexpr int ROW = 256;         // threads per entry of fork and truncate
constexpr int COPY = 256;        // threads of the copying kernels
constexpr int MOVE_BYTES = 32768;  // of a page that a block moves at a time
constexpr int MOVE_PER_SM = 4;

constexpr size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// Whether entry i's slot is one that no other entry of the call names: bounds,
// and a whole-block search for duplicates (and for `other`, nullable).
__device__ bool entry_alone(const KvView& kv, const int32_t* __restrict__ a, const int32_t* __restrict__ other,
                            int64_t n, int64_t i) {
  const int slot = a[i];
  bool bad = slot < 0 || slot >= kv.c.slots;
  for (int64_t j = threadIdx.x; j < n; j += blockDim.x) bad |= (j != i && a[j] == slot) || (other && other[j] == slot);
  return !__syncthreads_or(bad);
}

__device__ __forceinline__ bool length_ok(const KvView& kv, int len) { return len >= 0 && len <= kv.max_len; }

__device__ __forceinline__ void drop(const KvView& kv, int page) {
  if (page >= 0 && page < kv.c.pages) atomicSub(kv.c.refs + page, 1);
}

// A block per entry.  Counts change by sums, whose order does not matter.
__global__ __launch_bounds__(ROW) void k_kv_fork(KvView kv, const int32_t* __restrict__ dst,
                                                 const int32_t* __restrict__ src, int64_t n) {
  const int64_t i = blockIdx.x;
  const int from = src[i];
  bool ok = entry_alone(kv, dst, src, n, i) && from >= 0 && from < kv.c.slots;
  const int to = dst[i];
  const int had = ok ? kv.c.lens[to] : 0, len = ok ? kv.c.lens[from] : 0;
  ok = ok && length_ok(kv, had) && length_ok(kv, len);
  if (!ok) {
    if (threadIdx.x == 0) kv_status(kv, kKvBadEntry);
    return;
  }
  __syncthreads();  // (every thread has read lens[to])
  if (threadIdx.x == 0) kv.c.lens[to] = len;
  const int64_t old_pages = kv.pages_of(had), pages = kv.pages_of(len);
  int32_t* row = kv.c.table + to * kv.c.max_pages;
  const int32_t* given = kv.c.table + from * kv.c.max_pages;
  for (int64_t p = threadIdx.x; p < max(old_pages, pages); p += ROW) {
    if (p < old_pages) drop(kv, row[p]);
    int page = -1;
    if (p < pages) {
      page = given[p];
      if (page >= 0 && page < kv.c.pages) atomicAdd(kv.c.refs + page, 1);
    }
    row[p] = page;
  }
}

__global__ __launch_bounds__(ROW) void k_kv_truncate(KvView kv, const int32_t* __restrict__ slots,
                                                     const int32_t* __restrict__ lens, int64_t n) {
  const int64_t i = blockIdx.x;
  bool ok = entry_alone(kv, slots, nullptr, n, i);
  const int slot = slots[i], len = lens[i];
  const int had = ok ? kv.c.lens[slot] : 0;
  ok = ok && length_ok(kv, had) && len >= 0 && len <= had;
  if (!ok) {
    if (threadIdx.x == 0) kv_status(kv, kKvBadEntry);
    return;
  }
  __syncthreads();
  if (threadIdx.x == 0) kv.c.lens[slot] = len;
  int32_t* row = kv.c.table + slot * kv.c.max_pages;
  for (int64_t p = kv.pages_of(len) + threadIdx.x; p < kv.pages_of(had); p += ROW) {
    drop(kv, row[p]);
    row[p] = -1;
  }
}

// Exclusive sum over the block's threads of x; `total` receives the block's sum.
__device__ int64_t block_before(int64_t x, int64_t* warp_sums, int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t sum = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += y;
  }
  if (lane == 31) warp_sums[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    int64_t s = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  const int64_t before = warp ? warp_sums[warp - 1] : 0;
  total = warp_sums[ONE / 32 - 1];
  __syncthreads();
  return before + sum - x;
}

// Walks pages [0, end) in ascending order, each thread 16 neighbours at a time,
// and calls put(page, rank) for those whose count is free (or used), rank
// counting from 0.  Returns how many there are; stops once `most` are found.
template <bool USED, typename F>
__device__ int64_t ranked_pages(const KvView& kv, int64_t begin, int64_t end, int64_t most, int64_t* warp_sums, F put) {
  int64_t found = 0;
  for (int64_t base = begin & ~(int64_t)15; base < end && found < most; base += ONE * 16) {
    const int64_t p = base + (int64_t)threadIdx.x * 16;
    uint32_t bits = 0;
    // the counts' array is 4-byte aligned by contract: 16 plain loads, all in flight
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int64_t at = p + j;
      const int r = at >= begin && at < end ? kv.c.refs[at] : (USED ? 0 : 1);
      bits |= (uint32_t)((r > 0) == USED) << j;
    }
    int64_t total;
    int64_t rank = found + block_before(__popc(bits), warp_sums, total);
    while (bits) {
      const int j = __ffs(bits) - 1;
      bits &= bits - 1;
      if (rank < most) put(p + j, rank);
      ++rank;
    }
    found += total;
  }
  return found;
}

// What tq_kv_extend leaves for its copies and keeps while it settles.
struct ExtendWork {
  int64_t* before;     // [n + 1] pages that the entries in front take
  int32_t *from, *to;  // [n] page to copy for an entry, or -1
  int32_t* blocks;     // [n] its used blocks
  int32_t* list;       // [pages] free pages, ascending
};

ExtendWork extend_work(const KvView& kv, int64_t n, void* ws, size_t* bytes) {
  ExtendWork w;
  char* p = static_cast<char*>(ws);
  size_t off = 0;
  auto take = [&](size_t b) {
    char* at = p + off;
    off = align_up(off + b);
    return at;
  };
  w.before = reinterpret_cast<int64_t*>(take((n + 1) * sizeof(int64_t)));
  w.from = reinterpret_cast<int32_t*>(take(n * sizeof(int32_t)));
  w.to = reinterpret_cast<int32_t*>(take(n * sizeof(int32_t)));
  w.blocks = reinterpret_cast<int32_t*>(take(n * sizeof(int32_t)));
  w.list = reinterpret_cast<int32_t*>(take(kv.c.pages * sizeof(int32_t)));
  if (bytes) *bytes = off;
  return w;
}

__global__ __launch_bounds__(ONE) void k_kv_extend(KvView kv, const int32_t* __restrict__ slots,
                                                   const int32_t* __restrict__ counts, int64_t n, ExtendWork w) {
  __shared__ int64_t warp_sums[ONE / 32];
  __shared__ uint32_t seen[kKvMaxSlots / 32];
  griddep_launch_dependents();
  for (int i = threadIdx.x; i < kKvMaxSlots / 32; i += ONE) seen[i] = 0;
  __syncthreads();
  bool bad = false;
  int64_t wanted = 0;
  for (int64_t base = 0; base < n; base += ONE) {
    const int64_t i = base + threadIdx.x;
    int64_t mine = 0;
    if (i < n) {
      const int slot = slots[i], count = counts[i];
      w.from[i] = w.to[i] = -1;
      w.blocks[i] = 0;
      if (slot < 0 || slot >= kv.c.slots || count < 0 ||
          (atomicOr(&seen[slot >> 5], 1u << (slot & 31)) >> (slot & 31) & 1u)) {
        bad = true;
      } else {
        const int len = kv.c.lens[slot];
        if (!length_ok(kv, len) || (int64_t)len + count > kv.max_len) {
          bad = true;
        } else {
          const int64_t held = kv.pages_of(len);
          mine = kv.pages_of((int64_t)len + count) - held;
          const int part = len & (kv.c.page_tokens - 1);
          if (part && count) {
            const int last = kv.c.table[slot * kv.c.max_pages + held - 1];
            if (last < 0 || last >= kv.c.pages) {
              bad = true;
            } else if (kv.c.refs[last] > 1) {
              ++mine;
              w.from[i] = last;
              w.blocks[i] = (part + kKvBlock - 1) / kKvBlock;
            }
          }
        }
      }
    }
    int64_t total;
    const int64_t before = wanted + block_before(mine, warp_sums, total);
    if (i < n) w.before[i] = before;
    wanted += total;
  }
  if (threadIdx.x == 0) w.before[n] = wanted;
  const bool refused = __syncthreads_or(bad);
  const int64_t found =
      refused || !wanted
          ? 0
          : ranked_pages<false>(kv, 0, kv.c.pages, wanted, warp_sums,
                                [&](int64_t page, int64_t rank) { w.list[rank] = (int32_t)page; });
  if (refused || found < wanted) {
    for (int64_t i = threadIdx.x; i < n; i += ONE) w.from[i] = -1;
    if (threadIdx.x == 0) kv_status(kv, refused ? kKvBadEntry : kKvNoPages);
    return;
  }
  __syncthreads();  // the list, the entries' sums
  for (int64_t e = threadIdx.x; e < wanted; e += ONE) {
    int64_t lo = 0, hi = n;  // the entry that page e of the list goes to: the last with before <= e
    while (hi - lo > 1) {
      const int64_t mid = (lo + hi) / 2;
      (w.before[mid] <= e ? lo : hi) = mid;
    }
    const int slot = slots[lo], page = w.list[e];
    const int64_t held = kv.pages_of(kv.c.lens[slot]), nth = e - w.before[lo];
    const bool copy = w.from[lo] >= 0;
    kv.c.table[slot * kv.c.max_pages + held - copy + nth] = page;
    kv.c.refs[page] = 1;
    if (copy && nth == 0) {
      w.to[lo] = page;
      atomicSub(kv.c.refs + w.from[lo], 1);
    }
  }
  __syncthreads();  // every thread has read the lengths
  for (int64_t i = threadIdx.x; i < n; i += ONE) kv.c.lens[slots[i]] += counts[i];
}

// Copies the used blocks of the pages that tq_kv_extend replaced: a block of
// threads per entry, layer, and K or V, which has all heads' pieces of a column
// of threads on their way together.
__global__ __launch_bounds__(COPY) void k_kv_copy_parts(KvView kv, ExtendWork w) {
  const int64_t i = blockIdx.x;
  griddep_wait();
  const int from = w.from[i];
  if (from < 0) return;
  const int to = w.to[i], blocks = w.blocks[i];
  const int heads = kv.c.kv_heads, pieces = blocks * kv.c.head_dim;  // of 16 bytes, of a head
  const int64_t head_pieces = (int64_t)kv.c.page_tokens * kv.c.head_dim / 16;
  for (int64_t j = blockIdx.y; j < (int64_t)2 * kv.c.layers; j += gridDim.y) {
    const bool is_v = j & 1;
    const int layer = (int)(j >> 1);
    uint8_t* codes = is_v ? kv.c.v : kv.c.k;
    const uint4* a = reinterpret_cast<const uint4*>(codes + kv.codes_at(layer, from, 0));
    uint4* b = reinterpret_cast<uint4*>(codes + kv.codes_at(layer, to, 0));
    for (int e = threadIdx.x; e < pieces; e += COPY)
      for (int h = 0; h < heads; h += 8) {
        uint4 x[8];
#pragma unroll
        for (int y = 0; y < 8; ++y)
          if (h + y < heads) x[y] = a[(h + y) * head_pieces + e];
#pragma unroll
        for (int y = 0; y < 8; ++y)
          if (h + y < heads) b[(h + y) * head_pieces + e] = x[y];
      }
    float* scale = is_v ? kv.c.v_scale : kv.c.k_scale;
    for (int e = threadIdx.x; e < heads * blocks; e += COPY)
      scale[kv.scales_at(layer, to, e / blocks) + e % blocks] = scale[kv.scales_at(layer, from, e / blocks) + e % blocks];
  }
}

struct CompactWork {
  int64_t* sizes;        // pages in use, pages that move
  int32_t *from, *to;    // [pages] pages that move, and where to, ascending
  int32_t* name;         // [pages] new page of a moved one
};

CompactWork compact_work(const KvView& kv, void* ws, size_t* bytes) {
  CompactWork w;
  char* p = static_cast<char*>(ws);
  const size_t each = align_up(kv.c.pages * sizeof(int32_t));
  w.sizes = reinterpret_cast<int64_t*>(p);
  w.from = reinterpret_cast<int32_t*>(p + 256);
  w.to = reinterpret_cast<int32_t*>(p + 256 + each);
  w.name = reinterpret_cast<int32_t*>(p + 256 + 2 * each);
  if (bytes) *bytes = 256 + 3 * each;
  return w;
}

__global__ __launch_bounds__(ONE) void k_kv_compact(KvView kv, CompactWork w, int32_t* used) {
  __shared__ int64_t warp_sums[ONE / 32];
  griddep_launch_dependents();
  const int64_t pages = kv.c.pages;
  const int64_t live = ranked_pages<true>(kv, 0, pages, pages, warp_sums, [](int64_t, int64_t) {});
  const int64_t holes = ranked_pages<false>(kv, 0, live, pages, warp_sums,
                                            [&](int64_t page, int64_t rank) { w.to[rank] = (int32_t)page; });
  // as many used pages lie past `live` as free ones below it
  ranked_pages<true>(kv, live, pages, pages, warp_sums,
                     [&](int64_t page, int64_t rank) { w.from[rank] = (int32_t)page; });
  if (threadIdx.x == 0) {
    w.sizes[0] = live;
    w.sizes[1] = holes;
    if (used) *used = (int32_t)live;
  }
  __syncthreads();
  for (int64_t i = threadIdx.x; i < holes; i += ONE) {
    const int from = w.from[i], to = w.to[i];
    w.name[from] = to;
    kv.c.refs[to] = kv.c.refs[from];
    kv.c.refs[from] = 0;
  }
}

// Moves pages: pieces of MOVE_BYTES of (page, layer, K or V), in turn over the
// grid, each loaded whole before it is stored: 32 KB in flight per block, four
// blocks per SM.  The pages of the next piece are looked up beside the copy.
__global__ __launch_bounds__(COPY, MOVE_PER_SM) void k_kv_move(KvView kv, CompactWork w) {
  griddep_launch_dependents();
  griddep_wait();
  const int64_t moves = w.sizes[1];
  const int bytes = kv.c.kv_heads * kv.c.page_tokens * kv.c.head_dim;
  const int scales = kv.c.kv_heads * kv.c.page_tokens / kKvBlock;
  const int pieces = (bytes + MOVE_BYTES - 1) / MOVE_BYTES;
  const int per_page = pieces * 2 * kv.c.layers;
  const int64_t all = moves * per_page;
  int from = 0, to = 0;
  if (blockIdx.x < all) {
    from = w.from[blockIdx.x / per_page];
    to = w.to[blockIdx.x / per_page];
  }
  for (int64_t j = blockIdx.x; j < all; j += gridDim.x) {
    const int r = (int)(j % per_page), at = r % pieces * MOVE_BYTES;
    const bool is_v = r / pieces & 1;
    const int layer = r / pieces / 2;
    uint8_t* codes = is_v ? kv.c.v : kv.c.k;
    const uint4* a = reinterpret_cast<const uint4*>(codes + kv.codes_at(layer, from, 0) + at);
    uint4* b = reinterpret_cast<uint4*>(codes + kv.codes_at(layer, to, 0) + at);
    const int n = min(MOVE_BYTES, bytes - at) / 16;
    uint4 x[MOVE_BYTES / 16 / COPY];
#pragma unroll
    for (int i = 0; i < MOVE_BYTES / 16 / COPY; ++i) {
      const int e = i * COPY + threadIdx.x;
      if (e < n) x[i] = __ldcs(a + e);
    }
    if (at == 0) {
      float* scale = is_v ? kv.c.v_scale : kv.c.k_scale;
      for (int e = threadIdx.x; e < scales; e += COPY)
        scale[kv.scales_at(layer, to, 0) + e] = scale[kv.scales_at(layer, from, 0) + e];
    }
    if (j + gridDim.x < all) {
      from = w.from[(j + gridDim.x) / per_page];
      to = w.to[(j + gridDim.x) / per_page];
    }
#pragma unroll
    for (int i = 0; i < MOVE_BYTES / 16 / COPY; ++i) {
      const int e = i * COPY + threadIdx.x;
      if (e < n) __stcs(b + e, x[i]);
    }
  }
}

__global__ __launch_bounds__(COPY) void k_kv_rename(KvView kv, CompactWork w) {
  griddep_wait();
  const int64_t live = w.sizes[0], n = kv.c.slots * kv.c.max_pages;
  for (int64_t e = (int64_t)blockIdx.x * COPY + threadIdx.x; e < n; e += (int64_t)gridDim.x * COPY) {
    const int page = kv.c.table[e];
    if (page >= live && page < kv.c.pages) kv.c.table[e] = w.name[page];
  }
}

}  // namespace

cudaError_t launch_kv_fork(const KvView& kv, const int32_t* dst, const int32_t* src, int64_t n, cudaStream_t s) {
  k_kv_fork<<<(unsigned)n, ROW, 0, s>>>(kv, dst, src, n);
  return cudaGetLastError();
}

cudaError_t launch_kv_truncate(const KvView& kv, const int32_t* slots, const int32_t* lens, int64_t n,
                               cudaStream_t s) {
  k_kv_truncate<<<(unsigned)n, ROW, 0, s>>>(kv, slots, lens, n);
  return cudaGetLastError();
}

size_t kv_extend_workspace(const KvView& kv, int64_t n) {
  size_t bytes = 0;
  extend_work(kv, n, nullptr, &bytes);
  return bytes;
}

cudaError_t launch_kv_extend(const KvView& kv, const int32_t* slots, const int32_t* counts, int64_t n,
                             void* workspace, cudaStream_t s) {
  const ExtendWork w = extend_work(kv, n, workspace, nullptr);
  k_kv_extend<<<1, ONE, 0, s>>>(kv, slots, counts, n, w);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int64_t parts = (int64_t)2 * kv.c.layers;
  return launch_maybe_pdl(true, k_kv_copy_parts, dim3((unsigned)n, (unsigned)std::min<int64_t>(parts, 65535)),
                          dim3(COPY), 0, s, kv, w);
}

size_t kv_compact_workspace(const KvView& kv) {
  size_t bytes = 0;
  compact_work(kv, nullptr, &bytes);
  return bytes;
}

cudaError_t launch_kv_compact(const KvView& kv, int32_t* used, void* workspace, cudaStream_t s) {
  const CompactWork w = compact_work(kv, workspace, nullptr);
  const int sms = device_sm_count();
  k_kv_compact<<<1, ONE, 0, s>>>(kv, w, used);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  if ((e = launch_maybe_pdl(true, k_kv_move, dim3(sms * MOVE_PER_SM), dim3(COPY), 0, s, kv, w)) != cudaSuccess) return e;
  const int64_t entries = kv.c.slots * kv.c.max_pages;
  return launch_maybe_pdl(true, k_kv_rename, dim3((unsigned)std::min<int64_t>((entries + COPY - 1) / COPY, sms * 8)),
                          dim3(COPY), 0, s, kv, w);
}

}  // namespace tq
