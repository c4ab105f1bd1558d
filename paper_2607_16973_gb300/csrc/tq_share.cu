// tq_kv_share: which neighbouring requests of a batch hold the same first pages,
// and how many tokens those are.
//
//   c_i = min(b_i, b_(i+1), page_tokens * (leading pages that both tables name alike)),
//   b = the tokens that a request held before its new ones
//
// Requests with c_i > 0 between them are one group; its tokens are the smallest of its
// c_i.  k_share_pairs takes a warp per pair of neighbours, 128 pages at a time, down to
// the first difference; k_share_groups goes over the c_i with one block, 1,024 at a
// time, by segmented sums.
//
// Bound: latency of two launches and of the chain slot -> length -> table; the tables are
// read once or, from L2, twice.  2,000 requests of up to 1,000 pages (5 MB of tables): 14 to 16
// us a call on a GB300, 16 requests 13 to 15.
//
// k_share_entries says what a given plan's entries come to (tq_kv_attend_shared): a
// group counts where all its entries name it, so that no two groups' queries are the
// same.  Whether they do is seen without going over the group's entries for each of
// them: entries are compared with the ones in front, and a prefix sum of those that
// differ is alike at both ends.  Of the group that a block's first or last entry is
// in, the block compares what lies outside of it.  Bound: latency, the chain plan -> slot
// -> length: 3 to 4 us of a call.
#include "tq_kv.cuh"
#include "tq_topk.cuh"

namespace tq {
namespace {

constexpr int PAIRS = 4;       // warps of a block
constexpr int GROUPS = 1024;   // threads of the block that finds the groups
constexpr int AT_ONCE = 4;     // pages of a lane on their way

// Tokens before the new ones of request i; -1: it is left out.
__device__ __forceinline__ int64_t held_before(const KvView& kv, const int32_t* slots, const int32_t* starts, int64_t i,
                                               KvSeq& s) {
  return kv_seq(kv, slots, starts, i, INT32_MAX, false, s) ? s.len - s.count : -1;
}

// c_i to plan[2][i]; c of the last request is 0.
__global__ __launch_bounds__(PAIRS * 32) void k_share_pairs(KvView kv, const int32_t* __restrict__ slots,
                                                            const int32_t* __restrict__ starts, int64_t n,
                                                            int32_t* __restrict__ plan) {
  const int64_t i = (int64_t)blockIdx.x * PAIRS + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  griddep_launch_dependents();
  if (i >= n) return;
  KvSeq a, b;
  const int64_t before = held_before(kv, slots, starts, i, a);
  if (before < 0 && lane == 0) kv_status(kv, kKvBadEntry);
  int64_t common = 0;
  if (i + 1 < n) {
    const int64_t both = min(before, held_before(kv, slots, starts, i + 1, b));
    if (both > 0) {
      const int32_t *ta = kv.c.table + a.slot * kv.c.max_pages, *tb = kv.c.table + b.slot * kv.c.max_pages;
      const int64_t pages = kv.pages_of(both);
      int64_t same = pages;
      for (int64_t base = 0; base < pages; base += 32 * AT_ONCE) {
        int x[AT_ONCE], y[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
          const int64_t p = base + k * 32 + lane;
          x[k] = p < pages ? ta[p] : 0;
          y[k] = p < pages ? tb[p] : 0;
        }
        int64_t first = -1;
#pragma unroll
        for (int k = AT_ONCE - 1; k >= 0; --k) {
          const unsigned differ = __ballot_sync(FULL, x[k] != y[k] || x[k] < 0 || x[k] >= kv.c.pages);
          if (differ) first = base + k * 32 + __ffs(differ) - 1;
        }
        if (first >= 0) {
          same = first;
          break;
        }
      }
      common = min(both, same << kv.page_shift);
    }
  }
  if (lane == 0) plan[2 * n + i] = (int)common;
}

// A request in its group, up to the last of those seen: where the group began, the
// smallest c between its members.
struct Member {
  int first, least;
};
// What stands behind `a` in the same group or a later one (b.first = -1: b says nothing
// of where a group begins, but that it goes on).
__device__ __forceinline__ Member behind(const Member& a, const Member& b) {
  return b.first >= 0 ? b : Member{a.first, min(a.least, b.least)};
}

__global__ __launch_bounds__(GROUPS) void k_share_groups(int64_t n, int32_t* plan) {
  __shared__ Member warps[GROUPS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  griddep_wait();
  Member carry = {0, INT32_MAX};
  for (int64_t base = 0; base < n; base += GROUPS) {
    const int64_t i = base + threadIdx.x;
    const int link = i < n && i > 0 ? plan[2 * n + i - 1] : 0;  // to the one in front
    const int next = i < n ? plan[2 * n + i] : 0;
    Member m = link > 0 ? Member{-1, link} : Member{(int)i, INT32_MAX};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Member x = {__shfl_up_sync(FULL, m.first, o), __shfl_up_sync(FULL, m.least, o)};
      if (lane >= o) m = behind(x, m);
    }
    if (lane == 31) warps[warp] = m;
    __syncthreads();  // (and every c of these requests has been read)
    Member front = carry;
    for (int w = 0; w < GROUPS / 32; ++w) {
      if (w == warp) m = behind(front, m);
      front = behind(front, warps[w]);
    }
    carry = front;
    if (i < n) {
      plan[i] = m.first;
      if (next == 0) {  // the group's last: its size and tokens go to its first
        plan[n + m.first] = (int)i - m.first + 1;
        // (the first's c is needed no more: the next request's link was read with it, or lies in this group)
        plan[2 * n + m.first] = m.first < i ? m.least : 0;
      }
    }
    __syncthreads();
  }
  for (int64_t i = threadIdx.x; i < n; i += GROUPS) {
    const int first = plan[i];
    if (first < i) {
      plan[n + i] = plan[n + first];
      plan[2 * n + i] = plan[2 * n + first];
    }
  }
}

struct Entry {
  int first, members, tokens;
  __device__ __forceinline__ bool operator==(const Entry& x) const {
    return first == x.first && members == x.members && tokens == x.tokens;
  }
};

__global__ __launch_bounds__(GROUPS) void k_share_entries(KvView kv, const int32_t* __restrict__ slots,
                                                          const int32_t* __restrict__ starts,
                                                          const int32_t* __restrict__ plan, int64_t n, int64_t total,
                                                          KvShared* __restrict__ entries) {
  __shared__ int changes[GROUPS];  // of this block's entries up to each one: how many differ from the one in front
  __shared__ int warps[GROUPS / 32];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int64_t base = (int64_t)blockIdx.x * GROUPS, last = min(n, base + GROUPS) - 1, i = base + t;
  auto entry = [&](int64_t j) { return Entry{plan[j], plan[n + j], plan[2 * n + j]}; };
  const Entry e = i <= last ? entry(i) : Entry{0, 0, 0}, head = entry(base), tail = entry(last);
  // this request, its group's first, and where the group's queries end (all asked for before anything is waited for)
  KvSeq s, lead;
  const int64_t end = (int64_t)e.first + e.members;
  const bool there = i <= last && kv_seq(kv, slots, starts, i, total, true, s);
  const bool inside = i <= last && e.first >= 0 && e.first <= i && i < end && end <= n;
  const bool led = inside && kv_seq(kv, slots, starts, e.first, total, true, lead);
  const int stop = inside ? starts[end] : 0;
  const unsigned differ = __ballot_sync(FULL, t > 0 && i <= last && !(entry(i - 1) == e));
  if (lane == 31) warps[warp] = __popc(differ);
  __syncthreads();
  int front = 0;
  for (int w = 0; w < warp; ++w) front += warps[w];
  changes[t] = front + __popc(differ & (2u << lane) - 1u);
  // the groups of the block's first and last entries, outside of it
  bool same = true;
  for (int64_t j = max(head.first, 0) + t; j < base; j += GROUPS) same &= entry(j) == head;
  const bool left = __syncthreads_and(same);  // (and the changes are there)
  same = true;
  for (int64_t j = last + 1 + t; j < min(n, (int64_t)tail.first + tail.members); j += GROUPS) same &= entry(j) == tail;
  const bool right = __syncthreads_and(same);
  if (i > last) return;
  KvShared out = {0, 0};
  bool bad = there && e.tokens < 0;  // (where there is no such request the attention says so)
  if (there && e.tokens > 0 && e.members > 1) {
    // the first one's pages hold the tokens, the group's queries lie side by side, this one's among them
    const bool fits = led && changes[min(end - 1, last) - base] == changes[max((int64_t)e.first, base) - base] &&
                      (e.first >= base || left) && (end - 1 <= last || right) && lead.len - lead.count >= e.tokens &&
                      s.len - s.count >= e.tokens && stop <= total && lead.token + lead.count <= stop &&
                      s.token >= lead.token && s.token + s.count <= stop;
    if (fits) out = {e.tokens, e.first == i ? stop - s.token : 0};
    bad = !fits;
  }
  if (bad) kv_status(kv, kKvBadEntry);
  entries[i] = out;
}

}  // namespace

cudaError_t launch_kv_entries(const KvView& kv, const int32_t* slots, const int32_t* starts, const int32_t* plan,
                              int64_t n, int64_t total, KvShared* entries, cudaStream_t s) {
  k_share_entries<<<(unsigned)((n + GROUPS - 1) / GROUPS), GROUPS, 0, s>>>(kv, slots, starts, plan, n, total, entries);
  return cudaGetLastError();
}

cudaError_t launch_kv_share(const KvView& kv, const int32_t* slots, const int32_t* starts, int64_t n, int32_t* plan,
                            cudaStream_t s) {
  k_share_pairs<<<(unsigned)((n + PAIRS - 1) / PAIRS), PAIRS * 32, 0, s>>>(kv, slots, starts, n, plan);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_maybe_pdl(true, k_share_groups, dim3(1), dim3(GROUPS), 0, s, n, plan);
}

}  // namespace tq
