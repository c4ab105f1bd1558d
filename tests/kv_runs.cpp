// The cut of attention's work into runs (tq_kv_attend.cuh), run on the CPU: a
// block's threads are fibers that change places only where the CUDA code waits
// for others (a barrier of the block, a vote or a shuffle of a warp).  Warp
// `ahead` goes on whenever it can, so it runs as far in front of the others as
// the code lets it.
//
// stdin:  kernel ahead grid n group kv_heads window max_pages page_tokens, then n
//         times: tokens held, new ones
// stdout: "run c u end" of every block that has one, "segment c token tile head
//         b_first b_last blocks first place_lo place_hi whole row0 rows" of each of
//         its segments, "split c first last token head row0 rows"
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <type_traits>
#include <vector>

#include <ucontext.h>

// ---- a block of threads -----------------------------------------------------
namespace emu {
constexpr size_t STACK = 64 * 1024;
struct Group {  // of threads that wait for one another
  int size, arrived = 0;
  uint64_t round = 0;
  uint64_t slot[2][32];  // what a warp's threads hand over
};
struct Fiber {
  ucontext_t at;
  std::vector<char> stack = std::vector<char>(STACK);
  Group* waits = nullptr;
  uint64_t round = 0;
  bool done = false;
};
std::vector<Fiber> fibers;
std::vector<Group> warps;
Group block;
ucontext_t scheduler;
int now, ahead;
void (*body)();

// Waits for the group's other threads.
void meet(Group& g) {
  const uint64_t round = g.round;
  if (++g.arrived == g.size) {
    g.arrived = 0;
    ++g.round;
  } else {
    fibers[now].waits = &g;
    fibers[now].round = round;
  }
  swapcontext(&fibers[now].at, &scheduler);  // (the last one too: who goes on is the scheduler's choice)
}
Group& warp() { return warps[now / 32]; }
// Each thread of a warp gives x; returns everyone's.
const uint64_t* trade(uint64_t x) {
  Group& g = warp();
  const uint64_t round = g.round;
  g.slot[round & 1][now & 31] = x;
  meet(g);
  return g.slot[round & 1];
}
void enter() {
  body();
  fibers[now].done = true;
  swapcontext(&fibers[now].at, &scheduler);
}
// False if some threads wait for others that have left.
bool run(int threads) {
  fibers = std::vector<Fiber>(threads);
  warps.assign(threads / 32, Group{32});
  block = Group{threads};
  for (Fiber& f : fibers) {
    getcontext(&f.at);
    f.at.uc_stack.ss_sp = f.stack.data();
    f.at.uc_stack.ss_size = f.stack.size();
    f.at.uc_link = nullptr;
    makecontext(&f.at, enter, 0);
  }
  for (;;) {
    int next = -1, left = 0;
    for (int i = 0; i < threads; ++i) {
      const int t = (ahead * 32 + 31 - i + threads) % threads;
      Fiber& f = fibers[t];
      left += !f.done;
      if (f.done || (f.waits && f.waits->round == f.round)) continue;
      next = t;
      break;
    }
    if (next < 0) return left == 0;
    now = next;
    fibers[now].waits = nullptr;
    swapcontext(&scheduler, &fibers[now].at);
  }
}
template <typename T> uint64_t bits(T x) {
  uint64_t u = 0;
  memcpy(&u, &x, sizeof x);
  return u;
}
template <typename T> T value(uint64_t u) {
  T x;
  memcpy(&x, &u, sizeof x);
  return x;
}
struct Thread {
  struct X {
    operator int() const { return now; }
  } x;
};
}  // namespace emu

// ---- what of CUDA the header uses ---------------------------------------------
static emu::Thread threadIdx;
static struct { int x, y; } blockIdx, gridDim;
static struct { int x; } blockDim;
static void __syncthreads() { emu::meet(emu::block); }
static void __syncwarp() { emu::meet(emu::warp()); }
static unsigned __ballot_sync(unsigned, bool p) {
  const uint64_t* all = emu::trade(p);
  unsigned r = 0;
  for (int i = 0; i < 32; ++i) r |= (unsigned)all[i] << i;
  return r;
}
template <typename T> T __shfl_sync(unsigned, T x, int from) { return emu::value<T>(emu::trade(emu::bits(x))[from & 31]); }
template <typename T> T __shfl_up_sync(unsigned, T x, int by) {
  const int lane = emu::now & 31;
  return emu::value<T>(emu::trade(emu::bits(x))[lane >= by ? lane - by : lane]);
}
static int __clz(unsigned x) { return x ? __builtin_clz(x) : 32; }
static int __ffs(unsigned x) { return __builtin_ffs((int)x); }
static int atomicOr(int* p, int x) { return __sync_fetch_and_or(p, x); }
static unsigned __float_as_uint(float x) { return emu::value<unsigned>(emu::bits(x)); }
static unsigned __byte_perm(unsigned, unsigned, unsigned) { abort(); }  // (not reached)
static unsigned __vmaxu2(unsigned, unsigned) { abort(); }
static float __uint_as_float(unsigned) { abort(); }
template <typename A, typename B> typename std::common_type<A, B>::type min(A a, B b) { return a < b ? a : b; }
template <typename A, typename B> typename std::common_type<A, B>::type max(A a, B b) { return a > b ? a : b; }

#undef __launch_bounds__
#define __launch_bounds__(...)
#include "tq_kv_attend.cuh"

// ---- the kernels' use of it -----------------------------------------------------
static tq::AttendArgs args;
static tq::Units units;
static tq::Run the_run;
static bool has[1024];

template <class P>
void block_body() {
  const int t = threadIdx.x;
  has[t] = tq::my_run<P>(args, units, the_run);
  if (!has[t]) return;
  if (t == 0) printf("run %d %lld %lld\n", blockIdx.x, (long long)the_run.u, (long long)the_run.end);
  while (the_run.u < the_run.end) {
    tq::next_segment<P>(args, units, the_run);
    if (t == 0) {
      const tq::Segment& g = the_run.seg;
      printf("segment %d %d %d %d %d %d %d %d %d %d %d %d %d\n", blockIdx.x, g.it.s.token, g.it.tile, g.it.head, g.b_first,
             g.b_last, g.it.span.blocks, g.it.span.first, g.it.span.place_lo, g.it.span.place_hi, (int)g.whole, g.row0, g.rows);
    }
    __syncthreads();
    if (t == 0) the_run.u = the_run.seg.next;
    __syncthreads();
  }
}

int main() {
  char kernel[16];
  long long n, max_pages;
  int grid, group, kv_heads, window, page;
  if (scanf("%15s %d %d %lld %d %d %d %lld %d", kernel, &emu::ahead, &grid, &n, &group, &kv_heads, &window, &max_pages,
            &page) != 9)
    return 2;
  std::vector<int32_t> slots(n), starts(n + 1), lens(n);
  for (long long i = 0; i < n; ++i) {
    int count;
    if (scanf("%d %d", &lens[i], &count) != 2) return 2;
    slots[i] = (int)i;
    starts[i + 1] = starts[i] + count;
  }
  int32_t status = 0;
  std::vector<tq::Split> splits(grid);
  args = {};
  args.kv.c.slots = n;
  args.kv.c.lens = lens.data();
  args.kv.c.status = &status;
  args.kv.c.kv_heads = kv_heads;
  args.kv.c.max_pages = max_pages;
  args.kv.c.page_tokens = page;
  args.kv.max_len = max_pages * page;
  args.slots = slots.data();
  args.starts = starts.data();
  args.n = n;
  args.total = starts[n];
  args.heads = group * kv_heads;
  args.group = group;
  args.window = window;
  args.splits = splits.data();
  gridDim = {grid, 1};
  int threads = 128;
  if (!strcmp(kernel, "stream8")) emu::body = block_body<tq::Cut<8, 16, 16, 4>>;
  else if (!strcmp(kernel, "stream16")) emu::body = block_body<tq::Cut<16, 16, 16, 4>>;
  else if (!strcmp(kernel, "tile")) emu::body = block_body<tq::Cut<256, 128, 4, 1>>, threads = 384;
  else return 2;
  blockDim.x = threads;
  for (int c = 0; c < grid; ++c) {
    blockIdx = {c, 0};
    memset(&units, 0xCC, sizeof units);  // (shared memory holds anything at a block's start)
    memset(&the_run, 0xCC, sizeof the_run);
    if (!emu::run(threads)) {
      printf("stuck %d\n", c);
      return 0;
    }
    const tq::Split& s = splits[c];
    if (s.first >= 0) printf("split %d %d %d %d %d %d %d\n", c, s.first, s.last, s.token, s.head, s.row0, s.rows);
  }
  printf("status %d\n", status);
  return 0;
}
