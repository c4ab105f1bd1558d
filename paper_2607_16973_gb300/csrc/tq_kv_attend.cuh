// What the two attention kernels of the 8-bit cache share: the call's arguments,
// the cut of its work into equal runs, and the join of what the cuts leave.
//
// Work: items (sequence, tile of rows, key head), laid end to end, each as long as
// the blocks of tokens that its rows see (and a fixed amount for its setup), cut
// into runs of equal length, one for each block of threads, so that ragged
// batches and single long sequences load every SM alike.  A row is a query of
// one head: row r of a sequence is query r / group of head (key head) * group +
// r % group.
#pragma once

#include <type_traits>

#include "tq_kv.cuh"
#include "tq_topk.cuh"

namespace tq {

struct AttendArgs {
  KvView kv;
  int layer;
  const int32_t *slots, *starts;
  int64_t n, total;
  KvRows q;
  bool q_wide;           // every row of q starts on a 16-byte boundary
  int heads, group;
  float scale;
  int window;
  void* out;
  float* lse;
  float* parts;          // [2 * grid][rows * (D + 2)]: partial O, m, l
  struct Split* splits;  // [grid]
};

// The item that a run continues, left for k_kv_join by the first run that does.
struct Split {
  int first, last;      // runs that have a part of it; first = -1: none to join
  int token, head;      // first token of its sequence, its key head
  int row0, rows;       // first row of its tile, rows of its sequence
};

// Rows per key head that a sequence of the call brings on average.
inline int64_t attend_rows(const KvView& kv, int64_t n, int64_t total, int heads) {
  return n > 0 ? (total + n - 1) / n * (heads / kv.c.kv_heads) : 0;
}

// The tensor-core tiles (tq_kv_tile.cu).
bool kv_tile_supported(const KvView& kv, int64_t n, int64_t total, int heads);
size_t kv_tile_workspace(const KvView& kv);
cudaError_t launch_kv_tile(AttendArgs a, int type, void* workspace, cudaStream_t s);

namespace {

constexpr int CHUNK = 512;  // sequences whose units are kept in shared memory at a time
constexpr int SCAN = 128;   // threads that sum them
constexpr float LN2 = 0.6931471805599453f, LOG2E = 1.4426950408889634f;

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A kernel's cut: ROWS rows to a tile, blocks of BLOCK tokens, an item's setup in
// blocks, and the fewest blocks that are worth a run.
template <int ROWS_, int BLOCK_, int ITEM_, int MIN_>
struct Cut {
  static constexpr int ROWS = ROWS_, BLOCK = BLOCK_, ITEM = ITEM_, MIN = MIN_;
};

// Blocks that the rows of a tile see: [first, first + blocks).
struct Span {
  int first, blocks;
  int place_lo, place_hi;  // places of its first and last row
};

template <class P>
__device__ __forceinline__ Span tile_span(const AttendArgs& a, const KvSeq& s, int tile) {
  Span w;
  const unsigned group = (unsigned)a.group, row0 = (unsigned)tile * P::ROWS;
  const unsigned last = min((unsigned)s.count * group, row0 + P::ROWS) - 1;
  w.place_lo = s.len - s.count + (int)(row0 / group);
  w.place_hi = s.len - s.count + (int)(last / group);
  // (a row in front of the sequence's first token sees nothing; its place may be as far below 0 as int reaches)
  w.first = a.window ? max(0, max(0, w.place_lo) - a.window + 1) / P::BLOCK : 0;
  w.blocks = w.place_hi < 0 ? 0 : max(0, w.place_hi / P::BLOCK + 1 - w.first);
  return w;
}

// (rows of a sequence fit in 31 bits: the call's queries times heads do)
template <class P>
__device__ __forceinline__ int tiles_of(const AttendArgs& a, const KvSeq& s) {
  return (int)(((unsigned)s.count * (unsigned)a.group + P::ROWS - 1) / P::ROWS);
}

// Sums of the sequences' units, found by a whole block: before[i] is what lies
// in front of sequence base + i.
struct Units {
  int64_t before[CHUNK + 1];
  KvSeq seq[CHUNK];
  int64_t warp_sums[SCAN / 32];
  int64_t base, total;
};

template <class P>
__device__ void load_chunk(const AttendArgs& a, Units& u, int64_t base, int64_t sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();  // (a warp may still look an item up in the chunk that this one replaces)
  for (int j0 = 0; j0 < CHUNK; j0 += SCAN) {
    if (base + j0 >= a.n && j0) break;
    const int j = j0 + threadIdx.x;
    int64_t mine = 0, run = 0;
    if (threadIdx.x < SCAN) {
      if (base + j < a.n) {
        KvSeq s;
        if (!kv_seq(a.kv, a.slots, a.starts, base + j, a.total, true, s)) {
          if (blockIdx.x == 0) kv_status(a.kv, kKvBadEntry);
          s.len = 0;
          if (s.token < 0 || s.count < 0 || s.count > a.total || s.token > a.total - s.count) s.count = 0;
        }
        u.seq[j] = s;
        const int tiles = tiles_of<P>(a, s);
        for (int t = 0; t < tiles; ++t) mine += P::ITEM + tile_span<P>(a, s, t).blocks;
        mine *= a.kv.c.kv_heads;
      }
      run = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(FULL, run, o);
        if (lane >= o) run += y;
      }
      if (lane == 31) u.warp_sums[warp] = run;
    }
    __syncthreads();
    int64_t front = 0, all = 0;
#pragma unroll
    for (int w = 0; w < SCAN / 32; ++w) {
      if (w < warp) front += u.warp_sums[w];
      all += u.warp_sums[w];
    }
    if (threadIdx.x < SCAN) u.before[j] = sum + front + run - mine;
    sum += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    u.base = base;
    u.total = sum;
  }
  __syncthreads();
}

// The units of the whole call; the first chunk is loaded last.
template <class P>
__device__ int64_t load_units(const AttendArgs& a, Units& u) {
  load_chunk<P>(a, u, 0, 0);
  if (a.n <= CHUNK) return u.total;
  int64_t sum = u.total;
  for (int64_t base = CHUNK; base < a.n; base += CHUNK) {
    load_chunk<P>(a, u, base, sum);
    sum = u.total;
  }
  load_chunk<P>(a, u, 0, 0);
  return sum;
}

// The item that unit x falls into, found by a warp; the chunk with x is loaded.
struct Item {
  KvSeq s;
  Span span;
  int64_t begin;  // its first unit
  int tile, head, units;
};

template <class P>
__device__ Item find_item(const AttendArgs& a, const Units& u, int64_t x) {
  const int lane = threadIdx.x & 31;
  const int64_t i = warp_last_not_above(min((int64_t)CHUNK, a.n - u.base), x, [&](int64_t j) { return u.before[j]; });
  Item it;
  it.s = u.seq[i];
  const int tiles = tiles_of<P>(a, it.s);
  int64_t in = x - u.before[i];
  for (int base = 0;; base += 32) {  // a tile per lane
    const int64_t mine = base + lane < tiles ? (int64_t)(P::ITEM + tile_span<P>(a, it.s, base + lane).blocks) * a.kv.c.kv_heads : 0;
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(FULL, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned past = __ballot_sync(FULL, upto > in);
    if (past || base + 32 >= tiles) {
      const int at = past ? __ffs(past) - 1 : 0;
      in -= __shfl_sync(FULL, upto - mine, at);
      it.tile = base + at;
      break;
    }
    in -= __shfl_sync(FULL, upto, 31);
  }
  it.span = tile_span<P>(a, it.s, it.tile);
  it.units = P::ITEM + it.span.blocks;
  it.head = (int)(in / it.units);
  it.begin = x - in % it.units;
  return it;
}

// Loads the chunk that unit x falls into; x does not go back behind the one that is
// loaded.  By the whole block.
template <class P>
__device__ __forceinline__ void chunk_of(const AttendArgs& a, Units& u, int64_t x) {
  while (x >= u.total) load_chunk<P>(a, u, u.base + CHUNK, u.total);  // (uniform: x and u are the block's)
}

// Runs that share `units`; where run c starts if nothing is in the way; the last
// run that starts at or in front of a unit, the first at or behind it.
template <class P>
__device__ __forceinline__ int64_t runs(int64_t units, int64_t grid) {
  return max((int64_t)1, min(grid, units / P::MIN));
}
__device__ __forceinline__ int64_t run_start(int64_t c, int64_t units, int64_t n) { return c * units / n; }
__device__ __forceinline__ int64_t last_run(int64_t unit, int64_t units, int64_t n) { return ((unit + 1) * n - 1) / units; }
__device__ __forceinline__ int64_t first_run(int64_t unit, int64_t units, int64_t n) { return (unit * n + units - 1) / units; }

// Where run c really starts: not within MIN blocks of an item's ends, but at that
// end.  Items of less than 2 MIN blocks are never cut, so that where the cuts fall
// does not change a short sequence's result.  (The batch still does through the rows
// that its sequences bring on average: they decide on the kernel and its row tiles,
// which round weights differently.)
template <class P>
__device__ int64_t run_cut(const AttendArgs& a, Units& u, int64_t c, int64_t units, int64_t n) {
  const int64_t x = run_start(c, units, n);
  if (x >= units) return units;
  chunk_of<P>(a, u, x);
  const Item it = find_item<P>(a, u, x);
  const int64_t in = x - it.begin;
  return in < P::ITEM + P::MIN ? it.begin : it.units - in < P::MIN ? it.begin + it.units : x;
}

// A segment of a run: blocks [b_first, b_last) of an item, a whole item if both are
// its ends.
struct Segment {
  Item it;
  int b_first, b_last;
  bool whole;
  int row0, rows;
  int64_t next;  // the unit behind it
};

// A block's run [u, end), in shared memory: what is only needed between segments
// takes no registers within them.
struct Run {
  int64_t all, n_runs, u, end;
  Segment seg;
};

// Sets this block's run up: false if it has none.  Leaves the chunk of its start
// loaded, and its entry of `splits` empty.
template <class P>
__device__ bool my_run(const AttendArgs& a, Units& units, Run& run) {
  const int64_t all = load_units<P>(a, units), n_runs = runs<P>(all, gridDim.x);
  if (threadIdx.x == 0) a.splits[blockIdx.x].first = -1;
  if (blockIdx.x >= n_runs) return false;
  const int64_t u = run_cut<P>(a, units, blockIdx.x, all, n_runs);
  const int64_t chunk = units.base, sum = units.before[0];
  const int64_t end = run_cut<P>(a, units, blockIdx.x + 1, all, n_runs);
  if (units.base != chunk) load_chunk<P>(a, units, chunk, sum);  // (uniform)
  if (threadIdx.x == 0) {
    run.all = all;
    run.n_runs = n_runs;
    run.u = u;
    run.end = end;
  }
  __syncthreads();
  return run.u < run.end;
}

// Finds the next segment of the run, in run.seg; the caller moves run.u on, behind
// a barrier.  Notes an item that this run is the first to continue.
template <class P>
__device__ __forceinline__ void next_segment(const AttendArgs& a, Units& units, Run& run) {
  chunk_of<P>(a, units, run.u);
  if (threadIdx.x < 32) {
    const int64_t u = run.u;
    Segment g;
    g.it = find_item<P>(a, units, u);
    const int in = (int)(u - g.it.begin);
    g.b_first = max(0, in - P::ITEM);
    g.b_last = (int)min((int64_t)g.it.span.blocks, in + (run.end - u) - P::ITEM);
    g.whole = g.b_first == 0 && g.b_last == g.it.span.blocks;
    g.row0 = g.it.tile * P::ROWS;
    g.rows = g.it.s.count * a.group;
    g.next = u + P::ITEM + g.b_last - in;
    if (threadIdx.x == 0) {
      run.seg = g;
      if (g.b_first) {
        const int first = (int)first_run(g.it.begin + P::ITEM + P::MIN, run.all, run.n_runs) - 1;
        if (first + 1 == (int)blockIdx.x)
          a.splits[blockIdx.x] = {first,         (int)last_run(g.it.begin + g.it.units - P::MIN, run.all, run.n_runs),
                                  g.it.s.token, g.it.head, g.row0, g.rows};
      }
    }
  }
  __syncthreads();
}

// Where this segment's partial sums go: a run has one that continues an item at
// most, and one that begins an item and does not end it.
template <int D, int ROWS>
__device__ __forceinline__ float* part_of(const AttendArgs& a, const Segment& g) {
  return a.parts + ((int64_t)blockIdx.x * 2 + (g.b_first == 0)) * (ROWS * (D + 2));
}
// Output row (token, head) of row r of a sequence.
__device__ __forceinline__ int64_t out_row(const AttendArgs& a, int token, int head, int r) {
  return (int64_t)(token + r / a.group) * a.heads + head * a.group + r % a.group;
}
// (l = 0: nothing was seen; NaN: the query is not finite)
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -INFINITY : m * LN2 + logf(l); }

// Joins the items that several runs share, in the runs' order: a block per run
// that continues one and 8 of its rows.  A warp takes every 8th part, the 8
// rows of it at once, so that many parts are on their way together (every 4th at
// head_dim 256).  A part in which a row saw nothing has m = -inf and l = 0 and is
// left out; m = -inf beside another l is a row of NaN, which joins to NaN.
//
// PAD more columns of blocks write the queries that no sequence brings, in front
// of the first one's and behind the last one's (a call padded to a size that is
// kept): what a query that sees nothing gets.  (Asked by every block it was 1 us
// of every call: they start where the attention's blocks end.)
constexpr int PAD = 16;
constexpr int join_warps(int dim) { return dim == 256 ? 4 : 8; }  // (their sums take 32 KB of shared memory)
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(join_warps(D) * 32) void k_kv_join(AttendArgs a) {
  constexpr int JOIN_WARPS = join_warps(D);
  constexpr int E = D / 32;  // elements of a lane
  using Vec = typename std::conditional<E == 2, float2, float4>::type;
  constexpr int V = E * 4 / sizeof(Vec);
  __shared__ float sh_o[JOIN_WARPS][8][D];
  __shared__ float sh_l[JOIN_WARPS][8], sh_m[JOIN_WARPS][8];
  if (blockIdx.x < PAD) {
    const int64_t front = min(max((int64_t)a.starts[0], (int64_t)0), a.total);
    const int64_t behind = min(max((int64_t)a.starts[a.n], front), a.total);
    const int pieces = a.heads * (D / 8);  // of 16 bytes, of a token
    griddep_wait();
    for (int64_t e = ((int64_t)blockIdx.y * PAD + blockIdx.x) * blockDim.x + threadIdx.x;
         e < (front + a.total - behind) * pieces; e += (int64_t)gridDim.y * PAD * blockDim.x) {
      const int64_t nth = e / pieces, token = nth < front ? nth : behind + nth - front;
      const int piece = (int)(e - nth * pieces);
      static_cast<uint4*>(a.out)[token * pieces + piece] = make_uint4(0, 0, 0, 0);
      if (a.lse && piece % (D / 8) == 0) a.lse[token * a.heads + piece / (D / 8)] = -INFINITY;
    }
    return;
  }
  griddep_wait();
  const Split sp = a.splits[blockIdx.x - PAD];
  const int row0 = blockIdx.y * 8;
  if (sp.first < 0 || sp.row0 + row0 >= sp.rows) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int live = min(8, sp.rows - sp.row0 - row0);
  auto part = [&](int x) { return a.parts + ((int64_t)x * 2 + (x == sp.first)) * (ROWS * (D + 2)); };
  float o[8][E], m[8], l[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[r][e] = 0.0f;
  }
  for (int x = sp.first + warp; x <= sp.last; x += JOIN_WARPS) {
    const float* p = part(x);
    union {
      Vec v[V];
      float f[E];
    } z[8];
    float mm[8], ll[8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (r < live) {
#pragma unroll
        for (int v = 0; v < V; ++v) z[r].v[v] = *reinterpret_cast<const Vec*>(p + (row0 + r) * D + lane * E + v * (int)(sizeof(Vec) / 4));
        mm[r] = p[ROWS * D + row0 + r];
        ll[r] = p[ROWS * (D + 1) + row0 + r];
      }
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (r < live && (mm[r] > -INFINITY || ll[r] != 0.0f)) {
        const float top = fmaxf(m[r], mm[r]), keep = ex2(m[r] - top), f = ex2(mm[r] - top);
        m[r] = top;
        l[r] = l[r] * keep + ll[r] * f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[r][e] = o[r][e] * keep + z[r].f[e] * f;
      }
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
#pragma unroll
    for (int e = 0; e < E; ++e) sh_o[warp][r][lane * E + e] = o[r][e];
    if (lane == 0) {
      sh_m[warp][r] = m[r];
      sh_l[warp][r] = l[r];
    }
  }
  __syncthreads();
  for (int r = warp; r < live; r += JOIN_WARPS) {
    float top = -INFINITY, sum = 0.0f, y[E];
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = 0.0f;
#pragma unroll
    for (int x = 0; x < JOIN_WARPS; ++x) top = fmaxf(top, sh_m[x][r]);
#pragma unroll
    for (int x = 0; x < JOIN_WARPS; ++x) {
      const float f = top > -INFINITY ? ex2(sh_m[x][r] - top) : 1.0f;  // (1: sums of 0, or NaN)
      sum += f * sh_l[x][r];
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] += f * sh_o[x][r][lane * E + e];
    }
    const int64_t at = out_row(a, sp.token, sp.head, sp.row0 + row0 + r);
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    T* out = static_cast<T*>(a.out) + at * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = from_float<T>(y[e] * inv);
    if (a.lse && lane == 0) a.lse[at] = lse_of(top, sum);
  }
}

// Workspace: Split [grid] | partial sums.
template <typename T, int D, int ROWS>
cudaError_t launch_join(const AttendArgs& a, int grid, cudaStream_t s) {
  return launch_maybe_pdl(true, k_kv_join<T, D, ROWS>, dim3(PAD + grid, ROWS / 8), dim3(join_warps(D) * 32), 0, s, a);
}

inline size_t split_bytes(int grid) { return ((size_t)grid * sizeof(Split) + 255) / 256 * 256; }
inline size_t attend_workspace(int grid, int rows, int dim) {
  return split_bytes(grid) + (size_t)grid * 2 * rows * (dim + 2) * sizeof(float);
}
inline void take_workspace(AttendArgs& a, int grid, void* workspace) {
  a.splits = static_cast<Split*>(workspace);
  a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + split_bytes(grid));
}

}  // namespace
}  // namespace tq
