// tq_kv_attend: causal attention of the last tokens of each sequence over the
// 8-bit cache, in one pass over the codes.
//
//   out = sum_j e^(s_j) v_j / sum_j e^(s_j),   s_j = scale * q . k_j
//
// The queries that read one key head (its group of query heads, times the new
// tokens) are the columns of two small products with a block of 16 tokens,
//
//   S^T [16 tokens x rows] = K [16 x D] Q^T,     O^T [D x rows] += V^T [D x 16] P^T
//
// with the codes as the A operands, converted in registers (exact in fp16),
// so that a lane loads exactly the 16-byte pieces it needs, straight from HBM
// to registers: no shared memory, no layout but the plain one.  The order of
// the contraction index is free as long as both operands agree on it, which is
// what makes plain 16-byte loads fit the fragments:
//   K: lane (g, t) loads bytes 16t .. 16t+15 of tokens g and g + 8 (and the same
//      64, 128, 192 further on); word s of a piece is contraction step s;
//   V: lane (g, t) loads bytes 16g .. of tokens 2t, 2t+1, 2t+8, 2t+9; two byte
//      permutes pair the tokens of one element.
// The probabilities go from the layout of S^T to that of the B operand by
// movmatrix.  Scales: a block of keys has one factor, applied to the scores; a
// block of values has one, applied to the block's product, which is therefore
// taken by itself and added in float32.
//
// The softmax keeps a reference m per row that only moves when a score passes
// the one it was set to by LAZY: most blocks need no reduction over the warp.
//
// Bound: HBM, 2 (D + 1/4) bytes per token and key head.  200,001 tokens and 8 key
// heads (410 MB): 85 us, 4.8 TB/s of 6.8 measured; 100,001 tokens 57, 400,001 143:
// about 28 us for the start, the first loads, the sums and the join, and the rest at
// 7 TB/s.  128 sequences of 1,000 to 4,096 (663 MB): 119 us, 5.6 TB/s.
//
// The same code serves tq_kv_cross (every row sees all tokens) and tq_kv_attend_shared: there
// it, or the tiles, runs once over the shared tokens with the rows of all requests of a
// group, whose sums stay in float32, and once over each request's own, where the joined
// sums are written.  96 readers over 1,250 to 5,000 tokens (617 MB): 132 us, 4.7 TB/s; 64
// requests over 4 contexts of up to 12,000 tokens (157 MB read, 16 times as much without
// sharing): 116 us, of which the shared tokens take 57 and their join 12, each request's
// own 40 and their join 8 (one by one).
#include <algorithm>

#include "tq_kv_attend.cuh"

namespace tq {
namespace {

constexpr int WARPS = 4;
constexpr int THREADS = WARPS * 32;
// Weights are held as 2^(s - m) with the reference m LEAD below the largest score
// that it was last set to, and moved again when a score passes that by LAZY:
// they stay under 2^15, fp16's largest, and those down to 2^-24 of the largest
// one keep all of fp16's bits.
constexpr float LEAD = 10.0f, LAZY = 5.0f;
constexpr int AHEAD = 1;         // blocks of a warp on their way to L2 beyond the one on its way to registers (none: 102 us
                                 // for 200,001 tokens, 1: 84, 2: 85, 4: 98, 10: 123, what is on its way then fills L2)

// Rows come in tiles of 8 or 16; a run is worth 4 blocks (2: 12.4 us for one query
// over 1,031 tokens, 4: 11.6, 8: 12.8), and an item costs about as much as 16
// beside its own: looking it up, its queries, its sums (128 ragged sequences: 138 us
// counted as 4, 124 as 8, 114 as 16 to 32, 116 as 48).
template <int NT, bool CAUSAL>
using StreamCut = Cut<8 * NT, kKvBlock, 16, 4, CAUSAL>;

// Two pairs of fp16 values from the four codes of a word: every code is exact.
template <int CODES>
__device__ __forceinline__ void to_half4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (CODES == TQ_KV_INT8) {
    const uint32_t u = w ^ 0x80808080u;  // code + 128
    const __half2 bias = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));  // 1024 + 128
    union { uint32_t r; __half2 h; } x;
    x.r = __byte_perm(u, 0x64646464u, 0x4140);  // 1024 + byte
    x.h = __hsub2(x.h, bias);
    lo = x.r;
    x.r = __byte_perm(u, 0x64646464u, 0x4342);
    x.h = __hsub2(x.h, bias);
    hi = x.r;
  } else {
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
  }
}

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int D>
struct Piece {  // what a lane loads of a row: K pieces of 16 bytes, V pieces of 16 (8 at D = 64)
  static constexpr int K = D / 64;
  static constexpr int VW = D == 64 ? 2 : 4;      // words of a V piece
  static constexpr int V = D == 256 ? 2 : 1;
};

// Blocks of threads per SM, by the registers that the accumulators leave.
constexpr int per_sm(int dim, int nt) { return dim == 256 ? 2 : nt == 1 ? 4 : 3; }

template <typename T, int D, int CODES, int NT, bool CAUSAL>
__global__ __launch_bounds__(THREADS, per_sm(D, NT)) void k_kv_attend(AttendArgs a) {
  using P = StreamCut<NT, CAUSAL>;
  constexpr int ROWS = P::ROWS;
  constexpr int KP = Piece<D>::K, VP = Piece<D>::V, VW = Piece<D>::VW;
  constexpr int MT = D / 16;  // m-tiles of O^T
  __shared__ UnitsOf<CAUSAL> units;
  __shared__ Run run;
  __shared__ alignas(16) float sh_o[WARPS][ROWS][D + 4];  // (read two at a time)
  __shared__ float sh_m[WARPS][ROWS], sh_l[WARPS][ROWS];

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const KvView& kv = a.kv;
  griddep_launch_dependents();
  if (!my_run<P>(a, units, run)) return;

  while (run.u < run.end) {
    next_segment<P>(a, units, run);
    const KvSeq sq = run.seg.it.s;
    const Span span = run.seg.it.span;
    const int from = CAUSAL ? 0 : run.seg.it.from;
    const int head = run.seg.it.head, row0 = run.seg.row0, rows = run.seg.rows;

    if (run.seg.b_first == run.seg.b_last) {  // no row sees a token
      for (int e = threadIdx.x; e < min(ROWS, rows - row0) * D; e += THREADS) {
        const int64_t at = out_row(a, sq.token, head, row0 + e / D);
        static_cast<T*>(a.out)[at * D + e % D] = from_float<T>(0.0f);
        if (a.lse && e % D == 0) a.lse[at] = -INFINITY;
      }
      __syncthreads();
      if (threadIdx.x == 0) run.u = run.seg.next;
      __syncthreads();
      continue;
    }

    // the queries, scaled by a power of two to fp16's middle: row n = g of each 8.  A row
    // that is not finite becomes NaN throughout, and so do its scores, whatever the codes.
    uint32_t qf[NT][KP * 4][2];
    float unscale[NT][2];         // of rows 2t and 2t + 1: scores in log2 units
    int place[NT][2];             // last token that they see; -1: none
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = row0 + nt * 8 + g;
      const bool real = row < rows;
      const int64_t token = sq.token + row / a.group;
      const T* p = static_cast<const T*>(a.q.p) + token * a.q.token_stride +
                   (int64_t)(head * a.group + row % a.group) * a.q.head_stride + 16 * t;
      union { uint4 v[2]; T e[16]; } x[KP];
      uint32_t bits = 0;
#pragma unroll
      for (int c = 0; c < KP; ++c) {
        x[c].v[0] = x[c].v[1] = make_uint4(0, 0, 0, 0);
        if (real) {
          if (((uintptr_t)(p + 64 * c) & 15) == 0) {
            x[c].v[0] = __ldg(reinterpret_cast<const uint4*>(p + 64 * c));
            x[c].v[1] = __ldg(reinterpret_cast<const uint4*>(p + 64 * c) + 1);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[c].e[e] = p[64 * c + e];
          }
        }
        bits = max_magnitude<T>(max_magnitude<T>(bits, x[c].v[0]), x[c].v[1]);
      }
      bits = max_magnitude<T>(bits, __shfl_xor_sync(FULL, bits, 1));
      bits = max_magnitude<T>(bits, __shfl_xor_sync(FULL, bits, 2));
      const float top = magnitude<T>(bits);
      // the largest element to [2^8, 2^9): both factors are powers of two within float32's normal range
      const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -110), 127);
      const float up = top < INFINITY ? __uint_as_float((uint32_t)(127 + min(8 - e, 118)) << 23) : NAN;
      const float down = a.scale * LOG2E / up;
#pragma unroll
      for (int c = 0; c < KP; ++c)
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            qf[nt][c * 4 + s][h] =
                pack_half2(to_float(x[c].e[4 * s + 2 * h]) * up, to_float(x[c].e[4 * s + 2 * h + 1]) * up);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        unscale[nt][h] = __shfl_sync(FULL, down, (2 * t + h) * 4);
        const int r = row0 + nt * 8 + 2 * t + h;
        place[nt][h] = r < rows ? max(-1, dense<P>(a) ? sq.len - 1 : sq.len - sq.count + r / a.group) : -1;
      }
    }
    const int blk = span.first + run.seg.b_first, blk_end = span.first + run.seg.b_last;
    // blocks that every row of the tile sees whole
    const int whole_from = !CAUSAL ? (from + kKvBlock - 1) / kKvBlock
                           : a.window && span.place_hi >= a.window ? (span.place_hi - a.window) / kKvBlock + 1 : 0;
    const int whole_to = span.place_lo >= 0 ? (span.place_lo + 1) / kKvBlock : 0;

    float o[NT][MT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < MT; ++j) o[nt][j][0] = o[nt][j][1] = o[nt][j][2] = o[nt][j][3] = 0.0f;
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.0f;
    }

    // This warp's blocks: blk + warp, + WARPS, ...; lane l looks up the place and the
    // scales of the l-th of 32 of them, 32 to 64 blocks before they are scored.
    const int32_t* table = kv.c.table + sq.slot * kv.c.max_pages;
    // (line: a block's place in the pool; they are of 1 KB at least, and 2^31 of them more than any memory)
    struct Lines {
      int line;
      float ks, vs;
    };
    auto look_up = [&](int it) {
      Lines x = {-1, 0.0f, 0.0f};
      const int b = blk + warp + (it + lane) * WARPS;
      if (b < blk_end) {
        const int64_t tok = (int64_t)b * kKvBlock;
        const int page = table[tok >> kv.page_shift];
        if (page >= 0 && page < kv.c.pages) {
          x.line = (int)(kv.scales_at(a.layer, page, head) + ((tok & (kv.c.page_tokens - 1)) / kKvBlock));
          x.ks = __ldg(kv.c.k_scale + x.line);
          x.vs = __ldg(kv.c.v_scale + x.line);
        } else {
          kv_status(kv, kKvBadEntry);
        }
      }
      return x;
    };
    uint4 kr[KP][2];
    uint32_t vr[VP][4][VW];
    auto load_k = [&](int ln) {
      const uint8_t* p = kv.c.k + (int64_t)ln * (kKvBlock * D) + g * D + 16 * t;
#pragma unroll
      for (int c = 0; c < KP; ++c) {
        kr[c][0] = __ldg(reinterpret_cast<const uint4*>(p + 64 * c));
        kr[c][1] = __ldg(reinterpret_cast<const uint4*>(p + 64 * c + 8 * D));
      }
    };
    auto load_v = [&](int ln) {
      const uint8_t* p = kv.c.v + (int64_t)ln * (kKvBlock * D) + 2 * t * D + (D == 64 ? 8 : 16) * g;
#pragma unroll
      for (int c = 0; c < VP; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint8_t* x = p + 128 * c + ((r & 1) + (r >> 1) * 8) * D;
          if (VW == 2) {
            const uint2 y = __ldg(reinterpret_cast<const uint2*>(x));
            vr[c][r][0] = y.x, vr[c][r][1] = y.y;
          } else {
            const uint4 y = __ldg(reinterpret_cast<const uint4*>(x));
            vr[c][r][0] = y.x, vr[c][r][1] = y.y, vr[c][r][VW - 2] = y.z, vr[c][r][VW - 1] = y.w;
          }
        }
    };
    // a block's keys are 2 or 4 KB in one piece, its values too: half of the lanes
    // fetch each, 128 bytes apart
    auto fetch = [&](int ln) {
      const uint8_t* p = (lane < 16 ? kv.c.k : kv.c.v) + (int64_t)ln * (kKvBlock * D) + (lane & 15) * 128;
#pragma unroll
      for (int x = 0; x < kKvBlock * D; x += 2048)
        if (x + (lane & 15) * 128 < kKvBlock * D) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + x));
    };
    const int steps = (blk_end - blk - warp + WARPS - 1) / WARPS;  // (<= 0: none)
    // the 32 blocks that lanes stand for now, and the 32 behind them
    Lines batch = look_up(0), after = look_up(32);
    int now = __shfl_sync(FULL, batch.line, 0);
    if (now >= 0) {
      load_k(now);
      load_v(now);
    }
    for (int x = 1; x <= AHEAD; ++x) {
      const int ln = __shfl_sync(FULL, batch.line, x);
      if (ln >= 0) fetch(ln);
    }
    for (int it = 0; it < steps; ++it) {
      const float k_scale = __shfl_sync(FULL, batch.ks, it & 31), v_scale = __shfl_sync(FULL, batch.vs, it & 31);
      if (((it + 1) & 31) == 0) {
        batch = after;
        after = look_up(it + 33);
      }
      // (the blocks behind the last have no line)
      const int next = __shfl_sync(FULL, batch.line, (it + 1) & 31);
      const int far = ((it + 1) & 31) + AHEAD;
      const int ln = __shfl_sync(FULL, far < 32 ? batch.line : after.line, far & 31);
      if (ln >= 0) fetch(ln);
      const int b = blk + warp + it * WARPS;
      float s[NT][4];
      if (now >= 0) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.0f;
#pragma unroll
        for (int c = 0; c < KP; ++c) {
          const uint32_t x[4] = {kr[c][0].x, kr[c][0].y, kr[c][0].z, kr[c][0].w};
          const uint32_t y[4] = {kr[c][1].x, kr[c][1].y, kr[c][1].z, kr[c][1].w};
#pragma unroll
          for (int st = 0; st < 4; ++st) {
            uint32_t a0, a1, a2, a3;
            to_half4<CODES>(x[st], a0, a2);
            to_half4<CODES>(y[st], a1, a3);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma16816(s[nt], a0, a1, a2, a3, qf[nt][c * 4 + st][0], qf[nt][c * 4 + st][1]);
          }
        }
      }
      if (next >= 0) load_k(next);
      if (now >= 0) {
        bool rise = false;
        const bool whole = b >= whole_from && b < whole_to;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int h = x & 1;
            float y = s[nt][x] * (k_scale * unscale[nt][h]);
            if (!whole) {
              const int tok = b * kKvBlock + g + (x >> 1) * 8;
              if (tok > place[nt][h] || (!CAUSAL ? tok < from : a.window && tok <= place[nt][h] - a.window)) y = -INFINITY;
            }
            s[nt][x] = y;
            rise |= y > m[nt][h] + (LEAD + LAZY);
          }
        if (__any_sync(FULL, rise)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float top = fmaxf(m[nt][h], fmaxf(s[nt][h], s[nt][2 + h]) - LEAD);
              top = fmaxf(top, __shfl_xor_sync(FULL, top, 4));
              top = fmaxf(top, __shfl_xor_sync(FULL, top, 8));
              top = fmaxf(top, __shfl_xor_sync(FULL, top, 16));
              const float keep = top > m[nt][h] ? ex2(m[nt][h] - top) : 1.0f;
              m[nt][h] = top;
              l[nt][h] *= keep;
#pragma unroll
              for (int j = 0; j < MT; ++j) {
                o[nt][j][h] *= keep;
                o[nt][j][2 + h] *= keep;
              }
            }
        }
        if (CODES == TQ_KV_E4M3 && !whole) {
          // bytes that no token owns may be NaN, and 0 times that is not 0
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (b * kKvBlock + 2 * t + (r & 1) + (r >> 1) * 8 >= sq.len) {
#pragma unroll
              for (int c = 0; c < VP; ++c)
#pragma unroll
                for (int x = 0; x < VW; ++x) vr[c][r][x] = 0;
            }
        }
        uint32_t pf[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float m0 = m[nt][0] == -INFINITY ? 0.0f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.0f : m[nt][1];
          const float p0 = ex2(s[nt][0] - m0), p1 = ex2(s[nt][1] - m1);
          const float p2 = ex2(s[nt][2] - m0), p3 = ex2(s[nt][3] - m1);
          l[nt][0] += p0 + p2;
          l[nt][1] += p1 + p3;
          pf[nt][0] = transpose8x8(pack_half2(p0, p1));
          pf[nt][1] = transpose8x8(pack_half2(p2, p3));
        }
#pragma unroll
        for (int c = 0; c < VP; ++c)
#pragma unroll
          for (int x = 0; x < VW; ++x)
#pragma unroll
            for (int half = 0; half < 2; ++half) {  // elements 0, 1 and 2, 3 of the word
              const uint32_t sel = half ? 0x7362 : 0x5140;
              uint32_t a0, a1, a2, a3;
              to_half4<CODES>(__byte_perm(vr[c][0][x], vr[c][1][x], sel), a0, a1);
              to_half4<CODES>(__byte_perm(vr[c][2][x], vr[c][3][x], sel), a2, a3);
              const int j = (c * VW + x) * 2 + half;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                mma16816(y, a0, a1, a2, a3, pf[nt][0], pf[nt][1]);
#pragma unroll
                for (int z = 0; z < 4; ++z) o[nt][j][z] = fmaf(y[z], v_scale, o[nt][j][z]);
              }
            }
      }
      if (next >= 0) load_v(next);
      now = next;
    }

    // the warps' sums to shared memory, as [row][element]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = l[nt][h];
        sum += __shfl_xor_sync(FULL, sum, 4);
        sum += __shfl_xor_sync(FULL, sum, 8);
        sum += __shfl_xor_sync(FULL, sum, 16);
        const int row = nt * 8 + 2 * t + h;
        if (g == 0) {
          sh_m[warp][row] = m[nt][h];
          sh_l[warp][row] = sum;
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          constexpr int PER = VW * 2;  // m-tiles of a V piece, two elements each
          const int d = j / PER * 128 + (D == 64 ? 8 : 16) * g + j % PER * 2;
          *reinterpret_cast<float2*>(&sh_o[warp][row][d]) = make_float2(o[nt][j][h], o[nt][j][2 + h]);
        }
      }
    __syncthreads();
    // joined; whole items go to the output, the others to the partial sums
    const Segment& done = run.seg;
    float* part = part_of<D, ROWS>(a, done);
    for (int row = threadIdx.x / 32; row < ROWS; row += WARPS) {
      if (done.row0 + row >= done.rows) break;
      float top = -INFINITY, sum = 0.0f, f[WARPS];
#pragma unroll
      for (int x = 0; x < WARPS; ++x) top = fmaxf(top, sh_m[x][row]);
#pragma unroll
      for (int x = 0; x < WARPS; ++x) {
        f[x] = top == -INFINITY ? 0.0f : ex2(sh_m[x][row] - top);
        sum += f[x] * sh_l[x][row];
      }
      const int64_t at = out_row(a, done.it.s.token, done.it.head, done.row0 + row);
      const bool sums = !CAUSAL && a.sees == KvSees::SHARED;
      const int joined = !CAUSAL && done.whole ? done.it.from : 0;
      const Both both = join_shared(a, D, at, joined, top, sum);
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
      for (int d = lane * 2; d < D; d += 64) {
        float y0 = 0.0f, y1 = 0.0f;
#pragma unroll
        for (int x = 0; x < WARPS; ++x) {
          const float2 z = *reinterpret_cast<const float2*>(&sh_o[x][row][d]);
          y0 += f[x] * z.x;
          y1 += f[x] * z.y;
        }
        if (done.whole && sums) {
          *reinterpret_cast<float2*>(a.sums + at * D + d) = make_float2(y0, y1);
        } else if (done.whole) {
          if (joined > 0) {
            const float2 z = *reinterpret_cast<const float2*>(a.sums + at * D + d);
            y0 = y0 * both.own + z.x * both.shared;
            y1 = y1 * both.own + z.y * both.shared;
          }
          T* out = static_cast<T*>(a.out) + at * D + d;
          out[0] = from_float<T>(y0 * inv);
          out[1] = from_float<T>(y1 * inv);
        } else {
          *reinterpret_cast<float2*>(part + row * D + d) = make_float2(y0, y1);
        }
      }
      if (lane == 0) {
        if (!done.whole) {
          part[ROWS * D + row] = top;
          part[ROWS * (D + 1) + row] = sum;
        } else if (sums) {
          *sums_m(a, D, at) = top;
          *sums_l(a, D, at) = sum;
        } else if (a.lse) {
          a.lse[at] = lse_of(top, sum);
        }
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) run.u = done.next;
    __syncthreads();
  }
}

// Rows of a tile, in eights: 16 where the sequences bring more than 8 on average
// and the accumulators of 16 fit (head_dim up to 128).  (32 at head_dim 64, with
// two blocks of threads per SM: 71 us for 24 sequences of 25 rows over 4,096
// tokens, 58 us as two tiles of 16.)
int row_tiles_of(const KvView& kv, int64_t n, int64_t total, int heads) {
  return attend_rows(kv, n, total, heads) > 8 && kv.c.head_dim <= 128 ? 2 : 1;
}

template <typename T, int D, int NT, bool CAUSAL>
cudaError_t attend(AttendArgs a, void* workspace, cudaStream_t s) {
  const int grid = device_sm_count() * per_sm(D, NT);
  take_workspace(a, grid, workspace);
  (a.kv.c.codes == TQ_KV_INT8 ? k_kv_attend<T, D, TQ_KV_INT8, NT, CAUSAL> : k_kv_attend<T, D, TQ_KV_E4M3, NT, CAUSAL>)
      <<<grid, THREADS, 0, s>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_join<T, D, StreamCut<NT, CAUSAL>>(a, grid, s);
}

template <typename T, bool CAUSAL>
cudaError_t attend_for(const AttendArgs& a, int nt, void* workspace, cudaStream_t s) {
  switch (a.kv.c.head_dim) {
    case 64:
      return (nt == 1 ? attend<T, 64, 1, CAUSAL> : attend<T, 64, 2, CAUSAL>)(a, workspace, s);
    case 128:
      return (nt == 1 ? attend<T, 128, 1, CAUSAL> : attend<T, 128, 2, CAUSAL>)(a, workspace, s);
    default:
      return attend<T, 256, 1, CAUSAL>(a, workspace, s);
  }
}

}  // namespace

size_t kv_attend_needs(const KvView& kv, int64_t n, int64_t total, int heads) {
  if (kv_tile_supported(kv, n, total, heads)) return kv_tile_workspace(kv);
  const int nt = row_tiles_of(kv, n, total, heads);
  return attend_workspace(device_sm_count() * per_sm(kv.c.head_dim, nt), 8 * nt, kv.c.head_dim);
}

// The kernel and its row tiles go by the rows that a sequence brings on average, and
// fewer sequences may bring as many queries: the most that any of them needs.
size_t kv_attend_workspace(const KvView& kv, int64_t n, int64_t total, int heads) {
  size_t need = kv_attend_needs(kv, 1, std::min<int64_t>(total, 1), kv.c.kv_heads);  // (one row: in eights)
  if (n == 0 || total == 0) return need;
  if (row_tiles_of(kv, 1, total, heads) == 2)
    need = std::max(need, attend_workspace(device_sm_count() * per_sm(kv.c.head_dim, 2), 16, kv.c.head_dim));
  return kv_tile_supported(kv, 1, total, heads) ? std::max(need, kv_tile_workspace(kv)) : need;
}

namespace {

cudaError_t launch(const AttendArgs& a, int type, int64_t sequences, void* workspace, cudaStream_t s) {
  if (kv_tile_supported(a.kv, sequences, a.total, a.heads)) return launch_kv_tile(a, type, workspace, s);
  const int nt = row_tiles_of(a.kv, sequences, a.total, a.heads);
  const bool bf16 = type == TQ_BF16;
  return (a.sees == KvSees::CAUSAL ? bf16 ? attend_for<__nv_bfloat16, true> : attend_for<__half, true>
          : bf16                   ? attend_for<__nv_bfloat16, false>
                                   : attend_for<__half, false>)(a, nt, workspace, s);
}

size_t sums_bytes(const KvView& kv, int64_t total, int heads) {
  return ((size_t)total * heads * (kv.c.head_dim + 2) * sizeof(float) + 255) / 256 * 256;
}
size_t entries_bytes(int64_t n) { return ((size_t)n * sizeof(KvShared) + 255) / 256 * 256; }

}  // namespace

cudaError_t launch_kv_attend(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts, int64_t n,
                             const KvRows& q, int type, int64_t total, int heads, float scale, int window, void* out,
                             float* lse, void* workspace, cudaStream_t s, bool all) {
  const AttendArgs a = {kv, layer, slots, starts, n, total, q, false, heads, heads / kv.c.kv_heads, scale, window, out,
                        lse, nullptr, nullptr, all ? KvSees::ALL : KvSees::CAUSAL, nullptr, nullptr};
  return launch(a, type, n, workspace, s);
}

// Workspace: the shared tokens' sums | what the plan's entries come to | what either attention
// needs (one after the other).
size_t kv_shared_workspace(const KvView& kv, int64_t n, int64_t total, int heads) {
  return sums_bytes(kv, total, heads) + entries_bytes(n) + kv_attend_workspace(kv, n, total, heads);
}

// The shared tokens first, each group's once for all its queries, their sums left in
// float32; then each request's own, which its last kernel joins with them.
cudaError_t launch_kv_attend_shared(const KvView& kv, int layer, const int32_t* slots, const int32_t* starts,
                                    const int32_t* plan, int64_t n, int64_t groups, const KvRows& q, int type,
                                    int64_t total, int heads, float scale, void* out, float* lse, void* workspace,
                                    cudaStream_t s) {
  char* behind = static_cast<char*>(workspace) + sums_bytes(kv, total, heads);
  KvShared* entries = reinterpret_cast<KvShared*>(behind);
  void* rest = behind + entries_bytes(n);
  AttendArgs a = {kv, layer, slots, starts, n, total, q, false, heads, heads / kv.c.kv_heads, scale, 0, out, lse,
                  nullptr, nullptr, KvSees::SHARED, entries, static_cast<float*>(workspace)};
  cudaError_t e = launch_kv_entries(kv, slots, starts, plan, n, total, entries, s);
  if (e == cudaSuccess) e = launch(a, type, groups, rest, s);
  if (e != cudaSuccess) return e;
  a.sees = KvSees::OWN;
  return launch(a, type, n, rest, s);
}

}  // namespace tq
