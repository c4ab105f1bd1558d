// tq_kv_attend for many queries per key head (prompts, drafts): the products on
// the tensor cores by tcgen05, in tiles of 256 rows x 128 tokens.
//
//   S = Q K^T,   P = 2^(f S + log2(g) - m),   O += P V,   l += sum P / g
//
// in fp16 with float32 sums: codes are exact, queries scaled by a power of two; f
// is the block's key scale times the row's factor, g the block's value scale.
// The weight of a token thus is what it adds to the output, and the reference m
// follows the largest of those, so that P keeps fp16's bits whatever factors lie
// between the blocks' scales; the softmax's own sum is taken of the same numbers,
// per block, divided by g.  (g below 2^-100 counts as 2^-100.  Blocks whose scales lie
// up to 2^100 apart lose no weight above 2^-36 of the largest: 2^-126 is where a
// weight's float32 ends.)
//
// One CTA per SM, 12 warps (168 registers each):
//   0-7   softmax: warps 0-3 the first 128 rows, 4-7 the others; a thread per row.
//         (Up to 128 rows: both have them all and take tiles of tokens in turn.)
//         S is read from tensor memory 64 columns at a time (four blocks of
//         tokens): the second half's and the first half's maxima, the first half's
//         weights, and the second half again for its own.  P goes over the columns
//         of S as the A operand of the second product.  The reference m only
//         moves when a weight passes it by 2^15; then the row's O is scaled in
//         tensor memory (LEAD, LAZY: as in tq_kv_attend.cu).
//         The first warp of each four issues their MMAs: P V once all four have
//         written P, then, when that product is complete (S and P share columns),
//         the scores of the next tokens.  While one row tile's softmax runs, the
//         other's products do.
//   8-11  converters: codes from HBM to registers (the next half tile's loads
//         go out before the present one is converted), to keys [token][d] and
//         values transposed to [d][token] in fp16, both K-major with a 128-byte
//         swizzle, two stages each.
//
// Tensor memory (512 columns): S/P of the two row tiles, 128 each, O of the two.
//
// Bound: the chain softmax -> P V -> S of a row tile, half of which the other's
// fills.  Per 256 x 128 tile (head_dim 128) about 5,000 cycles: 3,300 of MMAs (32 of
// M128 N128 K16, ~100 each) and per row tile 620 for the maxima and 1,400 for the
// weights.  (Weighing in one pass with the old reference and again where it has to
// move was slower: 448 us against 418 for two prompts, for want of registers.)
// A prompt of 2,048 tokens and the last 2,046 of 6,000 (201 GFLOP): 307 us, 655
// TFLOP/s, 0.34 of the measured rate.  Up to 128 rows the converters bound it: 255 MB of codes in
// 154 us.
#include <algorithm>
#include <cstddef>

#include "tq_kv_attend.cuh"
#include "tq_tc.cuh"

namespace tq {
namespace {

constexpr int SOFT = 8, CONV = 4;  // warps
constexpr int TILE_THREADS = (SOFT + CONV) * 32;
constexpr int TOKENS = 128;
constexpr float LEAD = 10.0f, LAZY = 5.0f;
constexpr int AHEAD = 3;       // tiles on their way to L2 (less than four: see the converters' look-ups)
constexpr int SCALE_RING = 4;  // tiles whose scales are held (two being converted, two in the softmax)

// A run is worth a tile of tokens; an item costs about as much as four beside its
// own (two long prompts: 383 us counted as two, 313 as four, 318 as six).
template <bool CAUSAL>
using TileCut = Cut<256, TOKENS, 4, 1, CAUSAL>;

template <int D>
struct TileSmem {
  static constexpr int Q = 128 * D * 2;     // one row tile
  static constexpr int K = TOKENS * D * 2;  // one stage
  static constexpr int q = 0, k = q + 2 * Q, v = k + 2 * K, rest = v + 2 * K, total = rest + 18432 + 1024;
};

template <bool CAUSAL>
struct TileShared {  // behind the operands
  UnitsOf<CAUSAL> units;
  Run run;
  // of a tile's blocks: K's scale, log2 of V's, 1 / V's; a block without tokens, or
  // one that cannot be read, has 0, -inf, 0
  alignas(16) float scales[SCALE_RING][3][8];  // (read four at a time)
  float row_m[2][128], row_l[2][128];  // what the softmax ends with
  float unscale[256];  // factor of a row's scores, in log2 units
  uint64_t q_full[2], k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_full[2], fin;
  uint32_t tmem;
  int abort_flag, err;
};
static_assert(offsetof(TileShared<true>, scales) % 16 == 0 && offsetof(TileShared<false>, scales) % 16 == 0,
              "scales are read four at a time");
static_assert(sizeof(TileShared<true>) <= 18432 && sizeof(TileShared<false>) <= 18432, "shared memory behind the operands");

__host__ __device__ constexpr uint32_t tile_idesc(int n) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

// D (f32, tensor memory) += A x B, both in shared memory.
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}

__device__ __forceinline__ void tmem_put32(uint32_t at, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// Four floats of shared memory that another warp has written, read here and now.
__device__ __forceinline__ void lds4(const float* p, float (&x)[4]) {
  asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3])
               : "r"(smem_u32(p))
               : "memory");
}
__device__ __forceinline__ void tmem_put16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// Ties registers of a load to the wait in front of this (see tmem_wait16).
__device__ __forceinline__ void tmem_hold16(uint32_t (&r)[16]) {
  asm volatile(""
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}
__device__ __forceinline__ void tmem_wait_put() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Four codes of a word as fp16 pairs, exactly.
template <int CODES>
__device__ __forceinline__ void to_fp16x4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (CODES == TQ_KV_INT8) {
    const uint32_t u = w ^ 0x80808080u;
    const __half2 bias = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
    union {
      uint32_t r;
      __half2 h;
    } x, y;
    x.r = __byte_perm(u, 0x64646464u, 0x4140);
    y.r = __byte_perm(u, 0x64646464u, 0x4342);
    x.h = __hsub2(x.h, bias);
    y.h = __hsub2(y.h, bias);
    lo = x.r, hi = y.r;
  } else {
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
  }
}

__device__ __forceinline__ uint32_t pack_fp16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T, int D, int CODES, bool CAUSAL>
__global__ __launch_bounds__(TILE_THREADS, 1) void k_kv_tile(AttendArgs a) {
  using P = TileCut<CAUSAL>;
  using M = TileSmem<D>;
  extern __shared__ unsigned char raw_smem[];
  unsigned char* sm = raw_smem + ((1024u - (smem_u32(raw_smem) & 1023u)) & 1023u);
  TileShared<CAUSAL>& sh = *reinterpret_cast<TileShared<CAUSAL>*>(sm + M::rest);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const KvView& kv = a.kv;

  griddep_launch_dependents();
  if (threadIdx.x == 0) {
    mbar_init(&sh.fin, 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(sh.k_full + i, CONV);
      mbar_init(sh.v_full + i, CONV);
      mbar_init(sh.q_full + i, SOFT / 2);
      mbar_init(sh.k_empty + i, 2);  // (both row tiles' products; one's twice where it is alone)
      mbar_init(sh.v_empty + i, 2);
      mbar_init(sh.s_full + i, 1);
      mbar_init(sh.p_full + i, SOFT / 2);
      mbar_init(sh.o_full + i, 1);
    }
    sh.abort_flag = sh.err = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (!my_run<P>(a, sh.units, sh.run)) return;  // (the whole block)

  if (warp == SOFT) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sh.tmem)));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  volatile int* abort_flag = &sh.abort_flag;
  int* err = &sh.err;

  // Tiles of tokens done by this CTA, and by this half of the softmax: their
  // barriers' phases.
  int done = 0, mine = 0, segments = 0;
  while (sh.run.u < sh.run.end) {
    next_segment<P>(a, sh.units, sh.run);
    const Segment& seg = sh.run.seg;
    const KvSeq sq = seg.it.s;
    const int from = CAUSAL ? 0 : seg.it.from;
    const int head = seg.it.head;
    const int tiles = seg.b_last - seg.b_first, first = seg.it.span.first + seg.b_first;  // tiles of tokens
    // Two row tiles, each with its half of the softmax; or one, whose tiles of tokens
    // the halves take in turn, their sums joined at the end.
    const bool two = seg.rows - seg.row0 > 128;

    if (warp < SOFT) {
      // ------------------------------------------------------------ softmax
      const int w = warp >> 2, rt = two ? w : 0, row = (warp & 3) * 32 + lane, r = seg.row0 + rt * 128 + row;
      const bool real = r < seg.rows;
      const int j0 = two ? 0 : w, step_j = two ? 1 : 2;
      if (w == 0 || two) {
        // The warp's 32 rows of queries, D / 8 lanes to a row, each row scaled so that
        // its largest element lies in [2^8, 2^9).  A row that is not finite becomes NaN
        // throughout, and so do its scores, whatever the codes.
        constexpr int LANES = D / 8, STEP = 32 / LANES;
        const int c = lane % LANES;
        union Chunk {
          uint4 v;
          T e[8];
        };
        // N rows, y, y + STEP, ...: their reductions run side by side
        auto put_rows = [&](int y, const auto& in) {
          constexpr int N = sizeof(in) / sizeof(Chunk);
          uint32_t bits[N];
#pragma unroll
          for (int x = 0; x < N; ++x) bits[x] = max_magnitude<T>(0u, in[x].v);
#pragma unroll
          for (int o = LANES / 2; o; o >>= 1)
#pragma unroll
            for (int x = 0; x < N; ++x) bits[x] = max_magnitude<T>(bits[x], __shfl_xor_sync(FULL, bits[x], o));
#pragma unroll
          for (int x = 0; x < N; ++x) {
            const float top = magnitude<T>(bits[x]);
            const int e2 = min(max((int)(__float_as_uint(top) >> 23) - 127, -110), 127), at = y + x * STEP;
            const float up = top < INFINITY ? __uint_as_float((uint32_t)(127 + min(8 - e2, 118)) << 23) : NAN;
            const float f = a.scale < 0.0f ? -up : up;  // (the scale's sign goes with the queries)
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = pack_fp16(to_float(in[x].e[2 * e]) * f, to_float(in[x].e[2 * e + 1]) * f);
            *reinterpret_cast<uint4*>(sm + M::q + w * M::Q + (c >> 3) * 16384 + sw128_offset(at, c & 7)) =
                make_uint4(h[0], h[1], h[2], h[3]);
            if (c == 0) sh.unscale[w * 128 + at] = fabsf(a.scale) * LOG2E * __uint_as_float((uint32_t)(127 - min(8 - e2, 118)) << 23);
          }
        };
        int y = (warp & 3) * 32 + lane / LANES;
        int token = (seg.row0 + w * 128 + y) / a.group, member = (seg.row0 + w * 128 + y) % a.group;
        auto step = [&]() {  // to the lane's next row; returns the present one's address
          const T* p = static_cast<const T*>(a.q.p) + (int64_t)(sq.token + token) * a.q.token_stride +
                       (int64_t)(head * a.group + member) * a.q.head_stride + 8 * c;
          for (member += STEP; member >= a.group; member -= a.group) ++token;
          return p;
        };
        const int ys = seg.rows - seg.row0 - w * 128;  // (rows from ys on do not exist)
        if (a.q_wide) {
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {  // 16 rows on their way at a time
            Chunk in[16 / STEP];
#pragma unroll
            for (int x = 0; x < 16 / STEP; ++x) {
              const T* p = step();
              in[x].v = make_uint4(0, 0, 0, 0);
              if (y + x * STEP < ys) in[x].v = __ldg(reinterpret_cast<const uint4*>(p));
            }
            put_rows(y, in);
            y += 16;
          }
        } else {
#pragma unroll 1
          for (int x = 0; x < 32; x += STEP, y += STEP) {
            const T* p = step();
            Chunk in[1];
            in[0].v = make_uint4(0, 0, 0, 0);
            if (y < ys) {
#pragma unroll
              for (int e = 0; e < 8; ++e) in[0].e[e] = p[e];
            }
            put_rows(y, in);
          }
        }
        fence_proxy_async();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(sh.q_full + w);

      const uint32_t ts = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(w * TOKENS);
      float m = -INFINITY, l = 0.0f;
      bool ok = all_wait(sh.q_full + rt, segments & 1, abort_flag, err, 6);
      const float unscale = sh.unscale[rt * 128 + row];
      const int place = real ? max(-1, dense<P>(a) ? sq.len - 1 : sq.len - sq.count + r / a.group) : -1;
      // what the first warp issues for the four
      const bool issuer = (warp & 3) == 0;
      const uint32_t tm = __shfl_sync(FULL, tmem, 0), sm0 = __shfl_sync(FULL, smem_u32(sm), 0);
      auto scores = [&](int n) {  // of tile n of this CTA
        if (elect_one()) {
          const uint64_t qd = sw128_desc(sm0 + M::q + rt * M::Q), kd = sw128_desc(sm0 + M::k + (n & 1) * M::K);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t off = (uint64_t)((kk >> 2) * (16384 >> 4) + (kk & 3) * 2);
            mma_f16_ss(tm + (uint32_t)(w * TOKENS), qd + off, kd + off, tile_idesc(TOKENS), kk ? 1u : 0u);
          }
          mma_commit(sh.s_full + w);
          mma_commit(sh.k_empty + (n & 1));
          if (!two) mma_commit(sh.k_empty + (n & 1));
        }
        __syncwarp();
      };
      auto values = [&](int n, bool more) {
        if (elect_one()) {
          const uint64_t vd = sw128_desc(sm0 + M::v + (n & 1) * M::K);
#pragma unroll
          for (int kk = 0; kk < TOKENS / 16; ++kk)
            mma_f16_ta(tm + (uint32_t)(2 * TOKENS + w * D), tm + (uint32_t)(w * TOKENS + kk * 8),
                       vd + (uint64_t)((kk >> 2) * (D * 128 >> 4) + (kk & 3) * 2), tile_idesc(D), kk || more ? 1u : 0u);
          mma_commit(sh.o_full + w);
          mma_commit(sh.v_empty + (n & 1));
          if (!two) mma_commit(sh.v_empty + (n & 1));
        }
        __syncwarp();
      };
      if (ok && issuer && j0 < tiles) {
        const int n = done + j0;
        if ((ok = all_wait(sh.k_full + (n & 1), (n >> 1) & 1, abort_flag, err, 7))) {
          tc_fence_after();
          scores(n);
        }
      }
      for (int j = j0; ok && j < tiles;) {
        if (!(ok = all_wait(sh.s_full + w, mine & 1, abort_flag, err, 1))) break;
        tc_fence_after();
        if (__any_sync(FULL, real)) {  // (else P of these lanes is whatever S was: nobody reads their O)
          const float(*sc)[8] = sh.scales[(done + j) % SCALE_RING];
          const int t0 = (first + j) * TOKENS;
          // columns [lo, hi) are seen; they are looked at only where some row does not see them
          // all.  (lo may wrap around only for hi <= 0, where nothing is seen whatever it is.)
          const int hi = place - t0 + 1, lo = !CAUSAL ? max(0, from - t0) : a.window ? (int)((unsigned)hi - (unsigned)a.window) : 0;
          const bool edge = __any_sync(FULL, real && (hi < TOKENS || lo > 0));
          // Half of S at a time (64 columns, 4 blocks): the second half's maximum, the
          // first half's, its weights, and the second half read again for its.  P goes
          // over columns of the first half.
          uint32_t x[4][16];
          auto load = [&](int half) {
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld16_issue(ts + half * 64 + 16 * c, x[c]);
            tmem_wait16(x[0]);
#pragma unroll
            for (int c = 1; c < 4; ++c) tmem_hold16(x[c]);
            if (edge) {
#pragma unroll
              for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  const int at = half * 64 + 16 * c + i;
                  if (at >= hi || at < lo) x[c][i] = 0xFF800000u;  // -inf
                }
            }
          };
          float f[4], add[4];  // of the half's blocks
          auto factors = [&](int half) {
            lds4(sc[0] + half * 4, f);
            lds4(sc[1] + half * 4, add);
            // positive even for a zero scale (whose scores are 0), so that -inf stays
#pragma unroll
            for (int c = 0; c < 4; ++c) f[c] = fmaxf(f[c] * unscale, 1e-30f);
          };
          float top = -INFINITY;
#pragma unroll 1
          for (int half = 1; half >= 0; --half) {
            factors(half);
            load(half);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              float y[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) y[i] = __uint_as_float(x[c][i]);
#pragma unroll
              for (int i = 4; i < 16; ++i) y[i & 3] = fmaxf(y[i & 3], __uint_as_float(x[c][i]));
              top = fmaxf(top, fmaf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), f[c], add[c]));
            }
          }
          if (__any_sync(FULL, top > m + (LEAD + LAZY))) {
            const float to_m = fmaxf(m, top - LEAD), keep = to_m > m ? ex2(m - to_m) : 1.0f;
            m = to_m;
            l *= keep;
            if (j > j0) {  // O so far, once its product is complete
              if (!(ok = all_wait(sh.o_full + w, (mine - 1) & 1, abort_flag, err, 2))) break;
              tc_fence_after();
              const uint32_t to = ts + (uint32_t)(2 * TOKENS + w * D - w * TOKENS);
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                uint32_t y[16];
                tmem_ld16_issue(to + c, y);
                tmem_wait16(y);
#pragma unroll
                for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * keep);
                tmem_put16(to + c, y);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            float inv[4];
            lds4(sc[2] + half * 4, inv);
            if (half) {
              factors(1);
              load(1);
            }
            uint32_t out[32];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float plus = add[c] - ref;
              float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                const float p0 = ex2(fmaf(__uint_as_float(x[c][i]), f[c], plus));
                const float p1 = ex2(fmaf(__uint_as_float(x[c][i + 1]), f[c], plus));
                sum[i & 2] += p0;
                sum[(i & 2) + 1] += p1;
                out[c * 8 + i / 2] = pack_fp16(p0, p1);
              }
              l = fmaf((sum[0] + sum[1]) + (sum[2] + sum[3]), inv[c], l);
            }
            tmem_put32(ts + half * 32, out);
          }
          tmem_wait_put();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.p_full + w);
        if (issuer) {
          const int n = done + j, next = n + step_j;
          if (!(ok = all_wait(sh.v_full + (n & 1), (n >> 1) & 1, abort_flag, err, 8) &&
                     all_wait(sh.p_full + w, mine & 1, abort_flag, err, 9)))
            break;
          tc_fence_after();
          values(n, j > j0);
          if (j + step_j < tiles) {  // the next scores overwrite P: its product has to be complete
            if (!(ok = all_wait(sh.k_full + (next & 1), (next >> 1) & 1, abort_flag, err, 10) &&
                       all_wait(sh.o_full + w, mine & 1, abort_flag, err, 11)))
              break;
            tc_fence_after();
            scores(next);
          }
        }
        j += step_j;
        ++mine;
      }
      if (ok && j0 < tiles) all_wait(sh.o_full + w, (mine - 1) & 1, abort_flag, err, 3);
      sh.row_m[w][row] = m;
      sh.row_l[w][row] = l;
    } else {
      // --------------------------------------------------------- converters
      const int cw = warp - SOFT;
      const int32_t* table = kv.c.table + sq.slot * kv.c.max_pages;
      // Lane l looks up the l-th of the 32 blocks of four tiles: its place in the pool
      // and what the softmax takes of its scales; the next four tiles' are looked up
      // while these are converted.
      struct Lines {
        int line;  // (blocks are of 1 KB at least: 2^31 of them are more than any memory)
        float ks, log_g, inv_g;
      } now, ahead;
      auto look_up = [&](int j) {
        Lines x = {-1, 0.0f, -INFINITY, 0.0f};
        const int64_t tok = (int64_t)(first + j) * TOKENS + lane * kKvBlock;
        if (j + (lane >> 3) < tiles && tok < sq.len) {
          const int page = table[tok >> kv.page_shift];
          if (page >= 0 && page < kv.c.pages) {
            x.line = (int)(kv.scales_at(a.layer, page, head) + ((tok & (kv.c.page_tokens - 1)) / kKvBlock));
            x.ks = __ldg(kv.c.k_scale + x.line);
            const float g = fmaxf(__ldg(kv.c.v_scale + x.line), 0x1p-100f);
            x.log_g = log2f(g);
            x.inv_g = 1.0f / g;
          } else {
            kv_status(kv, kKvBadEntry);
          }
        }
        return x;
      };
      auto line_of = [&](int j, int block, const Lines& x) { return __shfl_sync(FULL, x.line, (j & 3) * 8 + block); };
      // A tile's codes on their way to L2: a warp takes half of each of the 8 blocks of K
      // or V, four lanes a block.
      auto fetch = [&](int j, const Lines& x) {
        const int ln = line_of(j, lane >> 2, x);
        if (ln >= 0) {
          const uint8_t* p = (cw & 1 ? kv.c.v : kv.c.k) + (int64_t)ln * (kKvBlock * D) + ((cw >> 1) * 4 + (lane & 3)) * (D * 2);
#pragma unroll
          for (int y = 0; y < D * 2; y += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + y));
        }
      };
      // keys: warp cw takes blocks 2 cw and 2 cw + 1; lane: 16-byte piece (lane & 3) of each
      // 64 bytes, tokens lane >> 2 and 8 more.  A block that is not there reads block 0
      // of the pool and is zeroed when it is converted.
      constexpr int KN = D / 64;
      uint4 kr[2][2][KN];
      bool k_there[2];
      auto load_k = [&](int j, const Lines& x) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int ln = line_of(j, cw * 2 + b, x);
          k_there[b] = ln >= 0;
          const uint8_t* p = kv.c.k + (int64_t)max(ln, 0) * (kKvBlock * D) + (lane >> 2) * D + (lane & 3) * 16;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < KN; ++c) kr[b][h][c] = __ldg(reinterpret_cast<const uint4*>(p + h * 8 * D + c * 64));
        }
      };
      // values: 64 tokens x 64 elements a warp (x 32 at head_dim 64); lane: 8 tokens (lane & 7), VB elements.
      // Bytes that no token owns may be NaN, and 0 times that is not 0: zeroed too.
      constexpr int VB = D / 8;  // bytes of a lane's row: 16 or 8
      const int half = cw >> 1, v_octet = lane & 7, v_el = (cw & 1) * (D / 2) + (lane >> 3) * VB;
      uint32_t vr[8][VB / 4];
      int v_tokens;  // that are there
      auto load_v = [&](int j, const Lines& x) {
        const int ln = line_of(j, half * 4 + (v_octet >> 1), x);
        v_tokens = ln >= 0 ? sq.len - ((first + j) * TOKENS + half * 64 + v_octet * 8) : 0;
        const uint8_t* p = kv.c.v + (int64_t)max(ln, 0) * (kKvBlock * D) + (v_octet & 1) * 8 * D + v_el;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (VB == 16) {
            const uint4 y = __ldg(reinterpret_cast<const uint4*>(p + i * D));
            vr[i][0] = y.x, vr[i][1] = y.y, vr[i][VB / 4 - 2] = y.z, vr[i][VB / 4 - 1] = y.w;
          } else {
            const uint2 y = __ldg(reinterpret_cast<const uint2*>(p + i * D));
            vr[i][0] = y.x, vr[i][1] = y.y;
          }
        }
      };
      now = look_up(0);
      ahead = look_up(4);
      if (tiles) load_k(0, now);
      for (int j = 1; j < AHEAD; ++j) fetch(j, now);
      for (int j = 0; j < tiles; ++j) {
        const int n = done + j, st = n & 1;
        load_v(j, now);
        if ((j & 3) + AHEAD < 4)
          fetch(j + AHEAD, now);
        else
          fetch(j + AHEAD, ahead);
        if (n >= 2 && !all_wait(sh.k_empty + st, ((n >> 1) - 1) & 1, abort_flag, err, 4)) break;
        if (cw == 0 && lane >> 3 == (j & 3)) {
          // (the softmax of the tile that had this place in the ring is over: S two tiles on waited for it)
          float* sc = &sh.scales[n % SCALE_RING][0][lane & 7];
          sc[0] = now.ks;
          sc[8] = now.log_g;
          sc[16] = now.inv_g;
        }
        unsigned char* sk = sm + M::k + st * M::K;
        if (!__all_sync(FULL, k_there[0] && k_there[1])) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int c = 0; c < KN; ++c)
                if (!k_there[b]) kr[b][h][c] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int c = 0; c < KN; ++c) {
              const int tok = cw * 32 + b * 16 + x * 8 + (lane >> 2), at = (lane & 3) * 2;
              const uint32_t y[4] = {kr[b][x][c].x, kr[b][x][c].y, kr[b][x][c].z, kr[b][x][c].w};
              uint32_t h[8];
#pragma unroll
              for (int e = 0; e < 4; ++e) to_fp16x4<CODES>(y[e], h[2 * e], h[2 * e + 1]);
              *reinterpret_cast<uint4*>(sk + c * 16384 + sw128_offset(tok, at)) = make_uint4(h[0], h[1], h[2], h[3]);
              *reinterpret_cast<uint4*>(sk + c * 16384 + sw128_offset(tok, at + 1)) = make_uint4(h[4], h[5], h[6], h[7]);
            }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.k_full + st);
        if ((j & 3) == 3) {
          now = ahead;
          ahead = look_up(j + 5);
        }
        if (j + 1 < tiles) load_k(j + 1, now);
        if (n >= 2 && !all_wait(sh.v_empty + st, ((n >> 1) - 1) & 1, abort_flag, err, 5)) break;
        if (__any_sync(FULL, v_tokens < 8)) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int x = 0; x < VB / 4; ++x)
              if (i >= v_tokens) vr[i][x] = 0;
        }
        unsigned char* sv = sm + M::v + st * M::K + half * (D * 128);
#pragma unroll
        for (int x = 0; x < VB / 4; ++x)
#pragma unroll
          for (int e = 0; e < 2; ++e) {  // elements 0, 1 and 2, 3 of the word, eight tokens of each
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              to_fp16x4<CODES>(__byte_perm(vr[2 * i][x], vr[2 * i + 1][x], e ? 0x7362 : 0x5140), lo[i], hi[i]);
            const int d = v_el + 4 * x + 2 * e;
            *reinterpret_cast<uint4*>(sv + sw128_offset(d, v_octet)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            *reinterpret_cast<uint4*>(sv + sw128_offset(d + 1, v_octet)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.v_full + st);
      }
    }
    done += tiles;
    ++segments;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*abort_flag) break;  // (uniform behind the barrier)

    // ------------------------------------------------------------ the sums
    // O of this thread's row, 16 elements at a time (none where no tile was seen).
    const int w = (warp >> 2) & 1, rt = two ? w : 0, row = (warp & 3) * 32 + lane, r = seg.row0 + rt * 128 + row;
    const bool real = r < seg.rows, seen = two ? tiles > 0 : w < tiles, some = warp < SOFT && __any_sync(FULL, real);
    const uint32_t to = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(2 * TOKENS + w * D);
    auto load_o = [&](int c, uint32_t(&x)[16]) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0;
      if (seen) {
        tmem_ld16_issue(to + c, x);
        tmem_wait16(x);
      }
    };
    float* other = reinterpret_cast<float*>(sm + M::k);  // [D][128], the second half's O (the keys are done with)
    if (!two) {
      if (w == 1 && some) {
#pragma unroll 1
        for (int c = 0; c < D; c += 16) {
          uint32_t x[16];
          load_o(c, x);
#pragma unroll
          for (int i = 0; i < 16; ++i) other[(c + i) * 128 + row] = __uint_as_float(x[i]);
        }
      }
      __syncthreads();
    }
    float m = sh.row_m[w][row], l = sh.row_l[w][row], keep0 = 1.0f, keep1 = 0.0f;
    if (!two) {
      const float m1 = sh.row_m[1][row], top = fmaxf(m, m1);
      keep0 = top > -INFINITY ? ex2(m - top) : 0.0f;
      keep1 = top > -INFINITY ? ex2(m1 - top) : 0.0f;
      m = top;
      l = l * keep0 + sh.row_l[1][row] * keep1;
    }
    if (some && (two || w == 0)) {
      const int64_t at = real ? out_row(a, sq.token, head, r) : 0;
      const bool sums = !CAUSAL && a.sees == KvSees::SHARED;
      const int joined = !CAUSAL && real && seg.whole ? from : 0;
      const Both both = join_shared(a, D, at, joined, m, l);
      const float inv = l > 0.0f ? 1.0f / l : 0.0f;
      float* part = part_of<D, P::ROWS>(a, seg);
      const int prow = rt * 128 + row;
#pragma unroll 1
      for (int c = 0; c < D; c += 16) {
        uint32_t x[16];
        load_o(c, x);
        if (!two) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            x[i] = __float_as_uint(__uint_as_float(x[i]) * keep0 + other[(c + i) * 128 + row] * keep1);
        }
        if (!real) continue;
        if (seg.whole && !sums) {
          if (joined > 0) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 z = *reinterpret_cast<const float4*>(a.sums + at * D + c + i);
              const float y[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) x[i + e] = __float_as_uint(__uint_as_float(x[i + e]) * both.own + y[e] * both.shared);
            }
          }
          union {
            T e[16];
            uint4 v[2];
          } y;
#pragma unroll
          for (int i = 0; i < 16; ++i) y.e[i] = from_float<T>(__uint_as_float(x[i]) * inv);
          uint4* o = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + at * D + c);
          o[0] = y.v[0];
          o[1] = y.v[1];
        } else {
          uint4* o = reinterpret_cast<uint4*>(seg.whole ? a.sums + at * D + c : part + prow * D + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        }
      }
      if (real && seg.whole && sums) {
        *sums_m(a, D, at) = m;
        *sums_l(a, D, at) = l;
      } else if (real && seg.whole && a.lse) {
        a.lse[at] = lse_of(m, l);
      }
      if (real && !seg.whole) {
        part[P::ROWS * D + prow] = m;
        part[P::ROWS * (D + 1) + prow] = l;
      }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (threadIdx.x == 0) sh.run.u = sh.run.seg.next;
    __syncthreads();
  }
  if (warp == 0 || warp == SOFT / 2) {
    if (elect_one()) {  // never leave with MMAs in flight
      mma_commit(&sh.fin);
      mbar_wait_drain(&sh.fin, 0);
    }
    __syncwarp();
  }
  if (threadIdx.x == 0 && sh.err) kv_status(kv, kKvTimeout);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == SOFT) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <typename T, int D, int CODES, bool CAUSAL>
cudaError_t tile(const AttendArgs& a, int grid, cudaStream_t s) {
  auto* kernel = k_kv_tile<T, D, CODES, CAUSAL>;
  cudaError_t e = set_max_dynamic_smem(reinterpret_cast<const void*>(kernel), TileSmem<D>::total);
  if (e != cudaSuccess) return e;
  kernel<<<grid, TILE_THREADS, TileSmem<D>::total, s>>>(a);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  return launch_join<T, D, TileCut<CAUSAL>>(a, grid, s);
}

template <typename T, bool CAUSAL>
cudaError_t tile_for(const AttendArgs& a, int grid, cudaStream_t s) {
  const bool i8 = a.kv.c.codes == TQ_KV_INT8;
  if (a.kv.c.head_dim == 64) return (i8 ? tile<T, 64, TQ_KV_INT8, CAUSAL> : tile<T, 64, TQ_KV_E4M3, CAUSAL>)(a, grid, s);
  return (i8 ? tile<T, 128, TQ_KV_INT8, CAUSAL> : tile<T, 128, TQ_KV_E4M3, CAUSAL>)(a, grid, s);
}

}  // namespace

// From where on the tiles are faster than the stream (tq_kv_attend.cu), in rows per
// key head, for 24 sequences of 2,000 to 8,190 tokens and 8 key heads: at head_dim
// 128 25 rows take 152 us here and 140 there, 28 rows 153 and 165, 40 rows 155 and
// 218; at head_dim 64 40 rows take 110 and 106, 48 rows 110 and 111, 64 rows 111
// and 137.  (The operands of 256 rows fit beside two stages up to head_dim 128.)
bool kv_tile_supported(const KvView& kv, int64_t n, int64_t total, int heads) {
  const int dim = kv.c.head_dim;
  return dim <= 128 && attend_rows(kv, n, total, heads) > (dim == 128 ? 26 : 40);
}

size_t kv_tile_workspace(const KvView& kv) {
  return attend_workspace(device_sm_count(), TileCut<true>::ROWS, kv.c.head_dim);
}

cudaError_t launch_kv_tile(AttendArgs a, int type, void* workspace, cudaStream_t s) {
  const int grid = device_sm_count();
  take_workspace(a, grid, workspace);
  a.q_wide = aligned16(a.q.p) && a.q.token_stride % 8 == 0 && a.q.head_stride % 8 == 0;
  const bool bf16 = type == TQ_BF16;
  return (a.sees == KvSees::CAUSAL ? bf16 ? tile_for<__nv_bfloat16, true> : tile_for<__half, true>
          : bf16                   ? tile_for<__nv_bfloat16, false>
                                   : tile_for<__half, false>)(a, grid, s);
}

}  // namespace tq
