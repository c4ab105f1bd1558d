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
// per block, divided by g.  (g below 2^-100 counts as 2^-100.)
//
// One CTA per SM, 13 warps:
//   0-7   softmax: warps 0-3 the first 128 rows, 4-7 the others; a thread per row.
//         S is read from tensor memory twice, for the maximum and for the
//         weights, 16 columns (one block of tokens, one scale) at a time; P goes
//         back over the columns of S as the A operand of the second product.
//         The reference m only moves when a weight passes it by 2^15; then the row's
//         O is scaled in tensor memory (LEAD, LAZY: as in tq_kv_attend.cu).
//   8-11  converters: codes from HBM to registers (the next half tile's loads
//         go out before the present one is converted), to keys [token][d] and
//         values transposed to [d][token] in fp16, both K-major with a 128-byte
//         swizzle, two stages each.
//   12    issues the MMAs.  While one 128 rows' softmax runs, the other's products
//         do: S and P of a row tile share their columns, so S of the next tokens
//         waits for the product that reads P.
//
// Tensor memory (512 columns): S/P of the two row tiles, 128 each, O of the two.
//
// Bound: per 256 x 128 tile (head_dim 128) about 2,200 cycles of MMAs, 2 x 128
// columns of softmax per scheduler (about 1,600 issue slots) and the converters'
// 500; for few rows the chain S -> softmax -> O.
#include <algorithm>

#include "tq_kv_attend.cuh"
#include "tq_tc.cuh"

namespace tq {
namespace {

constexpr int SOFT = 8, CONV = 4, ISSUE = SOFT + CONV;  // warps
constexpr int TILE_THREADS = (ISSUE + 1) * 32;
constexpr int TOKENS = 128;
constexpr float LEAD = 10.0f, LAZY = 5.0f;
constexpr int SCALE_RING = 4;  // tiles whose scales are held (two being converted, two in the softmax)

// A run is worth a tile of tokens; an item costs about as much as two beside its own.
using TileCut = Cut<256, TOKENS, 2, 1>;

template <int D>
struct TileSmem {
  static constexpr int Q = 128 * D * 2;     // one row tile
  static constexpr int K = TOKENS * D * 2;  // one stage
  static constexpr int q = 0, k = q + 2 * Q, v = k + 2 * K, rest = v + 2 * K, total = rest + 16384 + 1024;
};

struct TileShared {  // behind the operands
  Units units;
  // of a tile's blocks: K's scale, log2 of V's, 1 / V's; a block without tokens, or
  // one that cannot be read, has 0, -inf, 0
  float scales[SCALE_RING][3][8];
  uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2], o_full[2], fin;
  uint32_t tmem;
  int abort_flag, err;
};
static_assert(sizeof(TileShared) <= 16384, "shared memory behind the operands");

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

__device__ __forceinline__ void tmem_put8(uint32_t at, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
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

template <typename T, int D, int CODES>
__global__ __launch_bounds__(TILE_THREADS, 1) void k_kv_tile(AttendArgs a) {
  using P = TileCut;
  using M = TileSmem<D>;
  extern __shared__ unsigned char raw_smem[];
  unsigned char* sm = raw_smem + ((1024u - (smem_u32(raw_smem) & 1023u)) & 1023u);
  TileShared& sh = *reinterpret_cast<TileShared*>(sm + M::rest);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const KvView& kv = a.kv;

  griddep_launch_dependents();
  if (threadIdx.x == 0) {
    mbar_init(&sh.q_full, SOFT);
    mbar_init(&sh.fin, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(sh.k_full + i, CONV);
      mbar_init(sh.v_full + i, CONV);
      mbar_init(sh.k_empty + i, 1);
      mbar_init(sh.v_empty + i, 1);
      mbar_init(sh.s_full + i, 1);
      mbar_init(sh.p_full + i, SOFT / 2);
      mbar_init(sh.o_full + i, 1);
    }
    sh.abort_flag = sh.err = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  int64_t all, n_runs, u, end;
  if (!my_run<P>(a, sh.units, all, n_runs, u, end)) return;  // (the whole block)

  if (warp == ISSUE) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sh.tmem)));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  volatile int* abort_flag = &sh.abort_flag;
  int* err = &sh.err;

  // Tiles done by this CTA, and by its second row tile: their barriers' phases.
  int done = 0, done2 = 0, segments = 0;
  while (u < end) {
    const Segment seg = next_segment<P>(a, sh.units, all, n_runs, u, end);
    const KvSeq& sq = seg.it.s;
    const Span& span = seg.it.span;
    const int head = seg.it.head;
    const int tiles = seg.b_last - seg.b_first, first = span.first + seg.b_first;  // tiles of tokens
    const bool two = seg.rows - seg.row0 > 128;

    if (warp < SOFT) {
      // ------------------------------------------------------------ softmax
      const int w = warp >> 2, row = (warp & 3) * 32 + lane;
      const int64_t r = seg.row0 + w * 128 + row;
      const bool real = r < seg.rows;
      float unscale = 0.0f;
      if (w == 0 || two) {
        // the row of queries, scaled so that its largest element lies in [2^8, 2^9)
        const T* p = static_cast<const T*>(a.q.p) + (sq.token + r / a.group) * a.q.token_stride +
                     (int64_t)(head * a.group + (int)(r % a.group)) * a.q.head_stride;
        const bool wide = ((uintptr_t)p & 15) == 0;
        union {
          uint4 v;
          T e[8];
        } x;
        auto load = [&](int c) {
          x.v = make_uint4(0, 0, 0, 0);
          if (!real) return;
          if (wide) {
            x.v = __ldg(reinterpret_cast<const uint4*>(p + 8 * c));
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x.e[e] = p[8 * c + e];
          }
        };
        float top = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
          load(c);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(to_float(x.e[e])));
        }
        const int e2 = min(max((int)(__float_as_uint(top) >> 23) - 127, -110), 127);
        const float up = __uint_as_float((uint32_t)(127 + min(8 - e2, 118)) << 23);
        unscale = fabsf(a.scale) * LOG2E / up;  // (>= 0: the scale's sign goes with the queries)
        const float f = a.scale < 0.0f ? -up : up;
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
          load(c);
          uint32_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const __half2 y = __floats2half2_rn(to_float(x.e[2 * e]) * f, to_float(x.e[2 * e + 1]) * f);
            h[e] = *reinterpret_cast<const uint32_t*>(&y);
          }
          *reinterpret_cast<uint4*>(sm + M::q + w * M::Q + (c >> 3) * 16384 + sw128_offset(row, c & 7)) =
              make_uint4(h[0], h[1], h[2], h[3]);
        }
        fence_proxy_async();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.q_full);

      if (w == 0 || two) {
        const int place = real ? sq.len - sq.count + (int)(r / a.group) : -1;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem + lanes + (uint32_t)(w * TOKENS), to = tmem + lanes + (uint32_t)(2 * TOKENS + w * D);
        int phase = w ? done2 : done;
        float m = -INFINITY, l = 0.0f;
        bool ok = true;
        for (int j = 0; j < tiles; ++j, ++phase) {
          if (!(ok = all_wait(sh.s_full + w, phase & 1, abort_flag, err, 1))) break;
          tc_fence_after();
          const volatile float(*sc)[8] = sh.scales[(done + j) % SCALE_RING];
          const int t0 = (first + j) * TOKENS;
          // columns [lo, hi) are seen; the warp looks at each only where some row does not see them all
          const int hi = place - t0 + 1, lo = a.window ? place - a.window + 1 - t0 : 0;
          const bool edge = __any_sync(FULL, real && (hi < TOKENS || lo > 0));
          float top = -INFINITY;
          uint32_t r0[16], r1[16];
          auto block_top = [&](int c, const uint32_t(&x)[16]) {
            const float f = sc[0][c] * unscale;  // (>= 0)
            float y = -INFINITY;
            if (edge) {
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (16 * c + i < hi && 16 * c + i >= lo) y = fmaxf(y, __uint_as_float(x[i]) * f);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) y = fmaxf(y, __uint_as_float(x[i]));
              y *= f;
            }
            top = fmaxf(top, y + sc[1][c]);
          };
          tmem_ld16_issue(ts, r0);
#pragma unroll
          for (int c = 0; c < 8; c += 2) {
            tmem_wait16(r0);
            tmem_ld16_issue(ts + 16 * (c + 1), r1);
            block_top(c, r0);
            tmem_wait16(r1);
            tmem_ld16_issue(ts + 16 * ((c + 2) & 7), r0);  // (at the end the first block again, for the weights)
            block_top(c + 1, r1);
          }
          if (__any_sync(FULL, top > m + (LEAD + LAZY))) {
            const float to_m = fmaxf(m, top - LEAD), keep = to_m > m ? ex2(m - to_m) : 1.0f;
            m = to_m;
            l *= keep;
            if (j) {  // O so far, once its product is complete
              tmem_wait16(r0);
              if (!(ok = all_wait(sh.o_full + w, (phase - 1) & 1, abort_flag, err, 2))) break;
              tc_fence_after();
#pragma unroll
              for (int c = 0; c < D; c += 16) {
                tmem_ld16_issue(to + c, r0);
                tmem_wait16(r0);
#pragma unroll
                for (int i = 0; i < 16; ++i) r0[i] = __float_as_uint(__uint_as_float(r0[i]) * keep);
                tmem_put16(to + c, r0);
              }
              tmem_wait_put();
              tmem_ld16_issue(ts, r0);
            }
          }
          const float ref = m == -INFINITY ? 0.0f : m;
          auto weights = [&](int c, const uint32_t(&x)[16]) {
            const float f = sc[0][c] * unscale, add = sc[1][c] - ref;
            float sum = 0.0f;
            uint32_t out[8];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              float p0 = ex2(fmaf(__uint_as_float(x[i]), f, add)), p1 = ex2(fmaf(__uint_as_float(x[i + 1]), f, add));
              if (edge) {
                const int at = 16 * c + i;
                if (at >= hi || at < lo) p0 = 0.0f;
                if (at + 1 >= hi || at + 1 < lo) p1 = 0.0f;
              }
              sum += p0 + p1;
              out[i / 2] = pack_fp16(p0, p1);
            }
            l = fmaf(sum, sc[2][c], l);
            tmem_put8(ts + 8 * c, out);  // (columns of S that have been read)
          };
#pragma unroll
          for (int c = 0; c < 8; c += 2) {
            tmem_wait16(r0);
            tmem_ld16_issue(ts + 16 * (c + 1), r1);
            weights(c, r0);
            tmem_wait16(r1);
            if (c + 2 < 8) tmem_ld16_issue(ts + 16 * (c + 2), r0);
            weights(c + 1, r1);
          }
          tmem_wait_put();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(sh.p_full + w);
        }
        if (ok && tiles && (ok = all_wait(sh.o_full + w, (phase - 1) & 1, abort_flag, err, 3))) tc_fence_after();
        if (ok && __any_sync(FULL, real)) {
          const float inv = l > 0.0f ? 1.0f / l : 0.0f;
          const int64_t at = out_row(a, sq.token, head, r);
          float* part = part_of<D, P::ROWS>(a, seg);
          const int prow = w * 128 + row;
#pragma unroll
          for (int c = 0; c < D; c += 16) {
            uint32_t x[16];
            if (tiles) {
              tmem_ld16_issue(to + c, x);
              tmem_wait16(x);
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) x[i] = 0;
            }
            if (!real) continue;
            if (seg.whole) {
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
              uint4* o = reinterpret_cast<uint4*>(part + prow * D + c);
#pragma unroll
              for (int i = 0; i < 4; ++i) o[i] = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
            }
          }
          if (real && seg.whole && a.lse) a.lse[at] = lse_of(m, l);
          if (real && !seg.whole) {
            part[P::ROWS * D + prow] = m;
            part[P::ROWS * (D + 1) + prow] = l;
          }
        }
      }
    } else if (warp < ISSUE) {
      // --------------------------------------------------------- converters
      const int cw = warp - SOFT;
      const int32_t* table = kv.c.table + sq.slot * kv.c.max_pages;
      // lane b < 8 looks up block b of a tile: its 16 rows in the pool and its scales
      int64_t line = -1, line_next = -1;
      float ks = 0.0f, vs = 0.0f, ks_next = 0.0f, vs_next = 0.0f;
      auto look_up = [&](int j) {
        line_next = -1;
        ks_next = vs_next = 0.0f;
        const int64_t tok = (int64_t)(first + j) * TOKENS + lane * kKvBlock;
        if (lane < 8 && j < tiles && tok < sq.len) {
          const int page = table[tok >> kv.page_shift];
          if (page >= 0 && page < kv.c.pages) {
            line_next = kv.scales_at(a.layer, page, head) + ((tok & (kv.c.page_tokens - 1)) / kKvBlock);
            ks_next = __ldg(kv.c.k_scale + line_next);
            vs_next = __ldg(kv.c.v_scale + line_next);
          } else {
            kv_status(kv, kKvBadEntry);
          }
        }
      };
      // keys: warp cw takes tokens 32 cw ..; lane: 16-byte piece (lane & 3) of each 64 bytes, token lane >> 2 of 8
      constexpr int KN = D / 64 * 4;
      uint4 kr[KN];
      auto load_k = [&]() {
#pragma unroll
        for (int i = 0; i < KN; ++i) {
          const int tok = cw * 32 + (i & 3) * 8 + (lane >> 2);
          const int64_t ln = __shfl_sync(FULL, line, tok >> 4);
          kr[i] = make_uint4(0, 0, 0, 0);
          if (ln >= 0)
            kr[i] = __ldg(reinterpret_cast<const uint4*>(kv.c.k + (ln * kKvBlock + (tok & 15)) * D + (i >> 2) * 64 + (lane & 3) * 16));
        }
      };
      // values: 64 tokens x 64 elements a warp (half of them at head_dim 64: 64 x 32); lane: 8 tokens (lane & 7), VB elements
      constexpr int VB = D / 8;  // bytes of a lane's row: 16 or 8
      const int half = cw >> 1, v_octet = lane & 7, v_el = (cw & 1) * (D / 2) + (lane >> 3) * VB;
      uint32_t vr[8][VB / 4];
      auto load_v = [&](int j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int tok = half * 64 + v_octet * 8 + i;
          int64_t ln = __shfl_sync(FULL, line, tok >> 4);
          // bytes that no token owns may be NaN, and 0 times that is not 0
          if ((first + j) * TOKENS + tok >= sq.len) ln = -1;
          const uint8_t* p = kv.c.v + (ln * kKvBlock + (tok & 15)) * D + v_el;
#pragma unroll
          for (int x = 0; x < VB / 4; ++x) vr[i][x] = 0;
          if (ln >= 0) {
            if (VB == 16) {
              const uint4 y = __ldg(reinterpret_cast<const uint4*>(p));
              vr[i][0] = y.x, vr[i][1] = y.y, vr[i][VB / 4 - 2] = y.z, vr[i][VB / 4 - 1] = y.w;
            } else {
              const uint2 y = __ldg(reinterpret_cast<const uint2*>(p));
              vr[i][0] = y.x, vr[i][1] = y.y;
            }
          }
        }
      };
      look_up(0);
      line = line_next, ks = ks_next, vs = vs_next;
      if (tiles) load_k();
      for (int j = 0; j < tiles; ++j) {
        const int n = done + j, st = n & 1;
        load_v(j);
        look_up(j + 1);
        if (n >= 2 && !all_wait(sh.k_empty + st, ((n >> 1) - 1) & 1, abort_flag, err, 4)) break;
        if (cw == 0 && lane < 8) {
          // (the softmax of the tile that had this place in the ring is over: S two tiles on waited for it)
          const float g = fmaxf(vs, 0x1p-100f);
          sh.scales[n % SCALE_RING][0][lane] = ks;
          sh.scales[n % SCALE_RING][1][lane] = line >= 0 ? log2f(g) : -INFINITY;
          sh.scales[n % SCALE_RING][2][lane] = line >= 0 ? 1.0f / g : 0.0f;
        }
        unsigned char* sk = sm + M::k + st * M::K;
#pragma unroll
        for (int i = 0; i < KN; ++i) {
          const int tok = cw * 32 + (i & 3) * 8 + (lane >> 2), c = (lane & 3) * 2;
          uint32_t h[8];
          const uint32_t x[4] = {kr[i].x, kr[i].y, kr[i].z, kr[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) to_fp16x4<CODES>(x[e], h[2 * e], h[2 * e + 1]);
          unsigned char* to = sk + (i >> 2) * 16384;
          *reinterpret_cast<uint4*>(to + sw128_offset(tok, c)) = make_uint4(h[0], h[1], h[2], h[3]);
          *reinterpret_cast<uint4*>(to + sw128_offset(tok, c + 1)) = make_uint4(h[4], h[5], h[6], h[7]);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(sh.k_full + st);
        line = line_next, ks = ks_next, vs = vs_next;
        if (j + 1 < tiles) load_k();
        if (n >= 2 && !all_wait(sh.v_empty + st, ((n >> 1) - 1) & 1, abort_flag, err, 5)) break;
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
    } else {
      // --------------------------------------------------------- MMA issuer
      const uint32_t tm = __shfl_sync(FULL, tmem, 0);
      const uint64_t q0 = sw128_desc(__shfl_sync(FULL, smem_u32(sm + M::q), 0));
      const uint64_t k0 = sw128_desc(__shfl_sync(FULL, smem_u32(sm + M::k), 0));
      const uint64_t v0 = sw128_desc(__shfl_sync(FULL, smem_u32(sm + M::v), 0));
      // S of row tile w and tile n of this CTA
      auto scores = [&](int w, int n) {
        if (elect_one()) {
          const uint64_t qd = q0 + (uint64_t)(w * (M::Q >> 4)), kd = k0 + (uint64_t)((n & 1) * (M::K >> 4));
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint64_t off = (uint64_t)((kk >> 2) * (16384 >> 4) + (kk & 3) * 2);
            mma_f16_ss(tm + (uint32_t)(w * TOKENS), qd + off, kd + off, tile_idesc(TOKENS), kk ? 1u : 0u);
          }
          mma_commit(sh.s_full + w);
        }
        __syncwarp();
      };
      auto values = [&](int w, int n, bool more) {
        if (elect_one()) {
          const uint64_t vd = v0 + (uint64_t)((n & 1) * (M::K >> 4));
#pragma unroll
          for (int kk = 0; kk < TOKENS / 16; ++kk)
            mma_f16_ta(tm + (uint32_t)(2 * TOKENS + w * D), tm + (uint32_t)(w * TOKENS + kk * 8),
                       vd + (uint64_t)((kk >> 2) * (D * 128 >> 4) + (kk & 3) * 2), tile_idesc(D), kk || more ? 1u : 0u);
          mma_commit(sh.o_full + w);
        }
        __syncwarp();
      };
      auto release = [&](uint64_t* bar) {
        if (elect_one()) mma_commit(bar);
        __syncwarp();
      };
      bool ok = all_wait(&sh.q_full, segments & 1, abort_flag, err, 6);
      if (ok && tiles) {
        ok = all_wait(sh.k_full + (done & 1), (done >> 1) & 1, abort_flag, err, 7);
        if (ok) {
          tc_fence_after();
          scores(0, done);
          if (two) scores(1, done);
          release(sh.k_empty + (done & 1));
        }
        for (int j = 0; ok && j < tiles; ++j) {
          const int n = done + j;
          if (!(ok = all_wait(sh.v_full + (n & 1), (n >> 1) & 1, abort_flag, err, 8) &&
                     all_wait(sh.p_full, n & 1, abort_flag, err, 9)))
            break;
          tc_fence_after();
          values(0, n, j > 0);
          if (two) {
            if (!(ok = all_wait(sh.p_full + 1, (done2 + j) & 1, abort_flag, err, 10))) break;
            tc_fence_after();
            values(1, n, j > 0);
          }
          release(sh.v_empty + (n & 1));
          if (j + 1 == tiles) break;
          // the next scores overwrite P: its product has to be complete
          if (!(ok = all_wait(sh.k_full + ((n + 1) & 1), ((n + 1) >> 1) & 1, abort_flag, err, 11) &&
                     all_wait(sh.o_full, n & 1, abort_flag, err, 12)))
            break;
          tc_fence_after();
          scores(0, n + 1);
          if (two) {
            if (!(ok = all_wait(sh.o_full + 1, (done2 + j) & 1, abort_flag, err, 13))) break;
            tc_fence_after();
            scores(1, n + 1);
          }
          release(sh.k_empty + ((n + 1) & 1));
        }
      }
    }
    done += tiles;
    if (two) done2 += tiles;
    ++segments;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*abort_flag) break;  // (uniform behind the barrier)
  }
  if (warp == ISSUE) {
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
  if (warp == ISSUE) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

template <typename T, int D, int CODES>
cudaError_t tile(const AttendArgs& a, int grid, cudaStream_t s) {
  auto* kernel = k_kv_tile<T, D, CODES>;
  cudaError_t e = set_max_dynamic_smem(reinterpret_cast<const void*>(kernel), TileSmem<D>::total);
  if (e != cudaSuccess) return e;
  kernel<<<grid, TILE_THREADS, TileSmem<D>::total, s>>>(a);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  return launch_join<T, D, TileCut::ROWS>(a, grid, s);
}

template <typename T>
cudaError_t tile_for(const AttendArgs& a, int grid, cudaStream_t s) {
  const bool i8 = a.kv.c.codes == TQ_KV_INT8;
  if (a.kv.c.head_dim == 64) return (i8 ? tile<T, 64, TQ_KV_INT8> : tile<T, 64, TQ_KV_E4M3>)(a, grid, s);
  return (i8 ? tile<T, 128, TQ_KV_INT8> : tile<T, 128, TQ_KV_E4M3>)(a, grid, s);
}

}  // namespace

// Where the sequences bring more than 16 rows on average (and the operands of 256
// rows fit beside two stages: head_dim up to 128).
bool kv_tile_supported(const KvView& kv, int64_t n, int64_t total, int heads) {
  return n > 0 && kv.c.head_dim <= 128 && (total + n - 1) / n * (heads / kv.c.kv_heads) > 16;
}

size_t kv_tile_workspace(const KvView& kv) {
  return attend_workspace(device_sm_count(), TileCut::ROWS, kv.c.head_dim);
}

cudaError_t launch_kv_tile(AttendArgs a, int type, void* workspace, cudaStream_t s) {
  const int grid = device_sm_count();
  take_workspace(a, grid, workspace);
  return type == TQ_BF16 ? tile_for<__nv_bfloat16>(a, grid, s) : tile_for<__half>(a, grid, s);
}

}  // namespace tq
