// tree_attention.cu -- spinq_tree_attention_kv4 and spinq_window_attention_kv4:
// the last tokens of each sequence (a tree of drafted ones, or one) over the
// paged 4-bit cache.
//
// Sequence b has n tokens in the cache, the last nq of them its queries' own.  Query
// i sees the context, tokens 0 .. n - nq - 1, its ancestors by `parents`, and
// itself; with a window only those of them whose position (a context token's
// place, a node's n - nq + depth) is less than `window` before its own or below
// `sinks`.  Scores, weights and sums as in prefix_attention.cu:
//   t = scale log2(e) q . k + log2 alpha',  w = 2^(t - M),
//   o = [ sum w (u' - 8) + sum w (8 + beta' / alpha') ] / sum w / alpha'
// with the codes as exact fp16 operands and w in two fp16 parts.
//
// Work.  A job is ROWS rows (query x head of a kv head's group, in that order) of a
// sequence and a kv head; its keys are cut into units of UNIT tokens: the sinks, and
// from the first that a window reaches to the end.  The units of all jobs in a row
// are dealt to the CTAs in equal runs, so lengths may differ as they like: a CTA
// finds its run by a sum over the batch, and has at most one job that it continues
// and one that it begins but does not end.  Those two go to the workspace and
// tree_combine_kernel joins them, in the order of the keys; every other job is
// complete in its CTA.
#include <cuda_fp16.h>
#include <float.h>

#include "../../include/spinq.h"
#include "attn_tc.cuh"
#include "kv4_attn.cuh"
#include "launch_util.h"
#include "spinq_internal.h"
#include "tree_attention.cuh"

namespace spinq {
namespace {

constexpr int kRowsWarps = 4;
// Parts of a job on an average, at most: the runs are no more than this times the batch's jobs.  An even batch's jobs
// have no more each; a long one among short ones has, as those leave it their share (30000 tokens of one kv head
// beside 39 sequences of 10: 118 parts, 17.5 us; alone, in 20, 16.4).  (4 rows of D 128, one sequence of 4000 tokens: 9.9 us with 20, 11.2 with 60; of 8000 14.1
// and 13.7; of 16000 15.3 and 15.8; two of 16000 19.2 and 21.3)
constexpr int kRowsParts = 20;
constexpr int kCombineThreads = 256;

// Shared memory: each warp's ring (after a job's loop: float o [ROWS][D]), a stage the
// value rows, key rows (D/2 bytes each) and scales of 16 T tokens.  Three CTAs with two
// stages of 64 tokens (D 128) fill an SM.
template <int D, int T>
struct RowsRing {
  static constexpr int STAGES = T == 1 ? 4 : (T == 2 || D == 64 ? 3 : 2), KB = 16 * T * (D / 2), SB = 256 * T, KEYS = STAGES * KB, SCALES = 2 * KEYS,
                       WARP = SCALES + STAGES * SB, BYTES = kRowsWarps * WARP;
};

// ------------------------------------------------ few rows: warps and mma.sync
// A job is 8 NB rows, a unit 64 T tokens.  A warp takes 16 T tokens of each unit, whose
// rows of codes are one run of memory (two where pages have 16 tokens), copied ahead into the
// warp's ring.  Fragments of lane 4 g + c: key rows g and g + 8, bytes [c D/8, (c+1) D/8);
// of the values a transposing load of 8 rows x 16 bytes, which gives it dimensions 4 g ..
// 4 g + 3 of the 32 for tokens 2c and 2c + 1.  Those rows' pieces are moved about, so that
// eight of them lie in different banks.  Scores: tokens on M, rows on N; values: head_dim on M,
// tokens on K, rows on N.
// HALF: four rows at most; the second parts of the weights are the product's columns 4 .. 7 and
// cost no product of their own.
// T tiles of tokens a step: their chains of products and exponentials overlap, and the step's own
// cost is shared (4 rows of D 128, 128 windows of 4096 tokens: 140 us with one, 120.5 with two, 113.4
// with four; 16 rows of D 64, 32 x 8000: 71 and 63 with one and two).  16 rows of D 128 have no registers for two.
// Bound: instructions (262 for 16 tokens and a warp, 56 % of the issue slots at 3 warps a scheduler) beside the
// bytes: that case's 582 MB in 113.4 us with the join are 5.13 TB/s, 77 % of the measured copy rate.
// Bulk copies by one lane (the values' with a tensor map's swizzle) are faster alone (104 us for them, 118 to
// 131 for these), but cost more instructions: 131 us in all where these took 124.  5 CTAs an SM (spills) 149
// against 145; two chains of products for the scores 146 against 144; the scores multiplied a step ahead 170 against 151.
template <int D, int NB, int T, bool HALF>
__global__ void __launch_bounds__(kRowsWarps * 32, NB == 1 && T < 4 ? 4 : 3) tree_rows_kernel(const TreeParams p) {
  constexpr int KW = D / 32, NM = D / 16, ROWS = 8 * NB, UNIT = 16 * T * kRowsWarps;
  const TreeArgs& a = p.a;
  using Ring = RowsRing<D, T>;
  extern __shared__ __align__(512) uint8_t ring_s[];
  static_assert(Ring::WARP % 512 == 0 && Ring::KB % 512 == 0, "whole tiles of moved pieces");
  static_assert(ROWS * D * 4 <= Ring::WARP, "the output fits in the ring");
  __shared__ float m_s[kRowsWarps][ROWS], l_s[kRowsWarps][ROWS];
  __shared__ int parent_s[kTreeNodes];
  __shared__ TreeRow row_s[ROWS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  uint8_t* const ring = ring_s + warp * Ring::WARP;
  // a value row's 16-byte piece (of the first 16 rows; the rest repeat them)
  auto value_at = [](int row, int piece) { return row * (D / 2) + ((piece ^ (row / (256 / D) & (D / 32 - 1))) << 4); };
  // what the lane copies, and the row it names in a transposing load: matrix m has rows 8 (m % 2) .. and piece m / 2
  const uint32_t copy_k = smem_u32(ring) + Ring::KEYS + lane * 16, copy_s = smem_u32(ring) + Ring::SCALES + lane * 16;
  const uint32_t copy_v = smem_u32(ring) + value_at(lane / (D / 32), lane % (D / 32));
  const uint32_t load_v = smem_u32(ring) + value_at(lane & 15, lane >> 4);
  // a step's tokens lie in 2^pieces pages
  constexpr int STEP_LOG2 = T == 4 ? 6 : T + 3;
  static_assert(16 * T == 1 << STEP_LOG2, "tokens of a step");
  const int run_log2 = min(p.shift, STEP_LOG2), pieces = STEP_LOG2 - run_log2;
  pdl_wait();
  pdl_trigger();
  TreeWalk walk(tree_run<kRowsWarps * 32, kRowsParts>(p, blockIdx.x), blockIdx.x);
  for (TreeJob j; walk.next(p, j);) {
    const TreeSeq& s = j.s;
    const int rows = j.rows;
    const int nstep = j.v1 - j.v0;
    auto token_of = [&](int i) {   // first token of this warp's step i
      return j.token(j.v0 + i, UNIT) + 16 * T * warp;
    };
    const int32_t* table = a.table + (int64_t)j.b * a.table_width;
    // tokens before `none` that are not sinks are in no row's window: steps of them are passed over
    const int none = p.window > 0 && s.ctx >= p.window ? s.ctx - p.window + 1 : 0;
    auto unseen = [&](int t) { return T == 4 && t + 16 * T <= none && t >= p.sinks; };
    // Lane k holds a page of the warp's step 32 j + k (of two or four pages a step: 16 j + k / 2,
    // 8 j + k / 4): one look-up for many steps.
    int page = 0;
    int ks = 0, kr = 0;   // stages of the next step to copy, of the next to use
    auto issue = [&](int i) {   // copies of step i
      const int t = token_of(i);
      if (i >= nstep || t >= s.n) {   // an empty group keeps the count
        asm volatile("cp.async.commit_group;\n" ::: "memory");
        return;
      }
      const int at_lane = (i << pieces) & 31;
      if (at_lane == 0) {
        const int ti = token_of(min(i + (lane >> pieces), nstep - 1)) + ((lane & ((1 << pieces) - 1)) << run_log2);
        page = ti < s.n ? (int)tree_page(a, table, ti, p.shift) : 0;
      }
      if (!unseen(t)) {
        auto place = [&](int u) {   // of tile u, which begins a page or the step
          const int pg = __shfl_sync(0xffffffffu, page, at_lane + (16 * u >> run_log2));
          return ((int64_t)pg * a.Hkv + j.hk) * a.page_size + ((t + 16 * u) & (a.page_size - 1));
        };
        auto codes = [&](int u, int64_t at) {
          const int64_t x = at * (D / 2) + lane * 16;
#pragma unroll
          for (int k = 0; k < D / 64; ++k) {
            own_copy16(copy_k + ks * Ring::KB + u * (Ring::KB / T) + 512 * k, a.k_codes + x + 512 * k);
            own_copy16(copy_v + ks * Ring::KB + u * (Ring::KB / T) + 512 * k, a.v_codes + x + 512 * k);
          }
        };
        auto scales = [&](int u, int64_t at, int64_t next) {   // of tile u in the first half of the lanes, and the next in the others
          if (lane < 16 || (u + 1 < T && t + 16 * (u + 1) < s.n))
            own_copy16(copy_s + ks * Ring::SB + u * 256, a.scales + ((lane < 16 ? at : next - 16) + lane) * 4);
        };
        int64_t at = place(0);
        if (pieces == 0) {
#pragma unroll
          for (int u = 0; u < T; ++u) {
            if (u > 0 && t + 16 * u >= s.n) break;
            codes(u, at + 16 * u);
            if (u % 2 == 0) scales(u, at + 16 * u, at + 16 * (u + 1));
          }
        } else {
#pragma unroll
          for (int u = 0; u < T; u += 2) {
            if (u > 0 && t + 16 * u >= s.n) break;
            if (u > 0) at = place(u);   // (a step has two pages at least: one begins here)
            codes(u, at);
            int64_t next = at + 16;
            if (u + 1 < T && t + 16 * (u + 1) < s.n) {
              if (run_log2 == 4) next = place(u + 1);
              codes(u + 1, next);
            }
            scales(u, at, next);
          }
        }
      }
      asm volatile("cp.async.commit_group;\n" ::: "memory");
      ks = ks + 1 == Ring::STAGES ? 0 : ks + 1;
    };
    // (before the set-up, which takes as long as a copy)
#pragma unroll
    for (int i = 0; i < Ring::STAGES - 1; ++i) issue(i);
    // what the rows see
    tree_parents(p, s, parent_s, kRowsWarps * 32);
    __syncthreads();
    if (tid < ROWS) {
      TreeRow r = {};
      if (tid < rows) r = tree_row(p, s, parent_s, tree_node(p, j.r0 + tid));
      row_s[tid] = r;
    }
    // query fragments (k order as the codes come), their sums.  A key
    // code is masked out of its word in place: as fp16 bits the nibbles at bits 0 and 16
    // are u 2^-24, those at bits 4 and 20 are 16 u 2^-24, both exact operands; each
    // kind has a product of its own, the latter's is divided by 16 in fp32.
    uint32_t qb[NB][KW][4];
    float qsk[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = 8 * nb + g;
      const __half* qh = reinterpret_cast<const __half*>(a.q) + j.row_at(p, r < rows ? r : 0) * D + c * (D / 4);
      float qs = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        uint4 y = __ldg(reinterpret_cast<const uint4*>(qh + 8 * w));
        if (r >= rows) y = make_uint4(0, 0, 0, 0);
        const uint32_t ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&ys[q]));
          qs += f.x + f.y;
        }
        qb[nb][w][0] = __byte_perm(y.x, y.z, 0x5410);
        qb[nb][w][1] = __byte_perm(y.y, y.w, 0x5410);
        qb[nb][w][2] = __byte_perm(y.x, y.z, 0x7632);
        qb[nb][w][3] = __byte_perm(y.y, y.w, 0x7632);
      }
      qs += __shfl_xor_sync(0xffffffffu, qs, 1);
      qs += __shfl_xor_sync(0xffffffffu, qs, 2);
      qsk[nb][0] = p.scale_log2 * __shfl_sync(0xffffffffu, qs, 8 * c);
      qsk[nb][1] = p.scale_log2 * __shfl_sync(0xffffffffu, qs, 8 * c + 4);
    }
    const float ks24 = p.scale_log2 * 16777216.f;
    __syncthreads();   // rows' views written
    // tokens that every row sees: those below `ctx`, from the last row's window on or in the sinks
    int low = 0;
    for (int r = 0; r < rows; ++r) low = max(low, row_s[r].low);

    float o[NB][NM][4], m[NB][2], off[NB][2], l[NB][2], z[NB][2];   // m: M
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int mu = 0; mu < NM; ++mu) o[nb][mu][0] = o[nb][mu][1] = o[nb][mu][2] = o[nb][mu][3] = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) m[nb][e] = -INFINITY, off[nb][e] = l[nb][e] = z[nb][e] = 0.f;
    }
    for (int i = 0; i < nstep; ++i) {
      const int t0 = token_of(i);
      if (t0 >= s.n) break;   // (nothing was copied)
      asm volatile("cp.async.wait_group %0;\n" ::"n"(Ring::STAGES - 2) : "memory");
      __syncwarp();   // step i has landed for every lane, and step i - 1's stage has been read
      issue(i + Ring::STAGES - 1);
      if (unseen(t0)) {
        if (++kr == Ring::STAGES) kr = 0;
        continue;
      }
      const uint8_t* st = ring + Ring::KEYS + kr * Ring::KB + g * (D / 2) + c * (D / 8);
      const uint8_t* sp = ring + Ring::SCALES + kr * Ring::SB + g * 16;
      const uint32_t va = load_v + kr * Ring::KB;
      float sa[T][NB][4] = {}, s16[T][NB][4] = {};
#pragma unroll
      for (int u = 0; u < T; ++u) {
        uint32_t kx[2][KW];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint8_t* k = st + (16 * u + 8 * h) * (D / 2);
          if constexpr (KW == 4) {
            const uint4 w = *reinterpret_cast<const uint4*>(k);
            kx[h][0] = w.x, kx[h][1] = w.y, kx[h][2] = w.z, kx[h][3] = w.w;
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(k);
            kx[h][0] = w.x, kx[h][1] = w.y;
          }
        }
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          const uint32_t x0 = kx[0][w], x1 = kx[1][w], y0 = x0 >> 8, y1 = x1 >> 8;
          const uint32_t a0[4] = {x0 & 0x000F000Fu, x1 & 0x000F000Fu, y0 & 0x000F000Fu, y1 & 0x000F000Fu};
          const uint32_t a1[4] = {x0 & 0x00F000F0u, x1 & 0x00F000F0u, y0 & 0x00F000F0u, y1 & 0x00F000F0u};
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma_16816_f16_f32_acc(sa[u][nb], a0, qb[nb][w][0], qb[nb][w][1]);
            mma_16816_f16_f32_acc(s16[u][nb], a1, qb[nb][w][2], qb[nb][w][3]);
          }
        }
      }
      if (++kr == Ring::STAGES) kr = 0;
      // t = s + log2 alpha' (base 2) of tokens g, g + 8, .. for rows 8 nb + 2c, + 1
      float t[NB][2 * T][2], rv[2 * T], vz[2 * T];
#pragma unroll
      for (int h = 0; h < 2 * T; ++h) {
        const float4 sc = *reinterpret_cast<const float4*>(sp + h * 128);
        const float ka = ks24 * sc.x;
        const float av = value_scale(sc.z), la = log2_of_scale(av);
        rv[h] = one_over_scale(av);
        vz[h] = fmaf(rv[h], sc.w, 8.f);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            t[nb][h][e] = fmaf(ka, fmaf(0.0625f, s16[h >> 1][nb][2 * (h & 1) + e], sa[h >> 1][nb][2 * (h & 1) + e]),
                               fmaf(sc.y, qsk[nb][e], la));
      }
      // Not every row sees every token: -inf.  Factors that are not finite (a slot that was never
      // written, a page given back, a row of NaN) would give 0 times them: they are 0 here, and the
      // score of a row that does see the token is not a number.
      if (t0 + 16 * T > s.ctx || (t0 < low && t0 + 16 * T > p.sinks)) {
#pragma unroll
        for (int h = 0; h < 2 * T; ++h) {
          const bool bad = !(fabsf(rv[h]) <= FLT_MAX && fabsf(vz[h]) <= FLT_MAX);
          if (bad) rv[h] = vz[h] = 0.f;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t bits = tree_sees(p, s, row_s[8 * nb + 2 * c + e], t0 + 32 * (h >> 2)) >> (g + 8 * (h & 3));
              t[nb][h][e] = bits & 1u ? (bad ? __int_as_float(0x7fc00000) : t[nb][h][e]) : -INFINITY;
            }
        }
      }
      bool grow = false;
      float mx[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          mx[nb][e] = fmaxf(t[nb][0][e], t[nb][1][e]);
#pragma unroll
          for (int h = 2; h < 2 * T; ++h) mx[nb][e] = fmaxf(mx[nb][e], t[nb][h][e]);
          grow |= mx[nb][e] > m[nb][e] + kAttnSlack;
        }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) mx[nb][e] = fmaxf(mx[nb][e], __shfl_xor_sync(0xffffffffu, mx[nb][e], w));
            const float mn = mx[nb][e] > m[nb][e] + kAttnSlack ? mx[nb][e] : m[nb][e];
            const float to = mn == -INFINITY ? 0.f : mn;
            f[e] = m[nb][e] == -INFINITY ? 0.f : attn_exp2(off[nb][e] - to);
            // (a sum so far that is not a number stays one)
            if (m[nb][e] == -INFINITY && l[nb][e] != l[nb][e]) f[e] = 1.f;
            m[nb][e] = mn;
            off[nb][e] = to;
            l[nb][e] *= f[e];
            z[nb][e] *= f[e];
            if constexpr (HALF) f[e] = __shfl_sync(0xffffffffu, f[e], lane & 29);   // second parts: their rows' factor
          }
#pragma unroll
          for (int mu = 0; mu < NM; ++mu) {
            o[nb][mu][0] *= f[0], o[nb][mu][2] *= f[0];
            o[nb][mu][1] *= f[1], o[nb][mu][3] *= f[1];
          }
        }
      }
      // the weights as two fp16 parts, the second what the first leaves: with one part the
      // few weights that carry a row would all but double its error
      uint32_t p0[NB][2 * T], p1[NB][2 * T];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float w[2 * T][2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int h = 0; h < 2 * T; ++h) {
            w[h][e] = attn_exp2(t[nb][h][e] - off[nb][e]);
            l[nb][e] = fmaf(w[h][e], rv[h], l[nb][e]);
            z[nb][e] = fmaf(w[h][e], vz[h], z[nb][e]);
          }
#pragma unroll
        for (int h = 0; h < 2 * T; ++h) {
          const uint32_t hi = pack_half2_bits(w[h][0], w[h][1]);
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hi));
          const uint32_t lo = pack_half2_bits(w[h][0] - f.x, w[h][1] - f.y);
          if constexpr (HALF) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, lo, 2);
            p0[nb][h] = own_transpose(c & 2 ? other : hi);
          } else {
            p0[nb][h] = own_transpose(hi);
            p1[nb][h] = own_transpose(lo);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < T; ++u)
#pragma unroll
        for (int v = 0; v < D / 64; ++v) {
          uint32_t vx[4];   // two bytes of tokens 2c and 2c + 1, 2c + 8 and 2c + 9 in piece 2 v, then in piece 2 v + 1
          ldmatrix_x4_trans(vx, (va + u * 16 * (D / 2)) ^ (32 * v));
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            // one dimension of both tokens in a pair
            // (as u - 8: the values' sums would lose bits on the numbers that fp16 has below its normal ones)
            const uint4 ya = code_pairs1(vx[2 * q]), yb = code_pairs1(vx[2 * q + 1]);
            const uint32_t a0[4] = {ya.x, ya.y, yb.x, yb.y}, a1[4] = {ya.z, ya.w, yb.z, yb.w};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              mma_16816_f16_f32_acc(o[nb][4 * v + 2 * q], a0, p0[nb][2 * u], p0[nb][2 * u + 1]);
              mma_16816_f16_f32_acc(o[nb][4 * v + 2 * q + 1], a1, p0[nb][2 * u], p0[nb][2 * u + 1]);
              if constexpr (!HALF) {
                mma_16816_f16_f32_acc(o[nb][4 * v + 2 * q], a0, p1[nb][2 * u], p1[nb][2 * u + 1]);
                mma_16816_f16_f32_acc(o[nb][4 * v + 2 * q + 1], a1, p1[nb][2 * u], p1[nb][2 * u + 1]);
              }
            }
          }
        }
    }
    // join the lanes' shares, then the warps
    asm volatile("cp.async.wait_group 0;\n" ::: "memory");
    __syncwarp();   // the ring is free
    float* o_w = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float ls = l[nb][e], zs = z[nb][e];
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) {
          ls += __shfl_xor_sync(0xffffffffu, ls, w);
          zs += __shfl_xor_sync(0xffffffffu, zs, w);
        }
        const int r = 8 * nb + 2 * c + e;
        if constexpr (HALF) {
#pragma unroll
          for (int mu = 0; mu < NM; ++mu) {
            o[nb][mu][e] += __shfl_xor_sync(0xffffffffu, o[nb][mu][e], 2);
            o[nb][mu][2 + e] += __shfl_xor_sync(0xffffffffu, o[nb][mu][2 + e], 2);
          }
        }
#pragma unroll
        for (int q = 0; q < D / 32; ++q)
          *reinterpret_cast<float4*>(o_w + r * D + 32 * q + 4 * g) =
              make_float4(o[nb][2 * q][e] + zs, o[nb][2 * q][2 + e] + zs, o[nb][2 * q + 1][e] + zs, o[nb][2 * q + 1][2 + e] + zs);
        if (g == 0) {
          m_s[warp][r] = m[nb][e];
          l_s[warp][r] = ls;
        }
      }
    __syncthreads();
    const bool whole = j.whole();
    const int64_t slot = j.slot(blockIdx.x);
    for (int i = tid; i < rows * (D / 4); i += kRowsWarps * 32) {   // four values of a row
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kRowsWarps; ++w) M = fmaxf(M, m_s[w][r]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float ls = 0.f;
#pragma unroll
      for (int w = 0; w < kRowsWarps; ++w) {
        const float lw = l_s[w][r];
        if (lw == 0.f) continue;
        const float f = attn_exp2(m_s[w][r] - M);
        const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(ring_s + w * Ring::WARP) + r * D + d);
        v.x = fmaf(f, y.x, v.x), v.y = fmaf(f, y.y, v.y), v.z = fmaf(f, y.z, v.z), v.w = fmaf(f, y.w, v.w);
        ls = fmaf(f, lw, ls);
      }
      if (whole) {
        const float inv = ls != 0.f ? 1.f / ls : 0.f;
        *reinterpret_cast<uint2*>(reinterpret_cast<__half*>(a.out) + j.row_at(p, r) * D + d) =
            make_uint2(pack_half2_bits(v.x * inv, v.y * inv), pack_half2_bits(v.z * inv, v.w * inv));
      } else {
        *reinterpret_cast<float4*>(p.o + (slot * ROWS + r) * D + d) = v;
        if (d == 0) p.ml[slot * ROWS + r] = make_float2(M, ls);
      }
    }
    __syncthreads();   // the ring and the rows' views serve the next job
  }
}

// Joins the parts of a job that several CTAs share, in their order.  Block (c, y): the job that
// the runs' border c cuts first, its y-th group of rows; D / 4 lanes share a row, each has four of its
// values and looks every (D / 4)th part's numbers up for all of them.  Bound: latency; the first eight
// parts' values are under way before their numbers are there.
template <int D, int PARTS>
__global__ void __launch_bounds__(kCombineThreads) tree_combine_kernel(const TreeParams p) {
  constexpr int LPR = D / 4, RPB = kCombineThreads / LPR;
  static_assert(LPR <= 32 && LPR % 8 == 0, "lanes of a row");
  const TreeArgs& a = p.a;
  const int c = blockIdx.x + 1;
  // (the attention kernel started behind what wrote the lengths, and this one behind its start)
  const TreeRun run = tree_run<kCombineThreads, PARTS>(p, c);
  const TreeSeq& s = run.s;
  const int64_t x = c < run.ctas ? run.bound(c) : run.base, in = x - run.base;
  const int64_t job = in <= INT32_MAX ? (uint32_t)in / (uint32_t)max(1, s.units) : in / s.units;
  const int64_t begin = run.base + job * s.units, end = begin + s.units;
  pdl_wait();
  pdl_trigger();
  if (c >= run.ctas) return;
  if (x == begin || run.bound(c - 1) > begin || (int)(threadIdx.x / LPR) >= 1 << p.rows_log2) return;   // no job cut, or cut before
  const int rows = 1 << p.rows_log2;
  const int hk = (int)job / s.rts, r = blockIdx.y * RPB + threadIdx.x / LPR, k0 = threadIdx.x % LPR, d = 4 * k0;
  const int row = (((int)job - hk * s.rts) << p.rows_log2) + r;
  const bool valid = row < s.nq * p.G;
  // parts: the one that CTA c - 1 left, then those that c, c + 1, .. continued
  auto slot = [&](int i) { return (int64_t)(i ? 2 * (c - 1 + i) : 2 * (c - 1) + 1) * rows + r; };
  const int parts = run.owner(end - 1) - (c - 1) + 1;
  float4 o[8];
  auto load = [&](int i0) {   // eight parts' values under way at once (the last one's again past the end)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];\n"
                   : "=f"(o[i].x), "=f"(o[i].y), "=f"(o[i].z), "=f"(o[i].w)
                   : "l"(p.o + slot(min(i0 + i, parts - 1)) * D + d));
  };
  auto numbers = [&](int i) {   // M and sum of part i (the row of a part past the queries' end was not written)
    float2 y = make_float2(0.f, 0.f);
    if (valid && i < parts) asm volatile("ld.global.v2.f32 {%0, %1}, [%2];\n" : "=f"(y.x), "=f"(y.y) : "l"(p.ml + slot(i)));
    return y;
  };
  float2 y = numbers(k0);
  load(0);
  float M = y.y != 0.f ? y.x : -INFINITY;
  for (int i = k0 + LPR; i < parts; i += LPR) {
    const float2 z = numbers(i);
    if (z.y != 0.f) M = fmaxf(M, z.x);
  }
#pragma unroll
  for (int w = 1; w < LPR; w <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, w));
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  float l = 0.f;
  for (int i0 = 0; i0 < parts; i0 += 8) {
    if (i0 % LPR == 0 && i0) y = numbers(i0 + k0);
    const float mine = y.y != 0.f ? attn_exp2(y.x - M) : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = (i0 + i) % LPR;
      const float f = __shfl_sync(0xffffffffu, mine, k, LPR), t = __shfl_sync(0xffffffffu, y.y, k, LPR);
      // (A part without a key that the row sees, or past the last one, has the sum 0.  One whose sum is not a number has
      // no maximum or any: its factor may be 0, and the product with it keeps the sum what it is.)
      if (t != 0.f) {
        v.x = fmaf(f, o[i].x, v.x), v.y = fmaf(f, o[i].y, v.y), v.z = fmaf(f, o[i].z, v.z), v.w = fmaf(f, o[i].w, v.w);
        l = fmaf(f, t, l);
      }
    }
    if (i0 + 8 < parts) load(i0 + 8);
  }
  if (!valid) return;
  const float inv = l != 0.f ? 1.f / l : 0.f;
  const int node = tree_node(p, row), head = row - node * p.G;
  *reinterpret_cast<uint2*>(reinterpret_cast<__half*>(a.out) + ((int64_t)(s.q0 + node) * a.Hq + hk * p.G + head) * D + d) =
      make_uint2(pack_half2_bits(v.x * inv, v.y * inv), pack_half2_bits(v.z * inv, v.w * inv));
}

int64_t align256(int64_t v) { return (v + 255) / 256 * 256; }

// The variant for these sizes and its grid.
struct TreePlan {
  int rows_log2, unit_log2, ctas, least;   // ctas of the largest grid
};
TreePlan tree_plan(const TreeArgs& a) {
  const int64_t rows = a.max_q * (a.Hq / a.Hkv);
  // (D 64, 24 sequences of 25 rows: 1000 tokens 24.0 us on warps in two jobs, 28.3 on the tensor core, 8000 tokens
  // 93 and 101 (with one tile a step); D 128, 8 x 2000 tokens and 32 rows 29.8 and 25.1, 32 x 8000 198 and 145; 16 rows 107 and 144)
  if (rows > (a.D == 64 ? 32 : 16)) return {rows <= 32 ? 5 : (rows <= 64 ? 6 : 7), kTreeTcUnitLog2, device_sm_count(), 2};
  // A warp's step is four tiles of 16 tokens where there are jobs for the whole grid, of few jobs two
  // (D 128, 4 rows: 32 x 8000 tokens 57.0 us with four, 61.8 with two; one sequence of 16000 16.9 and 15.1, of 500
  // 8.4 and 7.6)
  if (rows <= 8) {
    if (a.B * a.Hkv * kRowsParts >= device_sm_count() * 3) return {3, 8, device_sm_count() * 3, 1};
    return {3, 7, device_sm_count() * 4, 1};
  }
  if (a.D == 64) return {4, 7, device_sm_count() * 3, 1};
  return {4, 6, device_sm_count() * 3, 2};
}

// M and sums, then the weighted sums of values.
int64_t tree_sums_bytes(const TreePlan& t) { return align256(((int64_t)2 * t.ctas << t.rows_log2) * 8); }

template <int D>
cudaError_t launch_t(const TreeArgs& a, cudaStream_t stream) {
  const TreePlan t = tree_plan(a);
  TreeParams p{};
  p.a = a;
  p.G = (int)(a.Hq / a.Hkv);
  p.g_inv = p.G > 1 ? (uint32_t)(((1ull << 32) + p.G - 1) / p.G) : 0;
  while ((1 << p.shift) < a.page_size) ++p.shift;
  p.window = (int)a.window;
  p.sinks = (int)a.sinks;
  p.cap = (int)(a.table_width << p.shift);
  p.ctas = t.ctas;
  p.rows_log2 = t.rows_log2;
  p.unit_log2 = t.unit_log2;
  p.least = t.least;
  p.scale_log2 = a.scale * kAttnLog2e;
  p.ml = static_cast<float2*>(a.workspace);
  p.o = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + tree_sums_bytes(t));
  cudaError_t e;
  if (t.rows_log2 >= 5) {
    e = launch_tree_tc(p, stream);
  } else {
    const bool half = a.max_q * p.G <= 4;
    void (*kernel)(TreeParams) = tree_rows_kernel<D, 2, D == 64 ? 2 : 1, false>;
    int bytes = RowsRing<D, D == 64 ? 2 : 1>::BYTES;
    if (t.rows_log2 == 3 && t.unit_log2 == 8) {
      kernel = half ? tree_rows_kernel<D, 1, 4, true> : tree_rows_kernel<D, 1, 4, false>;
      bytes = RowsRing<D, 4>::BYTES;
    } else if (t.rows_log2 == 3) {
      kernel = half ? tree_rows_kernel<D, 1, 2, true> : tree_rows_kernel<D, 1, 2, false>;
      bytes = RowsRing<D, 2>::BYTES;
    }
    int per_sm = 0;
    e = prepare_launch(kernel, kRowsWarps * 32, bytes, &per_sm);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kernel, dim3((unsigned)t.ctas), dim3(kRowsWarps * 32), bytes, stream, 1, p);
  }
  if (e != cudaSuccess) return e;
  constexpr int rpb = kCombineThreads / (D / 4);   // rows of a block
  auto combine = t.rows_log2 >= 5 ? tree_combine_kernel<D, 0> : tree_combine_kernel<D, kRowsParts>;
  e = launch_pdl(combine, dim3((unsigned)(t.ctas - 1), (unsigned)(((1 << t.rows_log2) + rpb - 1) / rpb)), dim3(kCombineThreads), 0,
                 stream, 1, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

int64_t tree_attention_workspace(const TreeArgs& a) {
  const TreePlan t = tree_plan(a);
  return tree_sums_bytes(t) + ((int64_t)2 * t.ctas << t.rows_log2) * a.D * 4;
}

cudaError_t launch_tree_attention(const TreeArgs& a, cudaStream_t stream) {
  if (a.D == 128) return launch_t<128>(a, stream);
  if (a.D == 64) return launch_t<64>(a, stream);
  return cudaErrorNotSupported;
}

}  // namespace spinq
