// tree_attention_tc.cu -- the many rows of spinq_tree_attention_kv4 on the
// 5th-generation tensor core (tree_attention.cu has the mathematics and how the
// work is dealt).
//
// A job is up to 32 NE rows of a sequence and a kv head, in groups of 8 dealt to the four
// lane quarters of the MMAs' 128 lanes, so that few rows are little work for every
// warp instead of all of it for one.  Two warpgroups take 64 tokens each of a tile of 128, with
// an accumulator, maximum and sums of their own until the job's end: nothing passes
// between them before.  A lane holds 4 rows (NE 4) of a quarter of its warp's tokens, so that
// the tokens' numbers, which come from shared memory at a quarter of its rate, are loaded for
// all of them at once.
// The second fp16 parts of the weights lie on lanes without rows (NE 1: 8 .. 15 of each quarter,
// NE 2: 16 .. 31) and cost no product; with NE 4 they are columns behind the first's.
// Scores of two tiles in tensor memory (with the accumulators its 512 columns) let the
// products run ahead of the softmax.
// Warp roles: 0-7 softmax; 8 one thread that issues the MMAs; 9 and 10 copy the codes of values
// and keys, a bulk copy per 16 tokens, two tiles ahead; 11 one thread that walks the CTA's
// jobs and writes them down for the others; 12-15 expand the codes into operand tiles, a
// token per thread, keys two tiles ahead of values.
//
// 32 sequences of 9001 to 16384 tokens with 64 nodes each (32 / 8 heads, D 128, jobs of 128 rows): 545 us, 759
// TFLOP/s, where the products alone would take 217 and the codes' bytes 74.  A tile is 1536 cycles of MMAs in about
// 3000 (two fp16 parts of the weights: the values' product counts twice); the softmax and the expansion of
// the codes take 59 % of the issue slots and wait for tensor memory and shared memory in between.
// The same case with one part 505 us (error 0.00028 for 0.00021); rows split between the warpgroups 642; tokens split, one
// maximum for both 663; a thread each for the two products 661; the numbers loaded a tile ahead 580; in the tree of these
// steps each against 565.  32 rows (NE 1), 32 x 8000 tokens: 145 us.
//
// Every wait is bounded; one that gives up raises the CTA's abort flag, the MMAs and
// copies in flight are drained and the status word is set.
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

__device__ uint64_t g_tree_wait_ns = kAttnWaitLimitNs;
constexpr int kTreeSite = 33;   // wait site recorded on a time-out

// Four warpgroups: two of softmax with 184 registers a thread, one with the MMAs and
// copies (56), one that expands the codes (88): 512 = 4 * 128, what the launch holds.
constexpr int kTreeThreads = 512;
constexpr int kJobSlots = 4;
// a job's readers: two copy warps, the MMA thread, four expanding and eight softmax warps
constexpr int kJobReaders = 15;
constexpr int kTreeTcUnit = 1 << kTreeTcUnitLog2;

// A job as the roles read it.
struct TreeJobSlot {
  int more;   // 0: no further job
  int low;    // from here on (or in the sinks) the windows of all its rows reach
  TreeJob j;
};

template <int D>
struct TreeCfg {
  static constexpr int TILE = 128 * D * 2;   // bytes of a Q, K or V operand tile
  static constexpr int NSTG = 2;             // tiles of keys, and of values
  static constexpr int NS = 2;               // tiles of scores; keys are expanded as far ahead of values
  // Tiles of per-token numbers.  Tile n + 2's are written when tile n's scores are done; those
  // came behind tile n - 2's weights.
  static constexpr int NCOL = 4;
  static constexpr int NRAW = D == 128 ? 2 : 4;
  // codes and scales as copied: keys' codes of NRAW tiles, the values', the scales
  static constexpr int CODES = 128 * (D / 2), SCALES = 128 * 16;
  // a tile's numbers: 64 pairs of tokens' score scales and offsets, 64 pairs of the factors
  // of the two sums, 64 pairs of log2 alpha'
  static constexpr int COL_V = 1024, COL_LOG = 2048, COL = 2560;
  static constexpr int OFF_K = TILE, OFF_V = OFF_K + NSTG * TILE;
  static constexpr int OFF_RAW = OFF_V + NSTG * TILE;
  static constexpr int OFF_COL = OFF_RAW + NRAW * (2 * CODES + SCALES);
  static constexpr int NVIEW = 2;                                    // jobs whose queries' views are kept
  static constexpr int OFF_VIEW = OFF_COL + NCOL * COL;              // TreeRow [NVIEW][128], of a job's queries
  static constexpr int OFF_PARENT = OFF_VIEW + NVIEW * 128 * (int)sizeof(TreeRow);
  static constexpr int OFF_X = OFF_PARENT + kTreeNodes * 4;          // float [2][3][128]: the warpgroups' M, l, z; query sums
  static constexpr int OFF_JOB = OFF_X + 6 * 128 * 4;
  static constexpr int OFF_BAR = (OFF_JOB + kJobSlots * (int)sizeof(TreeJobSlot) + 7) / 8 * 8;
  // q, full, free [2][NSTG], raw, rawfree [2][NRAW], s [NS], p, o [2][NS], drain, job, taken [kJobSlots], view, viewed [NVIEW]
  static constexpr int NBAR = 1 + 4 * NSTG + 4 * NRAW + 5 * NS + 1 + 2 * kJobSlots + 2 * NVIEW;
  static constexpr int OFF_MISC = OFF_BAR + NBAR * 8;
  static constexpr int BYTES = OFF_MISC + 16 + 1024;
  static_assert(OFF_BAR % 8 == 0 && BYTES <= 232448, "shared memory");
};

// O[tmem] (+)= P V of 64 tokens: their weights on 32 columns, the second parts (`part` = 1) on the 32
// behind them, 4 K steps of 16 tokens.
template <int D>
__device__ __forceinline__ void tree_mma_pv(uint32_t o_tmem, uint32_t p_tmem, uint32_t v_lo, int part, bool accumulate) {
  constexpr uint32_t idesc = umma_idesc_f16_f32_bmn(128, D);
  const uint32_t w = p_tmem + 32 * part;
  if (accumulate)
    attn_mma_ts<true>(o_tmem, w, v_lo, idesc);
  else
    attn_mma_ts<false>(o_tmem, w, v_lo, idesc);
#pragma unroll
  for (int ks = 1; ks < 4; ++ks) attn_mma_ts<true>(o_tmem, w + ks * 8, v_lo + ks * (2048 >> 4), idesc);
}

// attn_wait for whatever `ready` asks for.
template <typename F>
__device__ __forceinline__ bool attn_wait_until(F ready, volatile int* abort_flag, uint64_t limit_ns) {
  uint64_t t0 = 0;
  while (true) {
#pragma unroll 1
    for (int k = 0; k < 512; ++k)
      if (ready()) return true;
    if (*abort_flag) return false;
    const uint64_t t = globaltimer_ns();
    if (t0 == 0) t0 = t;
    if (t - t0 > limit_ns) {
      *abort_flag = 1;
      return false;
    }
  }
}

constexpr int kSoftmaxBarrier = 1;   // named barrier of the 256 softmax threads

template <int D, int NE>
__global__ void __launch_bounds__(kTreeThreads, 1) tree_tc_kernel(const TreeParams p) {
  using C = TreeCfg<D>;
  constexpr int NSTG = C::NSTG, NCOL = C::NCOL, NRAW = C::NRAW, NS = C::NS;
  constexpr int NH = NE == 4 ? 2 : 1;   // 16-lane halves of a quarter that hold rows
  const TreeArgs& a = p.a;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* qbar = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);   // a job's queries are in (8 warps)
  uint64_t* kfull = qbar + 1;       // key tile and per-token numbers written (4 warps)
  uint64_t* vfull = kfull + NSTG;   // value tile
  uint64_t* kfree = vfull + NSTG;   // its products are done
  uint64_t* vfree = kfree + NSTG;
  uint64_t* raw = vfree + NSTG;     // a tile's key codes and scales copied; NRAW further on: its value codes
  uint64_t* rawfree = raw + 2 * NRAW;   // and read (4 warps)
  uint64_t* sbar = rawfree + 2 * NRAW;  // a tile's scores written, and its per-token numbers before
  uint64_t* pbar = sbar + NS;       // weights of warpgroup i written (4 warps), at i NS ..
  uint64_t* obar = pbar + 2 * NS;   // their products done
  uint64_t* drain = obar + 2 * NS;  // every MMA done
  uint64_t* jbar = drain + 1;       // job written
  uint64_t* taken = jbar + kJobSlots;   // and no longer read
  TreeJobSlot* job_s = reinterpret_cast<TreeJobSlot*>(smem + C::OFF_JOB);
  uint64_t* vbar = taken + kJobSlots;   // views of a job's queries written
  uint64_t* viewed = vbar + C::NVIEW;   // and no longer read (8 warps)
  int* parent_s = reinterpret_cast<int*>(smem + C::OFF_PARENT);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  int* copied = reinterpret_cast<int*>(smem + C::OFF_MISC + 8);   // tiles whose keys' and values' copies were issued
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    mbar_init(qbar, 8);
    for (int s = 0; s < 2 * NSTG; ++s) {
      mbar_init(&kfull[s], 4);
      mbar_init(&kfree[s], 1);
    }
    for (int s = 0; s < 2 * NRAW; ++s) {
      mbar_init(&raw[s], 1);
      mbar_init(&rawfree[s], 4);
    }
    for (int s = 0; s < NS; ++s) mbar_init(&sbar[s], 1);
    for (int s = 0; s < 2 * NS; ++s) {
      mbar_init(&pbar[s], 4);
      mbar_init(&obar[s], 1);
    }
    mbar_init(drain, 1);
    for (int s = 0; s < kJobSlots; ++s) {
      mbar_init(&jbar[s], 1);
      mbar_init(&taken[s], kJobReaders);
    }
    for (int s = 0; s < C::NVIEW; ++s) {
      mbar_init(&vbar[s], 1);
      mbar_init(&viewed[s], 8);
    }
    *abort_flag = 0;
    copied[0] = copied[1] = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = 0;   // all 512 columns are this CTA's: they start at column 0
  constexpr uint32_t OCOL = NS * 128;
  pdl_wait();
  pdl_trigger();
  TreeWalk walk(tree_run<kTreeThreads, 0>(p, blockIdx.x), blockIdx.x);   // (of the thread that uses it)
  const uint32_t sb = smem_u32(smem);
  // Job number `it` for a whole warp, or for the one thread that asks: its slot stays as it is until job_done.
  auto next_job = [&](int it, bool warp_wide) -> const TreeJob* {
    uint64_t* bar = &jbar[it % kJobSlots];
    const uint32_t parity = (uint32_t)(it / kJobSlots) & 1u;
    const bool there = warp_wide ? attn_wait_warp(bar, parity, abort_flag, g_tree_wait_ns)
                                 : attn_wait(bar, parity, abort_flag, g_tree_wait_ns);
    const TreeJobSlot* x = &job_s[it % kJobSlots];
    return there && x->more ? &x->j : nullptr;
  };
  auto job_done = [&](int it) { mbar_arrive(&taken[it % kJobSlots]); };
  // For the second and later users of stage n % N: the one before has left it.
  auto wait_free = [&](uint64_t* bars, int n, int N) {
    return n < N || attn_wait_warp(&bars[n % N], (uint32_t)(n / N - 1) & 1u, abort_flag, g_tree_wait_ns);
  };
  auto wait_full = [&](uint64_t* bars, int n, int N) {
    return attn_wait_warp(&bars[n % N], (uint32_t)(n / N) & 1u, abort_flag, g_tree_wait_ns);
  };

  if (warp >= 12) {
    // ---------------- one thread per token of a tile: codes to operand rows
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;\n");
    const int t = tid & 127;
    constexpr int NW = D / 32;   // 16-byte pieces of a row of codes
    // (a thread starts with another piece than its neighbours: eight rows' pieces fall in different banks)
    auto load = [&](const uint8_t* src, uint4* w) {
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const int piece = NW == 4 ? (k + (t >> 1)) & 3 : (k + (t >> 2)) & 1;
        w[k] = *reinterpret_cast<const uint4*>(src + t * (D / 2) + piece * 16);
      }
    };
    auto expand = [&](const uint4* w, uint8_t* tile, uint64_t* bar) {
      uint8_t* dst = tile + t * 128;
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const int piece = NW == 4 ? (k + (t >> 1)) & 3 : (k + (t >> 2)) & 1;
        const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int ch = 4 * piece + q;   // 16-byte chunk (8 values) of the row
          *reinterpret_cast<uint4*>(dst + (ch >> 3) * kAttnAtom + (((ch & 7) ^ (t & 7)) << 4)) = code_pairs1(x[q]);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    // Keys are expanded two tiles ahead of values: those wait for products behind a
    // softmax, and the next scores would wait with them.  A step is the keys of tile n and the
    // values of tile n - 2, all it waits for asked for at once: an answer takes some 200
    // cycles, and four in a row were 800 of a step's 2100 for a few rows.
    auto value_tile = [&](int m) {
      uint4 w[NW];
      load(smem + C::OFF_RAW + (NRAW + m % NRAW) * C::CODES, w);
      __syncwarp();
      if (lane == 0) mbar_arrive(&rawfree[NRAW + m % NRAW]);
      expand(w, smem + C::OFF_V + (m % NSTG) * C::TILE, &vfull[m % NSTG]);
    };
    // phases complete: a tile's codes there, its stage free (from the third tile on)
    auto there = [&](uint64_t* bars, int m, int N) { return attn_test(&bars[m % N], (uint32_t)(m / N) & 1u); };
    auto left = [&](uint64_t* bars, int m, int N) { return m < N || attn_test(&bars[m % N], (uint32_t)(m / N - 1) & 1u); };
    int n = 0;   // tiles so far
    bool ok = true;
    for (int it = 0; ok; ++it) {
      const TreeJob* job = next_job(it, true);
      if (!job) break;
      const int v1 = job->v1, tokens = job->s.n, front = job->s.front, skip = job->s.skip;
      int v = job->v0;
      __syncwarp();
      if (lane == 0) job_done(it);
      for (; v < v1; ++v, ++n) {
        const int m = n - 2;
        ok = attn_wait_until(
            [&]() {
              const bool a0 = there(raw, n, NRAW), a1 = left(kfree, n, NSTG);
              const bool a2 = m < 0 || there(raw + NRAW, m, NRAW), a3 = m < 0 || left(vfree, m, NSTG);
              return a0 & a1 & a2 & a3;
            },
            abort_flag, g_tree_wait_ns);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        uint4 w[NW];
        load(smem + C::OFF_RAW + (n % NRAW) * C::CODES, w);
        const float4 sc =
            *reinterpret_cast<const float4*>(smem + C::OFF_RAW + 2 * NRAW * C::CODES + (n % NRAW) * C::SCALES + t * 16);
        __syncwarp();
        if (lane == 0) mbar_arrive(&rawfree[n % NRAW]);
        const bool in = (v < front ? v : v + skip) * kTreeTcUnit + t < tokens;
        uint8_t* cols = smem + C::OFF_COL + (n % NCOL) * C::COL;
        float* col = reinterpret_cast<float*>(cols) + (t >> 1) * 4 + (t & 1);
        col[0] = in ? p.scale_log2 * sc.x : 0.f;
        col[2] = in ? p.scale_log2 * fmaf(8.f, sc.x, sc.y) : 0.f;
        const float va = in ? value_scale(sc.z) : 1.f, rv = one_over_scale(va), vz = in ? fmaf(rv, sc.w, 8.f) : 0.f;
        // Factors that are not finite would give rows that do not see the token 0 times them:
        // they are 0 here, and the score of a row that does see it is not a number.
        const bool bad = !(fabsf(rv) <= FLT_MAX && fabsf(vz) <= FLT_MAX);
        col[C::COL_V / 4] = bad ? 0.f : rv;
        col[C::COL_V / 4 + 2] = bad ? 0.f : vz;
        // (in the order of the lanes: pairs c of groups 2 k and 2 k + 1 of eight tokens in one load)
        const int to = (t & 64) + (t >> 4 & 3) * 16 + (t >> 1 & 3) * 4 + (t >> 3 & 1) * 2 + (t & 1);
        reinterpret_cast<float*>(cols + C::COL_LOG)[to] = bad ? __int_as_float(0x7fc00000) : log2_of_scale(va);
        expand(w, smem + C::OFF_K + (n % NSTG) * C::TILE, &kfull[n % NSTG]);
        if (m >= 0) value_tile(m);
      }
    }
    if (ok)
      for (int m = max(0, n - 2); m < n; ++m) {
        if (!wait_full(raw + NRAW, m, NRAW) || !wait_free(vfree, m, NSTG)) break;
        value_tile(m);
      }
  } else if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;\n");
    if (warp == 8) {
      // ---------------- MMAs
      if (attn_elect()) {
        constexpr uint32_t idesc = umma_idesc_f16_f32(128, 128, false);
        const uint32_t q_lo = attn_desc_k(sb), k_lo = attn_desc_k(sb + C::OFF_K), v_lo = attn_desc_mn(sb + C::OFF_V);
        int n = 0;   // tiles so far
        bool ok = true;
        auto wait = [&](uint64_t* bars, int m, int N) {
          return ok = ok && attn_wait(&bars[m % N], (uint32_t)(m / N) & 1u, abort_flag, g_tree_wait_ns);
        };
        auto scores = [&](int m) {   // (its columns' weights were taken by products issued before)
          tc_fence_after();
          attn_mma_qk<D>((m % NS) * 128, q_lo, k_lo + (m % NSTG) * (C::TILE >> 4), idesc);
          tc_commit(&sbar[m % NS]);
          tc_commit(&kfree[m % NSTG]);
        };
        for (int it = 0; ok; ++it) {
          const TreeJob* job = next_job(it, false);
          if (!job) break;
          const int end = n + job->v1 - job->v0, first = n;
          job_done(it);
          if (!wait(qbar, it, 1)) break;
          for (int m = n; m < min(end, n + NS) && wait(kfull, m, NSTG); ++m) scores(m);
#pragma unroll 1
          for (; ok && n < end; ++n) {
            // (values and the first weights asked for at once; the keys two tiles on were written before the values)
            if (!(ok = attn_wait_until(
                      [&]() {
                        const bool a0 = attn_test(&vfull[n % NSTG], (uint32_t)(n / NSTG) & 1u);
                        const bool a1 = attn_test(&pbar[n % NS], (uint32_t)(n / NS) & 1u);
                        return a0 & a1;
                      },
                      abort_flag, g_tree_wait_ns)))
              break;
            const uint32_t vd = v_lo + (n % NSTG) * (C::TILE >> 4), pt = (n % NS) * 128;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              if (i && !wait(pbar + NS, n, NS)) break;
              tc_fence_after();
              tree_mma_pv<D>(OCOL + i * D, pt + 64 * i, vd + 4 * i * (2048 >> 4), 0, n > first);
              if (NE == 4) tree_mma_pv<D>(OCOL + i * D, pt + 64 * i, vd + 4 * i * (2048 >> 4), 1, true);
              tc_commit(&obar[i * NS + n % NS]);
            }
            if (!ok) break;
            tc_commit(&vfree[n % NSTG]);
            if (n + NS < end) scores(n + NS);
          }
        }
        tc_commit(drain);   // what is in flight finishes before tensor memory is given up
        mbar_wait_bounded(drain, 0, kAttnWaitLimitNs);
      }
    } else if (warp < 11) {
      // ---------------- copies of values (warp 9) or keys: lanes 0 .. 7 the tile's runs of 16 tokens
      const bool keys = warp == 10;
      uint64_t *there = keys ? raw : raw + NRAW, *left = keys ? rawfree : rawfree + NRAW;
      uint8_t* dst = smem + C::OFF_RAW + (keys ? 0 : NRAW * C::CODES);
      const uint8_t* codes = keys ? a.k_codes : a.v_codes;
      int n = 0;
      bool ok = !p.debug_stall;
      for (int it = 0; ok; ++it) {
        const TreeJob* job = next_job(it, true);
        if (!job) break;
        const int v0 = job->v0, v1 = job->v1, front = job->s.front, skip = job->s.skip, tokens = job->s.n, hk = job->hk;
        const int32_t* table = a.table + (int64_t)job->b * a.table_width;
        __syncwarp();
        if (lane == 0) job_done(it);
        int64_t place = 0;
        for (int v = v0; v < v1; ++v, ++n) {
          // lane 8 w + k looks run k of the tile w further on up: one look-up for four tiles
          if (((v - v0) & 3) == 0) {
            const int vt = v + (lane >> 3);
            const int tok = vt < v1 ? (vt < front ? vt : vt + skip) * kTreeTcUnit + 16 * (lane & 7) : tokens;
            place = tok < tokens ? (tree_page(a, table, tok, p.shift) * a.Hkv + hk) * a.page_size + (tok & (a.page_size - 1)) : -1;
          }
          const int64_t at = __shfl_sync(0xffffffffu, place, 8 * ((v - v0) & 3) + (lane & 7));
          const int runs = __popc(__ballot_sync(0xffffffffu, lane < 8 && at >= 0));
          const int st = n % NRAW;
          if (!(ok = wait_free(left, n, NRAW))) break;
          if (lane == 0) {
            mbar_arrive_expect_tx(&there[st], (uint32_t)runs * (8 * D + (keys ? 256 : 0)));
            copied[keys ? 0 : 1] = n + 1;
          }
          __syncwarp();
          if (lane < 8 && at >= 0) {
            bulk_load(dst + st * C::CODES + lane * 8 * D, codes + at * (D / 2), 8 * D, &there[st]);
            if (keys)
              bulk_load(dst + 2 * NRAW * C::CODES + st * C::SCALES + lane * 256, a.scales + at * 4, 256, &there[st]);
          }
        }
      }
    } else {
      // ---------------- jobs: written down by lane 0; then what their queries see, a query per lane
      bool more = true;
      for (int it = 0; more; ++it) {
        TreeJob j = {};
        more = walk.next(p, j);   // (every lane walks)
        if (!wait_free(taken, it, kJobSlots)) break;
        TreeJobSlot* x = &job_s[it % kJobSlots];
        // the window of the deepest query that there can be
        const int deepest = j.s.ctx + min(j.s.nq - 1, tree_node(p, max(0, j.r0 + j.rows - 1)));
        if (lane == 0) {
          x->more = more;
          x->low = p.window > 0 && deepest >= p.window ? deepest - p.window + 1 : 0;
          x->j = j;
          mbar_arrive(&jbar[it % kJobSlots]);
        }
        if (!more) break;
        for (int i = lane; i < j.s.nq; i += 32) parent_s[i] = a.parents ? __ldg(a.parents + j.s.q0 + i) : i - 1;
        if (!wait_free(viewed, it, C::NVIEW)) break;
        __syncwarp();
        const int first = tree_node(p, j.r0), last = tree_node(p, j.r0 + j.rows - 1);
        TreeRow* view = reinterpret_cast<TreeRow*>(smem + C::OFF_VIEW) + (it % C::NVIEW) * 128;
        for (int i = first + lane; i <= last; i += 32) view[i - first] = tree_row(p, j.s, parent_s, i);
        __syncwarp();
        if (lane == 0) mbar_arrive(&vbar[it % C::NVIEW]);
      }
    }
  } else {
    // ---------------- softmax.  Warpgroup i has tokens 64 i .. of a tile; lane 4 g + c holds rows
    // g + 8 e of its quarter and tokens 8 k + 2 c, + 1.
    asm volatile("setmaxnreg.inc.sync.aligned.u32 184;\n");
    const int i = warp >> 2, quad = warp & 3, g = lane >> 2, c = lane & 3;
    const uint32_t quarter = (uint32_t)(quad * 32) << 16, ot = tmem + OCOL + i * D + quarter;
    float* xs = reinterpret_cast<float*>(smem + C::OFF_X);
    // the job's row on lane l of quarter q, or -1
    auto row_of = [&](int q, int l) { return l < 8 * NE ? (l >> 3) * 32 + q * 8 + (l & 7) : -1; };
    // OR of a predicate over the softmax threads, a barrier for them.
    auto named_or = [&](bool x) {
      uint32_t r;
      asm volatile(
          "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, 256, p;\n selp.u32 %0, 1, 0, q;\n}\n"
          : "=r"(r)
          : "r"((uint32_t)x), "n"(kSoftmaxBarrier)
          : "memory");
      return r != 0;
    };
    int n = 0;   // tiles so far
    bool ok = true;
    for (int it = 0; ok; ++it) {
      const TreeJob* job = next_job(it, true);
      // (a warp that gave the wait up still meets the others at the barriers: all of them leave there)
      if (named_or(!job && *abort_flag)) break;
      if (!job) break;
      const TreeJob& j = *job;
      const TreeSeq& s = j.s;
      // (every thread is here past the last job's end: its sums and queries are free)
      // The queries, their pairs in the order of code_pairs, and their sums: D / 8 lanes share a
      // row, warp w has MMA lanes 16 w .. 16 w + 15.
      {
        constexpr int LPR = D / 8, RPL = 32 / LPR;   // lanes per row, rows per load
        const int ch = lane % LPR;
        uint4 w[16 / RPL];
#pragma unroll
        for (int k = 0; k < 16 / RPL; ++k) {
          const int m = 16 * warp + k * RPL + lane / LPR, r = row_of(m >> 5, m & 31);
          w[k] = r >= 0 && r < j.rows
                     ? __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __half*>(a.q) + j.row_at(p, r) * D) + ch)
                     : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < 16 / RPL; ++k) {
          const int m = 16 * warp + k * RPL + lane / LPR;
          const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
          float sum = 0.f;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[q]));
            sum += f.x + f.y;
          }
#pragma unroll
          for (int o = 1; o < LPR; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          if (ch == 0) xs[m] = sum;
          *reinterpret_cast<uint4*>(smem + (ch >> 3) * kAttnAtom + m * 128 + (((ch & 7) ^ (m & 7)) << 4)) =
              make_uint4(__byte_perm(x[0], x[2], 0x5410), __byte_perm(x[0], x[2], 0x7632), __byte_perm(x[1], x[3], 0x5410),
                         __byte_perm(x[1], x[3], 0x7632));
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(qbar);
      }
      named_bar_sync(kSoftmaxBarrier, 256);   // the sums are written
      float qs[NE];
#pragma unroll
      for (int e = 0; e < NE; ++e) qs[e] = xs[quad * 32 + 8 * e + g];
      named_bar_sync(kSoftmaxBarrier, 256);   // and read
      const int ctx = s.ctx, low = job_s[it % kJobSlots].low;
      // the view of this lane's row, where there is one
      const int my_row = row_of(quad, lane);
      const TreeRow* view = reinterpret_cast<const TreeRow*>(smem + C::OFF_VIEW) + (it % C::NVIEW) * 128 +
                            (my_row >= 0 && my_row < j.rows ? tree_node(p, j.r0 + my_row) - tree_node(p, j.r0) : 0);
      bool viewing = false;

      float m[NE], l[NE], z[NE];   // M; l, z: of this lane's tokens
#pragma unroll
      for (int e = 0; e < NE; ++e) m[e] = -INFINITY, l[e] = z[e] = 0.f;
      const int end = n + j.v1 - j.v0, start = n, v0 = j.v0, front = s.front, skip = s.skip;
#pragma unroll 1
      for (; n < end; ++n) {
        const int v = v0 + n - start, at = (v < front ? v : v + skip) * kTreeTcUnit + 64 * i;
        const uint32_t st = tmem + (n % NS) * 128 + quarter + 64 * i;
        if (!(ok = wait_full(sbar, n, NS))) break;
        tc_fence_after();
        // the numbers of tokens 8 k + 2 c, 8 k + 2 c + 1
        const uint8_t* cols = smem + C::OFF_COL + (n % NCOL) * C::COL;
        const ulonglong2* ab = reinterpret_cast<const ulonglong2*>(cols + i * 512) + c;
        const ulonglong2* fv = reinterpret_cast<const ulonglong2*>(cols + C::COL_V + i * 512) + c;
        const ulonglong2* la = reinterpret_cast<const ulonglong2*>(cols + C::COL_LOG + i * 256) + c;
        uint32_t x[NH][32];   // x[h][4 k + 2 e + y]: row 16 h + 8 e + g, token 8 k + 2 c + y
#pragma unroll
        for (int h = 0; h < NH; ++h) tmem_ld_16x256b_x8(st + ((16u * h) << 16), x[h]);
#pragma unroll
        for (int h = 0; h < NH; ++h) tmem_ld_wait_all<32>(x[h]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const ulonglong2 w = ab[4 * k], l2 = la[4 * (k >> 1)];
          const F2 lg = F2{k & 1 ? l2.y : l2.x};
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            uint32_t* y = &x[e >> 1][4 * k + 2 * (e & 1)];
            float t0, t1;
            f2_split(f2_fma(f2_from_bits(y[0], y[1]), F2{w.x}, f2_fma(F2{w.y}, f2_make(qs[e], qs[e]), lg)), t0, t1);
            y[0] = __float_as_uint(t0);
            y[1] = __float_as_uint(t1);
          }
        }
        if (at + 64 > ctx || (at < low && at + 64 > p.sinks)) {
          // not every row sees every token: lane r has a bit per token for its row
          if (!viewing && !(ok = wait_full(vbar, it, C::NVIEW))) break;
          viewing = true;
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t seen = tree_sees(p, s, *view, at + 32 * w);
#pragma unroll
            for (int e = 0; e < NE; ++e) {
              const uint32_t bits = __shfl_sync(0xffffffffu, seen, 8 * e + g) >> (2 * c);
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                  if (!((bits >> (8 * k + y)) & 1u)) x[e >> 1][4 * (4 * w + k) + 2 * (e & 1) + y] = 0xFF800000u;   // -inf
            }
          }
        }
        float mx[NE];
        bool grow = false;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const uint32_t* y = &x[e >> 1][2 * (e & 1)];
          float p0 = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])), p1 = fmaxf(__uint_as_float(y[4]), __uint_as_float(y[5]));
#pragma unroll
          for (int k = 2; k < 8; k += 2) {
            p0 = attn_max3(p0, __uint_as_float(y[4 * k]), __uint_as_float(y[4 * k + 1]));
            p1 = attn_max3(p1, __uint_as_float(y[4 * k + 4]), __uint_as_float(y[4 * k + 5]));
          }
          mx[e] = fmaxf(p0, p1);
          grow |= mx[e] > m[e] + kAttnSlack;
        }
        if (__any_sync(0xffffffffu, grow)) {   // seldom: M moves
          float f[4];
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 1));
            mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
            const float mn = mx[e] > m[e] + kAttnSlack ? mx[e] : m[e];
            // (a row without a maximum has no weights, or sums that are not numbers and stay so)
            f[e] = m[e] == -INFINITY || mn == m[e] ? 1.f : attn_exp2(m[e] - mn);
            m[e] = mn;
            l[e] *= f[e];
            z[e] *= f[e];
          }
          if constexpr (NE == 1) f[1] = f[0];   // the second parts' rows
          if constexpr (NE == 2) f[2] = f[0], f[3] = f[1];
          if (n > start) {
            if (!(ok = wait_full(obar + i * NS, n - 1, NS))) break;   // the products so far are done
            tc_fence_after();
#pragma unroll 1
            for (int d = 0; d < D; d += 16) {
#pragma unroll
              for (int h = 0; h < (NE == 1 ? 1 : 2); ++h) {
                uint32_t y[8];
                tmem_ld_16x256b_x2(ot + ((16u * h) << 16) + d, y);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * f[2 * h + ((k >> 1) & 1)]);
                tmem_st_16x256b_x2(ot + ((16u * h) << 16) + d, y);
              }
            }
          }
        }
        uint32_t w0[NH][16], w1[NH][16];   // first and second parts: 32-bit columns 4 k + c
        F2 of2[NE], sum[NE], zs[NE];
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const float off = m[e] == -INFINITY ? 0.f : -m[e];
          of2[e] = f2_make(off, off);
          sum[e] = f2_make(l[e], 0.f);
          zs[e] = f2_make(z[e], 0.f);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const ulonglong2 f = fv[4 * k];
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const uint32_t* y = &x[e >> 1][4 * k + 2 * (e & 1)];
            float t0, t1;
            f2_split(f2_add(f2_from_bits(y[0], y[1]), of2[e]), t0, t1);
            const F2 ex = f2_make(attn_exp2(t0), attn_exp2(t1));
            sum[e] = f2_fma(ex, F2{f.x}, sum[e]);
            zs[e] = f2_fma(ex, F2{f.y}, zs[e]);
            f2_split(ex, t0, t1);
            const uint32_t hi = pack_half2_bits(t0, t1);
            const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&hi));
            f2_split(f2_sub(ex, f2_make(r.x, r.y)), t0, t1);
            const uint32_t lo = pack_half2_bits(t0, t1);
            w0[e >> 1][2 * k + (e & 1)] = hi;
            if (NE == 1)
              w0[0][2 * k + 1] = lo;
            else
              w1[e >> 1][2 * k + (e & 1)] = lo;
          }
        }
#pragma unroll
        for (int h = 0; h < NH; ++h) {
          tmem_st_16x128b_x8(st + ((16u * h) << 16), w0[h]);
          if (NE == 2) tmem_st_16x128b_x8(st + (16u << 16), w1[h]);
          if (NE == 4) tmem_st_16x128b_x8(st + ((16u * h) << 16) + 32, w1[h]);
        }
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          float t0, t1;
          f2_split(sum[e], t0, t1);
          l[e] = t0 + t1;
          f2_split(zs[e], t0, t1);
          z[e] = t0 + t1;
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pbar[i * NS + n % NS]);
      }
      if (ok) ok = wait_full(obar + i * NS, end - 1, NS);
      // the rows' numbers, and whether a wait was given up
#pragma unroll
      for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int w = 1; w < 4; w <<= 1) {
          l[e] += __shfl_xor_sync(0xffffffffu, l[e], w);
          z[e] += __shfl_xor_sync(0xffffffffu, z[e], w);
        }
      if (c == 0) {
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          float* y = xs + 384 * i + quad * 32 + 8 * e + g;
          y[0] = m[e], y[128] = l[e], y[256] = z[e];
        }
      }
      ok = !named_or(!ok);
      if (!ok) break;
      tc_fence_after();
      // a row per lane, half of D per warpgroup
      {
        const int r = row_of(quad, lane);
        const bool mine = r >= 0 && r < j.rows;
        const float* y = xs + quad * 32 + lane;
        const float l0 = mine ? y[128] : 0.f, l1 = mine ? y[384 + 128] : 0.f;
        const float m0 = l0 != 0.f ? y[0] : -INFINITY, m1 = l1 != 0.f ? y[384] : -INFINITY, M = fmaxf(m0, m1);
        const float f0 = l0 != 0.f ? attn_exp2(m0 - M) : 0.f, f1 = l1 != 0.f ? attn_exp2(m1 - M) : 0.f;
        const float ls = fmaf(f1, l1, f0 * l0), zz = fmaf(f1, mine ? y[384 + 256] : 0.f, f0 * (mine ? y[256] : 0.f));
        const bool whole = j.whole();
        const float inv = whole ? (ls != 0.f ? 1.f / ls : 0.f) : 1.f;
        const int64_t slot = j.slot(blockIdx.x) * (32 * NE) + r;
        const int64_t at = mine ? j.row_at(p, r) : 0;
        if (mine && !whole && i == 0) p.ml[slot] = make_float2(M, ls);
#pragma unroll 1
        for (int q = 0; q < D / 2; q += 16) {
          const int d0 = i * (D / 2) + q;
          uint32_t o0[16], o1[16];
          tmem_ld_32x32b_x16(tmem + OCOL + quarter + d0, o0);
          tmem_ld_32x32b_x16(tmem + OCOL + D + quarter + d0, o1);
          tmem_ld_wait(o0);
          tmem_ld_wait(o1);
          float o[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float u = __uint_as_float(o0[k]), w = __uint_as_float(o1[k]);
            if (NE < 4) {   // and what the second parts gave
              u += __shfl_down_sync(0xffffffffu, u, NE == 1 ? 8 : 16);
              w += __shfl_down_sync(0xffffffffu, w, NE == 1 ? 8 : 16);
            }
            o[k] = fmaf(f1, w, fmaf(f0, u, zz)) * inv;
          }
          if (mine) {   // column 0, 1, .. of eight holds value 0, 4, 1, 5, 2, 6, 3, 7
#pragma unroll
            for (int k = 0; k < 16; k += 8) {
              if (whole) {
                *reinterpret_cast<uint4*>(reinterpret_cast<__half*>(a.out) + at * D + d0 + k) =
                    make_uint4(pack_half2_bits(o[k], o[k + 2]), pack_half2_bits(o[k + 4], o[k + 6]),
                               pack_half2_bits(o[k + 1], o[k + 3]), pack_half2_bits(o[k + 5], o[k + 7]));
              } else {
                float4* dst = reinterpret_cast<float4*>(p.o + slot * D + d0 + k);
                dst[0] = make_float4(o[k], o[k + 2], o[k + 4], o[k + 6]);
                dst[1] = make_float4(o[k + 1], o[k + 3], o[k + 5], o[k + 7]);
              }
            }
          }
        }
        tc_fence_before();
      }
      __syncwarp();
      if (lane == 0) {
        job_done(it);
        mbar_arrive(&viewed[it % C::NVIEW]);
      }
      named_bar_sync(kSoftmaxBarrier, 256);   // the rows' numbers have been read
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // the copies in flight land before the memory is given up
    if (tid == 0) {
      for (int k = 0; k < 2; ++k)
        for (int n = max(0, copied[k] - NRAW); n < copied[k]; ++n)
          mbar_wait_bounded(&raw[k * NRAW + n % NRAW], (uint32_t)(n / NRAW) & 1u, kAttnWaitLimitNs);
      if (p.status && atomicCAS(p.status, 0, (int)SPINQ_ETIMEOUT) == 0) atomicExch(p.status + 1, kTreeSite);
    }
    __syncthreads();
  }
  tc_fence_after();
  if (warp == 8) tmem_dealloc(*tmem_slot, 512);
}

template <int D, int NE>
cudaError_t launch_t(const TreeParams& p, cudaStream_t stream) {
  int per_sm = 0;
  cudaError_t e = prepare_launch_tmem(tree_tc_kernel<D, NE>, kTreeThreads, TreeCfg<D>::BYTES, 512, &per_sm);
  if (e != cudaSuccess) return e;
  return launch_pdl(tree_tc_kernel<D, NE>, dim3((unsigned)p.ctas), dim3(kTreeThreads), TreeCfg<D>::BYTES, stream, 1, p);
}

template <int D>
cudaError_t launch_d(const TreeParams& p, cudaStream_t stream) {
  return p.rows_log2 == 5 ? launch_t<D, 1>(p, stream) : (p.rows_log2 == 6 ? launch_t<D, 2>(p, stream) : launch_t<D, 4>(p, stream));
}

}  // namespace

cudaError_t set_wait_limit_tree(uint64_t ns) { return cudaMemcpyToSymbol(g_tree_wait_ns, &ns, sizeof(ns)); }

cudaError_t launch_tree_tc(const TreeParams& params, cudaStream_t stream) {
  TreeParams p = params;
  p.status = device_status_word();
  p.debug_stall = take_debug_stall() ? 1 : 0;
  return p.a.D == 128 ? launch_d<128>(p, stream) : launch_d<64>(p, stream);
}

}  // namespace spinq
