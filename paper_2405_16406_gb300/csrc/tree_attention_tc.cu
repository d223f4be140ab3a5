// tree_attention_tc.cu -- the many rows of spinq_tree_attention_kv4 on the
// 5th-generation tensor core (tree_attention.cu has the mathematics and how the
// work is dealt).
//
// A job is up to 32 NE rows of a sequence and a kv head, in 8-row groups over the four
// warps of a warpgroup: row 8 i + g lies on lane 32 (i % 4) + 8 (i / 4) + g of the
// MMAs' 128, so that few rows are little work for every warp instead of all of it for
// one.  Two warpgroups take a job's tiles of 128 tokens in turn, each with its
// own scores, weights, output accumulator, maximum and sums, and join at the job's
// end: nothing passes between them per tile, and the tensor core works on one's
// products under the other's softmax.
// The second fp16 parts of the weights lie on lanes that have no rows (NE 1: 8 .. 15 of
// each warp, NE 2: 16 .. 31) and cost no product of their own; with NE 4 they lie in
// the columns behind the first's.
// Warp roles: 0-3 and 4-7 softmax (the even and the odd tiles); 8 and 9 one thread each
// that issues the MMAs of the even and the odd tiles; 10 copies the codes, one
// bulk copy per 16 tokens, two tiles ahead; 11 one thread that walks the CTA's jobs and
// writes them down for the others; 12-15 expand the codes into operand tiles, a token per thread.
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
// a job's readers: copy warp, two MMA threads, four expanding and eight softmax warps
constexpr int kJobReaders = 15;
constexpr int kTreeTcUnit = 1 << kTreeTcUnitLog2;

// A job as the roles read it.
struct TreeJobSlot {
  int more;   // 0: no further job
  TreeJob j;
};

template <int D>
struct TreeCfg {
  static constexpr int TILE = 128 * D * 2;   // bytes of a Q, K or V operand tile
  static constexpr int NSTG = 4;             // operand tiles: K and V of two tiles of tokens
  static constexpr int NCOL = 4;             // tiles of per-token numbers
  static constexpr int NRAW = D == 128 ? 2 : 4;
  static constexpr int RAW_V = 128 * (D / 2), RAW_S = 2 * RAW_V, RAW = RAW_S + 128 * 16;   // codes and scales as copied
  // a tile's numbers: 64 pairs of tokens' score scales and offsets, 64 pairs of the factors
  // of the two sums, 64 pairs of log2 alpha'
  static constexpr int COL_V = 1024, COL_LOG = 2048, COL = 2560;
  static constexpr int OFF_KV = TILE;
  static constexpr int OFF_RAW = OFF_KV + NSTG * TILE;
  static constexpr int OFF_COL = OFF_RAW + NRAW * RAW;
  static constexpr int OFF_ROW = OFF_COL + NCOL * COL;               // TreeRow [128]
  static constexpr int OFF_PARENT = OFF_ROW + 128 * (int)sizeof(TreeRow);
  static constexpr int OFF_X = OFF_PARENT + kTreeNodes * 4;          // float [2][3][128]: the warpgroups' M, l, z; query sums
  // q, full, free [NSTG], col [NCOL], raw, rawfree [NRAW], s, p, o, drain [2], job, taken [kJobSlots]
  static constexpr int OFF_JOB = OFF_X + 2 * 3 * 128 * 4;
  static constexpr int OFF_BAR = (OFF_JOB + kJobSlots * (int)sizeof(TreeJobSlot) + 7) / 8 * 8;
  static constexpr int NBAR = 1 + 2 * NSTG + NCOL + 2 * NRAW + 8 + 2 * kJobSlots;
  static constexpr int OFF_MISC = OFF_BAR + NBAR * 8;
  static constexpr int BYTES = OFF_MISC + 16 + 1024;
  static_assert(OFF_BAR % 8 == 0 && BYTES <= 232448, "shared memory");
};

// 16 lanes x 4 groups of 8 columns from tensor memory, and x 4 groups of 4 columns to it
// (as the forms for 8 groups in attn_tc.cuh).
__device__ __forceinline__ void tmem_ld_16x256b_x4(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st_16x128b_x4(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// O[tmem] (+)= P V: 32 tokens' weights on 16 columns, their second parts (`part` = 1) on the
// 16 behind them, 8 K steps of 16 tokens.
template <int D>
__device__ __forceinline__ void tree_mma_pv(uint32_t o_tmem, uint32_t p_tmem, uint32_t v_lo, int part, bool accumulate) {
  constexpr uint32_t idesc = umma_idesc_f16_f32_bmn(128, D);
  const uint32_t w = p_tmem + 16 * part;
  if (accumulate)
    attn_mma_ts<true>(o_tmem, w, v_lo, idesc);
  else
    attn_mma_ts<false>(o_tmem, w, v_lo, idesc);
#pragma unroll
  for (int ks = 1; ks < 8; ++ks)
    attn_mma_ts<true>(o_tmem, w + (ks >> 1) * 32 + (ks & 1) * 8, v_lo + ks * (2048 >> 4), idesc);
}

constexpr int kSoftmaxBarrier = 1;   // named barrier of the 256 softmax threads

template <int D, int NE>
__global__ void __launch_bounds__(kTreeThreads, 1) tree_tc_kernel(const TreeParams p) {
  using C = TreeCfg<D>;
  constexpr int NSTG = C::NSTG, NCOL = C::NCOL, NRAW = C::NRAW, NH = NE == 4 ? 2 : 1;
  const TreeArgs& a = p.a;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* qbar = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);   // a job's queries are in (8 warps)
  uint64_t* full = qbar + 1;        // operand tile written (4 warps)
  uint64_t* free_ = full + NSTG;    // its products are done
  uint64_t* cbar = free_ + NSTG;    // per-token numbers of a tile written (4 warps)
  uint64_t* raw = cbar + NCOL;      // codes of a tile copied
  uint64_t* rawfree = raw + NRAW;   // and read (4 warps)
  uint64_t* sbar = rawfree + NRAW;  // scores of warpgroup i written
  uint64_t* pbar = sbar + 2;        // its weights written (4 warps)
  uint64_t* obar = pbar + 2;        // its products of a job done
  uint64_t* drain = obar + 2;       // every MMA of thread i done
  uint64_t* jbar = drain + 2;       // job written
  uint64_t* taken = jbar + kJobSlots;   // and no longer read
  TreeJobSlot* job_s = reinterpret_cast<TreeJobSlot*>(smem + C::OFF_JOB);
  TreeRow* row_s = reinterpret_cast<TreeRow*>(smem + C::OFF_ROW);
  int* parent_s = reinterpret_cast<int*>(smem + C::OFF_PARENT);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  int* copied = reinterpret_cast<int*>(smem + C::OFF_MISC + 8);   // tiles whose copies were issued
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    mbar_init(qbar, 8);
    for (int s = 0; s < NSTG; ++s) {
      mbar_init(&full[s], 4);
      mbar_init(&free_[s], 1);
    }
    for (int s = 0; s < NCOL; ++s) mbar_init(&cbar[s], 4);
    for (int s = 0; s < NRAW; ++s) {
      mbar_init(&raw[s], 1);
      mbar_init(&rawfree[s], 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sbar[i], 1);
      mbar_init(&pbar[i], 4);
      mbar_init(&obar[i], 1);
      mbar_init(&drain[i], 1);
    }
    for (int s = 0; s < kJobSlots; ++s) {
      mbar_init(&jbar[s], 1);
      mbar_init(&taken[s], kJobReaders);
    }
    *abort_flag = 0;
    *copied = 0;
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
  pdl_wait();
  pdl_trigger();
  TreeWalk walk(tree_run<kTreeThreads>(p, blockIdx.x), blockIdx.x);   // (of the thread that uses it)
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
    auto expand = [&](const uint4* w, int n) {   // into operand tile n of the ring
      uint8_t* dst = smem + C::OFF_KV + (n % NSTG) * C::TILE + t * 128;
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const int piece = NW == 4 ? (k + (t >> 1)) & 3 : (k + (t >> 2)) & 1;
        const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int ch = 4 * piece + q;   // 16-byte chunk (8 values) of the row
          *reinterpret_cast<uint4*>(dst + (ch >> 3) * kAttnAtom + (((ch & 7) ^ (t & 7)) << 4)) = code_pairs(x[q]);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[n % NSTG]);
    };
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
        if (!(ok = attn_wait_warp(&raw[n % NRAW], (uint32_t)(n / NRAW) & 1u, abort_flag, g_tree_wait_ns))) break;
        const uint8_t* src = smem + C::OFF_RAW + (n % NRAW) * C::RAW;
        uint4 kw[NW], vw[NW];
        load(src, kw);
        load(src + C::RAW_V, vw);
        const float4 sc = *reinterpret_cast<const float4*>(src + C::RAW_S + t * 16);
        __syncwarp();
        if (lane == 0) mbar_arrive(&rawfree[n % NRAW]);
        const int o = 2 * n;
        if (o >= NSTG && !(ok = attn_wait_warp(&free_[o % NSTG], (uint32_t)(o / NSTG - 1) & 1u, abort_flag, g_tree_wait_ns)))
          break;
        // The tile's numbers: slot n % NCOL was last read for tile n - 4.  Tile n - 2's scores are
        // done (its K tile is free); they were issued behind tile n - 4's products, by the same
        // thread, or, where a job ended between, behind all softmax work on it.
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
        __syncwarp();
        if (lane == 0) mbar_arrive(&cbar[n % NCOL]);
        expand(kw, o);
        if (o + 1 >= NSTG &&
            !(ok = attn_wait_warp(&free_[(o + 1) % NSTG], (uint32_t)((o + 1) / NSTG - 1) & 1u, abort_flag, g_tree_wait_ns)))
          break;
        expand(vw, o + 1);
      }
    }
  } else if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;\n");
    const int i = warp - 8;
    if (i < 2) {
      // ---------------- MMAs of the even or the odd tiles of a job
      if (attn_elect()) {
        constexpr uint32_t idesc = umma_idesc_f16_f32(128, 128, false);
        const uint32_t q_lo = attn_desc_k(sb), k_lo = attn_desc_k(sb + C::OFF_KV), v_lo = attn_desc_mn(sb + C::OFF_KV);
        int n0 = 0, nq = 0, np = 0;   // tiles before this job, jobs, weight tiles so far
        bool ok = true;
        auto wait_tile = [&](int o) {   // operand tile o
          ok = attn_wait(&full[o % NSTG], (uint32_t)(o / NSTG) & 1u, abort_flag, g_tree_wait_ns);
        };
        for (; ok; ++nq) {
          const TreeJob* job = next_job(nq, false);
          if (!job) break;
          const int nt = job->v1 - job->v0;
          job_done(nq);
          if (!(ok = attn_wait(qbar, (uint32_t)nq & 1u, abort_flag, g_tree_wait_ns))) break;
          if (i < nt) {
            const int o0 = 2 * (n0 + i);
            wait_tile(o0);
            if (!ok) break;
            tc_fence_after();
            attn_mma_qk<D>(i * 128, q_lo, k_lo + (o0 % NSTG) * (C::TILE >> 4), idesc);
            tc_commit(&sbar[i]);
            tc_commit(&free_[o0 % NSTG]);
#pragma unroll 1
            for (int v = i; v < nt; v += 2) {
              const int o = 2 * (n0 + v), on = o + 4;
              const bool more = v + 2 < nt;
              wait_tile(o + 1);
              if (ok && more) wait_tile(on);   // ahead of the weights, as in the prompt kernel
              if (!ok || !(ok = attn_wait(&pbar[i], (uint32_t)np & 1u, abort_flag, g_tree_wait_ns))) break;
              ++np;
              tc_fence_after();
              const uint32_t vd = v_lo + ((o + 1) % NSTG) * (C::TILE >> 4);
              tree_mma_pv<D>(256 + i * D, i * 128, vd, 0, v > i);
              if (NE == 4) tree_mma_pv<D>(256 + i * D, i * 128, vd, 1, true);
              if (more) {
                attn_mma_qk<D>(i * 128, q_lo, k_lo + (on % NSTG) * (C::TILE >> 4), idesc);
                tc_commit(&sbar[i]);
                tc_commit(&free_[(o + 1) % NSTG]);
                tc_commit(&free_[on % NSTG]);
              } else {
                tc_commit(&obar[i]);
                tc_commit(&free_[(o + 1) % NSTG]);
              }
            }
          }
          n0 += nt;
        }
        tc_commit(&drain[i]);   // what is in flight finishes before tensor memory is given up
        mbar_wait_bounded(&drain[i], 0, kAttnWaitLimitNs);
      }
    } else if (i == 2 && !p.debug_stall) {
      // ---------------- copies: lanes 0 .. 7 the tile's runs of 16 tokens
      int n = 0;
      bool ok = true;
      for (int it = 0; ok; ++it) {
        const TreeJob* job = next_job(it, true);
        if (!job) break;
        const TreeJob j = *job;
        __syncwarp();
        if (lane == 0) job_done(it);
        const int32_t* table = a.table + (int64_t)j.b * a.table_width;
        int64_t place = 0;
        for (int v = j.v0; v < j.v1; ++v, ++n) {
          // lane 8 w + k looks run k of the tile w further on up: one look-up for four tiles
          if (((v - j.v0) & 3) == 0) {
            const int vt = v + (lane >> 3);
            const int tok = vt < j.v1 ? j.token(vt, kTreeTcUnit) + 16 * (lane & 7) : j.s.n;
            place = tok < j.s.n ? (tree_page(a, table, tok, p.shift) * a.Hkv + j.hk) * a.page_size + (tok & (a.page_size - 1)) : -1;
          }
          const int64_t at = __shfl_sync(0xffffffffu, place, 8 * ((v - j.v0) & 3) + (lane & 7));
          const int runs = __popc(__ballot_sync(0xffffffffu, lane < 8 && at >= 0));
          const int st = n % NRAW;
          if (n >= NRAW && !(ok = attn_wait_warp(&rawfree[st], (uint32_t)(n / NRAW - 1) & 1u, abort_flag, g_tree_wait_ns))) break;
          if (lane == 0) {
            mbar_arrive_expect_tx(&raw[st], (uint32_t)runs * (16 * D + 256));
            *copied = n + 1;
          }
          __syncwarp();
          if (lane < 8 && at >= 0) {
            uint8_t* dst = smem + C::OFF_RAW + st * C::RAW;
            bulk_load(dst + lane * 8 * D, a.k_codes + at * (D / 2), 8 * D, &raw[st]);
            bulk_load(dst + C::RAW_V + lane * 8 * D, a.v_codes + at * (D / 2), 8 * D, &raw[st]);
            bulk_load(dst + C::RAW_S + lane * 256, a.scales + at * 4, 256, &raw[st]);
          }
        }
      }
    } else if (i == 3 && attn_elect()) {
      // ---------------- jobs
      bool more = true;
      for (int it = 0; more; ++it) {
        TreeJob j = {};
        more = walk.next(p, j);
        if (it >= kJobSlots &&
            !attn_wait(&taken[it % kJobSlots], (uint32_t)(it / kJobSlots - 1) & 1u, abort_flag, g_tree_wait_ns))
          break;
        TreeJobSlot* x = &job_s[it % kJobSlots];
        x->more = more;
        x->j = j;
        mbar_arrive(&jbar[it % kJobSlots]);
      }
    }
  } else {
    // ---------------- softmax of the even (warps 0-3) and odd (4-7) tiles.  Lane 4 g + c
    // holds rows g + 8 e of its warp's lanes, e < NE, and tokens 8 k + 2 c, + 1.
    asm volatile("setmaxnreg.inc.sync.aligned.u32 184;\n");
    const int i = warp >> 2, quad = warp & 3, g = lane >> 2, c = lane & 3;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const uint32_t st = tmem + i * 128 + lanes, ot = tmem + 256 + i * D + lanes;
    float* xs = reinterpret_cast<float*>(smem + C::OFF_X);
    // the job's row on MMA lane `at` (quad, lane of the warp), 8 groups of 8 rows per e
    auto row_of = [&](int q, int l) { return (l >> 3) * 32 + q * 8 + (l & 7); };
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
    int ns = 0, nob = 0, n0 = 0;   // score tiles and jobs with an own tile so far, tiles before this job
    bool ok = true;
    for (int it = 0; ok; ++it) {
      const TreeJob* job = next_job(it, true);
      // (a warp that gave the wait up still meets the others at the barriers: all of them leave there)
      if (named_or(!job && *abort_flag)) break;
      if (!job) break;
      const TreeJob& j = *job;
      const TreeSeq& s = j.s;
      const int nt = j.v1 - j.v0, first = j.v0, front = s.front, skip = s.skip, ctx = s.ctx;
      // (every thread is here past the last job's end: its views, sums and queries are free)
      if (tid < s.nq) parent_s[tid] = a.parents ? __ldg(a.parents + s.q0 + tid) : tid - 1;
      // The queries, their pairs in the order of code_pairs, and their sums: D / 8 lanes share a
      // row, warp w has MMA lanes 16 w .. 16 w + 15.
      {
        constexpr int LPR = D / 8, RPL = 32 / LPR;   // lanes per row, rows per load
        const int ch = lane % LPR;
        uint4 w[16 / RPL];
#pragma unroll
        for (int k = 0; k < 16 / RPL; ++k) {
          const int m = 16 * warp + k * RPL + lane / LPR, r = row_of(m >> 5, m & 31);
          w[k] = r < j.rows
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
      named_bar_sync(kSoftmaxBarrier, 256);   // parents and sums written
      if (tid < 128) {
        const int r = row_of(quad, lane);
        TreeRow v = {};
        if (r < j.rows) v = tree_row(p, s, parent_s, (j.r0 + r) / p.G);
        row_s[tid] = v;
      }
      float qs[NE];
#pragma unroll
      for (int e = 0; e < NE; ++e) qs[e] = xs[quad * 32 + 8 * e + g];
      named_bar_sync(kSoftmaxBarrier, 256);   // the rows' views written, the sums read
      // tokens that every row sees: those below `ctx`, from the last row's window on or in the sinks
      int low = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) low = max(low, row_s[k * 32 + lane].low);
      low = (int)__reduce_max_sync(0xffffffffu, (unsigned)low);

      float m[NE], l[NE], z[NE];   // M; l, z: of this lane's tokens
#pragma unroll
      for (int e = 0; e < NE; ++e) m[e] = -INFINITY, l[e] = z[e] = 0.f;
#pragma unroll 1
      for (int v = i; v < nt; v += 2, ++ns) {
        const int n = n0 + v, base = (first + v < front ? first + v : first + v + skip) * kTreeTcUnit;
        if (!(ok = attn_wait_warp(&cbar[n % NCOL], (uint32_t)(n / NCOL) & 1u, abort_flag, g_tree_wait_ns))) break;
        // the numbers of tokens 8 k + 2 c, 8 k + 2 c + 1
        const uint8_t* cols = smem + C::OFF_COL + (n % NCOL) * C::COL;
        const ulonglong2* ab = reinterpret_cast<const ulonglong2*>(cols) + c;
        const ulonglong2* fv = reinterpret_cast<const ulonglong2*>(cols + C::COL_V) + c;
        const ulonglong2* la = reinterpret_cast<const ulonglong2*>(cols + C::COL_LOG) + c;
        if (!(ok = attn_wait_warp(&sbar[i], (uint32_t)ns & 1u, abort_flag, g_tree_wait_ns))) break;
        tc_fence_after();
        // 32 tokens at a time: this loop's code stays in the instruction cache
#pragma unroll 1
        for (int q = 0; q < 4; ++q, ab += 16, fv += 16, la += 8) {
          uint32_t x[NH][16];   // x[h][4 k + 2 e + y]: row 16 h + 8 e + g, token 32 q + 8 k + 2 c + y
#pragma unroll
          for (int h = 0; h < NH; ++h) tmem_ld_16x256b_x4(st + ((16u * h) << 16) + 32 * q, x[h]);
#pragma unroll
          for (int h = 0; h < NH; ++h) tmem_ld_wait(x[h]);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
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
          const int at = base + 32 * q;
          if (at + 32 > ctx || (at < low && at + 32 > p.sinks)) {
            // not every row sees every token: lane r has a bit per token for row r of the warp
            const uint32_t seen = tree_sees(p, s, row_s[quad * 32 + lane], at);
#pragma unroll
            for (int e = 0; e < NE; ++e) {
              const uint32_t bits = __shfl_sync(0xffffffffu, seen, 8 * e + g) >> (2 * c);
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                  if (!((bits >> (8 * k + y)) & 1u)) x[e >> 1][4 * k + 2 * (e & 1) + y] = 0xFF800000u;   // -inf
            }
          }
          float mx[NE];
          bool grow = false;
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const uint32_t* y = &x[e >> 1][2 * (e & 1)];
            mx[e] = fmaxf(attn_max3(__uint_as_float(y[0]), __uint_as_float(y[1]), __uint_as_float(y[4])),
                          attn_max3(__uint_as_float(y[5]), __uint_as_float(y[8]), __uint_as_float(y[9])));
            mx[e] = attn_max3(mx[e], __uint_as_float(y[12]), __uint_as_float(y[13]));
            grow |= mx[e] > m[e] + kAttnSlack;
          }
          if (__any_sync(0xffffffffu, grow)) {   // seldom: M moves
            float f[4];
#pragma unroll
            for (int e = 0; e < NE; ++e) {
              mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 1));
              mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
              // (whole numbers: the factor is a power of two, which leaves the weights' parts exact)
              const float mn = mx[e] > m[e] + kAttnSlack ? ceilf(mx[e]) : m[e];
              // (a row without a maximum has no weights, or sums that are not numbers and stay so)
              f[e] = m[e] == -INFINITY || mn == m[e] ? 1.f : __int_as_float(((int)fmaxf(m[e] - mn, -127.f) + 127) << 23);
              m[e] = mn;
              l[e] *= f[e];
              z[e] *= f[e];
            }
            if constexpr (NE == 1) f[1] = f[2] = f[3] = f[0];   // (lanes of second parts, and of no row)
            if constexpr (NE == 2) f[2] = f[0], f[3] = f[1];
            // the factor of lane r's row is with lanes 4 (r % 8) ..
            float fr = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float y = __shfl_sync(0xffffffffu, f[e], 4 * (lane & 7));
              if (lane >> 3 == e) fr = y;
            }
            // (the scores' barrier says that every product issued before them is done)
            if (v > i) attn_rescale<D>(ot, fr);
            // this tile's weights so far
#pragma unroll 1
            for (int t = 0; t < 32 * q; t += 16) {
              uint32_t w[16];
              tmem_st_wait();
              tmem_ld_32x32b_x16(st + t, w);
              tmem_ld_wait(w);
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
                w[k] = pack_half2_bits(y.x * fr, y.y * fr);
              }
              tmem_st_32x32b_x16(st + t, w);
            }
          }
          uint32_t w0[NH][8], w1[NH][8];   // first and second parts: 32-bit columns 4 k + c
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const float off = m[e] == -INFINITY ? 0.f : -m[e];
            const F2 of2 = f2_make(off, off);
            F2 sum = f2_make(l[e], 0.f), zs = f2_make(z[e], 0.f);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const ulonglong2 f = fv[4 * k];
              const uint32_t* y = &x[e >> 1][4 * k + 2 * (e & 1)];
              float t0, t1;
              f2_split(f2_add(f2_from_bits(y[0], y[1]), of2), t0, t1);
              t0 = attn_exp2(t0);
              t1 = attn_exp2(t1);
              const F2 ex = f2_make(t0, t1);
              sum = f2_fma(ex, F2{f.x}, sum);
              zs = f2_fma(ex, F2{f.y}, zs);
              const uint32_t hi = pack_half2_bits(t0, t1);
              const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&hi));
              const uint32_t lo = pack_half2_bits(t0 - r.x, t1 - r.y);
              w0[e >> 1][2 * k + (e & 1)] = hi;
              if (NE == 1)
                w0[0][2 * k + 1] = lo;
              else
                w1[e >> 1][2 * k + (e & 1)] = lo;
            }
            float t0, t1;
            f2_split(sum, t0, t1);
            l[e] = t0 + t1;
            f2_split(zs, t0, t1);
            z[e] = t0 + t1;
          }
#pragma unroll
          for (int h = 0; h < NH; ++h) {
            tmem_st_16x128b_x4(st + ((16u * h) << 16) + 32 * q, w0[h]);
            if (NE == 2) tmem_st_16x128b_x4(st + (16u << 16) + 32 * q, w1[h]);
            if (NE == 4) tmem_st_16x128b_x4(st + ((16u * h) << 16) + 32 * q + 16, w1[h]);
          }
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pbar[i]);
      }
      if (ok && i < nt) ok = attn_wait_warp(&obar[i], (uint32_t)nob++ & 1u, abort_flag, g_tree_wait_ns);
      // the warpgroups' numbers of every row, and whether either gave a wait up
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
          float* y = xs + i * 384 + quad * 32 + 8 * e + g;
          y[0] = m[e], y[128] = l[e], y[256] = z[e];
        }
      }
      ok = !named_or(!ok);
      if (!ok) break;
      tc_fence_after();
      // o = sum of the warpgroups' accumulators: this one's half of D, a row per lane
      {
        const int r = row_of(quad, lane);
        const bool mine = lane < 8 * NE && r < j.rows;
        const float* y = xs + quad * 32 + lane;
        const float l0 = mine ? y[128] : 0.f, l1 = mine ? y[384 + 128] : 0.f;
        const float m0 = l0 != 0.f ? y[0] : -INFINITY, m1 = l1 != 0.f ? y[384] : -INFINITY, M = fmaxf(m0, m1);
        const float f0 = l0 != 0.f ? attn_exp2(m0 - M) : 0.f, f1 = l1 != 0.f ? attn_exp2(m1 - M) : 0.f;
        float ls = l0 != 0.f ? f0 * l0 : 0.f, zz = l0 != 0.f ? f0 * y[256] : 0.f;
        if (l1 != 0.f) ls = fmaf(f1, l1, ls), zz = fmaf(f1, y[384 + 256], zz);
        const bool whole = j.whole();
        const float inv = whole ? (ls != 0.f ? 1.f / ls : 0.f) : 1.f;
        const int64_t slot = j.slot(blockIdx.x) * (32 * NE) + r;
        const int64_t at = mine ? j.row_at(p, r) : 0;
        if (mine && !whole && i == 0) p.ml[slot] = make_float2(M, ls);
#pragma unroll 1
        for (int q = 0; q < D / 2; q += 16) {
          const int d0 = i * (D / 2) + q;
          uint32_t o0[16], o1[16];
          tmem_ld_32x32b_x16(tmem + 256 + lanes + d0, o0);
          tmem_ld_32x32b_x16(tmem + 256 + D + lanes + d0, o1);
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
            // (an accumulator of a warpgroup without tokens that this row sees may hold anything)
            float val = l0 != 0.f ? fmaf(f0, u, zz) : zz;
            if (l1 != 0.f) val = fmaf(f1, w, val);
            o[k] = val * inv;
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
      n0 += nt;
      __syncwarp();
      if (lane == 0) job_done(it);
      named_bar_sync(kSoftmaxBarrier, 256);   // the rows' numbers have been read
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // the copies in flight land before the memory is given up
    if (tid == 0) {
      for (int n = max(0, *copied - NRAW); n < *copied; ++n)
        mbar_wait_bounded(&raw[n % NRAW], (uint32_t)(n / NRAW) & 1u, kAttnWaitLimitNs);
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
