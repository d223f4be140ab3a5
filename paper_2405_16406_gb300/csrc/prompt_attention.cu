// prompt_attention.cu -- spinq_prompt_attention: causal attention over packed
// prompts with grouped heads, on the 5th-generation tensor core.
//
//   o_i = sum_{j < n_i} softmax_j(scale q_i . k_j) v_j
//
// n_i = min(lk, i + 1 + lk - lq) with the causal mask (the queries are the
// last lq of the sequence's lk positions), else lk; a query that sees no key
// gives zeros.
//
// Rows.  The G query heads of a kv head share its keys, so an MMA's 128 rows
// are TPT = floor(128 / G) consecutive queries of all G heads (row = query *
// G + head): K and V are read once for the group, a short prompt fills the
// tile, and a causal tile spans TPT positions instead of 128.
//
// A work item is two such tiles of a kv head and a sequence.  S = Q K^T (128 x
// 128 fp32) and O (128 x D fp32) of both tiles fill tensor memory; P replaces S
// as fp16 and is the A operand of O += P V straight from there.  One CTA per SM;
// it starts with the item of its block index and takes further ones from the grid's
// blocks that have not started (cluster launch control), the last queries,
// which see the most keys, first: the next item's copies and first products run
// under this one's last weights, and O is read and stored after the next item's first
// weights (before them: 16 ragged sequences of 9454 tokens 91.4 us against 87.7, 4 x
// 4096 395 us against 386; with a block per item 4 x 4096 took 431), exchanged in quads so
// that it leaves in runs of 64 bytes (with 16 bytes of a row per lane 87.5 us against 78.8, 384
// against 365).  Blocks past a sequence's end are passed over; a grid that counts only the
// items there are took 103 us for 91 on the ragged batch, whose long items it starts later.  4 x
// 4096, 32 / 8 heads, D 128: 366 us run again and again on one state, 414 us with cold inputs (1.50 and
// 1.33 PFLOP/s; the measured rate of a large matrix product is 1.91).  The softmax bounds
// it: a step of 128 keys for both tiles is 2052 cycles of MMAs and about 3200 in all.
// P in one fp16 part is a choice: the output's error against 64 bits is 0.00022 to 0.00029 where
// its own rounding alone is 0.00021 (0.00031 in calls of a few rows).  Two parts, the second in
// the rows that tiles of 64 leave idle, made those calls exact to the output's rounding
// and 15 to 25 % slower (1 query behind 2168 tokens 26 and 31 us, 64 behind 32768 355 and 430).  Warp roles:
//  * warps 0-3 and 4-7: softmax of tile 0 and 1, one row per thread: running
//    maximum (base 2, moved only by more than 2^8, when the row's O is
//    rescaled) and sum in fp32 registers;
//  * warp 8: one thread copies Q, then the K and V tiles of 128 tokens into
//    a ring of stages by TMA (128-byte swizzle);
//  * warps 9 and 10: one thread each issues the MMAs of tile 0 and 1, PV then the
//    next QK.  An issue blocks while the tensor core is busy, and a wait on a
//    barrier costs 150 to 230 cycles beside MMAs that read shared memory at its full
//    rate: with one issuing thread for both tiles the tensor core idled
//    through those waits (4 x 4096: 484 us against 431 us);
//  * warp 11: one thread fetches the items and leaves out those past a
//    sequence's end.
// Floor: the tensor core (4 D flops per visible pair of a query head and a key).
//
// A sequence's last V tile may hold rows of the next sequence or of no
// sequence: they meet weights 0, which is not enough if they are not finite, so the
// softmax threads zero them; K's such rows only reach scores that the mask replaces.
//
// Every wait is bounded; one that gives up raises the CTA's abort flag, the
// MMAs and copies in flight are drained and the status word is set.
#include <cuda_fp16.h>

#include "../../include/spinq.h"
#include "attn_tc.cuh"
#include "launch_util.h"
#include "spinq_internal.h"
#include "tensor_map.h"

namespace spinq {
namespace {

__device__ uint64_t g_prompt_wait_ns = kAttnWaitLimitNs;
constexpr int kPromptSite = 31;   // wait site recorded on a time-out

struct PromptParams {
  const int32_t* cu_q;
  const int32_t* cu_k;
  __half* out;
  int64_t total_q, total_k;
  int Hq, Hkv, batch, G, tpt;   // tpt: queries per tile
  int tiles;                    // items along a sequence's queries
  bool causal;
  int window, sinks;            // the windowed form's (causal; window >= 1)
  float scale_log2;             // |scale| log2 e
  uint32_t idesc_qk;
  int* status;
  int debug_stall;
};

// A work item as the roles read it.
struct PromptItem {
  int more;   // 0: no further item
  int hk, t0, lq, lk, pad;
  int64_t q0, k0;
};

template <int D>
struct PromptCfg {
  static constexpr int TILE = 128 * D * 2;               // bytes of a Q, K or V tile
  static constexpr int NSTG = D == 128 ? 5 : 8;
  static constexpr int OFF_KV = 2 * TILE;
  static constexpr int OFF_ITEM = OFF_KV + NSTG * TILE;  // PromptItem [2]
  static constexpr int OFF_CLC = OFF_ITEM + 2 * (int)sizeof(PromptItem);   // 16 bytes: answer of the launch control
  static constexpr int OFF_BAR = OFF_CLC + 16;
  // full, free [NSTG], q, qfree, clc, item, taken [2], s, p, drain [2]
  static constexpr int OFF_MISC = OFF_BAR + (2 * NSTG + 3 + 4 + 6) * 8;
  static constexpr int BYTES = OFF_MISC + 16 + 1024;
  static_assert(OFF_CLC % 16 == 0 && BYTES <= 232448, "shared memory");
};
// three warpgroups: two of softmax with 216 registers a thread, one with the
// copies and the MMAs with 72; 2 * 216 + 72 = 3 * 168, what the launch holds
constexpr int kPromptThreads = 384;
constexpr int kSinkRows = 32;
// the item's readers: copy thread, two MMA threads, eight softmax warps
constexpr int kItemReaders = 11;

// WIN: a query at position p sees keys j <= p with p - j < window or j < sinks.  An item's keys are
// then a list: the sinks in whole groups of kSinkRows, and behind them those from the first that the
// window of the item's first query reaches, so that a few sinks cost a part of a tile and
// no tile starts before the window (2 x 32 queries with a window of 512 and 4 sinks: 5 tiles of
// 128; with a tile of sinks and tiles at whole multiples of 128 tokens 6.5: 16 ragged sequences of
// 32767 tokens 471 us so and 347 now, 0.92 PFLOP/s on visible pairs; 2 x 16384 with a window of 4096 1.31 ms, 1.48).
// Bound: the softmax, as above, and the masks: the window's two edges cross 2 of those 5 tiles.  Both
// tiles of an item work through its one list, so the second's first keys may lie before all of its windows (one
// head a group, no sinks: one tile of 6 with a window of 512).
template <int D, bool WIN>
__global__ void __launch_bounds__(kPromptThreads, 1)
    prompt_tc_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                     const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mks,
                     const __grid_constant__ CUtensorMap mvs, const PromptParams a) {
  using C = PromptCfg<D>;
  constexpr int NSTG = C::NSTG;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* free_ = full + NSTG;
  uint64_t* qbar = free_ + NSTG;   // an item's Q tiles are in
  uint64_t* qfree = qbar + 1;      // its last products with them are done
  uint64_t* clc = qfree + 1;       // answer of the launch control
  uint64_t* item = clc + 1;        // slot written
  uint64_t* taken = item + 2;      // slot read by every role
  uint64_t* sbar = taken + 2;      // scores of tile i written
  uint64_t* pbar = sbar + 2;       // weights of tile i written (4 warps)
  uint64_t* drain = pbar + 2;      // every MMA of tile i done
  const volatile PromptItem* items = reinterpret_cast<const volatile PromptItem*>(smem + C::OFF_ITEM);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  int* issued = reinterpret_cast<int*>(smem + C::OFF_MISC + 8);   // K and V tiles copied, items' Q tiles copied
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    for (int s = 0; s < NSTG; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&free_[s], 2);
    }
    mbar_init(qbar, 1);
    mbar_init(qfree, 2);
    mbar_init(clc, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&item[i], 1);
      mbar_init(&taken[i], kItemReaders);
      mbar_init(&sbar[i], 1);
      mbar_init(&pbar[i], 4);
      mbar_init(&drain[i], 1);
    }
    *abort_flag = 0;
    issued[0] = issued[1] = 0;
    fence_mbar_init();
    prefetch_tmap(&mq);
    prefetch_tmap(&mk);
    prefetch_tmap(&mv);
  }
  if (warp == 9) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = 0;   // all 512 columns are this CTA's: they start at column 0
  pdl_wait();
  pdl_trigger();
  const uint32_t sb = smem_u32(smem);

  // What a role knows of its item: the keys that tile i's last query sees and
  // the tiles of 128 tokens that hold them.
  struct Work {
    int hk, t0, lq, lk, nt[2], ntile;
    int64_t q0, k0;
    int front, from;   // WIN: rows of sinks at the list's start; the token behind them
  };
  auto read_item = [&](int slot, Work& w) {
    const volatile PromptItem& x = items[slot];
    w.hk = x.hk, w.t0 = x.t0, w.lq = x.lq, w.lk = x.lk, w.q0 = x.q0, w.k0 = x.k0;
    w.front = w.from = 0;
    if constexpr (WIN) {
      const int first = w.t0 + w.lk - w.lq;   // position of the item's first query
      const int low = first >= a.window ? first - a.window + 1 : 0;
      // (rows of the front are tokens before the window, and so of the sequence)
      const int64_t front = ((int64_t)a.sinks + kSinkRows - 1) / kSinkRows * kSinkRows;
      if (front <= low) {
        w.front = (int)front;
        w.from = low;
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int first = w.t0 + i * a.tpt, last = min(first + a.tpt, w.lq) - 1;
      const int nk = first < w.lq ? (a.causal ? max(0, min(w.lk, last + 1 + w.lk - w.lq)) : w.lk) : 0;
      // (WIN: a tile that sees a key sees it behind the window's start)
      w.nt[i] = ((WIN && nk > 0 ? nk - w.from + w.front : nk) + 127) / 128;
    }
    w.ntile = max(w.nt[0], w.nt[1]);
    return x.more != 0;
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;\n");
    if (warp == 8) {
      // ---------------- copies
      if (attn_elect() && !a.debug_stall) {
        int sk = 0, pk = 1;   // ring stage, parity of the phase that frees it (the first time: none)
        int nq = 0;           // items whose Q was copied
        for (int it = 0;; ++it) {
          if (!attn_wait(&item[it & 1], (uint32_t)(it >> 1) & 1u, abort_flag, g_prompt_wait_ns)) break;
          Work w;
          const bool more = read_item(it & 1, w);
          mbar_arrive(&taken[it & 1]);
          if (!more) break;
          if (w.ntile == 0) continue;
          if (nq > 0 && !attn_wait(qfree, (uint32_t)(nq - 1) & 1u, abort_flag, g_prompt_wait_ns)) break;
          mbar_arrive_expect_tx(qbar, (uint32_t)(a.G * a.tpt) * 128u * (D / 64) * 2u);
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int at = 0; at < D / 64; ++at)
              tma_load_3d(smem + i * C::TILE + at * kAttnAtom, &mq, qbar, at * 64, w.hk * a.G,
                          (int32_t)(w.q0 + w.t0 + i * a.tpt));
          issued[1] = ++nq;
          bool ok = true;
          for (int n = 0; n < 2 * w.ntile; ++n) {
            // (a fresh barrier answers the parity before its first phase at once)
            if (!(ok = attn_wait(&free_[sk], pk, abort_flag, g_prompt_wait_ns))) break;
            mbar_arrive_expect_tx(&full[sk], (uint32_t)C::TILE);
            const int row = (n >> 1) * 128;
            if (WIN && row < w.front && row + 128 > w.front) {
              // the last sinks and the window's first keys
#pragma unroll 1
              for (int r = 0; r < 128; r += kSinkRows)
#pragma unroll
                for (int at = 0; at < D / 64; ++at)
                  tma_load_3d(smem + C::OFF_KV + sk * C::TILE + at * kAttnAtom + r * 128, n & 1 ? &mvs : &mks, &full[sk], at * 64,
                              w.hk, (int32_t)(w.k0 + (row + r < w.front ? row + r : row + r - w.front + w.from)));
            } else {
              const int token = WIN && row >= w.front ? row - w.front + w.from : row;
#pragma unroll
              for (int at = 0; at < D / 64; ++at)
                tma_load_3d(smem + C::OFF_KV + sk * C::TILE + at * kAttnAtom, n & 1 ? &mv : &mk, &full[sk], at * 64, w.hk,
                            (int32_t)(w.k0 + token));
            }
            ++issued[0];
            if (++sk == NSTG) sk = 0, pk ^= 1;
          }
          if (!ok) break;
        }
      }
    } else if (warp < 11) {
      // ---------------- MMAs of tile i, by one thread
      const int i = warp - 9;
      if (attn_elect()) {
        const uint32_t q_lo = attn_desc_k(sb + i * C::TILE), k_lo = attn_desc_k(sb + C::OFF_KV),
                       v_lo = attn_desc_mn(sb + C::OFF_KV);
        int sk = 0, pk = 0;          // ring stage of the next K or V tile, its phase
        int nq = 0, np = 0;          // items with keys, weight tiles so far
        bool ok = true;
        auto wait_tile = [&]() {
          ok = attn_wait(&full[sk], pk, abort_flag, g_prompt_wait_ns);
          const int s = sk;
          if (++sk == NSTG) sk = 0, pk ^= 1;
          return s;
        };
#pragma unroll 1
        for (int it = 0; ok; ++it) {
          if (!(ok = attn_wait(&item[it & 1], (uint32_t)(it >> 1) & 1u, abort_flag, g_prompt_wait_ns))) break;
          Work w;
          const bool more = read_item(it & 1, w);
          mbar_arrive(&taken[it & 1]);
          if (!more) break;
          if (w.ntile == 0) continue;
          const int nti = i ? w.nt[1] : w.nt[0];
          if (!(ok = attn_wait(qbar, (uint32_t)nq & 1u, abort_flag, g_prompt_wait_ns))) break;
          ++nq;
          const int s0 = wait_tile();
          if (!ok) break;
          tc_fence_after();
          if (nti > 0) {
            attn_mma_qk<D>(i * 128, q_lo, k_lo + s0 * (C::TILE >> 4), a.idesc_qk);
            tc_commit(&sbar[i]);
          }
          if (nti <= 1) tc_commit(qfree);
          tc_commit(&free_[s0]);
#pragma unroll 1
          for (int j = 0; j < w.ntile; ++j) {
            const int sv = wait_tile();
            if (!ok) break;
            // everything else is waited for ahead of the weights: what follows
            // those is on the path from this tile's softmax to its next scores
            const int sn = j + 1 < w.ntile ? wait_tile() : -1;
            if (!ok) break;
            if (j < nti) {
              // (an item's first weights come after the last item's O has been read)
              if (!(ok = attn_wait(&pbar[i], (uint32_t)np & 1u, abort_flag, g_prompt_wait_ns))) break;
              ++np;
              tc_fence_after();
              attn_mma_pv<D>(256 + i * D, i * 128, v_lo + sv * (C::TILE >> 4), j > 0);
              if (j + 1 < nti) {
                attn_mma_qk<D>(i * 128, q_lo, k_lo + sn * (C::TILE >> 4), a.idesc_qk);
                tc_commit(&sbar[i]);
                if (j + 2 == nti) tc_commit(qfree);
              }
            }
            tc_commit(&free_[sv]);
            if (sn >= 0) tc_commit(&free_[sn]);
          }
        }
        tc_commit(&drain[i]);   // what is in flight finishes before tensor memory is given up
        mbar_wait_bounded(&drain[i], 0, kAttnWaitLimitNs);
      }
    } else if (attn_elect()) {
      // ---------------- items
      uint32_t id = blockIdx.x;
      int nc = 0, it = 0;
      bool more = true;
      while (true) {
        // the last queries first, over all heads and sequences
        const uint32_t heads = (uint32_t)(a.Hkv * a.batch), tile = id / heads, hb = id - tile * heads;
        const int b = (int)(hb / (uint32_t)a.Hkv), t0 = (a.tiles - 1 - (int)tile) * 2 * a.tpt;
        // (offsets outside the rows are clamped: nothing is written or read out of range)
        const int64_t q0 = max(0, __ldg(a.cu_q + b)), q1 = min((int64_t)__ldg(a.cu_q + b + 1), a.total_q);
        const int64_t k0 = max(0, __ldg(a.cu_k + b)), k1 = min((int64_t)__ldg(a.cu_k + b + 1), a.total_k);
        if (!more || q0 + t0 < q1) {
          if (it >= 2 && !attn_wait(&taken[it & 1], (uint32_t)((it >> 1) - 1) & 1u, abort_flag, g_prompt_wait_ns)) break;
          volatile PromptItem& x = const_cast<volatile PromptItem&>(items[it & 1]);
          x.more = more;
          x.hk = (int)(hb - (uint32_t)b * (uint32_t)a.Hkv);
          x.t0 = t0;
          x.lq = (int)(q1 - q0);
          x.lk = (int)max((int64_t)0, k1 - k0);
          x.q0 = q0;
          x.k0 = k0;
          mbar_arrive(&item[it & 1]);
          ++it;
          if (!more) break;
        }
        // the grid's next block that has not started, if there is one
        mbar_arrive_expect_tx(clc, 16);
        asm volatile(
            "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];\n" ::"r"(
                sb + C::OFF_CLC),
            "r"(smem_u32(clc))
            : "memory");
        if (!attn_wait(clc, (uint32_t)nc & 1u, abort_flag, g_prompt_wait_ns)) {
          mbar_wait_bounded(clc, (uint32_t)nc & 1u, kAttnWaitLimitNs);   // the answer is still to be written
          break;
        }
        ++nc;
        uint32_t got, x;
        asm volatile(
            "{\n .reg .b128 h;\n .reg .pred p;\n ld.shared.b128 h, [%2];\n"
            " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n selp.u32 %0, 1, 0, p;\n mov.u32 %1, 0;\n"
            " @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, h;\n}\n"
            : "=r"(got), "=r"(x)
            : "r"(sb + C::OFF_CLC)
            : "memory");
        fence_proxy_async_smem();   // the answer is read before the next one is asked for
        more = got != 0;
        if (more) id = x;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;\n");
    // ---------------- softmax: warps 4i .. 4i + 3 own tile i, thread = row
    const int i = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t st = tmem + i * 128 + lanes, ot = tmem + 256 + i * D + lanes;
    const int row_t = r / a.G, row_h = r - row_t * a.G;
    int kv = 0;            // K and V tiles before this item
    int ns = 0;            // score tiles so far
    // The last item's O stays in tensor memory until this item's first weights are
    // written: its products and its way out then run under the next item's scores.
    __half* out = nullptr;   // where this row of it goes, if it does
    float inv = 0.f;
    bool held = false;       // there is such an O
    // Four lanes exchange 16-byte pieces of their rows, so that a store is 64 bytes of eight rows (a piece
    // of 32 rows each took 3600 of the 22400 cycles of an item with a window of 512; 1900 of 20400 so).
    auto store = [&](const uint32_t* o) {
      __half* row[4];   // of the quad
#pragma unroll
      for (int k = 0; k < 4; ++k)
        row[k] = reinterpret_cast<__half*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(out), (lane & 28) + k));
#pragma unroll
      for (int e = 0; e < D; e += 32) {
        uint32_t v[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int q = 0; q < 4; ++q) {   // a row without a key: zeros, whatever is in O
            const int x = e + 8 * k + 2 * q;
            v[k][q] = inv != 0.f ? pack_half2_bits(__uint_as_float(o[x]) * inv, __uint_as_float(o[x + 1]) * inv) : 0u;
          }
#pragma unroll
        for (int bit = 1; bit < 4; bit <<= 1)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (!(k & bit)) {
              const bool up = (lane & bit) != 0;
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? v[k][q] : v[k | bit][q], bit);
                if (up) v[k][q] = got; else v[k | bit][q] = got;
              }
            }
        // v[k]: piece lane % 4 of these four of the quad's row k
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (row[k] != nullptr)
            *reinterpret_cast<uint4*>(row[k] + e + 8 * (lane & 3)) = make_uint4(v[k][0], v[k][1], v[k][2], v[k][3]);
      }
    };
    bool ok = true;
    for (int it = 0; ok; ++it) {
      if (!(ok = attn_wait_warp(&item[it & 1], (uint32_t)(it >> 1) & 1u, abort_flag, g_prompt_wait_ns))) break;
      int nti, lk, kv_after, n;   // n: keys of this row
      int low = 0;   // WIN: the list's first key of its window.  n and lk are places in the list too.
      {
        Work w;
        if (!read_item(it & 1, w)) break;
        nti = i ? w.nt[1] : w.nt[0];
        lk = w.lk;
        kv_after = kv + 2 * w.ntile;
        const int tok = w.t0 + i * a.tpt + row_t;
        n = r < a.G * a.tpt && tok < w.lq ? (a.causal ? min(lk, tok + 1 + lk - w.lq) : lk) : 128 * nti;
        if constexpr (WIN) {
          const int shift = w.front - w.from;   // of a window's key, from its token to its place
          lk += shift;
          if (r < a.G * a.tpt && tok < w.lq) {
            const int pos = tok + w.lk - w.lq;
            low = (pos >= a.window ? pos - a.window + 1 : 0) + shift;
            n += shift;
          }
        }
      }
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < nti; ++j, ++ns) {
        if (!(ok = attn_wait_warp(&sbar[i], (uint32_t)ns & 1u, abort_flag, g_prompt_wait_ns))) break;
        tc_fence_after();
        uint32_t s[128];
#pragma unroll
        for (int c = 0; c < 128; c += 32) tmem_ld_32x32b_x32(st + c, s + c);
        tmem_ld_wait_all<128>(s);
        const int seen = n - j * 128;
        if (__any_sync(0xffffffffu, seen < 128)) {
#pragma unroll
          for (int c = 0; c < 128; ++c)
            if (c >= seen) s[c] = 0xFF800000u;   // -inf
        }
        if constexpr (WIN) {
          // keys between the sinks and the row's window
          const int from = a.sinks - j * 128, to = low - j * 128;
          if (__any_sync(0xffffffffu, to > 0 && from < 128 && from < to)) {
#pragma unroll
            for (int c = 0; c < 128; ++c)
              if (c >= from && c < to) s[c] = 0xFF800000u;
          }
        }
        const float mx = attn_row_max(s) * a.scale_log2;
        const float mn = mx > m + kAttnSlack ? mx : m;
        if (__any_sync(0xffffffffu, mn != m) && j > 0) {
          // the scores' barrier says that every product issued before them,
          // this tile's last one included, is done
          const float f = mn != m ? attn_exp2(m - mn) : 1.f;
          l *= f;
          attn_rescale<D>(ot, f);
        }
        m = mn;
        const float off = m == -INFINITY ? 0.f : -m;   // a row without a key so far: weights 0
        const F2 sl2 = f2_make(a.scale_log2, a.scale_log2), of2 = f2_make(off, off);
        F2 sum[2] = {f2_make(l, 0.f), f2_make(0.f, 0.f)};
#pragma unroll
        for (int c = 0; c < 128; c += 2) {
          float x, y;
          f2_split(f2_fma(f2_from_bits(s[c], s[c + 1]), sl2, of2), x, y);
          x = attn_exp2(x);
          y = attn_exp2(y);
          sum[(c >> 1) & 1] = f2_add(sum[(c >> 1) & 1], f2_make(x, y));
          s[c >> 1] = pack_half2_bits(x, y);
        }
        float x, y;
        f2_split(f2_add(sum[0], sum[1]), x, y);
        l = x + y;
        tmem_st_32x32b_x32(st, s);
        tmem_st_32x32b_x32(st + 32, s + 32);
        if (j * 128 + 128 > lk) {
          // this V tile ends past the sequence: thread r zeroes row r if it lies there
          // (the threads of the other tile may write the same zeros)
          const int nv = kv + 2 * j + 1;
          if (!(ok = attn_wait_warp(&full[nv % NSTG], (uint32_t)(nv / NSTG) & 1u, abort_flag, g_prompt_wait_ns))) break;
          if (j * 128 + r >= lk) {
            const uint32_t vb = sb + C::OFF_KV + (nv % NSTG) * C::TILE + r * 128;
#pragma unroll
            for (int at = 0; at < D / 64; ++at)
#pragma unroll
              for (int o = 0; o < 128; o += 16) sts128(vb + at * kAttnAtom + o, make_uint4(0, 0, 0, 0));
          }
          fence_proxy_async_smem();
        }
        const bool take = j == 0 && held;
        if (take) {   // complete: its products were issued before these scores'
#pragma unroll
          for (int c = 0; c < D; c += 32) tmem_ld_32x32b_x32(ot + c, s + c);
          tmem_ld_wait_all<D>(s);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pbar[i]);
        if (take) {
          store(s);
          held = false;
        }
      }
      if (!ok) break;
      kv = kv_after;
      const volatile PromptItem& x = items[it & 1];
      const int tok = x.t0 + i * a.tpt + row_t;
      const bool live = r < a.G * a.tpt && tok < x.lq;
      __half* to = a.out + ((x.q0 + tok) * a.Hq + x.hk * a.G + row_h) * D;
      __syncwarp();
      if (lane == 0) mbar_arrive(&taken[it & 1]);
      if (nti > 0) {
        out = live ? to : nullptr;
        inv = l != 0.f ? 1.f / l : 0.f;
        held = true;
      } else if (live) {   // no query of the tile sees a key
#pragma unroll
        for (int e = 0; e < D; e += 8) *reinterpret_cast<uint4*>(to + e) = make_uint4(0, 0, 0, 0);
      }
    }
    if (ok && held && attn_wait_warp(&drain[i], 0, abort_flag, g_prompt_wait_ns)) {   // the last item's
      tc_fence_after();
      uint32_t o[D];
#pragma unroll
      for (int c = 0; c < D; c += 32) tmem_ld_32x32b_x32(ot + c, o + c);
      tmem_ld_wait_all<D>(o);
      store(o);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // the copies in flight land before the memory is given up
    if (tid == 0 && issued[1] > 0) mbar_wait_bounded(qbar, (uint32_t)(issued[1] - 1) & 1u, kAttnWaitLimitNs);
    if (tid == 0)
      for (int n = max(0, issued[0] - NSTG); n < issued[0]; ++n)
        mbar_wait_bounded(&full[n % NSTG], (uint32_t)(n / NSTG) & 1u, kAttnWaitLimitNs);
    if (tid == 0 && a.status && atomicCAS(a.status, 0, (int)SPINQ_ETIMEOUT) == 0) atomicExch(a.status + 1, kPromptSite);
    __syncthreads();
  }
  tc_fence_after();
  if (warp == 9) tmem_dealloc(*tmem_slot, 512);
}

// fp16 [tokens] rows of H heads of D values, ld elements apart, in boxes of 64
// values x heads x tokens.
bool encode_heads(EncodeTiledFn enc, CUtensorMap* map, const void* p, int64_t tokens, int64_t H, int D, int64_t ld,
                  int heads, int rows) {
  const cuuint64_t dim[3] = {(cuuint64_t)D, (cuuint64_t)H, (cuuint64_t)tokens};
  const cuuint64_t str[2] = {(cuuint64_t)D * 2, (cuuint64_t)ld * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)rows};
  const cuuint32_t one[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(p), dim, str, box, one,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool WIN>
cudaError_t launch_t(const PromptArgs& a, cudaStream_t stream) {
  using C = PromptCfg<D>;
  EncodeTiledFn enc = get_encode_fn();
  if (!enc) return cudaErrorNotSupported;
  PromptParams p{};
  p.G = (int)(a.Hq / a.Hkv);
  p.tpt = 128 / p.G;
  CUtensorMap mq, mk, mv, mks, mvs;
  // without any key no K or V tile is copied: their maps only have to be valid
  const bool keys = a.total_k > 0;
  if (!encode_heads(enc, &mq, a.q, a.total_q, a.Hq, D, a.ldq, p.G, p.tpt) ||
      !encode_heads(enc, &mk, keys ? a.k : a.q, keys ? a.total_k : 1, keys ? a.Hkv : 1, D, keys ? a.ldk : D, 1, 128) ||
      !encode_heads(enc, &mv, keys ? a.v : a.q, keys ? a.total_k : 1, keys ? a.Hkv : 1, D, keys ? a.ldv : D, 1, 128))
    return cudaErrorNotSupported;
  mks = mk, mvs = mv;
  if (WIN && keys && (!encode_heads(enc, &mks, a.k, a.total_k, a.Hkv, D, a.ldk, 1, kSinkRows) ||
                      !encode_heads(enc, &mvs, a.v, a.total_k, a.Hkv, D, a.ldv, 1, kSinkRows)))
    return cudaErrorNotSupported;
  p.cu_q = a.cu_q;
  p.cu_k = a.cu_k;
  p.out = static_cast<__half*>(a.out);
  p.total_q = a.total_q;
  p.total_k = a.total_k;
  p.Hq = (int)a.Hq;
  p.Hkv = (int)a.Hkv;
  p.batch = (int)a.batch;
  p.causal = a.causal;
  p.window = (int)(a.window < INT32_MAX ? a.window : INT32_MAX);
  p.sinks = (int)(a.sinks < INT32_MAX ? a.sinks : INT32_MAX);
  // a negative scale is |scale| times negated queries; zero makes every
  // weight equal, as any product too small to move 2^x does
  p.scale_log2 = fmaxf(fabsf(a.scale) * kAttnLog2e, 1e-30f);
  p.idesc_qk = umma_idesc_f16_f32(128, 128, a.scale < 0.f);
  p.status = device_status_word();
  p.debug_stall = take_debug_stall() ? 1 : 0;
  p.tiles = (int)((a.max_q + 2 * p.tpt - 1) / (2 * p.tpt));
  const int64_t items = (int64_t)p.tiles * a.Hkv * a.batch;
  if (items > INT32_MAX) return cudaErrorNotSupported;
  int per_sm = 0;
  cudaError_t e = prepare_launch_tmem(prompt_tc_kernel<D, WIN>, kPromptThreads, C::BYTES, 512, &per_sm);
  if (e != cudaSuccess) return e;
  e = launch_pdl(prompt_tc_kernel<D, WIN>, dim3((unsigned)items), dim3(kPromptThreads),
                 C::BYTES, stream, 1, mq, mk, mv, mks, mvs, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t set_wait_limit_prompt(uint64_t ns) { return cudaMemcpyToSymbol(g_prompt_wait_ns, &ns, sizeof(ns)); }

cudaError_t launch_prompt_attention(const PromptArgs& a, cudaStream_t stream) {
  if (a.D == 128) return a.window > 0 ? launch_t<128, true>(a, stream) : launch_t<128, false>(a, stream);
  if (a.D == 64) return a.window > 0 ? launch_t<64, true>(a, stream) : launch_t<64, false>(a, stream);
  return cudaErrorNotSupported;
}

}  // namespace spinq
