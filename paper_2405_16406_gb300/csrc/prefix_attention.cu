// prefix_attention.cu -- spinq_prefix_attention_kv4: one query per (sequence,
// head) over a prefix that every sequence shares and the sequence's own
// tokens, both in the paged 4-bit cache.
//
//   s_t = scale q . k_t,  k_t = alpha_t u_t + beta_t
//   o   = sum_t softmax_t(s) v_t,  v_t = alpha'_t u'_t + beta'_t
//
// The codes meet the tensor core as the whole numbers u - 8, exact in fp16, and the
// weights are those that the codes have in the output, w = 2^(s + log2 alpha' - M)
// with M the running maximum of s + log2 alpha' (base 2):
//   s_t = (scale alpha_t) (q . (u_t - 8)) + scale (beta_t + 8 alpha_t) sum_d q_d
//   o   = [ sum_t w_t (u'_t - 8) + sum_t w_t (8 + beta'_t / alpha'_t) ] / sum_t w_t / alpha'_t
// so the only rounding before the output is that of w to fp16, on codes about
// their middle (the two other sums stay in fp32); the own tokens and a prefix with few
// sequences carry w as two fp16 parts.  The token that weighs most has w near 1 (M moves
// only when a token outgrows it by 2^8): a large alpha' of a token without weight in the softmax
// does not push the others' w below fp16's range, as one scale for scores and one for
// alpha' apart would.
//
// Two or three kernels on the stream:
//   prefix_tc_kernel   the shared tokens, once for all sequences: an MMA's 128
//     rows are floor(128 / G) sequences of the G heads of a kv head, two such
//     tiles per CTA, the prefix split over the grid's z.  S = Q K^T and O += P V on
//     the 5th-generation tensor core as in the prompt kernel; four warps
//     expand the pages' codes into the operand tiles.
//     Bound: the softmax.  128 tokens for both tiles are 2052 cycles of MMAs and
//     about 6000 in all: two warps per scheduler, whose packed fp32 work is about 2800, and
//     waits between.  32768 tokens, 256 sequences, 32 / 8 heads, D 128, on 128 SMs: 209
//     us with an empty join, 0.66 PFLOP/s.
//   own_tokens_kernel  each sequence's own tokens, beside the prefix kernel where it
//     leaves SMs: G heads are too few rows for those tiles, so mma.sync with the
//     tokens on the M side, codes copied as they are.  Bound: latency (256 sequences of
//     523 tokens on average, 154 MB: 47 us alone, 3.3 TB/s, half of the copy rate; issue is at
//     36 %): a warp has 8 steps there, behind a page look-up and a filled ring and before a join.
//     8 sequences of 30000 tokens, 277 MB: 73 us, 3.8 TB/s.  Where one CTA has all of a
//     sequence's own tokens it may also join them with the prefix's parts.
//   prefix_combine_kernel  else joins the parts (maximum, sum, o) in a fixed order.
#include <cuda_fp16.h>
#include <float.h>

#include "../../include/spinq.h"
#include "attn_tc.cuh"
#include "launch_util.h"
#include "spinq_internal.h"

namespace spinq {
namespace {

__device__ uint64_t g_prefix_wait_ns = kAttnWaitLimitNs;
constexpr int kPrefixSite = 32;    // wait site recorded on a time-out
// A row of values with a smaller scale (equal values have 0) counts as one of this scale, 2^-40:
// 15 steps of it, 2^-36, are nothing beside fp16's smallest step, 2^-24, and w stays
// above 2^-126 beside any alpha' up to 2^80.  (A scale that is not a number stays one.)
constexpr float kMinValueScale = 9.094947017729282e-13f;
__device__ __forceinline__ float value_scale(float x) { return x < kMinValueScale ? kMinValueScale : x; }
__device__ __forceinline__ float log2_of_scale(float x) {   // within 2^-22; no subnormal numbers come here
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float one_over_scale(float x) {   // within 2^-23
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

// Parts of the result: part p of row (b, head) is M and sum of w / alpha' at ml[p][row] and
// the weighted sum of the values at o[p][row][D] (not written where the sum is 0).
struct PrefixParams {
  PrefixArgs a;
  int G;
  int tps;         // sequences per tile of 128 rows
  int nsplit;      // parts of the prefix
  int nchunk;      // parts of the sequences' own tokens
  bool join;       // the own-tokens kernel joins the parts itself
  float* o;
  float2* ml;
  float scale_log2;
  int* status;
  int debug_stall;
};

__device__ __forceinline__ int64_t page_at(const PrefixArgs& a, const int32_t* table, int64_t t, int shift) {
  const int64_t page = __ldg(table + (t >> shift));
  return page < 0 ? 0 : (page >= a.num_pages ? a.num_pages - 1 : page);
}

// Eight codes of a word as fp16 pairs u - 8: (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ uint32_t code_pair(uint32_t x) {   // nibbles at bits 0 and 16
  const uint32_t m = (x & 0x000F000Fu) | 0x64006400u;         // 1024 + u
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&m), __half2half2(__ushort_as_half(0x6408)));   // 1032
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 code_pairs(uint32_t x) {
  return make_uint4(code_pair(x), code_pair(x >> 4), code_pair(x >> 8), code_pair(x >> 12));
}

constexpr int kMaxSplits = 160;   // parts of the prefix at most

// --------------------------------------------------------------- the prefix
template <int D>
struct PrefixCfg {
  static constexpr int TILE = 128 * D * 2;
  static constexpr int NSTG = 4;                         // operand tiles in flight
  static constexpr int NCOL = 4;                         // tiles of per-token numbers
  static constexpr int OFF_KV = 2 * TILE;
  // a tile's numbers: 64 pairs of tokens' score scales and offsets, 64 pairs of the factors
  // of the two sums, 64 pairs of log2 alpha'
  static constexpr int COL_V = 1024, COL_LOG = 2048, COL = 2560;
  static constexpr int OFF_COL = OFF_KV + NSTG * TILE;
  static constexpr int OFF_BAR = OFF_COL + NCOL * COL;   // q, full, free [NSTG], col [NCOL], s, p, o, drain [2]
  static constexpr int OFF_MISC = OFF_BAR + (2 * NSTG + NCOL + 9) * 8;
  static constexpr int OFF_X = OFF_MISC + 16;            // 256 floats: query sums, then exchanged values
  static constexpr int BYTES = OFF_X + 1024 + 1024;
  static_assert(BYTES <= 232448, "shared memory");
};
// four warpgroups: two of softmax with 184 registers a thread, one with the
// MMAs (56), one that expands the codes (88): 512 = 4 * 128, what the launch holds
constexpr int kPrefixThreads = 512;

// TWO: the weights as two fp16 parts, the second (what the first leaves) in the
// columns of S behind the first's, with a product of its own; one tile of rows.
template <int D, bool TWO>
__global__ void __launch_bounds__(kPrefixThreads, 1) prefix_tc_kernel(const PrefixParams p) {
  using C = PrefixCfg<D>;
  constexpr int NSTG = C::NSTG, NCOL = C::NCOL;
  const PrefixArgs& a = p.a;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* qbar = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* full = qbar + 1;
  uint64_t* free_ = full + NSTG;
  uint64_t* cbar = free_ + NSTG;   // per-token numbers of a tile written
  uint64_t* sbar = cbar + NCOL;
  uint64_t* pbar = sbar + 2;
  uint64_t* obar = pbar + 2;
  uint64_t* drain = obar + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  const int b0 = blockIdx.x * 2 * p.tps;
  constexpr int NROW = TWO ? 1 : 2;
  const int nrow = !TWO && b0 + p.tps < (int)a.B ? 2 : 1;   // tiles of rows
  if (tid == 0) {
    mbar_init(qbar, 8);
    for (int s = 0; s < NSTG; ++s) {
      mbar_init(&full[s], 4);
      mbar_init(&free_[s], nrow);
    }
    for (int s = 0; s < NCOL; ++s) mbar_init(&cbar[s], 4);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sbar[i], 1);
      mbar_init(&pbar[i], 8);
      mbar_init(&obar[i], 1);
      mbar_init(&drain[i], 1);
    }
    *abort_flag = 0;
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
  // In this order: own_tokens_kernel starts at the trigger and relies on the work before this kernel being done.
  pdl_wait();
  pdl_trigger();

  const int hk = blockIdx.y;
  const int ntiles = (int)((a.prefix_len + 127) / 128);
  const int j0 = (int)((int64_t)ntiles * blockIdx.z / p.nsplit), j1 = (int)((int64_t)ntiles * (blockIdx.z + 1) / p.nsplit);
  const int nt = j1 - j0;                              // tiles of 128 tokens of this part
  const uint32_t sb = smem_u32(smem);

  if (warp >= 12) {
    // ---------------- one thread per token of a tile: codes to operand rows
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;\n");
    const int t = tid & 127, shift = __ffs(a.page_size) - 1;
    constexpr int NW = D / 32;   // 16-byte pieces of a row of codes
    auto row_of = [&](int j) {   // index of this thread's token in the page arrays (clamped to the prefix)
      int64_t tok = (int64_t)j * 128 + t;
      if (tok >= a.prefix_len) tok = a.prefix_len - 1;
      return (page_at(a, a.prefix_table, tok, shift) * a.Hkv + hk) * a.page_size + (tok & (a.page_size - 1));
    };
    auto expand = [&](const uint4* w, int n) {   // into operand tile n of the ring
      uint8_t* dst = smem + C::OFF_KV + (n % NSTG) * C::TILE + t * 128;
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int ch = 4 * k + q;   // 16-byte chunk (8 values) of the row
          *reinterpret_cast<uint4*>(dst + (ch >> 3) * kAttnAtom + (((ch & 7) ^ (t & 7)) << 4)) = code_pairs(x[q]);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[n % NSTG]);
    };
    uint4 kw[NW], vw[NW];
    float4 sc = make_float4(0.f, 0.f, 0.f, 0.f);
    int64_t at = 0;
    auto load_k = [&](int j) {
      at = row_of(j);
      const uint4* src = reinterpret_cast<const uint4*>(a.k_codes + at * (D / 2));
#pragma unroll
      for (int k = 0; k < NW; ++k) kw[k] = __ldg(src + k);
      sc = __ldg(reinterpret_cast<const float4*>(a.scales) + at);
    };
    auto load_v = [&]() {
      const uint4* src = reinterpret_cast<const uint4*>(a.v_codes + at * (D / 2));
#pragma unroll
      for (int k = 0; k < NW; ++k) vw[k] = __ldg(src + k);
    };
    const int expand_n = p.debug_stall ? 0 : nt;   // a test of the time-outs expands nothing
    if (nt > 0) {
      load_k(j0);
      load_v();
    }
    for (int j = 0; j < expand_n; ++j) {
      const int n = 2 * j;
      if (n >= NSTG && !attn_wait_warp(&free_[n % NSTG], (uint32_t)(n / NSTG - 1) & 1u, abort_flag, g_prefix_wait_ns)) break;
      // the tile's numbers: slot j % NCOL was last read for tile j - NCOL,
      // whose V tile has been released by now (NSTG operand tiles = 2 tiles of tokens)
      const bool in = (int64_t)(j0 + j) * 128 + t < a.prefix_len;
      uint8_t* cols = smem + C::OFF_COL + (j % NCOL) * C::COL;
      float* col = reinterpret_cast<float*>(cols) + (t >> 1) * 4 + (t & 1);
      col[0] = in ? p.scale_log2 * sc.x : 0.f;
      col[2] = in ? p.scale_log2 * fmaf(8.f, sc.x, sc.y) : 0.f;
      const float va = in ? value_scale(sc.z) : 1.f, rv = one_over_scale(va);
      col[C::COL_V / 4] = rv;
      col[C::COL_V / 4 + 2] = in ? fmaf(rv, sc.w, 8.f) : 0.f;
      // (in the order of the lanes: pairs c of groups 2 k and 2 k + 1 of eight tokens in one load)
      const int to = (t & 64) + (t >> 4 & 3) * 16 + (t >> 1 & 3) * 4 + (t >> 3 & 1) * 2 + (t & 1);
      reinterpret_cast<float*>(cols + C::COL_LOG)[to] = log2_of_scale(va);
      __syncwarp();
      if (lane == 0) mbar_arrive(&cbar[j % NCOL]);
      expand(kw, n);
      if (j + 1 < nt) load_k(j0 + j + 1);
      if (n + 1 >= NSTG &&
          !attn_wait_warp(&free_[(n + 1) % NSTG], (uint32_t)((n + 1) / NSTG - 1) & 1u, abort_flag, g_prefix_wait_ns))
        break;
      expand(vw, n + 1);
      if (j + 1 < nt) load_v();
    }
  } else if (warp >= 8) {
    // ---------------- MMAs
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;\n");
    const int i = warp - 8;   // tile of rows whose MMAs this warp's thread issues
    if (i < nrow && nt > 0 && attn_elect()) {
      constexpr uint32_t idesc = umma_idesc_f16_f32(128, 128, false);
      bool ok = attn_wait(qbar, 0, abort_flag, g_prefix_wait_ns);
      const uint32_t q_lo = attn_desc_k(sb + i * C::TILE), k_lo = attn_desc_k(sb + C::OFF_KV),
                     v_lo = attn_desc_mn(sb + C::OFF_KV);
      int sk = 0, pk = 0;   // ring stage of the next tile to wait for, its phase
      auto wait_tile = [&]() {
        ok = attn_wait(&full[sk], pk, abort_flag, g_prefix_wait_ns);
        const int s = sk;
        if (++sk == NSTG) sk = 0, pk ^= 1;
        return s;
      };
      const int s0 = ok ? wait_tile() : 0;
      if (ok) {
        tc_fence_after();
        attn_mma_qk<D>(i * 128, q_lo, k_lo + s0 * (C::TILE >> 4), idesc);
        tc_commit(&sbar[i]);
        tc_commit(&free_[s0]);
      }
#pragma unroll 1
      for (int j = 0; ok && j < nt; ++j) {
        const int sv = wait_tile();
        if (!ok) break;
        const int sn = j + 1 < nt ? wait_tile() : -1;   // ahead of the weights, as in the prompt kernel
        if (!ok || !(ok = attn_wait(&pbar[i], (uint32_t)j & 1u, abort_flag, g_prefix_wait_ns))) break;
        tc_fence_after();
        attn_mma_pv<D>(256 + i * D, i * 128, v_lo + sv * (C::TILE >> 4), j > 0);
        if (TWO) attn_mma_pv<D>(256 + i * D, i * 128 + 64, v_lo + sv * (C::TILE >> 4), true);
        if (sn >= 0) {
          attn_mma_qk<D>(i * 128, q_lo, k_lo + sn * (C::TILE >> 4), idesc);
          tc_commit(&sbar[i]);
          tc_commit(&free_[sv]);
          tc_commit(&free_[sn]);
        } else {
          tc_commit(&obar[i]);
        }
      }
      tc_commit(&drain[i]);   // what is in flight finishes before tensor memory is given up
      mbar_wait_bounded(&drain[i], 0, kAttnWaitLimitNs);
    }
  } else {
    // ---------------- softmax: either warpgroup hf owns tokens 64 hf ..
    // 64 hf + 63 of both tiles, in turn.  What a tile's weights wait for beside the
    // tensor core is then half a row's arithmetic (32768 x 256, this kernel: 224 us with a
    // warpgroup per tile and whole rows, 204 us so).  Lane 4 g + c holds rows g, g + 8,
    // g + 16, g + 24 of its warp and tokens 8 k + 2 c, 8 k + 2 c + 1: the per-token numbers
    // are loaded for a quarter of the tokens and serve four rows.  With a row
    // per lane those loads, beside MMAs that take shared memory's full rate, were 2048 of
    // 4750 of its passes per 128 tokens (204 us; 200 us so).
    asm volatile("setmaxnreg.inc.sync.aligned.u32 184;\n");
    const int hf = warp >> 2, r = tid & 127, pair = 1 + (warp & 3);   // named barrier of this warp and warp ^ 4
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    float* xs = reinterpret_cast<float*>(smem + C::OFF_X);
    int64_t row[2];    // this thread's row of tile i among all rows, or -1
    bool work[2];      // the warp has a row of tile i at all
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int b = b0 + i * p.tps + r / p.G;
      row[i] = r < p.G * p.tps && b < (int)a.B ? (int64_t)b * a.Hq + hk * p.G + r % p.G : -1;
      work[i] = __any_sync(0xffffffffu, row[i] >= 0);
    }
    // The warp's rows of Q of tile hf, their pairs in the order of code_pairs,
    // and their sums: D / 8 lanes share a row, every load is under way at once.
    {
      constexpr int LPR = D / 8, RPL = 32 / LPR;   // lanes per row, rows per load
      const int64_t at = hf ? row[1] : row[0];
      const int ch = lane % LPR;
      uint4 w[32 / RPL];
#pragma unroll
      for (int k = 0; k < 32 / RPL; ++k) {
        const int64_t src = __shfl_sync(0xffffffffu, at, k * RPL + lane / LPR);
        w[k] = src >= 0 ? __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __half*>(a.q) + src * D) + ch)
                        : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int k = 0; k < 32 / RPL; ++k) {
        const uint32_t x[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[q]));
          sum += f.x + f.y;
        }
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const int rr = (warp & 3) * 32 + k * RPL + lane / LPR;
        if (ch == 0) xs[hf * 128 + rr] = sum;
        *reinterpret_cast<uint4*>(smem + hf * C::TILE + (ch >> 3) * kAttnAtom + rr * 128 + (((ch & 7) ^ (rr & 7)) << 4)) =
            make_uint4(__byte_perm(x[0], x[2], 0x5410), __byte_perm(x[0], x[2], 0x7632), __byte_perm(x[1], x[3], 0x5410),
                       __byte_perm(x[1], x[3], 0x7632));
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(qbar);
    }
    named_bar_sync(pair, 64);   // the pair's warps hold the sums of tiles 0 and 1
    const int g = lane >> 2, c = lane & 3;
    float qs[2][4];   // of rows 8 e + g of the warp
#pragma unroll
    for (int e = 0; e < 4; ++e) qs[0][e] = xs[(warp & 3) * 32 + 8 * e + g], qs[1][e] = xs[128 + (warp & 3) * 32 + 8 * e + g];
    named_bar_sync(pair, 64);   // both have read them: the slots serve the exchanges from here on
    xs += (warp & 3) * 32;
    // a value of each of the lane's four rows (the same in a quad) as one per lane, of row 8 c + g
    auto gather = [&](const float (&v)[4]) { return c < 2 ? (c == 0 ? v[0] : v[1]) : (c == 2 ? v[2] : v[3]); };
    float m[2][4], l[2][4], z[2][4];   // M; l, z: of this lane's tokens
#pragma unroll
    for (int e = 0; e < 4; ++e) m[0][e] = m[1][e] = -INFINITY, l[0][e] = l[1][e] = z[0][e] = z[1][e] = 0.f;
    bool ok = true;
#pragma unroll 1
    for (int j = 0; ok && j < nt; ++j)
#pragma unroll
      for (int i = 0; i < NROW; ++i) {
        if (i >= nrow || !ok) continue;
        const uint32_t st = tmem + i * 128 + lanes;
        if (i == 0) ok = attn_wait_warp(&cbar[j % NCOL], (uint32_t)(j / NCOL) & 1u, abort_flag, g_prefix_wait_ns);
        if (!work[i]) {   // the same for both warps of a pair
          ok = ok && attn_wait_warp(&sbar[i], (uint32_t)j & 1u, abort_flag, g_prefix_wait_ns);
          ok = !attn_pair_or(!ok, pair);
          if (!ok) continue;
        } else {
          // the numbers of tokens 8 k + 2 c, 8 k + 2 c + 1: scale and offset of the scores,
          // k = 0 .. 7, then the factors of the sums; the latter are loaded as the former are used
          const uint8_t* cols = smem + C::OFF_COL + (j % NCOL) * C::COL;
          const ulonglong2* ab = reinterpret_cast<const ulonglong2*>(cols + hf * 512) + c;
          const ulonglong2* fv = reinterpret_cast<const ulonglong2*>(cols + C::COL_V + hf * 512) + c;
          const ulonglong2* la = reinterpret_cast<const ulonglong2*>(cols + C::COL_LOG + hf * 256) + c;
          ulonglong2 f[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) f[k] = ab[4 * k];
          ok = ok && attn_wait_warp(&sbar[i], (uint32_t)j & 1u, abort_flag, g_prefix_wait_ns);
          tc_fence_after();
          // (after a wait given up the columns are read all the same, in bounds, and discarded)
          uint32_t s[2][32];   // s[h][4 k + 2 e + x]: row 16 h + 8 e + g, token 8 k + 2 c + x
          tmem_ld_16x256b_x8(st + hf * 64, s[0]);
          tmem_ld_16x256b_x8(st + (16u << 16) + hf * 64, s[1]);
          tmem_ld_wait_all<32>(s[0]);
          tmem_ld_wait_all<32>(s[1]);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const ulonglong2 w = f[k], l2 = la[4 * (k >> 1)];
            const F2 lg = F2{k & 1 ? l2.y : l2.x};
            f[k] = fv[4 * k];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t* v = &s[e >> 1][4 * k + 2 * (e & 1)];
              float x, y;
              f2_split(f2_fma(f2_from_bits(v[0], v[1]), F2{w.x}, f2_fma(F2{w.y}, f2_make(qs[i][e], qs[i][e]), lg)), x, y);
              v[0] = __float_as_uint(x);
              v[1] = __float_as_uint(y);
            }
          }
          const int64_t left = a.prefix_len - (int64_t)(j0 + j) * 128 - hf * 64;
          if (left < 64) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
              for (int x = 0; x < 2; ++x)
                if (8 * k + 2 * c + x >= (int)left)
                  s[0][4 * k + x] = s[0][4 * k + 2 + x] = s[1][4 * k + x] = s[1][4 * k + 2 + x] = 0xFF800000u;   // -inf
          }
          float mx[4];
          bool grow = !ok;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t* v = &s[e >> 1][2 * (e & 1)];
            float p0 = fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1])), p1 = fmaxf(__uint_as_float(v[4]), __uint_as_float(v[5]));
#pragma unroll
            for (int k = 2; k < 8; k += 2) {
              p0 = attn_max3(p0, __uint_as_float(v[4 * k]), __uint_as_float(v[4 * k + 1]));
              p1 = attn_max3(p1, __uint_as_float(v[4 * k + 4]), __uint_as_float(v[4 * k + 5]));
            }
            mx[e] = fmaxf(p0, p1);
            grow |= mx[e] > m[i][e] + kAttnSlack;
          }
          // Seldom: a wait was given up, or M moves.  Also: both warps have read
          // their scores before either writes weights over them.
          if (attn_pair_or(grow, pair)) {
            ok = !attn_pair_or(!ok, pair);
            if (!ok) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 1));
              mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
            }
            const float other = attn_pair_swap(xs, gather(mx), hf, lane, pair);
            float fr[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float t = fmaxf(mx[e], __shfl_sync(0xffffffffu, other, (lane & 28) + e));
              const float mn = t > m[i][e] + kAttnSlack ? t : m[i][e];
              fr[e] = m[i][e] == -INFINITY ? 0.f : attn_exp2(m[i][e] - mn);
              m[i][e] = mn;
              l[i][e] *= fr[e];
              z[i][e] *= fr[e];
            }
            // the scores' barrier says that every product issued before them is done
            if (j > 0) attn_rescale_rows<D / 2>(tmem + 256 + i * D + hf * (D / 2) + lanes, fr);
          }
          F2 of2[4], sum[4], zs[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float off = m[i][e] == -INFINITY ? 0.f : -m[i][e];
            of2[e] = f2_make(off, off);
            sum[e] = f2_make(l[i][e], 0.f);
            zs[e] = f2_make(z[i][e], 0.f);
          }
          uint32_t rest[2][16];   // second parts
#pragma unroll
          for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t* v = &s[e >> 1][4 * k + 2 * (e & 1)];
              float x, y;
              f2_split(f2_add(f2_from_bits(v[0], v[1]), of2[e]), x, y);
              const F2 ex = f2_make(attn_exp2(x), attn_exp2(y));
              sum[e] = f2_fma(ex, F2{f[k].x}, sum[e]);
              zs[e] = f2_fma(ex, F2{f[k].y}, zs[e]);
              f2_split(ex, x, y);
              const uint32_t h = pack_half2_bits(x, y);
              s[e >> 1][2 * k + (e & 1)] = h;   // 32-bit column 4 k + c of this half's P
              if (TWO) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
                rest[e >> 1][2 * k + (e & 1)] = pack_half2_bits(x - f.x, y - f.y);
              }
            }
          if (TWO) {
            tmem_st_16x128b_x8(st + 64 + hf * 32, rest[0]);
            tmem_st_16x128b_x8(st + (16u << 16) + 64 + hf * 32, rest[1]);
          }
          tmem_st_16x128b_x8(st + hf * 32, s[0]);
          tmem_st_16x128b_x8(st + (16u << 16) + hf * 32, s[1]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x, y;
            f2_split(sum[e], x, y);
            l[i][e] = x + y;
            f2_split(zs[e], x, y);
            z[i][e] = x + y;
          }
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pbar[i]);
      }
#pragma unroll
    for (int i = 0; i < NROW; ++i) {
      if (!ok || i >= nrow || !work[i]) continue;
      if (nt > 0) ok = attn_wait_warp(&obar[i], 0, abort_flag, g_prefix_wait_ns);
      ok = !attn_pair_or(!ok, pair);
      if (!ok) continue;
      tc_fence_after();
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int w = 1; w < 4; w <<= 1) {
          l[i][e] += __shfl_xor_sync(0xffffffffu, l[i][e], w);
          z[i][e] += __shfl_xor_sync(0xffffffffu, z[i][e], w);
        }
      // of row 8 c + g, and from there to the row's lane
      float mi = gather(m[i]), li = gather(l[i]), zi = gather(z[i]);
      li += attn_pair_swap(xs, li, hf, lane, pair);
      zi += attn_pair_swap(xs, zi, hf, lane, pair);
      const int from = 4 * (lane & 7) + (lane >> 3);
      mi = __shfl_sync(0xffffffffu, mi, from);
      li = __shfl_sync(0xffffffffu, li, from);
      zi = __shfl_sync(0xffffffffu, zi, from);
      const int64_t rows = a.B * a.Hq, mine = row[i];
      if (mine >= 0 && hf == 0) p.ml[(int64_t)blockIdx.z * rows + mine] = make_float2(mi, li);
      if (nt == 0) continue;
      // D / 4 values of each row at a time through the tile's Q rows, which no
      // product reads any more, so that a row's values leave in one run
      const int64_t at = mine >= 0 ? ((int64_t)blockIdx.z * rows + mine) * D : -1;
      uint8_t* buf = smem + i * C::TILE + (warp & 7) * (C::TILE / 8);
      uint32_t o[D / 2];
#pragma unroll
      for (int c = 0; c < D / 2; c += 32) tmem_ld_32x32b_x32(tmem + 256 + i * D + hf * (D / 2) + lanes + c, o + c);
      tmem_ld_wait_all<D / 2>(o);
#pragma unroll
      for (int part = 0; part < D / 2; part += D / 4) {
        __syncwarp();
#pragma unroll
        for (int e = 0; e < D / 4; e += 8) {   // column 0, 1, .. of eight holds value 0, 4, 1, 5, 2, 6, 3, 7
          float v[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] = __uint_as_float(o[part + e + x]) + zi;
          uint8_t* dst = buf + lane * D;
          *reinterpret_cast<float4*>(dst + (((e >> 2) ^ (lane & (D / 16 - 1))) << 4)) = make_float4(v[0], v[2], v[4], v[6]);
          *reinterpret_cast<float4*>(dst + (((e >> 2) + 1 ^ (lane & (D / 16 - 1))) << 4)) =
              make_float4(v[1], v[3], v[5], v[7]);
        }
        __syncwarp();
        constexpr int LPR = D / 16, RPL = 32 / LPR;   // lanes per row, rows per store
#pragma unroll
        for (int k = 0; k < 32 / RPL; ++k) {
          const int rr = k * RPL + lane / LPR, ch = lane % LPR;
          const int64_t to = __shfl_sync(0xffffffffu, at, rr);
          const float4 v = *reinterpret_cast<const float4*>(buf + rr * D + ((ch ^ (rr & (D / 16 - 1))) << 4));
          if (to >= 0) *reinterpret_cast<float4*>(p.o + to + hf * (D / 2) + part + ch * 4) = v;
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (tid == 0 && p.status && atomicCAS(p.status, 0, (int)SPINQ_ETIMEOUT) == 0) atomicExch(p.status + 1, kPrefixSite);
  }
  tc_fence_after();
  if (warp == 8) tmem_dealloc(*tmem_slot, 512);
}

// ------------------------------------------------- the sequences' own tokens
constexpr int kOwnWarps = 4;

__device__ __forceinline__ uint32_t own_transpose(uint32_t x) {   // 8x8 fp16 transpose over the warp
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
  return y;
}

constexpr int kOwnStages = 4;

__device__ __forceinline__ void own_copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}

// A warp's ring of stages: 16 tokens' key rows, value rows (D/2 bytes each) and
// scales.  Key rows lie as in the page (a fragment load covers eight whole rows);
// a fragment load of the values takes 8 or 4 bytes of rows 0, 2, 4, 6 (or 1, 3,
// ..), so their 16-byte pieces are moved about to fall in different banks.
template <int D>
struct OwnRing {
  static constexpr int KB = 16 * (D / 2), STAGE = 2 * KB + 256, WARP = kOwnStages * STAGE;
  static constexpr int CPR = D / 32;   // 16-byte pieces of a row
  static __device__ __forceinline__ int value_at(int row, int piece) {   // byte offset of a value row's piece
    if (D == 128) {
      const int pair = row >> 1;
      return pair * 128 + (((row ^ pair) & 1) << 6) + ((piece ^ (pair & 2)) << 4);
    }
    return row * 32 + ((piece ^ ((row >> 2) & 1)) << 4);
  }
};

// grid (chunk, kv head x group of 8 query heads, sequence).  A warp takes
// steps of 16 tokens, which lie in one page, so its rows of codes are one run of
// memory, copied three steps ahead into the warp's ring.  Fragments of lane
// 4 g + c: key rows g and g + 8, bytes [c D/8, (c+1) D/8); value rows 2c, 2c+1, 2c+8,
// 2c+9, bytes [g D/16, (g+1) D/16).  Scores: tokens on M, heads on N; values:
// head_dim on M, tokens on K, heads on N.
template <int D>
__global__ void __launch_bounds__(kOwnWarps * 32, 4) own_tokens_kernel(const PrefixParams p, int hgroups, int chunk_len) {
  constexpr int KW = D / 32, VW = D / 64, NM = D / 16;
  const PrefixArgs& a = p.a;
  using Ring = OwnRing<D>;
  __shared__ __align__(16) uint8_t ring_s[kOwnWarps][Ring::WARP];   // after the loop: float o [8][D]
  static_assert(8 * D * 4 <= Ring::WARP, "the output fits in the ring");
  __shared__ float m_s[kOwnWarps][8], l_s[kOwnWarps][8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  const int hk = blockIdx.y / hgroups, hg = blockIdx.y % hgroups, b = blockIdx.z;
  const int heads = min(8, p.G - 8 * hg);   // query heads of this CTA
  // Behind a prefix this kernel starts beside it, on the SMs that it leaves: the
  // prefix kernel lets it start once all its CTAs have seen the end of the work before.
  if (p.nsplit == 0) pdl_wait();
  pdl_trigger();
  const int64_t cap = a.table_width * a.page_size;
  int64_t len = a.lens[b];
  len = len < 0 ? 0 : (len > cap ? cap : len);
  const int t0 = (int)min((int64_t)blockIdx.x * chunk_len, len), t1 = (int)min((int64_t)t0 + chunk_len, len);
  const int steps = (t1 - t0 + 15) / 16;
  const int nstep = steps > warp ? (steps - warp + kOwnWarps - 1) / kOwnWarps : 0;
  const int shift = __ffs(a.page_size) - 1;
  const int32_t* table = a.table + (int64_t)b * a.table_width;
  const int64_t row0 = (int64_t)b * a.Hq + hk * p.G + 8 * hg;

  // query fragments of head g (k order as the codes come), their sums.  A key
  // code is masked out of its word in place: as fp16 bits the nibbles at bits 0 and 16
  // are u 2^-24, those at bits 4 and 20 are 16 u 2^-24, both exact operands; each
  // kind has a product of its own, the latter's is divided by 16 in fp32.
  uint32_t qb[KW][4];
  float qs = 0.f;
  {
    const __half* qh = reinterpret_cast<const __half*>(a.q) + (row0 + (g < heads ? g : 0)) * D + c * (D / 4);
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      uint4 x = __ldg(reinterpret_cast<const uint4*>(qh + 8 * w));
      if (g >= heads) x = make_uint4(0, 0, 0, 0);
      const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&xs[q]));
        qs += f.x + f.y;
      }
      qb[w][0] = __byte_perm(x.x, x.z, 0x5410);
      qb[w][1] = __byte_perm(x.y, x.w, 0x5410);
      qb[w][2] = __byte_perm(x.x, x.z, 0x7632);
      qb[w][3] = __byte_perm(x.y, x.w, 0x7632);
    }
    qs += __shfl_xor_sync(0xffffffffu, qs, 1);
    qs += __shfl_xor_sync(0xffffffffu, qs, 2);
  }
  const float qsk[2] = {p.scale_log2 * __shfl_sync(0xffffffffu, qs, 8 * c),
                        p.scale_log2 * __shfl_sync(0xffffffffu, qs, 8 * c + 4)};
  const float ks24 = p.scale_log2 * 16777216.f;

  // Lane n holds the place in the page arrays of the warp's step 32 b + n (of
  // head hk, in tokens): one look-up for 32 steps.
  int64_t place = 0;
  const uint32_t ring = smem_u32(ring_s[warp]);
  auto issue = [&](int i) {   // copies of step i (an empty group past the end keeps the count)
    if (i < nstep) {
      if ((i & 31) == 0) {
        if (i + lane < nstep) {
          const int t = t0 + 16 * (warp + kOwnWarps * (i + lane));   // chunks start at multiples of 16
          place = (page_at(a, table, t, shift) * a.Hkv + hk) * a.page_size + (t & (a.page_size - 1));
        }
      }
      const int64_t at = __shfl_sync(0xffffffffu, place, i & 31);
      const uint32_t st = ring + (uint32_t)(i % kOwnStages) * Ring::STAGE;
      const uint8_t* kr = a.k_codes + at * (D / 2);
      const uint8_t* vr = a.v_codes + at * (D / 2);
#pragma unroll
      for (int n = 0; n < D / 64; ++n) {
        const int piece = lane + 32 * n;
        own_copy16(st + piece * 16, kr + piece * 16);
        own_copy16(st + Ring::KB + Ring::value_at(piece / Ring::CPR, piece % Ring::CPR), vr + piece * 16);
      }
      if (lane < 16) own_copy16(st + 2 * Ring::KB + lane * 16, a.scales + (at + lane) * 4);
    }
    asm volatile("cp.async.commit_group;\n" ::: "memory");
  };

  float o[NM][4];
#pragma unroll
  for (int mu = 0; mu < NM; ++mu) o[mu][0] = o[mu][1] = o[mu][2] = o[mu][3] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, off[2] = {0.f, 0.f}, l[2] = {0.f, 0.f}, z[2] = {0.f, 0.f};   // m: M
#pragma unroll
  for (int i = 0; i < kOwnStages - 1; ++i) issue(i);
  for (int i = 0; i < nstep; ++i) {
    asm volatile("cp.async.wait_group %0;\n" ::"n"(kOwnStages - 2) : "memory");
    __syncwarp();   // step i has landed for every lane, and step i - 1's stage has been read
    issue(i + kOwnStages - 1);
    const uint8_t* st = ring_s[warp] + (i % kOwnStages) * Ring::STAGE;
    struct {
      uint32_t k[2][KW], v[4][VW];
      float4 sc[2];
    } x;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint8_t* kr = st + (g + 8 * h) * (D / 2) + c * (D / 8);
      if constexpr (KW == 4) {
        const uint4 w = *reinterpret_cast<const uint4*>(kr);
        x.k[h][0] = w.x, x.k[h][1] = w.y, x.k[h][2] = w.z, x.k[h][3] = w.w;
      } else {
        const uint2 w = *reinterpret_cast<const uint2*>(kr);
        x.k[h][0] = w.x, x.k[h][1] = w.y;
      }
      x.sc[h] = *reinterpret_cast<const float4*>(st + 2 * Ring::KB + (g + 8 * h) * 16);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = 8 * (q >> 1) + 2 * c + (q & 1);
      const uint8_t* vr = st + Ring::KB + Ring::value_at(row, g * (D / 16) / 16) + g * (D / 16) % 16;
      if constexpr (VW == 2) {
        const uint2 w = *reinterpret_cast<const uint2*>(vr);
        x.v[q][0] = w.x, x.v[q][1] = w.y;
      } else {
        x.v[q][0] = *reinterpret_cast<const uint32_t*>(vr);
      }
    }
    float sa[4] = {0.f, 0.f, 0.f, 0.f}, s16[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const uint32_t x0 = x.k[0][w], x1 = x.k[1][w], y0 = x0 >> 8, y1 = x1 >> 8;
      const uint32_t a0[4] = {x0 & 0x000F000Fu, x1 & 0x000F000Fu, y0 & 0x000F000Fu, y1 & 0x000F000Fu};
      const uint32_t a1[4] = {x0 & 0x00F000F0u, x1 & 0x00F000F0u, y0 & 0x00F000F0u, y1 & 0x00F000F0u};
      mma_16816_f16_f32_acc(sa, a0, qb[w][0], qb[w][1]);
      mma_16816_f16_f32_acc(s16, a1, qb[w][2], qb[w][3]);
    }
    // s + log2 alpha' (base 2) of tokens g, g + 8 for heads 2c, 2c + 1; tokens past the
    // chunk (their slots may hold anything) get -inf and factors 0
    float t[2][2], rv[2], vz[2];
    const int left = t1 - (t0 + 16 * (warp + kOwnWarps * i));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float ka = ks24 * x.sc[h].x;
      const float va = value_scale(x.sc[h].z), la = log2_of_scale(va);
      rv[h] = one_over_scale(va);
      vz[h] = fmaf(rv[h], x.sc[h].w, 8.f);
#pragma unroll
      for (int e = 0; e < 2; ++e) t[h][e] = fmaf(ka, fmaf(0.0625f, s16[2 * h + e], sa[2 * h + e]), fmaf(x.sc[h].y, qsk[e], la));
    }
    if (left < 16) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (g + 8 * h >= left) t[h][0] = t[h][1] = -INFINITY, rv[h] = vz[h] = 0.f;
    }
    const float mx0 = fmaxf(t[0][0], t[1][0]), mx1 = fmaxf(t[0][1], t[1][1]);
    if (__any_sync(0xffffffffu, mx0 > m[0] + kAttnSlack || mx1 > m[1] + kAttnSlack)) {
      float mx[2] = {mx0, mx1};
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) {
        mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], w));
        mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], w));
      }
      float f[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float mn = mx[e] > m[e] + kAttnSlack ? mx[e] : m[e];
        const float to = mn == -INFINITY ? 0.f : mn;
        f[e] = m[e] == -INFINITY ? 0.f : attn_exp2(off[e] - to);
        m[e] = mn;
        off[e] = to;
        l[e] *= f[e];
        z[e] *= f[e];
      }
#pragma unroll
      for (int mu = 0; mu < NM; ++mu) {
        o[mu][0] *= f[0], o[mu][2] *= f[0];
        o[mu][1] *= f[1], o[mu][3] *= f[1];
      }
    }
    float w[2][2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        w[h][e] = attn_exp2(t[h][e] - off[e]);
        l[e] = fmaf(w[h][e], rv[h], l[e]);
        z[e] = fmaf(w[h][e], vz[h], z[e]);
      }
    // the weights as two fp16 parts, the second what the first leaves: with one part the
    // few weights that carry a short sequence's row would all but double its error
    const uint32_t h0 = pack_half2_bits(w[0][0], w[0][1]), h1 = pack_half2_bits(w[1][0], w[1][1]);
    const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&h0)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&h1));
    const uint32_t pb0 = own_transpose(h0), pb1 = own_transpose(h1);
    const uint32_t pc0 = own_transpose(pack_half2_bits(w[0][0] - f0.x, w[0][1] - f0.y));
    const uint32_t pc1 = own_transpose(pack_half2_bits(w[1][0] - f1.x, w[1][1] - f1.y));
#pragma unroll
    for (int vw = 0; vw < VW; ++vw)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        // two bytes of two tokens' rows: one dimension of both in a pair
        const uint32_t xa = __byte_perm(x.v[0][vw], x.v[1][vw], q ? 0x7632 : 0x5410);
        const uint32_t xb = __byte_perm(x.v[2][vw], x.v[3][vw], q ? 0x7632 : 0x5410);
        const uint4 ya = code_pairs(xa), yb = code_pairs(xb);
        const uint32_t a0[4] = {ya.x, ya.y, yb.x, yb.y}, a1[4] = {ya.z, ya.w, yb.z, yb.w};
        mma_16816_f16_f32_acc(o[4 * vw + 2 * q], a0, pb0, pb1);
        mma_16816_f16_f32_acc(o[4 * vw + 2 * q + 1], a1, pb0, pb1);
        mma_16816_f16_f32_acc(o[4 * vw + 2 * q], a0, pc0, pc1);
        mma_16816_f16_f32_acc(o[4 * vw + 2 * q + 1], a1, pc0, pc1);
      }
  }
  // join the lanes' shares, then the warps
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int w = 4; w < 32; w <<= 1) {
      l[e] += __shfl_xor_sync(0xffffffffu, l[e], w);
      z[e] += __shfl_xor_sync(0xffffffffu, z[e], w);
    }
  asm volatile("cp.async.wait_group 0;\n" ::: "memory");
  __syncwarp();   // the ring is free
  float* o_w = reinterpret_cast<float*>(ring_s[warp]);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int h = 2 * c + e;
#pragma unroll
    for (int mu = 0; mu < NM; ++mu) {
      o_w[h * D + g * (D / 8) + 2 * mu] = o[mu][e] + z[e];
      o_w[h * D + g * (D / 8) + 2 * mu + 1] = o[mu][2 + e] + z[e];
    }
    if (g == 0) {
      m_s[warp][h] = m[e];
      l_s[warp][h] = l[e];
    }
  }
  __syncthreads();
  const int64_t rows = a.B * a.Hq, part = (int64_t)p.nsplit + blockIdx.x;
  if (!p.join) {
    for (int e = threadIdx.x; e < heads * D; e += kOwnWarps * 32) {
      const int h = e / D, d = e % D;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kOwnWarps; ++w) M = fmaxf(M, m_s[w][h]);
      float val = 0.f, ls = 0.f;
#pragma unroll
      for (int w = 0; w < kOwnWarps; ++w) {
        const float f = l_s[w][h] != 0.f ? attn_exp2(m_s[w][h] - M) : 0.f;
        val = fmaf(f, reinterpret_cast<const float*>(ring_s[w])[h * D + d], val);
        ls = fmaf(f, l_s[w][h], ls);
      }
      p.o[(part * rows + row0 + h) * D + d] = val;
      if (d == 0) p.ml[part * rows + row0 + h] = make_float2(M, ls);
    }
    // one CTA stays until the prefix's parts are written, and with it the grid that the
    // combine kernel waits for
    if (p.nsplit > 0 && blockIdx.x == gridDim.x - 1 && blockIdx.y == gridDim.y - 1 && blockIdx.z == gridDim.z - 1) pdl_wait();
    return;
  }
  if (p.nsplit > 0) pdl_wait();   // the prefix's parts
  // The only part of these rows' own tokens: joined with the prefix's here.
  // f_s[h][0 .. 3] the warps' factors, then the prefix parts', all over the sum.
  __shared__ float f_s[8][kOwnWarps + kMaxSplits];
  for (int h = warp; h < heads; h += kOwnWarps) {
    const float2* ml = p.ml + row0 + h;
    float M = -INFINITY, sum = 0.f;
    for (int q = lane; q < kOwnWarps + p.nsplit; q += 32) {
      const float2 x = q < kOwnWarps ? make_float2(m_s[q][h], l_s[q][h]) : ml[(q - kOwnWarps) * rows];
      if (x.y != 0.f) M = fmaxf(M, x.x);
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, w));
    for (int q = lane; q < kOwnWarps + p.nsplit; q += 32) {
      const float2 x = q < kOwnWarps ? make_float2(m_s[q][h], l_s[q][h]) : ml[(q - kOwnWarps) * rows];
      const float f = x.y != 0.f ? attn_exp2(x.x - M) : 0.f;   // (a sum that is not a number stays one)
      f_s[h][q] = f;
      sum = fmaf(f, x.y, sum);
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    __syncwarp();
    for (int q = lane; q < kOwnWarps + p.nsplit; q += 32) f_s[h][q] *= inv;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < heads * (D / 4); e += kOwnWarps * 32) {   // four values of a row
    const int h = e / (D / 4), d = e % (D / 4) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float f, const float4& x) {
      v.x = fmaf(f, x.x, v.x), v.y = fmaf(f, x.y, v.y), v.z = fmaf(f, x.z, v.z), v.w = fmaf(f, x.w, v.w);
    };
    const float* parts = p.o + (row0 + h) * D + d;
#pragma unroll 8
    for (int q = 0; q < p.nsplit; ++q) {   // a part without a sum was not written
      const float f = f_s[h][kOwnWarps + q];
      const float4 x = *reinterpret_cast<const float4*>(parts + q * rows * D);
      if (f != 0.f) add(f, x);
    }
#pragma unroll
    for (int w = 0; w < kOwnWarps; ++w)
      add(f_s[h][w], *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(ring_s[w]) + h * D + d));
    *reinterpret_cast<uint2*>(reinterpret_cast<__half*>(a.out) + (row0 + h) * D + d) =
        make_uint2(pack_half2_bits(v.x, v.y), pack_half2_bits(v.z, v.w));
  }
}

// One warp per row joins its parts, in their order.
template <int D>
__global__ void __launch_bounds__(128) prefix_combine_kernel(const PrefixParams p) {
  constexpr int DPL = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t rows = p.a.B * p.a.Hq, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  pdl_wait();
  pdl_trigger();
  if (row >= rows) return;
  const int parts = p.nsplit + p.nchunk;
  float M = -INFINITY;
  for (int i = lane; i < parts; i += 32) {
    const float2 x = p.ml[i * rows + row];
    if (x.y != 0.f) M = fmaxf(M, x.x);
  }
#pragma unroll
  for (int w = 16; w > 0; w >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, w));
  float o[DPL] = {}, l = 0.f;
  for (int i = 0; i < parts; ++i) {
    const float2 x = p.ml[i * rows + row];
    if (x.y == 0.f) continue;
    const float f = attn_exp2(x.x - M);
    l = fmaf(f, x.y, l);
    const float* s = p.o + (i * rows + row) * D + lane * DPL;
#pragma unroll
    for (int e = 0; e < DPL; ++e) o[e] = fmaf(f, s[e], o[e]);
  }
  const float inv = l != 0.f ? 1.f / l : 0.f;
  __half* out = reinterpret_cast<__half*>(p.a.out) + row * D + lane * DPL;
#pragma unroll
  for (int e = 0; e < DPL; e += 2) *reinterpret_cast<__half2*>(out + e) = __floats2half2_rn(o[e] * inv, o[e + 1] * inv);
}

// ------------------------------------------------------------------- plan
int row_blocks(const PrefixArgs& a) {
  const int64_t tps = 128 / (a.Hq / a.Hkv);
  return (int)((a.B + 2 * tps - 1) / (2 * tps));
}

int prefix_splits(const PrefixArgs& a) {
  if (a.prefix_len == 0) return 0;
  const int64_t tiles = (a.prefix_len + 127) / 128;
  int64_t n = device_sm_count() / (row_blocks(a) * a.Hkv);   // one CTA per SM
  n = n < 1 ? 1 : (n > kMaxSplits ? kMaxSplits : n);
  // no more than the longest part's length asks for: fewer parts to write and join, and
  // SMs for the own tokens (8191 x 64, 64 tiles: 34.4 us in 19 parts where 16 took 33.4)
  const int64_t longest = (tiles + n - 1) / n;
  return (int)((tiles + longest - 1) / longest);
}

// Parts of the sequences' own tokens.  One, where that gives every SM a CTA: the
// kernel then joins its rows with the prefix's parts itself.  Else so many that
// there are eight CTAs per SM, of 256 tokens at least.
int own_chunks(const PrefixArgs& a) {
  const int64_t cap = a.table_width * a.page_size, sms = device_sm_count();
  const int64_t ctas = a.B * a.Hkv * ((a.Hq / a.Hkv + 7) / 8);
  if (cap <= 256 || ctas >= sms) return 1;
  const int64_t n = 8 * sms / ctas, by_len = (cap + 255) / 256;
  return (int)(n > by_len ? by_len : n);
}

// Whether the own-tokens kernel joins the parts.  Not where the prefix kernel
// leaves an eighth of the SMs or more and there are several waves of own-tokens CTAs:
// those that join wait for the prefix in their slots, the others pass through the idle
// SMs beside it (32768 x 256, 128 of 152 SMs: 247 us with the own tokens after the
// prefix and joined there, 222 us so; few CTAs save the third kernel's 3 us).
bool own_joins(const PrefixArgs& a) {
  if (own_chunks(a) > 1) return false;
  const int64_t sms = device_sm_count(), ctas = a.B * a.Hkv * ((a.Hq / a.Hkv + 7) / 8);
  return prefix_splits(a) == 0 || 8 * row_blocks(a) * a.Hkv * prefix_splits(a) > 7 * sms || ctas <= 8 * sms;
}

int64_t align256(int64_t v) { return (v + 255) / 256 * 256; }

template <int D>
cudaError_t launch_t(const PrefixArgs& a, cudaStream_t stream) {
  PrefixParams p{};
  p.a = a;
  p.G = (int)(a.Hq / a.Hkv);
  p.tps = 128 / p.G;
  p.nsplit = prefix_splits(a);
  p.nchunk = own_chunks(a);
  p.join = own_joins(a);
  const int64_t rows = a.B * a.Hq;
  p.ml = static_cast<float2*>(a.workspace);
  p.o = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + align256((p.nsplit + (p.join ? 0 : p.nchunk)) * rows * 8));
  p.scale_log2 = a.scale * kAttnLog2e;
  p.status = device_status_word();
  cudaError_t e = cudaSuccess;
  if (p.nsplit > 0) {
    p.debug_stall = take_debug_stall() ? 1 : 0;
    int per_sm = 0;
    // A few rows may be carried by few weights, whose rounding then nearly doubles the
    // error of the whole output; many rows average it (0.00028 against 0.00021 of the
    // output's own rounding).  So one tile of rows takes second parts (1000 x 4: 9.6 us
    // and 0.00022 with one part, 10.1 us and 0.00021 with two; 24000 x 32: 32.9 us and 0.00027, 38.8 us and
    // 0.00021); two tiles do not, whose softmax bounds their kernel (8191 x 64: 34.2 us with one
    // part, 37.2 with two; 32768 x 256: 227 and 276 us, 0.00028 and 0.00022).
    auto kernel = a.B <= p.tps ? prefix_tc_kernel<D, true> : prefix_tc_kernel<D, false>;
    e = prepare_launch_tmem(kernel, kPrefixThreads, PrefixCfg<D>::BYTES, 512, &per_sm);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kernel, dim3((unsigned)row_blocks(a), (unsigned)a.Hkv, (unsigned)p.nsplit),
                   dim3(kPrefixThreads), PrefixCfg<D>::BYTES, stream, 1, p);
    if (e != cudaSuccess) return e;
  }
  {
    const int64_t cap = a.table_width * a.page_size;
    const int chunk = (int)(((cap + p.nchunk - 1) / p.nchunk + 15) / 16 * 16);
    const int hgroups = (p.G + 7) / 8;
    e = launch_pdl(own_tokens_kernel<D>, dim3((unsigned)p.nchunk, (unsigned)(a.Hkv * hgroups), (unsigned)a.B),
                   dim3(kOwnWarps * 32), 0, stream, 1, p, hgroups, chunk);
    if (e != cudaSuccess || p.join) return e != cudaSuccess ? e : cudaGetLastError();
  }
  e = launch_pdl(prefix_combine_kernel<D>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, stream, 1, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t set_wait_limit_prefix(uint64_t ns) { return cudaMemcpyToSymbol(g_prefix_wait_ns, &ns, sizeof(ns)); }

int64_t prefix_attention_workspace(const PrefixArgs& a) {
  const int64_t parts = prefix_splits(a) + (own_joins(a) ? 0 : own_chunks(a)), rows = a.B * a.Hq;
  return align256(parts * rows * 8) + parts * rows * a.D * 4;
}

cudaError_t launch_prefix_attention(const PrefixArgs& a, cudaStream_t stream) {
  if (a.D == 128) return launch_t<128>(a, stream);
  if (a.D == 64) return launch_t<64>(a, stream);
  return cudaErrorNotSupported;
}

}  // namespace spinq
