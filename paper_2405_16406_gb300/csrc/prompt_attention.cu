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
// One CTA per (two such tiles, kv head, sequence).  S = Q K^T (128 x 128 fp32)
// and O (128 x D fp32) of both tiles fill tensor memory; P replaces S as fp16
// and is the A operand of O += P V straight from there.  Warp roles:
//  * warps 0-3 and 4-7: softmax of tile 0 and 1, one row per thread: running
//    maximum (base 2, moved only by more than 2^8, when the row's O is
//    rescaled) and sum in fp32 registers;
//  * warp 8: one thread copies Q, then the K and V tiles of 128 tokens into
//    a ring of stages by TMA (128-byte swizzle);
//  * warps 9 and 10: one thread each issues the MMAs of tile 0 and 1, PV then the
//    next QK.  An issue blocks while the tensor core is busy, and a wait on a
//    barrier costs 150 to 230 cycles beside MMAs that read shared memory at its full
//    rate: with one issuing thread for both tiles the tensor core idled
//    through those waits (4 x 4096: 484 us so, XXX with two);
//  * warp 11: zeroes the last V tile's rows past the sequence.
// Bound: the tensor core (4 D flops per visible pair of a query head and a
// key).
//
// A sequence's last V tile may hold rows of the next sequence or of no
// sequence: they meet weights 0, which is not enough if they are not finite, so they are
// zeroed; K's such rows only reach scores that the mask replaces.
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
  int Hq, G, tpt;       // tpt: queries per tile
  int tiles;            // pairs of tiles along the queries (the grid's x)
  bool causal;
  float scale_log2;     // |scale| log2 e
  uint32_t idesc_qk;
  int* status;
  int debug_stall;
};

template <int D>
struct PromptCfg {
  static constexpr int TILE = 128 * D * 2;               // bytes of a Q, K or V tile
  static constexpr int NSTG = D == 128 ? 5 : 8;
  static constexpr int OFF_KV = 2 * TILE;
  static constexpr int OFF_BAR = OFF_KV + NSTG * TILE;   // q, full[NSTG], free[NSTG], s[2], p[2], o[2], z[2], drain[2]
  static constexpr int OFF_MISC = OFF_BAR + (2 * NSTG + 11) * 8;
  static constexpr int BYTES = OFF_MISC + 16 + 1024;
  static_assert(BYTES <= 232448, "shared memory");
};
// three warpgroups: two of softmax with 216 registers a thread, one with the
// copies and the MMAs with 72; 2 * 216 + 72 = 3 * 168, what the launch holds
constexpr int kPromptThreads = 384;

template <int D>
__global__ void __launch_bounds__(kPromptThreads, 1)
    prompt_tc_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                     const __grid_constant__ CUtensorMap mv, const PromptParams a) {
  using C = PromptCfg<D>;
  constexpr int NSTG = C::NSTG;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* qbar = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* full = qbar + 1;
  uint64_t* free_ = full + NSTG;
  uint64_t* sbar = free_ + NSTG;   // scores of tile i written
  uint64_t* pbar = sbar + 2;       // weights of tile i written (4 warps)
  uint64_t* obar = pbar + 2;       // last product of tile i done
  uint64_t* zreq = obar + 2;       // the sequence's last V tile is in,
  uint64_t* zbar = zreq + 1;       // its rows past the sequence are zeroed
  uint64_t* drain = zbar + 1;      // every MMA of tile i done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  int* issued = reinterpret_cast<int*>(smem + C::OFF_MISC + 8);   // K and V tiles copied (0: Q neither)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    mbar_init(qbar, 1);
    for (int s = 0; s < NSTG; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&free_[s], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sbar[i], 1);
      mbar_init(&pbar[i], 4);
      mbar_init(&obar[i], 1);
      mbar_init(&drain[i], 1);
    }
    mbar_init(zreq, 1);
    mbar_init(zbar, 1);
    *abort_flag = 0;
    *issued = -1;
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

  // the sequence, and this CTA's two tiles of queries (the last positions,
  // which see the most keys, first)
  const int hk = blockIdx.y, b = blockIdx.z;
  const int64_t q0 = a.cu_q[b], k0 = a.cu_k[b];
  const int lq = (int)(min((int64_t)a.cu_q[b + 1], a.total_q) - q0);
  const int lk = max(0, (int)(min((int64_t)a.cu_k[b + 1], a.total_k) - k0));
  const int t0 = (a.tiles - 1 - (int)blockIdx.x) * 2 * a.tpt;
  // keys that tile i's last query sees
  int nk[2], nt[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int first = t0 + i * a.tpt, last = min(first + a.tpt, lq) - 1;
    nk[i] = first < lq ? (a.causal ? max(0, min(lk, last + 1 + lk - lq)) : lk) : 0;
    nt[i] = (nk[i] + 127) / 128;
  }
  const int ntile = max(nt[0], nt[1]);
  const uint32_t sb = smem_u32(smem);
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;\n");
    if (warp == 8) {
      // ---------------- copies
      if (lane == 0 && ntile > 0 && !a.debug_stall) {
        const uint32_t qbytes = (uint32_t)(a.G * a.tpt) * 128u * (D / 64) * 2u;
        mbar_arrive_expect_tx(qbar, qbytes);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int at = 0; at < D / 64; ++at)
            tma_load_3d(smem + i * C::TILE + at * kAttnAtom, &mq, qbar, at * 64, hk * a.G,
                        (int32_t)(q0 + t0 + i * a.tpt));
        *issued = 0;
        for (int n = 0; n < 2 * ntile; ++n) {
          const int s = n % NSTG;
          if (n >= NSTG && !attn_wait(&free_[s], (uint32_t)(n / NSTG - 1) & 1u, abort_flag, g_prompt_wait_ns)) break;
          mbar_arrive_expect_tx(&full[s], (uint32_t)C::TILE);
#pragma unroll
          for (int at = 0; at < D / 64; ++at)
            tma_load_3d(smem + C::OFF_KV + s * C::TILE + at * kAttnAtom, n & 1 ? &mv : &mk, &full[s], at * 64, hk,
                        (int32_t)(k0 + (n >> 1) * 128));
          *issued = n + 1;
        }
      }
    } else if (warp < 11) {
      // ---------------- MMAs of tile i, by one thread
      const int i = warp - 9, nti = i ? nt[1] : nt[0];
      if (ntile > 0 && attn_elect()) {
        bool ok = attn_wait(qbar, 0, abort_flag, g_prompt_wait_ns);
        const uint32_t q_lo = attn_desc_k(sb + i * C::TILE), k_lo = attn_desc_k(sb + C::OFF_KV),
                       v_lo = attn_desc_mn(sb + C::OFF_KV);
        int sk = 0, pk = 0;   // ring stage of the next K or V tile, its phase
        auto wait_tile = [&]() {
          ok = attn_wait(&full[sk], pk, abort_flag, g_prompt_wait_ns);
          const int s = sk;
          if (++sk == NSTG) sk = 0, pk ^= 1;
          return s;
        };
        const int s0 = ok ? wait_tile() : 0;
        if (ok) {
          tc_fence_after();
          if (nti > 0) {
            attn_mma_qk<D>(i * 128, q_lo, k_lo + s0 * (C::TILE >> 4), a.idesc_qk);
            tc_commit(&sbar[i]);
          }
          tc_commit(&free_[s0]);
        }
#pragma unroll 1
        for (int j = 0; ok && j < ntile; ++j) {
          const int sv = wait_tile();
          if (!ok) break;
          // everything else is waited for ahead of the weights: what follows
          // those is on the path from this tile's softmax to its next scores
          const int sn = j + 1 < ntile ? wait_tile() : -1;
          if (!ok) break;
          if (j < nti) {
            if (j * 128 + 128 > lk) {   // the sequence's last V tile ends past it
              if (i == 0 || nt[0] < ntile) mbar_arrive(zreq);
              if (!(ok = attn_wait(zbar, 0, abort_flag, g_prompt_wait_ns))) break;
            }
            if (!(ok = attn_wait(&pbar[i], (uint32_t)j & 1u, abort_flag, g_prompt_wait_ns))) break;
            tc_fence_after();
            attn_mma_pv<D>(256 + i * D, i * 128, v_lo + sv * (C::TILE >> 4), j > 0);
            if (j + 1 < nti) {
              attn_mma_qk<D>(i * 128, q_lo, k_lo + sn * (C::TILE >> 4), a.idesc_qk);
              tc_commit(&sbar[i]);
            } else {
              tc_commit(&obar[i]);
            }
          }
          tc_commit(&free_[sv]);
          if (sn >= 0) tc_commit(&free_[sn]);
        }
        tc_commit(&drain[i]);   // what is in flight finishes before tensor memory is given up
        mbar_wait_bounded(&drain[i], 0, kAttnWaitLimitNs);
      }
    } else {
      // ---------------- rows of the last V tile past the sequence: zeroed
      if (ntile * 128 > lk) {
        const int n = 2 * ntile - 1;
        if (attn_wait_warp(zreq, 0, abort_flag, g_prompt_wait_ns)) {   // the tile is in
          const uint32_t vb = sb + C::OFF_KV + (n % NSTG) * C::TILE, from = (lk - (ntile - 1) * 128) * 128;
          for (int at = 0; at < D / 64; ++at)
            for (uint32_t o = from + lane * 16; o < kAttnAtom; o += 512)
              sts128(vb + at * kAttnAtom + o, make_uint4(0, 0, 0, 0));
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(zbar);
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;\n");
    // ---------------- softmax: warps 4i .. 4i + 3 own tile i, thread = row
    const int i = warp >> 2, r = tid & 127, nti = i ? nt[1] : nt[0];
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t st = tmem + i * 128 + lanes, ot = tmem + 256 + i * D + lanes;
    const int tok = t0 + i * a.tpt + r / a.G, head = hk * a.G + r % a.G;
    const bool live = r < a.G * a.tpt && tok < lq;
    const int n = live ? (a.causal ? min(lk, tok + 1 + lk - lq) : lk) : 128 * nti;   // keys of this row
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int j = 0; j < nti; ++j) {
      if (!(ok = attn_wait_warp(&sbar[i], (uint32_t)j & 1u, abort_flag, g_prompt_wait_ns))) break;
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
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&pbar[i]);
    }
    if (ok && nti > 0) ok = attn_wait_warp(&obar[i], 0, abort_flag, g_prompt_wait_ns);
    if (ok) {
      tc_fence_after();
      const float inv = l > 0.f ? 1.f / l : 0.f;
      __half* out = a.out + ((q0 + tok) * a.Hq + head) * D;
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        if (nti > 0) {
          tmem_ld_32x32b_x32(ot + c, o);
          tmem_ld_wait_all<32>(o);
        }
        if (live) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint32_t w[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
              w[x] = l > 0.f ? pack_half2_bits(__uint_as_float(o[e + 2 * x]) * inv, __uint_as_float(o[e + 2 * x + 1]) * inv)
                             : 0u;
            *reinterpret_cast<uint4*>(out + c + e) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // the copies in flight land before the memory is given up
    if (tid == 0 && *issued >= 0) mbar_wait_bounded(qbar, 0, kAttnWaitLimitNs);
    if (tid == 0)
      for (int n = max(0, *issued - NSTG); n < *issued; ++n)
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

template <int D>
cudaError_t launch_t(const PromptArgs& a, cudaStream_t stream) {
  using C = PromptCfg<D>;
  EncodeTiledFn enc = get_encode_fn();
  if (!enc) return cudaErrorNotSupported;
  PromptParams p{};
  p.G = (int)(a.Hq / a.Hkv);
  p.tpt = 128 / p.G;
  CUtensorMap mq, mk, mv;
  // without any key no K or V tile is copied: their maps only have to be valid
  const bool keys = a.total_k > 0;
  if (!encode_heads(enc, &mq, a.q, a.total_q, a.Hq, D, a.ldq, p.G, p.tpt) ||
      !encode_heads(enc, &mk, keys ? a.k : a.q, keys ? a.total_k : 1, keys ? a.Hkv : 1, D, keys ? a.ldk : D, 1, 128) ||
      !encode_heads(enc, &mv, keys ? a.v : a.q, keys ? a.total_k : 1, keys ? a.Hkv : 1, D, keys ? a.ldv : D, 1, 128))
    return cudaErrorNotSupported;
  p.cu_q = a.cu_q;
  p.cu_k = a.cu_k;
  p.out = static_cast<__half*>(a.out);
  p.total_q = a.total_q;
  p.total_k = a.total_k;
  p.Hq = (int)a.Hq;
  p.causal = a.causal;
  // a negative scale is |scale| times negated queries; zero makes every
  // weight equal, as any product too small to move 2^x does
  p.scale_log2 = fmaxf(fabsf(a.scale) * kAttnLog2e, 1e-30f);
  p.idesc_qk = umma_idesc_f16_f32(128, 128, a.scale < 0.f);
  p.status = device_status_word();
  p.debug_stall = take_debug_stall() ? 1 : 0;
  p.tiles = (int)((a.max_q + 2 * p.tpt - 1) / (2 * p.tpt));
  int per_sm = 0;
  cudaError_t e = prepare_launch_tmem(prompt_tc_kernel<D>, kPromptThreads, C::BYTES, 512, &per_sm);
  if (e != cudaSuccess) return e;
  e = launch_pdl(prompt_tc_kernel<D>, dim3((unsigned)p.tiles, (unsigned)a.Hkv, (unsigned)a.batch),
                 dim3(kPromptThreads), C::BYTES, stream, 1, mq, mk, mv, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t set_wait_limit_prompt(uint64_t ns) { return cudaMemcpyToSymbol(g_prompt_wait_ns, &ns, sizeof(ns)); }

int64_t prompt_attention_workspace(const PromptArgs&) { return 0; }

cudaError_t launch_prompt_attention(const PromptArgs& a, cudaStream_t stream) {
  if (a.D == 128) return launch_t<128>(a, stream);
  if (a.D == 64) return launch_t<64>(a, stream);
  return cudaErrorNotSupported;
}

}  // namespace spinq
