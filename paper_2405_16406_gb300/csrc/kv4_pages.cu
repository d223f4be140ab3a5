// kv4_pages.cu -- the paged 4-bit cache: spinq_kv4_append (norm of each query
// and key head, rotary embedding, R3 and the 4-bit quantizer in one pass, K
// and V written into pages) and spinq_kv4_read (cached tokens expanded to
// packed fp16 K and V).
//
// Pages.  codes [page][kv head][slot][D/2], scales [page][kv head][slot][4]
// (k alpha, k beta, v alpha, v beta): the tokens of one head lie next to one
// another, so a reader of one head moves whole runs of a page.
//
// Append, per row x of D values (Sec. 3.1 R3; Eq. 1):
//   x <- x w / sqrt(mean x^2 + eps)        queries and keys, where a weight is given
//   x <- rotary embedding of the first R values
//   y = H_D x                               (1/sqrt(D) goes to alpha, beta and q_out)
//   u = rint((y - min y) (15 / (max y - min y)))
// in fp32 from the fp16 input to the code: only q_out (fp16) and the codes
// are rounded to fewer bits.  Every sum has a fixed order: index bit 0 first, then
// bit 1, ... (the norm's sum of squares and the butterflies alike), so the
// result does not depend on how the rows are spread over the lanes.
//
// Append layout.  A quad of lanes owns a row, a warp 8 rows of one kind (all
// query heads of all tokens, then key heads, then value heads).  The row's
// 8-value pieces go to the lanes in turn (a quad's loads and stores are runs of
// 64 bytes): lane c holds values D/2 s + 32 v + 8 c + e, as pairs (s = 0, s = 1) in
// packed fp32.  A rotate-half pair over the whole head is one register pair, every
// butterfly but the last works on packed pairs, and only bits 3 and 4 of
// the transform go through shuffles.  The next row's data are loaded before this
// one's are worked on.  Bound: the bytes come second to the shuffles, 64 per 8 rows, which
// with the loads hold L1/TEX at 69 % of its peak (issue at 54 %, with norm and RoPE).
// 32768 tokens, 32 / 8 heads, D 128, RoPE: 709 MB in 162 us, 4.4 TB/s (a row per
// warp took 251 us with the read below, packed pairs 211, pieces in turn and the next row
// ahead 198).
//
// Read layout.  A warp expands 16 tokens of one kv head, whose codes are one
// run of a page wherever the tokens are; the warps of a block take the heads of the same
// tokens, whose output rows lie next to one another.  Bound: the bytes, 711 MB in 129
// us, 5.5 TB/s (a token per warp: 196 us); in 777 tokens the latency of a table entry, a
// row of codes and a store, 3 us.
#include <cuda_fp16.h>
#include <float.h>

#include "launch_util.h"
#include "spinq_device.cuh"
#include "spinq_internal.h"

namespace spinq {
namespace {

constexpr int kAppendWarps = 4;
constexpr int kReadWarps = 8;

// The product of two packed pairs, rounded before whatever is added to it:
// a product written as such is fused with a following packed sum
// (one rounding instead of two), which the fixed order of this file's sums excludes.
__device__ __forceinline__ F2 f2_product(F2 a, F2 b) { return f2_fma(a, b, f2_make(0.f, 0.f)); }

enum RopeForm { kRopeNone = 0, kRopePairs = 1, kRopeHalves = 2, kRopePartHalves = 3 };

// D = head_dim, ROPE one of RopeForm:
//   kRopePairs       neighbouring pairs (2i, 2i+1) of the first R values;
//   kRopeHalves      pairs (i, i + D/2), R = D: one register pair;
//   kRopePartHalves  pairs (i, i + R/2), R < D: the partner's 8-value piece is
//                    loaded a second time (it is another lane's).
template <int D, bool CLAMP, int ROPE>
__global__ void __launch_bounds__(kAppendWarps * 32) kv4_append_kernel(AppendArgs a, uint32_t uq, uint32_t uk) {
  constexpr int V = D / 64;   // pieces of 8 values per lane and half of the row
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const uint32_t units = uq + 2 * uk, stride = gridDim.x * kAppendWarps;
  struct Row {
    int kind;        // the warp's rows: 0 queries, 1 keys, 2 values
    uint32_t row, t, h;
    bool valid;
    const __half* src;
    uint4 in[2][V];
    int pos;
  };
  auto fetch = [&](uint32_t u, Row& x) {
    x.kind = u < uq ? 0 : (u < uq + uk ? 1 : 2);
    const uint32_t H = (uint32_t)(x.kind == 0 ? a.Hq : a.Hkv);
    x.row = (x.kind == 0 ? u : (x.kind == 1 ? u - uq : u - uq - uk)) * 8 + g;
    x.t = x.row / H;
    x.h = x.row - x.t * H;
    x.valid = x.t < (uint32_t)a.T;
    x.src = reinterpret_cast<const __half*>(x.kind == 0 ? a.q : (x.kind == 1 ? a.k : a.v)) +
            (int64_t)x.t * (x.kind == 0 ? a.ldq : (x.kind == 1 ? a.ldk : a.ldv)) + x.h * D;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int v = 0; v < V; ++v)
        x.in[s][v] = x.valid ? __ldg(reinterpret_cast<const uint4*>(x.src + s * (D / 2)) + 4 * v + c)
                             : make_uint4(0, 0, 0, 0);
    x.pos = ROPE != kRopeNone && x.valid && x.kind != 2 ? __ldg(a.positions + x.t) : 0;
  };
  // packed pairs (piece of the first half, piece of the second) as fp32
  auto widen = [](const uint4& p, const uint4& q, F2* out) {
    const uint32_t lo[4] = {p.x, p.y, p.z, p.w}, hi[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo[j]));
      const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&hi[j]));
      out[2 * j] = f2_make(x.x, y.x);
      out[2 * j + 1] = f2_make(x.y, y.y);
    }
  };
  pdl_wait();
  pdl_trigger();
  Row next;
  uint32_t u = blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  if (u < units) fetch(u, next);
  for (; u < units; u += stride) {
    const Row x = next;
    if (u + stride < units) fetch(u + stride, next);
    F2 y[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) widen(x.in[0][v], x.in[1][v], y[v]);

    if (x.kind != 2) {
      // ---- norm of the head
      const __half* wt = reinterpret_cast<const __half*>(x.kind == 0 ? a.q_weight : a.k_weight);
      const uint4* w4 = reinterpret_cast<const uint4*>(wt);
      float r = 1.f;
      if (wt != nullptr) {
        float part[2];
        F2 sum[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          F2 sq[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) sq[i] = f2_product(y[v][i], y[v][i]);
#pragma unroll
          for (int w = 4; w >= 1; w >>= 1)   // neighbours first
#pragma unroll
            for (int i = 0; i < w; ++i) sq[i] = f2_add(sq[2 * i], sq[2 * i + 1]);
#pragma unroll
          for (int b = 1; b < 4; b <<= 1) {
            float p, q;
            f2_split(sq[0], p, q);
            sq[0] = f2_add(sq[0], f2_make(__shfl_xor_sync(0xffffffffu, p, b), __shfl_xor_sync(0xffffffffu, q, b)));
          }
          sum[v] = sq[0];
        }
        if (V == 2) sum[0] = f2_add(sum[0], sum[V - 1]);
        f2_split(sum[0], part[0], part[1]);
        const float ms = __fadd_rn(part[0], part[1]) * (1.f / D);   // D is a power of two: exact
        r = __frcp_rn(__fsqrt_rn(__fadd_rn(ms, a.eps)));
        const F2 rr = f2_make(r, r);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          F2 wf[8];
          widen(__ldg(w4 + 4 * v + c), __ldg(w4 + D / 16 + 4 * v + c), wf);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[v][i] = f2_product(f2_product(y[v][i], rr), wf[i]);
        }
      }

      // ---- rotary embedding of the first R values
      if (ROPE != kRopeNone) {
        const int half = a.rotary / 2;
        const int64_t pos = x.pos < 0 ? 0 : ((int64_t)x.pos >= a.max_pos ? a.max_pos - 1 : x.pos);
        const float2* cs = reinterpret_cast<const float2*>(a.cos_sin) + pos * half;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int e0 = 32 * v + 8 * c;   // first value of the piece (and e0 + D/2)
          if (ROPE == kRopePairs) {
            // angles e/2 and D/4 + e/2; past R: cos 1, sin 0
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              const int e = (e0 + i) / 2;
              const float2 f0 = e < half ? __ldg(cs + e) : make_float2(1.f, 0.f);
              const float2 f1 = e + D / 4 < half ? __ldg(cs + e + D / 4) : make_float2(1.f, 0.f);
              const F2 co = f2_make(f0.x, f1.x), si = f2_make(f0.y, f1.y);
              const F2 p = y[v][i], q = y[v][i + 1];
              y[v][i] = f2_sub(f2_product(p, co), f2_product(q, si));
              y[v][i + 1] = f2_add(f2_product(p, si), f2_product(q, co));
            }
          } else if (ROPE == kRopeHalves) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              const float4 f = __ldg(reinterpret_cast<const float4*>(cs + e0 + i));
              float p, q;
              f2_split(y[v][i], p, q);
              y[v][i] = f2_add(f2_product(y[v][i], f2_make(f.x, f.x)), f2_product(f2_make(q, p), f2_make(-f.y, f.y)));
              f2_split(y[v][i + 1], p, q);
              y[v][i + 1] =
                  f2_add(f2_product(y[v][i + 1], f2_make(f.z, f.z)), f2_product(f2_make(q, p), f2_make(-f.w, f.w)));
            }
          } else {
            float z[2][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f2_split(y[v][i], z[0][i], z[1][i]);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const int e = e0 + s * (D / 2);
              if (e < a.rotary) {
                const bool first = e < half;
                const int o = first ? e + half : e - half, f0 = first ? e : e - half;
                const uint4 xo = x.valid ? __ldg(reinterpret_cast<const uint4*>(x.src + o)) : make_uint4(0, 0, 0, 0);
                const uint4 wo = wt != nullptr ? __ldg(reinterpret_cast<const uint4*>(wt + o)) : make_uint4(0, 0, 0, 0);
                F2 xw[8];   // (partner value, its weight)
                widen(xo, wo, xw);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  float q, w;
                  f2_split(xw[i], q, w);
                  if (wt != nullptr) q = __fmul_rn(__fmul_rn(q, r), w);
                  const float2 f = __ldg(cs + f0 + i);
                  const float p = __fmul_rn(z[s][i], f.x), n = __fmul_rn(q, f.y);
                  z[s][i] = first ? __fsub_rn(p, n) : __fadd_rn(p, n);
                }
              }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) y[v][i] = f2_make(z[0][i], z[1][i]);
          }
        }
      }

      // ---- R3: bits 0-2 in the lane, the two lane bits, bit 5 (D = 128) and the pair's bit
#pragma unroll
      for (int v = 0; v < V; ++v) {
#pragma unroll
        for (int bit = 1; bit < 8; bit <<= 1)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (!(i & bit)) f2_bfly(y[v][i], y[v][i | bit]);
#pragma unroll
        for (int bit = 1; bit < 4; bit <<= 1) {
          const float sg = c & bit ? -1.f : 1.f;   // the upper lane's value enters with a minus sign (exact product)
          const F2 sg2 = f2_make(sg, sg);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float p, q;
            f2_split(y[v][i], p, q);
            y[v][i] =
                f2_fma(y[v][i], sg2, f2_make(__shfl_xor_sync(0xffffffffu, p, bit), __shfl_xor_sync(0xffffffffu, q, bit)));
          }
        }
      }
      if (V == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f2_bfly(y[0][i], y[V - 1][i]);
      }
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) f2_bfly_inner(y[v][i]);
    }

    if (x.kind == 0) {
      if (x.valid) {
        uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<__half*>(a.q_out) + (int64_t)x.row * D) + c;
        const F2 nn = f2_make(a.norm, a.norm);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          uint32_t w[2][4];
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            float p0, q0, p1, q1;
            f2_split(f2_product(y[v][i], nn), p0, q0);
            f2_split(f2_product(y[v][i + 1], nn), p1, q1);
            w[0][i / 2] = pack_half2_bits(p0, p1);
            w[1][i / 2] = pack_half2_bits(q0, q1);
          }
#pragma unroll
          for (int s = 0; s < 2; ++s) dst[s * (D / 16) + 4 * v] = make_uint4(w[s][0], w[s][1], w[s][2], w[s][3]);
        }
      }
      continue;
    }

    // ---- Eq. 1 over the row, into its slot.  A value that is not a number makes the extremes
    // and with them the row's scales NaN: the cache does not turn it into a number.
    float hi = -FLT_MAX, lo = FLT_MAX;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float p, q;
        f2_split(y[v][i], p, q);
        asm("max.NaN.f32 %0, %0, %1, %2;\n" : "+f"(hi) : "f"(p), "f"(q));
        asm("min.NaN.f32 %0, %0, %1, %2;\n" : "+f"(lo) : "f"(p), "f"(q));
      }
#pragma unroll
    for (int b = 1; b < 4; b <<= 1) {
      const float oh = __shfl_xor_sync(0xffffffffu, hi, b), ol = __shfl_xor_sync(0xffffffffu, lo, b);
      asm("max.NaN.f32 %0, %0, %1;\n" : "+f"(hi) : "f"(oh));
      asm("min.NaN.f32 %0, %0, %1;\n" : "+f"(lo) : "f"(ol));
    }
    if (CLAMP) {
      hi *= a.clip;
      lo *= a.clip;
    }
    const float span = __fsub_rn(hi, lo);
    // One reciprocal and product per row, a product per value, each rounded: within 3 * 2^-24 of the
    // quotient of the two differences, so a code differs from it only for a value within
    // 2^-18.5 (of a step) of the middle of two codes.  A value that lies exactly there, as those of V's
    // fp16 rows do now and then, may go either way: of 168 M codes of normal fp16 rows 3.2e-5
    // differ from Eq. 1 in 64 bits (4.7e-5 with the unpaged cache's y inv - lo inv).
    const float inv = span > 0.f ? __fmul_rn(__frcp_rn(span), 15.f) : 0.f;
    const F2 lo2 = f2_make(lo, lo), inv2 = f2_make(inv, inv), mg2 = f2_make(kRoundMagic, kRoundMagic);
    uint32_t word[4];   // codes of the pieces (s, v): word 2 s + v (D = 128) or s
#pragma unroll
    for (int v = 0; v < V; ++v) {
      uint32_t r[2][8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        F2 t = f2_product(f2_sub(y[v][i], lo2), inv2);
        float p, q;
        if (CLAMP) {
          f2_split(t, p, q);
          t = f2_make(fminf(fmaxf(p, 0.f), 15.f), fminf(fmaxf(q, 0.f), 15.f));
        }
        f2_split(f2_add(t, mg2), p, q);
        r[0][i] = __float_as_uint(p);
        r[1][i] = __float_as_uint(q);
      }
      word[v] = pack8_nibbles(r[0]);
      word[V + v] = pack8_nibbles(r[1]);
    }
    if (V == 2) {
      // 4 x 4 transpose over the quad: lane c ends with the words of piece
      // group c of all four lanes, 16 contiguous bytes of the row
#pragma unroll
      for (int bit = 1; bit < 4; bit <<= 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(i & bit)) {
            const bool up = (c & bit) != 0;
            const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? word[i] : word[i | bit], bit);
            if (up) word[i] = got; else word[i | bit] = got;
          }
      }
    }
    const int64_t slot = x.valid ? __ldg(a.slots + x.t) : -1;
    if (slot >= 0 && slot < a.num_slots) {
      const int64_t page = slot >> a.page_shift, in_page = slot & (a.page_size - 1);
      const int64_t at = (page * a.Hkv + x.h) * a.page_size + in_page;
      uint8_t* codes = (x.kind == 1 ? a.k_codes : a.v_codes) + at * (D / 2);
      if (V == 2) {
        *reinterpret_cast<uint4*>(codes + 16 * c) = make_uint4(word[0], word[1], word[2], word[3]);
      } else {
        *reinterpret_cast<uint32_t*>(codes + 4 * c) = word[0];
        *reinterpret_cast<uint32_t*>(codes + 16 + 4 * c) = word[1];
      }
      if (c == 0) {
        const float nrm = x.kind == 1 ? a.norm : 1.f;
        reinterpret_cast<float2*>(a.scales + at * 4)[x.kind - 1] =
            make_float2(__fmul_rn(__fdiv_rn(span, 15.f), nrm), __fmul_rn(lo, nrm));
      }
    }
  }
}

template <int D, bool CLAMP, int ROPE>
cudaError_t append_t(const AppendArgs& a, cudaStream_t stream) {
  const uint32_t uq = (uint32_t)((a.T * a.Hq + 7) / 8), uk = (uint32_t)((a.T * a.Hkv + 7) / 8);
  const int64_t units = (int64_t)uq + 2 * (int64_t)uk;
  int per_sm = 1;
  cudaError_t e = prepare_launch(kv4_append_kernel<D, CLAMP, ROPE>, kAppendWarps * 32, 0, &per_sm);
  if (e != cudaSuccess) return e;
  int64_t blocks = (units + kAppendWarps - 1) / kAppendWarps;
  const int64_t cap = (int64_t)device_sm_count() * per_sm;
  if (blocks > cap) blocks = cap;
  e = launch_pdl(kv4_append_kernel<D, CLAMP, ROPE>, dim3((unsigned)blocks), dim3(kAppendWarps * 32), 0, stream, 1, a,
                 uq, uk);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int D, bool CLAMP>
cudaError_t append_c(const AppendArgs& a, cudaStream_t stream) {
  if (a.rotary == 0) return append_t<D, CLAMP, kRopeNone>(a, stream);
  if (a.interleaved) return append_t<D, CLAMP, kRopePairs>(a, stream);
  return a.rotary == D ? append_t<D, CLAMP, kRopeHalves>(a, stream) : append_t<D, CLAMP, kRopePartHalves>(a, stream);
}

// A warp takes 16 output tokens of one kv head: lane n looks token n % 16 up
// and loads its scales, then D / 8 lanes share a row of codes (4 bytes, 8 values
// and one 16-byte store per lane), K and V side by side.
template <int D>
__global__ void __launch_bounds__(kReadWarps * 32) kv4_read_kernel(ReadArgs a, uint32_t units) {
  constexpr int LPR = D / 8;          // lanes per row
  constexpr int TPS = 32 / LPR / 2;   // tokens per step (K and V of each)
  const int lane = threadIdx.x & 31;
  const int part = lane % LPR, which = (lane / LPR) & 1, ts = lane / (2 * LPR);
  const uint32_t stride = gridDim.x * kReadWarps, heads = (uint32_t)a.Hkv;
  pdl_wait();
  pdl_trigger();
  const int end = __ldg(a.cu + a.batch);
  for (uint32_t u = blockIdx.x * kReadWarps + (threadIdx.x >> 5); u < units; u += stride) {
    const uint32_t grp = u / heads, h = u - grp * heads;
    const int64_t i0 = (int64_t)grp * 16, i = i0 + (lane & 15);
    int64_t at = -1;   // the token's place in the page arrays
    float4 sc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < a.total && i < end) {
      int lo = 0, hi = (int)a.batch - 1;   // the last sequence whose offset is <= i
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (__ldg(a.cu + mid) <= (int)i) lo = mid; else hi = mid - 1;
      }
      const int64_t t = i - __ldg(a.cu + lo) + (a.starts ? __ldg(a.starts + lo) : 0);
      const int64_t pi = t >> a.page_shift;
      if (t >= 0 && pi < a.table_width) {
        const int64_t page = __ldg(a.table + (int64_t)lo * a.table_width + pi);
        if (page >= 0 && page < a.num_pages) {
          at = (page * heads + h) * a.page_size + (t & (a.page_size - 1));
          sc = __ldg(reinterpret_cast<const float4*>(a.scales) + at);
        }
      }
    }
    const uint32_t* codes = reinterpret_cast<const uint32_t*>(which ? a.v_codes : a.k_codes) + part;
    uint32_t w[16 / TPS];
#pragma unroll
    for (int s = 0; s < 16 / TPS; ++s) {
      const int64_t ax = __shfl_sync(0xffffffffu, at, s * TPS + ts);
      w[s] = ax >= 0 ? __ldg(codes + ax * (D / 8)) : 0u;
    }
    __half* out = reinterpret_cast<__half*>(which ? a.v : a.k) + (i0 * heads + h) * D + part * 8;
#pragma unroll
    for (int s = 0; s < 16 / TPS; ++s) {
      const int n = s * TPS + ts;   // tokens without a page have scales 0 and read as zeros
      const float ka = __shfl_sync(0xffffffffu, sc.x, n), kb = __shfl_sync(0xffffffffu, sc.y, n);
      const float va = __shfl_sync(0xffffffffu, sc.z, n), vb = __shfl_sync(0xffffffffu, sc.w, n);
      const float al = which ? va : ka, be = which ? vb : kb;
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        o[j] = pack_half2_bits(fmaf((float)((w[s] >> (8 * j)) & 15u), al, be),
                               fmaf((float)((w[s] >> (8 * j + 4)) & 15u), al, be));
      if (i0 + n < a.total)
        *reinterpret_cast<uint4*>(out + (int64_t)n * heads * D) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

template <int D>
cudaError_t read_t(const ReadArgs& a, cudaStream_t stream) {
  int per_sm = 1;
  cudaError_t e = prepare_launch(kv4_read_kernel<D>, kReadWarps * 32, 0, &per_sm);
  if (e != cudaSuccess) return e;
  const int64_t units = (a.total + 15) / 16 * a.Hkv;
  int64_t blocks = (units + kReadWarps - 1) / kReadWarps;
  const int64_t cap = (int64_t)device_sm_count() * per_sm;
  if (blocks > cap) blocks = cap;
  e = launch_pdl(kv4_read_kernel<D>, dim3((unsigned)blocks), dim3(kReadWarps * 32), 0, stream, 1, a,
                 (uint32_t)units);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv4_append(const AppendArgs& a, cudaStream_t stream) {
  const bool clamp = a.clip < 1.f;
  if (a.D == 128) return clamp ? append_c<128, true>(a, stream) : append_c<128, false>(a, stream);
  if (a.D == 64) return clamp ? append_c<64, true>(a, stream) : append_c<64, false>(a, stream);
  return cudaErrorNotSupported;
}

cudaError_t launch_kv4_read(const ReadArgs& a, cudaStream_t stream) {
  if (a.D == 128) return read_t<128>(a, stream);
  if (a.D == 64) return read_t<64>(a, stream);
  return cudaErrorNotSupported;
}

}  // namespace spinq
