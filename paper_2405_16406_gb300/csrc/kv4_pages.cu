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
// Layout.  A quad of lanes owns a row, a warp 8 rows of one token.  Lane c
// holds the values [Cc, Cc + C) and [D/2 + Cc, D/2 + Cc + C), C = D/8: the
// pairs (i, i + D/2) of the rotate-half form over the whole head sit in one
// lane, as do neighbouring pairs, and only the two middle bits of the transform go
// through shuffles.
#include <cuda_fp16.h>
#include <float.h>

#include "launch_util.h"
#include "spinq_device.cuh"
#include "spinq_internal.h"

namespace spinq {
namespace {

constexpr int kAppendWarps = 4;
constexpr int kReadWarps = 8;

enum RopeForm { kRopeNone = 0, kRopePairs = 1, kRopeHalves = 2, kRopePartHalves = 3 };

// D = head_dim, ROPE one of RopeForm:
//   kRopePairs       neighbouring pairs (2i, 2i+1) of the first R values;
//   kRopeHalves      pairs (i, i + D/2), R = D: both in the lane;
//   kRopePartHalves  pairs (i, i + R/2), R < D a multiple of D/4: the partner
//                    is a whole C-value run of another lane of the quad.
template <int D, bool CLAMP, int ROPE>
__global__ void __launch_bounds__(kAppendWarps * 32) kv4_append_kernel(AppendArgs a, int64_t units, int groups) {
  constexpr int C = D / 8;    // values per run; a lane holds two runs
  constexpr int CV = C / 8;   // 16-byte loads per run
  const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int64_t stride = (int64_t)gridDim.x * kAppendWarps;
  pdl_wait();
  pdl_trigger();
  for (int64_t u = (int64_t)blockIdx.x * kAppendWarps + (threadIdx.x >> 5); u < units; u += stride) {
    const int64_t t = u / groups;
    const int row = (int)(u - t * groups) * 8 + g;   // query heads, then key heads, then value heads
    const int rows = (int)(a.Hq + 2 * a.Hkv);
    const bool valid = row < rows;
    const int kind = row < a.Hq ? 0 : (row < a.Hq + a.Hkv ? 1 : 2);
    const int h = kind == 0 ? row : (kind == 1 ? row - (int)a.Hq : row - (int)(a.Hq + a.Hkv));
    const __half* src = reinterpret_cast<const __half*>(kind == 0 ? a.q : (kind == 1 ? a.k : a.v)) +
                        t * (kind == 0 ? a.ldq : (kind == 1 ? a.ldk : a.ldv)) + (int64_t)h * D;
    float y[2][C];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < CV; ++i) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (valid) w = __ldg(reinterpret_cast<const uint4*>(src + s * (D / 2) + c * C) + i);
        const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&ws[j]));
          y[s][8 * i + 2 * j] = f.x;
          y[s][8 * i + 2 * j + 1] = f.y;
        }
      }

    // ---- norm of the head (queries and keys)
    const __half* wt = reinterpret_cast<const __half*>(kind == 0 ? a.q_weight : a.k_weight);
    const bool norm = valid && kind != 2 && wt != nullptr;
    if (__any_sync(0xffffffffu, norm)) {
      float part[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float sq[C];
#pragma unroll
        for (int i = 0; i < C; ++i) sq[i] = __fmul_rn(y[s][i], y[s][i]);
#pragma unroll
        for (int w = C / 2; w >= 1; w >>= 1)   // neighbours first
#pragma unroll
          for (int i = 0; i < w; ++i) sq[i] = __fadd_rn(sq[2 * i], sq[2 * i + 1]);
        part[s] = sq[0];
        part[s] = __fadd_rn(part[s], __shfl_xor_sync(0xffffffffu, part[s], 1));
        part[s] = __fadd_rn(part[s], __shfl_xor_sync(0xffffffffu, part[s], 2));
      }
      if (norm) {
        const float ms = __fadd_rn(part[0], part[1]) * (1.f / D);   // D is a power of two: exact
        const float r = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(ms, a.eps)));
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < CV; ++i) {
            const uint4 w = __ldg(reinterpret_cast<const uint4*>(wt + s * (D / 2) + c * C) + i);
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&ws[j]));
              y[s][8 * i + 2 * j] = __fmul_rn(__fmul_rn(y[s][8 * i + 2 * j], r), f.x);
              y[s][8 * i + 2 * j + 1] = __fmul_rn(__fmul_rn(y[s][8 * i + 2 * j + 1], r), f.y);
            }
          }
      }
    }

    // ---- rotary embedding of the first R values (queries and keys)
    if (ROPE != kRopeNone) {
      const int half = a.rotary / 2;
      int64_t pos = valid ? (int64_t)a.positions[t] : 0;
      pos = pos < 0 ? 0 : (pos >= a.max_pos ? a.max_pos - 1 : pos);
      const float2* cs = reinterpret_cast<const float2*>(a.cos_sin) + pos * half;
      if (ROPE == kRopePairs) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < C; i += 2) {
            const int e = s * (D / 2) + c * C + i;
            if (kind != 2 && e < a.rotary) {
              const float2 f = __ldg(cs + e / 2);
              const float p = y[s][i], q = y[s][i + 1];
              y[s][i] = __fsub_rn(__fmul_rn(p, f.x), __fmul_rn(q, f.y));
              y[s][i + 1] = __fadd_rn(__fmul_rn(p, f.y), __fmul_rn(q, f.x));
            }
          }
      } else if (ROPE == kRopeHalves) {
        if (kind != 2) {
#pragma unroll
          for (int i = 0; i < C; i += 2) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(cs + c * C + i));
            const float p0 = y[0][i], q0 = y[1][i], p1 = y[0][i + 1], q1 = y[1][i + 1];
            y[0][i] = __fsub_rn(__fmul_rn(p0, f.x), __fmul_rn(q0, f.y));
            y[1][i] = __fadd_rn(__fmul_rn(p0, f.y), __fmul_rn(q0, f.x));
            y[0][i + 1] = __fsub_rn(__fmul_rn(p1, f.z), __fmul_rn(q1, f.w));
            y[1][i + 1] = __fadd_rn(__fmul_rn(p1, f.w), __fmul_rn(q1, f.z));
          }
        }
      } else {
        // run number c + 4 s; the partner run is R/2 values away
        const int hop = half / C;
        float o[2][C];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int run = c + 4 * s, other = run < hop ? run + hop : run - hop;
          const int from = (lane & ~3) | (other & 3);
#pragma unroll
          for (int i = 0; i < C; ++i) {
            const float lo = __shfl_sync(0xffffffffu, y[0][i], from), hi = __shfl_sync(0xffffffffu, y[1][i], from);
            o[s][i] = other & 4 ? hi : lo;
          }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int run = c + 4 * s;
          if (kind != 2 && run < 2 * hop) {
            const bool first = run < hop;
            const float2* f0 = cs + (first ? run : run - hop) * C;
#pragma unroll
            for (int i = 0; i < C; ++i) {
              const float2 f = __ldg(f0 + i);
              const float p = __fmul_rn(y[s][i], f.x), q = __fmul_rn(o[s][i], f.y);
              y[s][i] = first ? __fsub_rn(p, q) : __fadd_rn(p, q);
            }
          }
        }
      }
    }

    // ---- R3: bits 0 .. log2 C - 1 in the lane, the two lane bits, the top bit in the lane
    if (__any_sync(0xffffffffu, valid && kind != 2)) {
      float z[2][C];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < C; ++i) z[s][i] = y[s][i];
#pragma unroll
      for (int bit = 1; bit < C; bit <<= 1)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < C; ++i)
            if (!(i & bit)) {
              const float p = z[s][i], q = z[s][i | bit];
              z[s][i] = __fadd_rn(p, q);
              z[s][i | bit] = __fsub_rn(p, q);
            }
#pragma unroll
      for (int bit = 1; bit < 4; bit <<= 1) {
        const float sg = c & bit ? -1.f : 1.f;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < C; ++i)   // the upper lane's value enters with a minus sign (exact product)
            z[s][i] = fmaf(z[s][i], sg, __shfl_xor_sync(0xffffffffu, z[s][i], bit));
      }
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const float p = z[0][i], q = z[1][i];
        z[0][i] = __fadd_rn(p, q);
        z[1][i] = __fsub_rn(p, q);
      }
      if (kind != 2) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int i = 0; i < C; ++i) y[s][i] = z[s][i];
      }
    }

    if (valid && kind == 0) {
      __half* dst = reinterpret_cast<__half*>(a.q_out) + (t * a.Hq + h) * D + c * C;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < CV; ++i) {
          uint4 w;
          w.x = pack_half2_bits(y[s][8 * i] * a.norm, y[s][8 * i + 1] * a.norm);
          w.y = pack_half2_bits(y[s][8 * i + 2] * a.norm, y[s][8 * i + 3] * a.norm);
          w.z = pack_half2_bits(y[s][8 * i + 4] * a.norm, y[s][8 * i + 5] * a.norm);
          w.w = pack_half2_bits(y[s][8 * i + 6] * a.norm, y[s][8 * i + 7] * a.norm);
          reinterpret_cast<uint4*>(dst + s * (D / 2))[i] = w;
        }
    }

    // ---- Eq. 1 over the row, into its slot
    if (__any_sync(0xffffffffu, valid && kind != 0)) {
      float hi = -FLT_MAX, lo = FLT_MAX;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < C; ++i) {
          hi = fmaxf(hi, y[s][i]);
          lo = fminf(lo, y[s][i]);
        }
#pragma unroll
      for (int b = 1; b < 4; b <<= 1) {
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, b));
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, b));
      }
      if (CLAMP) {
        hi *= a.clip;
        lo *= a.clip;
      }
      const float span = __fsub_rn(hi, lo);
      // one reciprocal per row, a product per value: a code differs from Eq. 1's
      // quotient only for a value within 2^-20 of the middle of two codes
      const float inv = span > 0.f ? __fmul_rn(__frcp_rn(span), 15.f) : 0.f;
      uint32_t words[2][CV];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < CV; ++i) {
          uint32_t r[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float v = __fmul_rn(__fsub_rn(y[s][8 * i + j], lo), inv);
            if (CLAMP) v = fminf(fmaxf(v, 0.f), 15.f);
            r[j] = round_bits(v);
          }
          words[s][i] = pack8_nibbles(r);
        }
      const int64_t slot = valid && kind != 0 ? a.slots[t] : -1;
      if (slot >= 0 && slot < a.num_slots) {
        const int64_t page = slot / a.page_size, in_page = slot - page * a.page_size;
        const int64_t at = (page * a.Hkv + h) * a.page_size + in_page;
        uint8_t* codes = (kind == 1 ? a.k_codes : a.v_codes) + at * (D / 2) + c * (C / 2);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          if (CV == 2)
            *reinterpret_cast<uint2*>(codes + s * (D / 4)) = make_uint2(words[s][0], words[s][1 % CV]);
          else
            *reinterpret_cast<uint32_t*>(codes + s * (D / 4)) = words[s][0];
        }
        if (c == 0) {
          const float nrm = kind == 1 ? a.norm : 1.f;
          reinterpret_cast<float2*>(a.scales + at * 4)[kind - 1] =
              make_float2(__fmul_rn(__fdiv_rn(span, 15.f), nrm), __fmul_rn(lo, nrm));
        }
      }
    }
  }
}

template <int D, bool CLAMP, int ROPE>
cudaError_t append_t(const AppendArgs& a, cudaStream_t stream) {
  const int groups = (int)((a.Hq + 2 * a.Hkv + 7) / 8);
  const int64_t units = a.T * groups;
  int per_sm = 1;
  cudaError_t e = prepare_launch(kv4_append_kernel<D, CLAMP, ROPE>, kAppendWarps * 32, 0, &per_sm);
  if (e != cudaSuccess) return e;
  int64_t blocks = (units + kAppendWarps - 1) / kAppendWarps;
  const int64_t cap = (int64_t)device_sm_count() * per_sm;
  if (blocks > cap) blocks = cap;
  e = launch_pdl(kv4_append_kernel<D, CLAMP, ROPE>, dim3((unsigned)blocks), dim3(kAppendWarps * 32), 0, stream, 1, a,
                 units, groups);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int D, bool CLAMP>
cudaError_t append_c(const AppendArgs& a, cudaStream_t stream) {
  if (a.rotary == 0) return append_t<D, CLAMP, kRopeNone>(a, stream);
  if (a.interleaved) return append_t<D, CLAMP, kRopePairs>(a, stream);
  return a.rotary == D ? append_t<D, CLAMP, kRopeHalves>(a, stream) : append_t<D, CLAMP, kRopePartHalves>(a, stream);
}

// One warp per output token: it looks the token's page up once and walks the
// kv heads.  D / 8 lanes share a row of codes (4 bytes, 8 values and one
// 16-byte store per lane); a warp covers 32 / (D / 8) rows, K and V side by
// side.
template <int D>
__global__ void __launch_bounds__(kReadWarps * 32) kv4_read_kernel(ReadArgs a) {
  constexpr int LPR = D / 8;          // lanes per row
  constexpr int HPS = 32 / LPR / 2;   // kv heads per step (K and V of each)
  const int lane = threadIdx.x & 31;
  const int part = lane % LPR, which = (lane / LPR) & 1, hs = lane / (2 * LPR);
  const int64_t stride = (int64_t)gridDim.x * kReadWarps;
  pdl_wait();
  pdl_trigger();
  for (int64_t i = (int64_t)blockIdx.x * kReadWarps + (threadIdx.x >> 5); i < a.total; i += stride) {
    // the last sequence whose offset is <= i
    int lo = 0, hi = (int)a.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((int64_t)__ldg(a.cu + mid) <= i) lo = mid; else hi = mid - 1;
    }
    const int64_t t = i - __ldg(a.cu + lo) + (a.starts ? __ldg(a.starts + lo) : 0);
    const int64_t pi = t >= 0 ? t / a.page_size : -1;
    int64_t page = -1;
    if (pi >= 0 && pi < a.table_width) page = __ldg(a.table + (int64_t)lo * a.table_width + pi);
    const bool in = page >= 0 && page < a.num_pages && i < __ldg(a.cu + a.batch);
    const int64_t at0 = in ? (page * a.Hkv) * a.page_size + (t - pi * a.page_size) : 0;
    const uint8_t* codes = which ? a.v_codes : a.k_codes;
    __half* out = reinterpret_cast<__half*>(which ? a.v : a.k) + i * a.Hkv * D + part * 8;
#pragma unroll 4
    for (int h = hs; h < a.Hkv; h += HPS) {
      uint4 w = make_uint4(0, 0, 0, 0);   // tokens without a page read as zeros
      if (in) {
        const int64_t at = at0 + (int64_t)h * a.page_size;
        const uint32_t c = __ldg(reinterpret_cast<const uint32_t*>(codes + at * (D / 2)) + part);
        const float2 f = __ldg(reinterpret_cast<const float2*>(a.scales + at * 4) + which);
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o[j] = pack_half2_bits(fmaf((float)((c >> (8 * j)) & 15u), f.x, f.y),
                                 fmaf((float)((c >> (8 * j + 4)) & 15u), f.x, f.y));
        w = make_uint4(o[0], o[1], o[2], o[3]);
      }
      *reinterpret_cast<uint4*>(out + (int64_t)h * D) = w;
    }
  }
}

template <int D>
cudaError_t read_t(const ReadArgs& a, cudaStream_t stream) {
  int per_sm = 1;
  cudaError_t e = prepare_launch(kv4_read_kernel<D>, kReadWarps * 32, 0, &per_sm);
  if (e != cudaSuccess) return e;
  int64_t blocks = (a.total + kReadWarps - 1) / kReadWarps;
  const int64_t cap = (int64_t)device_sm_count() * per_sm;
  if (blocks > cap) blocks = cap;
  e = launch_pdl(kv4_read_kernel<D>, dim3((unsigned)blocks), dim3(kReadWarps * 32), 0, stream, 1, a);
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
