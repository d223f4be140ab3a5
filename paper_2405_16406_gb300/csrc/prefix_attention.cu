// prefix_attention.cu -- spinq_prefix_attention_kv4: one query per (sequence,
// head) over a prefix that every sequence shares and the sequence's own
// tokens, both in the paged 4-bit cache.
//
//   s_t = scale q . k_t,  k_t = alpha_t u_t + beta_t
//   o   = sum_t softmax_t(s) v_t,  v_t = alpha'_t u'_t + beta'_t
//
// over the prefix's tokens, then the sequence's own lens[b].  One warp per
// (sequence, head): a lane takes a token's score, then D/32 values of the
// weighted sum; running maximum and sum in fp32.
#include <cuda_fp16.h>

#include "launch_util.h"
#include "spinq_device.cuh"
#include "spinq_internal.h"

namespace spinq {
namespace {

template <int D>
__global__ void __launch_bounds__(128) prefix_rows_kernel(PrefixArgs a) {
  constexpr int DPL = D / 32;
  __shared__ float q_s[4][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t stride = (int64_t)gridDim.x * 4;
  pdl_wait();
  pdl_trigger();
  for (int64_t u = (int64_t)blockIdx.x * 4 + warp; u < a.B * a.Hq; u += stride) {
    const int64_t b = u / a.Hq, h = u - b * a.Hq, hk = h / (a.Hq / a.Hkv);
    int64_t own = a.lens[b];
    own = own < 0 ? 0 : (own > a.table_width * a.page_size ? a.table_width * a.page_size : own);
    const int64_t n = a.prefix_len + own;
    __syncwarp();
    float qsum = 0.f;
    for (int d = lane; d < D; d += 32) {
      const float f = __half2float(reinterpret_cast<const __half*>(a.q)[(b * a.Hq + h) * D + d]) * a.scale;
      q_s[warp][d] = f;
      qsum += f;
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) qsum += __shfl_xor_sync(0xffffffffu, qsum, w);
    __syncwarp();
    float m = -INFINITY, l = 0.f, o[DPL] = {};
    for (int64_t j0 = 0; j0 < n; j0 += 32) {
      const int64_t j = j0 + lane;
      float s = -INFINITY;
      int64_t at = 0;
      if (j < n) {
        const int64_t t = j < a.prefix_len ? j : j - a.prefix_len;
        const int64_t pi = t / a.page_size;
        int64_t page = j < a.prefix_len ? a.prefix_table[pi] : a.table[b * a.table_width + pi];
        page = page < 0 ? 0 : (page >= a.num_pages ? a.num_pages - 1 : page);
        at = (page * a.Hkv + hk) * a.page_size + (t - pi * a.page_size);
        const uint32_t* kr = reinterpret_cast<const uint32_t*>(a.k_codes + at * (D / 2));
        float dot = 0.f;
        for (int e = 0; e < D / 8; ++e) {
          const uint32_t w = __ldg(kr + e);
#pragma unroll
          for (int x = 0; x < 8; ++x) dot = fmaf((float)((w >> (4 * x)) & 15u), q_s[warp][8 * e + x], dot);
        }
        s = a.scales[at * 4] * dot + a.scales[at * 4 + 1] * qsum;
      }
      float mx = s;
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float mn = fmaxf(m, mx);
      const float corr = __expf(m - mn), p = __expf(s - mn);
      l = l * corr + p;
#pragma unroll
      for (int e = 0; e < DPL; ++e) o[e] *= corr;
      const int cnt = n - j0 < 32 ? (int)(n - j0) : 32;
      for (int x = 0; x < cnt; ++x) {
        const float px = __shfl_sync(0xffffffffu, p, x);
        const int64_t ax = __shfl_sync(0xffffffffu, at, x);
        const float va = a.scales[ax * 4 + 2], vb = a.scales[ax * 4 + 3];
#pragma unroll
        for (int e = 0; e < DPL; ++e) {
          const int d = 32 * e + lane;
          const uint32_t code = (a.v_codes[ax * (D / 2) + d / 2] >> (4 * (d & 1))) & 15u;
          o[e] = fmaf(px, fmaf((float)code, va, vb), o[e]);
        }
      }
      m = mn;
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int e = 0; e < DPL; ++e)
      reinterpret_cast<__half*>(a.out)[(b * a.Hq + h) * D + 32 * e + lane] = __float2half_rn(o[e] * inv);
  }
}

template <int D>
cudaError_t launch_t(const PrefixArgs& a, cudaStream_t stream) {
  int64_t blocks = (a.B * a.Hq + 3) / 4;
  const int64_t cap = (int64_t)device_sm_count() * 16;
  if (blocks > cap) blocks = cap;
  const cudaError_t e = launch_pdl(prefix_rows_kernel<D>, dim3((unsigned)blocks), dim3(128), 0, stream, 1, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

int64_t prefix_attention_workspace(const PrefixArgs&) { return 0; }

cudaError_t launch_prefix_attention(const PrefixArgs& a, cudaStream_t stream) {
  if (a.D == 128) return launch_t<128>(a, stream);
  if (a.D == 64) return launch_t<64>(a, stream);
  return cudaErrorNotSupported;
}

}  // namespace spinq
