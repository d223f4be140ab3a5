// prompt_attention.cu -- spinq_prompt_attention: causal attention over packed
// prompts with grouped heads.
//
//   o_i = sum_{j < n_i} softmax_j(scale q_i . k_j) v_j
//
// n_i = min(lk, i + 1 + lk - lq) with the causal mask (the queries are the
// last lq of the sequence's lk positions), else lk; a query that sees no key
// gives zeros.  One warp per (query, head): a lane takes a key's score, then
// D/32 values of the weighted sum; running maximum and sum in fp32.
#include <cuda_fp16.h>

#include "launch_util.h"
#include "spinq_device.cuh"
#include "spinq_internal.h"

namespace spinq {
namespace {

template <int D>
__global__ void __launch_bounds__(128) prompt_rows_kernel(PromptArgs a) {
  constexpr int DPL = D / 32;
  __shared__ float q_s[4][D];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t stride = (int64_t)gridDim.x * 4;
  pdl_wait();
  pdl_trigger();
  for (int64_t u = (int64_t)blockIdx.x * 4 + warp; u < a.total_q * a.Hq; u += stride) {
    const int64_t i = u / a.Hq, h = u - i * a.Hq, hk = h / (a.Hq / a.Hkv);
    int lo = 0, hi = (int)a.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((int64_t)a.cu_q[mid] <= i) lo = mid; else hi = mid - 1;
    }
    if (i >= a.cu_q[a.batch]) break;   // a row after the last sequence
    const int64_t q0 = a.cu_q[lo], lq = a.cu_q[lo + 1] - q0, k0 = a.cu_k[lo], lk = a.cu_k[lo + 1] - k0;
    int64_t n = a.causal ? i - q0 + 1 + lk - lq : lk;
    n = n < 0 ? 0 : (n > lk ? lk : n);
    const __half* q = reinterpret_cast<const __half*>(a.q) + i * a.ldq + h * D;
    __syncwarp();
    for (int d = lane; d < D; d += 32) q_s[warp][d] = __half2float(q[d]) * a.scale;
    __syncwarp();
    const __half* kb = reinterpret_cast<const __half*>(a.k) + k0 * a.ldk + hk * D;
    const __half* vb = reinterpret_cast<const __half*>(a.v) + k0 * a.ldv + hk * D;
    float m = -INFINITY, l = 0.f, o[DPL] = {};
    for (int64_t j0 = 0; j0 < n; j0 += 32) {
      const int64_t j = j0 + lane;
      float s = -INFINITY;
      if (j < n) {
        s = 0.f;
        const uint4* kr = reinterpret_cast<const uint4*>(kb + j * a.ldk);
        for (int e = 0; e < D / 8; ++e) {
          const uint4 w = __ldg(kr + e);
          const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&ws[x]));
            s = fmaf(f.x, q_s[warp][8 * e + 2 * x], s);
            s = fmaf(f.y, q_s[warp][8 * e + 2 * x + 1], s);
          }
        }
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
#pragma unroll
        for (int e = 0; e < DPL; ++e) o[e] = fmaf(px, __half2float(vb[(j0 + x) * a.ldv + 32 * e + lane]), o[e]);
      }
      m = mn;
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int e = 0; e < DPL; ++e)
      reinterpret_cast<__half*>(a.out)[(i * a.Hq + h) * D + 32 * e + lane] = __float2half_rn(o[e] * inv);
  }
}

template <int D>
cudaError_t launch_t(const PromptArgs& a, cudaStream_t stream) {
  int64_t blocks = (a.total_q * a.Hq + 3) / 4;
  const int64_t cap = (int64_t)device_sm_count() * 16;
  if (blocks > cap) blocks = cap;
  const cudaError_t e = launch_pdl(prompt_rows_kernel<D>, dim3((unsigned)blocks), dim3(128), 0, stream, 1, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

int64_t prompt_attention_workspace(const PromptArgs&) { return 0; }

cudaError_t launch_prompt_attention(const PromptArgs& a, cudaStream_t stream) {
  if (a.D == 128) return launch_t<128>(a, stream);
  if (a.D == 64) return launch_t<64>(a, stream);
  return cudaErrorNotSupported;
}

}  // namespace spinq
