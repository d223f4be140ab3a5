// tree_attention.cuh -- what the kernels of spinq_tree_attention_kv4 share: what a
// row sees, and how the work is dealt to the CTAs (tree_attention.cu).
#pragma once

#include <stdint.h>

#include "spinq_device.cuh"
#include "spinq_internal.h"

namespace spinq {

constexpr int kTreeNodes = 128;   // queries of a sequence at most

struct TreeParams {
  TreeArgs a;
  int G, shift;            // query heads per kv head; page_size = 1 << shift
  uint32_t g_inv;          // ceil(2^32 / G); 0 for G = 1
  int window, sinks, cap;  // window 0: none; tokens that a row of the table has room for
  int ctas;                // of the attention kernel's grid
  int rows_log2, unit_log2;   // rows of a job, tokens of a unit
  int least;               // units a CTA gets at least
  float scale_log2;
  float* o;                // [2 * ctas][rows][D]: of CTA c the job it continues (2 c) and the one it leaves (2 c + 1)
  float2* ml;              // [2 * ctas][rows]: M, and sum of w / alpha'
  int* status;
  int debug_stall;
};

// x / G of a row number x < 2^16: x ceil(2^32 / G) is less than x + 2^32 / G off 2^32 x / G.
__device__ __forceinline__ int tree_node(const TreeParams& p, int x) { return p.g_inv ? (int)__umulhi((uint32_t)x, p.g_inv) : x; }

// What the lengths say of a sequence.
struct TreeSeq {
  int n, nq, ctx;     // tokens, queries, tokens before the queries' own (below 0: the first queries have none)
  int q0;
  int front, skip;    // units of sinks; units left out behind them
  int units, rts, jobs;
};

__device__ __forceinline__ TreeSeq tree_seq(const TreeParams& p, int b) {
  const TreeArgs& a = p.a;
  TreeSeq s;
  s.n = min(max(__ldg(a.lens + b), 0), p.cap);
  s.q0 = b;
  s.nq = 1;
  if (a.cu_q) {
    s.q0 = max(__ldg(a.cu_q + b), 0);
    s.nq = max(0, min(min(__ldg(a.cu_q + b + 1), (int)a.total_q) - s.q0, (int)a.max_q));
  }
  s.ctx = s.n - s.nq;
  const int reach = p.window > 0 && s.ctx >= p.window ? (s.ctx - p.window + 1) >> p.unit_log2 : 0;
  s.front = min((int)(((unsigned)p.sinks + (1u << p.unit_log2) - 1) >> p.unit_log2), reach);
  s.skip = reach - s.front;
  // one at least: a sequence without tokens has rows too
  s.units = max(1, ((s.n + (1 << p.unit_log2) - 1) >> p.unit_log2) - s.skip);
  s.rts = (s.nq * p.G + (1 << p.rows_log2) - 1) >> p.rows_log2;
  s.jobs = s.rts * (int)a.Hkv;
  return s;
}

// Where the units of run c of `ctas` lie: [bound(c), bound(c + 1)) of all; the first of them in
// sequence b, whose units begin at `base`.
struct TreeRun {
  int64_t per, base;
  int rest, ctas, b;
  TreeSeq s;   // of sequence b
  __device__ __forceinline__ int64_t bound(int c) const { return per * c + min(c, rest); }
  // the run that unit x is in
  __device__ __forceinline__ int owner(int64_t x) const {
    const int64_t longer = (per + 1) * rest;   // units of the runs that have one more
    const int64_t y = x < longer ? x : x - longer, by = x < longer ? per + 1 : per;
    const int c = y <= INT32_MAX && by <= INT32_MAX ? (int)((uint32_t)y / (uint32_t)by) : (int)(y / by);
    return x < longer ? c : rest + c;
  }
};

// PARTS > 0: at most that many runs per job of the batch, so that even jobs are cut into about that many
// at most (one that is far longer than the others into more).  The parts of a job are
// joined eight at a time, which for few jobs takes as long as their keys.
template <int THREADS, int PARTS>
__device__ __forceinline__ TreeRun tree_run(const TreeParams& p, int c) {
  __shared__ int64_t sums[THREADS / 32], base_s;
  __shared__ int jobs_s[PARTS > 0 ? THREADS / 32 : 1];
  __shared__ int b_s;
  __shared__ TreeSeq seq_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, B = (int)p.a.B;
  const int per = B <= THREADS ? 1 : (B + THREADS - 1) / THREADS, b0 = min(tid * per, B), b1 = min(b0 + per, B);
  int64_t mine = 0;
  int jobs = 0;   // (4096 stands for more: the limit is above any grid)
  TreeSeq s = {};
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    s = tree_seq(p, b);
    mine += (int64_t)s.units * s.jobs;
    jobs = min(jobs + min(s.jobs, 4096), 4096);
  }
  if constexpr (PARTS > 0) {
    jobs = __reduce_add_sync(0xffffffffu, jobs);
    if (lane == 0) jobs_s[warp] = jobs;
  }
  int64_t sum = mine;
#pragma unroll
  for (int w = 1; w < 32; w <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, sum, w);
    if (lane >= w) sum += y;
  }
  if (lane == 31) sums[warp] = sum;
  if (tid == 0) b_s = B;
  __syncthreads();
  int64_t at = sum - mine, all = 0;
  int ctas = p.ctas;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w == warp) at += all;
    all += sums[w];
  }
  if constexpr (PARTS > 0) {
    jobs = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) jobs += jobs_s[w];
    ctas = min(ctas, jobs * PARTS);
  }
  TreeRun r;
  if (all <= INT32_MAX) {   // (32-bit divisions: a wave of CTAs waits for these)
    const uint32_t n = (uint32_t)all;
    r.ctas = (int)min((uint32_t)ctas, (n + p.least - 1) / p.least);
    if (PARTS > 0 && n > (uint32_t)r.ctas && n < 4u * r.ctas) {   // (as few runs as the longest allows)
      const uint32_t longest = (n + r.ctas - 1) / (uint32_t)r.ctas;
      r.ctas = (int)((n + longest - 1) / longest);
    }
    r.per = r.ctas ? n / (uint32_t)r.ctas : 0;
  } else {
    r.ctas = ctas;
    r.per = all / ctas;
  }
  r.rest = (int)(all - r.per * r.ctas);
  if (c < r.ctas) {
    const int64_t x = r.bound(c);
    if (at <= x && x < at + mine) {
      int b = b0;
      if (per > 1) {
#pragma unroll 1
        for (; b < b1; ++b) {
          s = tree_seq(p, b);
          const int64_t t = (int64_t)s.units * s.jobs;
          if (x < at + t) break;
          at += t;
        }
      }
      b_s = b;
      base_s = at;
      seq_s = s;
    }
  }
  __syncthreads();
  r.b = b_s;
  r.base = base_s;
  r.s = seq_s;
  return r;
}

// A row's view of the keys.
struct TreeRow {
  uint32_t line[4];   // its ancestors that it sees, and itself
  int low;            // first context token that its window reaches
};

// The queries' parents in shared memory (all threads), then a thread's row of them.
__device__ __forceinline__ void tree_parents(const TreeParams& p, const TreeSeq& s, int* parent, int threads) {
  for (int i = threadIdx.x; i < s.nq; i += threads) parent[i] = p.a.parents ? __ldg(p.a.parents + s.q0 + i) : i - 1;
}
__device__ __forceinline__ TreeRow tree_row(const TreeParams& p, const TreeSeq& s, const int* parent, int node) {
  auto up = [&](int i) {   // (a parent comes before its node; any other number: none)
    const int x = parent[i];
    return x >= 0 && x < i ? x : -1;
  };
  TreeRow r;
  int depth = -1;
  r.line[0] = r.line[1] = r.line[2] = r.line[3] = 0;
  auto see = [&](int i) {
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (w == i >> 5) r.line[w] |= 1u << (i & 31);
  };
  const int window = p.window > 0 ? p.window : INT32_MAX;
  if (window >= s.nq) {   // (no line is longer)
    for (int i = node; i >= 0; i = up(i)) ++depth, see(i);
  } else {
    for (int i = node; i >= 0; i = up(i)) ++depth;
    for (int i = node, k = 0; i >= 0; i = up(i), ++k)
      if (k < window || s.ctx + depth - k < p.sinks) see(i);
  }
  r.low = p.window > 0 && s.ctx + depth >= p.window ? s.ctx + depth - p.window + 1 : 0;
  return r;
}

// Bits a .. b - 1 of the 32 from `at` on.
__device__ __forceinline__ uint32_t tree_span(int a, int b, int at) {
  const int lo = max(min(a - at, 32), 0), hi = max(min(b - at, 32), 0);
  return hi > lo ? (0xffffffffu >> (32 - (hi - lo))) << lo : 0u;
}
// What a row sees of tokens at .. at + 31, a bit per token.
__device__ __forceinline__ uint32_t tree_sees(const TreeParams& p, const TreeSeq& s, const TreeRow& r, int at) {
  uint32_t bits = tree_span(r.low, s.ctx, at) | tree_span(0, min(p.sinks, s.ctx), at);
  const int first = at - s.ctx, w = first >> 5, sh = first & 31;   // the node at `at`, its word and bit
  const uint32_t x = w >= 0 && w < 4 ? r.line[w & 3] : 0u, y = w >= -1 && w < 3 ? r.line[(w + 1) & 3] : 0u;
  return bits | __funnelshift_r(x, y, sh);
}

__device__ __forceinline__ int64_t tree_page(const TreeArgs& a, const int32_t* table, int t, int shift) {
  const int64_t page = __ldg(table + (t >> shift));
  return page < 0 ? 0 : (page >= a.num_pages ? a.num_pages - 1 : page);
}

// A job, or what of it a CTA has.
struct TreeJob {
  TreeSeq s;
  int b, hk, r0, rows;   // sequence, kv head, first row of the group's and how many
  int v0, v1;            // units of it that this CTA has
  __device__ __forceinline__ bool whole() const { return v0 == 0 && v1 == s.units; }
  __device__ __forceinline__ int64_t slot(int cta) const { return 2 * (int64_t)cta + (v0 == 0 ? 1 : 0); }
  // first token of unit v
  __device__ __forceinline__ int token(int v, int unit) const { return (v < s.front ? v : v + s.skip) * unit; }
  // a row's place among [query][head] rows
  __device__ __forceinline__ int64_t row_at(const TreeParams& p, int r) const {
    const int node = tree_node(p, r0 + r), head = r0 + r - node * p.G;
    return (int64_t)(s.q0 + node) * p.a.Hq + hk * p.G + head;
  }
};
// A CTA's way through its run.
struct TreeWalk {
  int64_t x, x1, base;
  int b;
  TreeSeq s;   // of sequence b
  __device__ __forceinline__ TreeWalk(const TreeRun& r, int c)
      : x(c < r.ctas ? r.bound(c) : 0), x1(c < r.ctas ? r.bound(c + 1) : 0), base(r.base), b(r.b), s(r.s) {}
  __device__ __forceinline__ bool next(const TreeParams& p, TreeJob& j) {
    while (x < x1 && b < (int)p.a.B) {
      j.s = s;
      const int64_t all = (int64_t)j.s.units * j.s.jobs, at = x - base;
      if (at >= all) {
        base += all;
        if (++b < (int)p.a.B) s = tree_seq(p, b);
        continue;
      }
      const int job = all <= INT32_MAX ? (int)((uint32_t)at / (uint32_t)j.s.units) : (int)(at / j.s.units);
      j.b = b;
      j.v0 = (int)(at - (int64_t)job * j.s.units);
      j.v1 = (int)min((int64_t)j.s.units, j.v0 + (x1 - x));
      j.hk = job / j.s.rts;
      j.r0 = (job - j.hk * j.s.rts) << p.rows_log2;
      j.rows = min(1 << p.rows_log2, j.s.nq * p.G - j.r0);
      x += j.v1 - j.v0;
      return true;
    }
    return false;
  }
};

// Many rows, on the 5th-generation tensor core (tree_attention_tc.cu): jobs of 32, 64 or 128
// rows, one CTA per SM.
constexpr int kTreeTcUnitLog2 = 7;
cudaError_t launch_tree_tc(const TreeParams& p, cudaStream_t stream);

}  // namespace spinq
