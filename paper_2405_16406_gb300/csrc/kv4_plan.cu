// kv4_plan.cu -- bookkeeping of the paged 4-bit cache on the GPU:
// spinq_kv4_plan (pages, positions and slots of a step's tokens from the
// requests' lengths) and spinq_kv4_keep (the accepted path of each drafted tree
// moves together).
//
// Plan.  With P tokens a page and, for sequence b,
//   start = max(lens - drop, 0),  kept = ceil(start / P),
//   freed = the entries kept .. ceil(lens / P) - 1 that are pages (not below 0: given back
//   before, as a window passed them),  need = ceil((start + add) / P) - kept,
// the free pages are a stack: freed page i of all (sequences in order, pages in
// order) lies i below its top, and page a of all that are needed is the a-th from
// the top, so a sequence that gives and takes gets its own pages back.  Three
// prefix sums over the batch (tokens, freed, needed pages) say where everything is:
// every CTA takes them by itself, in shared memory.
//  * Up to kPlanTokens rows: one kernel, of one CTA or a cluster, whose threads share the pages
//    and tokens.  The stack is written before a barrier and read behind it.  A few dropped entries of a
//    sequence are looked through by the thread that loads its lengths, many by a warp of the grid.
//  * More: the dropped entries are counted, a warp per sequence, by a kernel of its own; then the
//    tokens by a kernel that fills the GPU and reads the lists as they were, then
//    the lists and lengths by the one cluster (1000 sequences, 251 K tokens: 60 us in one
//    kernel, whose 4096 threads had 64 dependent look-ups each).
// Bound: latency (a chain of the lengths' loads and the dropped entries, three block-wide sums, a
// barrier, and two dependent loads).  Call after call in a graph: 8 sequences of one token 3.5 us, 512 of
// one 6.9, those 1000 sequences 23.4 (3.7 of them for the count; 29.4 with the copies that put the lengths
// back), 8 of 32768 tokens that end among 248 of one more 11.9, 256 that end among 256 95.8 (524 K pages of 16).
//
// Keep.  A path ascends, so a token never moves up and never onto one that is
// still to be read by a later part of its path: a CTA takes the 16-byte pieces of
// a sequence and a kv head in rounds, reads all of a round, then writes it.  Bound: latency
// (4 x 3 tokens 2.2 us, 256 x 11 of 8 heads 3.85 us: 6.5 MB, 1.7 TB/s).
#include "launch_util.h"
#include "spinq_device.cuh"
#include "spinq_internal.h"

namespace spinq {
namespace {

constexpr int kPlanCluster = 8;
constexpr int64_t kPlanTokens = 8192;
enum PlanPart { kPlanAll = 0, kPlanRows = 1, kPlanLists = 2 };
constexpr uint32_t kPlanOwn = 4;                 // dropped entries of a sequence that a thread looks through by itself
constexpr uint32_t kPlanLong = 0x80000000u;      // more of them (a sequence has fewer than 2^27 pages)

// Sums of whole numbers in [0, 2^31) that stay there.
constexpr uint32_t kPlanMost = 0x7fffffffu;
__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return min(a + b, kPlanMost); }

// Exclusive prefix sum of x over the block and the total; `part`: a word per warp.
template <int THREADS>
__device__ __forceinline__ uint32_t block_prefix(uint32_t x, uint32_t* part, uint32_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t s = x;
#pragma unroll
  for (int w = 1; w < 32; w <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, s, w);
    if (lane >= w) s = sat_add(s, y);
  }
  __syncthreads();   // the last sum's parts have been read
  if (lane == 31) part[warp] = s;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w == warp) before = all;
    all = sat_add(all, part[w]);
  }
  *total = all;
  uint32_t ex = __shfl_up_sync(0xffffffffu, s, 1);
  if (lane == 0) ex = 0;
  return sat_add(before, ex);
}

// The last i of [0, n) with start[i] <= x, where start ascends from 0.
__device__ __forceinline__ int last_at_most(const uint32_t* start, int n, uint32_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// How many of a sequence's entries e[0 .. n - 1] are pages (a warp).
__device__ __forceinline__ uint32_t count_pages(const int32_t* e, uint32_t n) {
  uint32_t have = 0;
#pragma unroll 16
  for (uint32_t i = threadIdx.x & 31; i < n; i += 32) have += __ldcg(e + i) >= 0;
  return __reduce_add_sync(0xffffffffu, have);
}

// Into cu_tokens, which the lists' kernel writes at its end: the pages that each sequence gives back, a warp each.
constexpr int kPlanCountThreads = 256;
__global__ void __launch_bounds__(kPlanCountThreads) kv4_plan_count_kernel(const PlanArgs a) {
  const int b = blockIdx.x * (kPlanCountThreads / 32) + (threadIdx.x >> 5);
  const uint32_t page1 = (1u << a.page_shift) - 1, cap = (uint32_t)(a.table_width << a.page_shift);
  pdl_wait();
  pdl_trigger();
  if (b >= (int)a.batch) return;
  const uint32_t len = min((uint32_t)max(a.lens[b], 0), cap), drop = (uint32_t)max(a.drop[b], 0);
  const uint32_t s = len > drop ? len - drop : 0u, kept = (s + page1) >> a.page_shift;
  const uint32_t have = count_pages(a.table + (int64_t)b * a.table_width + kept, ((len + page1) >> a.page_shift) - kept);
  if ((threadIdx.x & 31) == 0) a.cu_tokens[b] = (int32_t)have;
}

// PER: sequences per thread at most.
template <int THREADS, int PER, int PART>
__global__ void __launch_bounds__(THREADS, 1) kv4_plan_kernel(const PlanArgs a) {
  extern __shared__ uint32_t plan_smem[];
  __shared__ uint32_t part[THREADS / 32];
  __shared__ uint32_t holes[kPlanMaxBatch / 32], any_hole;   // sequences that drop entries which are no pages; whether one does
  __shared__ uint32_t lost[kPlanMaxBatch / 32];              // whose new tokens would begin in such an entry
  const int B = (int)a.batch;
  uint32_t* start = plan_smem;        // tokens that stay
  uint32_t* cu = start + B;           // tokens asked for before this sequence
  uint32_t* freed = cu + B;           // pages freed before it
  uint32_t* taken = freed + B;        // pages needed before it
  uint32_t* gets = taken + B;         // pages it gets, or kPlanMost: refused
  const int tid = threadIdx.x, shift = a.page_shift;
  const uint32_t stride = gridDim.x * THREADS, first = blockIdx.x * THREADS + tid;
  const uint32_t page1 = (1u << shift) - 1, cap = (uint32_t)(a.table_width << shift), total = (uint32_t)a.total;
  auto pages = [&](uint32_t tokens) { return (tokens + page1) >> shift; };   // tokens <= 2^31 - 256
  auto dropped = [&](int b) { return a.table + (int64_t)b * a.table_width + pages(start[b]); };   // the first dropped entry
  auto hole = [&](int b) { return (holes[b >> 5] >> (b & 31) & 1u) != 0; };
  auto count_is = [&](int b, uint32_t entries, uint32_t have) {   // of them are pages
    freed[b] = have;
    if (have != entries) {
      atomicOr(&holes[b >> 5], 1u << (b & 31));
      any_hole = 1;
    }
  };
  auto grid_sync = [&]() {   // what the grid, one cluster, has written can be read
    if (gridDim.x > 1) {
      __threadfence();
      asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;\n" ::: "memory");
    } else {
      __syncthreads();
    }
  };
  for (int i = tid; i < (B + 31) / 32; i += THREADS) holes[i] = lost[i] = 0;
  if (tid == 0) any_hole = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  const int32_t count0 = *a.free_count;
  bool many = false;
  for (int b = tid; b < B; b += THREADS) {
    const uint32_t len = min((uint32_t)max(a.lens[b], 0), cap), drop = a.drop ? (uint32_t)max(a.drop[b], 0) : 0u;
    const uint32_t s = len > drop ? len - drop : 0u, entries = pages(len) - pages(s);
    const uint32_t add = a.add ? (uint32_t)max(a.add[b], 0) : 0u;
    start[b] = s;
    cu[b] = add;
    if (add > 0 && (s & page1) && __ldcg(a.table + (int64_t)b * a.table_width + (s >> shift)) < 0)
      atomicOr(&lost[b >> 5], 1u << (b & 31));
    if (PART != kPlanAll) {
      count_is(b, entries, a.drop ? (uint32_t)__ldcg(a.cu_tokens + b) : 0u);
    } else if (entries <= kPlanOwn) {
      const int32_t* e = dropped(b);
      uint32_t have = 0;
#pragma unroll
      for (uint32_t k = 0; k < kPlanOwn; ++k)
        if (k < entries) have += __ldcg(e + k) >= 0;
      count_is(b, entries, have);
    } else {
      freed[b] = entries | kPlanLong;
      many = true;
    }
  }
  // (every CTA finds the same)
  if (__syncthreads_or(many)) {
    // counted by the grid's warps in turn, and passed on through cu_tokens, which is written last of all
    for (int b = (int)(first >> 5); b < B; b += (int)(stride >> 5))
      if (freed[b] & kPlanLong) {
        const uint32_t have = count_pages(dropped(b), freed[b] & ~kPlanLong);
        if ((tid & 31) == 0) a.cu_tokens[b] = (int32_t)have;
      }
    grid_sync();
    for (int b = tid; b < B; b += THREADS)
      if (freed[b] & kPlanLong) count_is(b, freed[b] & ~kPlanLong, (uint32_t)__ldcg(a.cu_tokens + b));
    __syncthreads();
  }
  // a thread's sequences lie next to one another
  const int per = (B + THREADS - 1) / THREADS, b0 = min(tid * per, B), b1 = min(b0 + per, B);
  uint32_t sum_add = 0, sum_freed = 0;
  for (int b = b0; b < b1; ++b) sum_add = sat_add(sum_add, cu[b]), sum_freed = sat_add(sum_freed, freed[b]);
  uint32_t all_add, all_freed, all_need;
  uint32_t at_add = block_prefix<THREADS>(sum_add, part, &all_add);
  uint32_t at_freed = block_prefix<THREADS>(sum_freed, part, &all_freed);
  uint32_t need[PER], sum_need = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    need[k] = 0;
    if (b0 + k < b1) {
      const int b = b0 + k;
      const uint32_t add = cu[b], f = freed[b];
      cu[b] = at_add;
      freed[b] = at_freed;
      at_add = sat_add(at_add, add);
      at_freed = sat_add(at_freed, f);
      // it fits the answer's arrays and its row of the table (start <= cap), and its last page is there
      const bool fits = add == 0 || (at_add <= total && add <= cap - start[b] && !(lost[b >> 5] >> (b & 31) & 1u));
      need[k] = fits ? pages(start[b] + add) - pages(start[b]) : 0u;
      gets[b] = fits ? need[k] : kPlanMost;
      sum_need = sat_add(sum_need, need[k]);
    }
  }
  uint32_t at_need = block_prefix<THREADS>(sum_need, part, &all_need);
  const uint32_t count = (uint32_t)min(max((int64_t)count0, (int64_t)0), a.free_capacity);
  const uint32_t there = (uint32_t)min((int64_t)sat_add(count, all_freed), a.free_capacity);   // free pages
  uint32_t given = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k)
    if (b0 + k < b1) {
      const int b = b0 + k;
      taken[b] = at_need;
      at_need = sat_add(at_need, need[k]);
      if (need[k] > 0) {
        if (at_need > there) gets[b] = kPlanMost;
        else given = at_need;
      }
    }
  // (pages needed so far ascend: the largest sum that was granted is what was handed out)
  given = __reduce_max_sync(0xffffffffu, given);
  __syncthreads();
  if ((tid & 31) == 0) part[tid >> 5] = given;
  __syncthreads();
  given = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) given = max(given, part[w]);

  // where freed page i of all lies, as long as the table has not been written
  auto freed_page = [&](uint32_t i) -> const int32_t* {
    const int b = last_at_most(freed, B, i);
    const int32_t *e = dropped(b), *last = a.table + (int64_t)(b + 1) * a.table_width - 1;
    uint32_t k = i - freed[b];
    if (!hole(b)) return e + k;
    while (e < last && (__ldcg(e) < 0 || k-- > 0)) ++e;   // (it has more than k pages)
    return e;
  };
  if (PART != kPlanRows) {
    // freed pages onto the stack (where a list that is too short left room for them)
    const uint32_t room = there - count;
    for (uint32_t i = first; i < all_freed && i < room; i += stride) {
      const int b = last_at_most(freed, B, i);
      if (!hole(b)) a.free_pages[there - 1 - i] = __ldcg(dropped(b) + i - freed[b]);
    }
    if (any_hole) {   // a warp looks the others' entries through
      for (int b = (int)(first >> 5); b < B; b += (int)(stride >> 5)) {
        if (!hole(b)) continue;
        const int32_t* e = dropped(b);
        const uint32_t end = b + 1 < B ? freed[b + 1] : all_freed, width = (uint32_t)a.table_width - pages(start[b]);
        uint32_t i = freed[b];
        for (uint32_t k = tid & 31; i < end && (k & ~31u) < width; k += 32) {
          const int32_t page = k < width ? __ldcg(e + k) : -1;   // (what lies behind the last dropped one comes too late)
          const uint32_t has = __ballot_sync(0xffffffffu, page >= 0);
          const uint32_t at = i + __popc(has & ((1u << (tid & 31)) - 1));
          if (page >= 0 && at < end && at < room) a.free_pages[there - 1 - at] = page;
          i += __popc(has);
        }
      }
    }
    grid_sync();
    // pages from its top into the tables
    for (uint32_t i = first; i < given; i += stride) {
      const int b = last_at_most(taken, B, i);
      a.table[(int64_t)b * a.table_width + pages(start[b]) + i - taken[b]] = __ldcg(a.free_pages + (there - 1 - i));
    }
  }
  // positions and slots
  if (PART != kPlanLists) {
    for (uint32_t t = first; t < total; t += stride) {
      int64_t slot = -1, pos = 0;
      if (t < all_add) {
        const int b = last_at_most(cu, B, t);
        const uint32_t s = start[b], i = t - cu[b], at = s + i, kept = pages(s);
        pos = min(max((int64_t)s + (a.depths ? (int64_t)a.depths[t] : (int64_t)i) + a.position_offset, (int64_t)0),
                  (int64_t)INT32_MAX);
        if (gets[b] != kPlanMost) {
          const uint32_t p = at >> shift, k = taken[b] + p - kept;   // a new page: number k from the stack's top
          const int32_t* where = p < kept ? a.table + (int64_t)b * a.table_width + p : a.free_pages + (there - 1 - k);
          if (PART == kPlanRows && p >= kept && there - 1 - k >= count) where = freed_page(k);   // not on the stack yet
          slot = ((int64_t)__ldcg(where) << shift) + (at & page1);
        }
      }
      a.positions[t] = (int32_t)pos;
      a.slots[t] = slot;
    }
  }
  // the batch's numbers, the last of all: every CTA has read the lengths
  if (PART != kPlanRows) {
    for (uint32_t b = first; b <= (uint32_t)B; b += stride) {
      if (b == (uint32_t)B) {
        a.cu_tokens[B] = (int32_t)min(all_add, total);
        *a.free_count = (int32_t)(there - given);
        break;
      }
      const bool ok = gets[b] != kPlanMost;
      const uint32_t next = b + 1 < (uint32_t)B ? cu[b + 1] : all_add;
      a.cu_tokens[b] = (int32_t)min(cu[b], total);
      if (a.granted) a.granted[b] = ok;
      a.lens[b] = (int32_t)(start[b] + (ok ? next - cu[b] : 0u));
    }
  }
}

constexpr int kKeepThreads = 128;

template <int D>
__global__ void __launch_bounds__(kKeepThreads) kv4_keep_kernel(const KeepArgs a) {
  constexpr int CP = D / 32, PIECES = 2 * CP + 1;   // 16-byte pieces of a token's codes, and its scales
  const int64_t b = blockIdx.x / (uint32_t)a.Hkv, h = blockIdx.x - b * a.Hkv;
  pdl_wait();
  pdl_trigger();
  const int n = min(max(__ldg(a.counts + b), 0), (int)a.path_width);
  const int64_t start = __ldg(a.starts + b);
  const int32_t* path = a.path + b * a.path_width;
  const int32_t* table = a.table + b * a.table_width;
  // the token's place in the page arrays, or -1
  auto place = [&](int64_t t) {
    if (t < 0 || (t >> a.page_shift) >= a.table_width) return (int64_t)-1;
    const int64_t page = __ldg(table + (t >> a.page_shift));
    return page < 0 || page >= a.num_pages ? (int64_t)-1 : (page * a.Hkv + h) * a.page_size + (t & (a.page_size - 1));
  };
  auto piece = [&](int64_t at, int k) {
    return k < CP ? reinterpret_cast<uint4*>(a.k_codes + at * (D / 2)) + k
                  : (k < 2 * CP ? reinterpret_cast<uint4*>(a.v_codes + at * (D / 2)) + (k - CP)
                                : reinterpret_cast<uint4*>(a.scales) + at);
  };
  const int64_t items = (int64_t)n * PIECES;
  for (int64_t i0 = 0; i0 < items; i0 += kKeepThreads) {
    const int64_t i = i0 + threadIdx.x;
    uint4* to = nullptr;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (i < items) {
      const int64_t token = i / PIECES;
      const int k = (int)(i - token * PIECES);
      const int64_t node = __ldg(path + token);
      if (node != token && node >= 0) {
        const int64_t from = place(start + node), at = place(start + token);
        if (from >= 0 && at >= 0) {
          x = *piece(from, k);
          to = piece(at, k);
        }
      }
    }
    __syncthreads();
    if (to) *to = x;
    __syncthreads();
  }
}

}  // namespace

template <int THREADS, int PER, int PART>
static cudaError_t launch_plan_t(const PlanArgs& a, int ctas, int cluster, cudaStream_t stream) {
  int per_sm = 1;
  cudaError_t e = prepare_launch(kv4_plan_kernel<THREADS, PER, PART>, THREADS, THREADS * PER * 5 * 4, &per_sm);
  if (e != cudaSuccess) return e;
  return launch_pdl(kv4_plan_kernel<THREADS, PER, PART>, dim3((unsigned)ctas), dim3(THREADS), (size_t)a.batch * 5 * 4,
                    stream, cluster, a);
}

cudaError_t launch_kv4_plan(const PlanArgs& a, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  if (a.total + a.batch * 4 <= 1024) {   // one small CTA: short sums, no cluster's barrier
    e = launch_plan_t<128, 2, kPlanAll>(a, 1, 1, stream);
  } else if (a.total <= kPlanTokens) {
    e = launch_plan_t<512, 8, kPlanAll>(a, kPlanCluster, kPlanCluster, stream);
  } else {
    const int64_t want = (a.total + 511) / 512, most = device_sm_count();
    constexpr int kWarps = kPlanCountThreads / 32;
    if (a.drop && a.batch > 0)
      e = launch_pdl(kv4_plan_count_kernel, dim3((unsigned)((a.batch + kWarps - 1) / kWarps)), dim3(kPlanCountThreads), 0, stream, 1, a);
    if (e == cudaSuccess) e = launch_plan_t<512, 8, kPlanRows>(a, (int)(want < most ? want : most), 1, stream);
    if (e == cudaSuccess) e = launch_plan_t<512, 8, kPlanLists>(a, kPlanCluster, kPlanCluster, stream);
  }
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv4_keep(const KeepArgs& a, cudaStream_t stream) {
  auto kernel = a.D == 128 ? kv4_keep_kernel<128> : kv4_keep_kernel<64>;
  const cudaError_t e = launch_pdl(kernel, dim3((unsigned)(a.batch * a.Hkv)), dim3(kKeepThreads), 0, stream, 1, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace spinq
