// attn_tc.cuh -- what the attention kernels on the 5th-generation tensor core
// share: bounded waits, tensor-memory stores, MMAs that take their A operand
// from tensor memory, and the arithmetic of the running softmax.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "spinq_device.cuh"

namespace spinq {

constexpr uint64_t kAttnWaitLimitNs = 2000000000ull;
constexpr float kAttnLog2e = 1.4426950408889634f;
// The running maximum moves only when a score exceeds it by more than this
// (base 2): the weights stay below 2^8 and the accumulator is rescaled rarely.
constexpr float kAttnSlack = 8.f;

// Non-blocking probe of the phase with `parity`.
__device__ __forceinline__ bool attn_test(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}

// Bounded wait that polls; false, with the abort flag up, after `limit_ns`, and false
// soon after another warp raised it.  The clock and the flag are looked at only
// every 512 polls: reading the timer costs hundreds of cycles, which a wait on
// the path from the scores to the weights would pay on every tile.
__device__ __forceinline__ bool attn_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, uint64_t limit_ns) {
  uint64_t t0 = 0;
  while (true) {
#pragma unroll 1
    for (int k = 0; k < 512; ++k)
      if (attn_test(bar, parity)) return true;
    if (*abort_flag) return false;
    const uint64_t t = globaltimer_ns();
    if (t0 == 0) t0 = t;
    if (t - t0 > limit_ns) {
      *abort_flag = 1;
      return false;
    }
  }
}

// The same by a whole warp, with one answer for all its lanes.
__device__ __forceinline__ bool attn_wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag,
                                               uint64_t limit_ns) {
  return __all_sync(0xffffffffu, attn_wait(bar, parity, abort_flag, limit_ns));
}

__device__ __forceinline__ float attn_exp2(float x) {   // 2^x: relative error below 2^-22, 0 for -inf
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float attn_max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// 32 lanes x 32 consecutive 32-bit columns to tensor memory.
__device__ __forceinline__ void tmem_st_32x32b_x32(uint32_t taddr, const uint32_t r[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t r[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

// 16 lanes x 8 groups of 8 columns from tensor memory: lane 4 g + c gets columns
// 8 k + 2 c and + 1 of row g in r[4 k], r[4 k + 1], of row g + 8 in r[4 k + 2], r[4 k + 3].
__device__ __forceinline__ void tmem_ld_16x256b_x8(uint32_t taddr, uint32_t r[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
// The same of 2 groups, with the wait.
__device__ __forceinline__ void tmem_ld_16x256b_x2(uint32_t taddr, uint32_t r[8]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n tcgen05.wait::ld.sync.aligned;\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_st_16x256b_x2(uint32_t taddr, const uint32_t r[8]) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// 16 lanes x 8 groups of 4 columns to tensor memory: lane 4 g + c gives column
// 4 k + c of row g in r[2 k], of row g + 8 in r[2 k + 1].
__device__ __forceinline__ void tmem_st_16x128b_x8(uint32_t taddr, const uint32_t r[16]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
               "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}

// Waits for the tensor-memory loads of r[N] (N a multiple of 16).
template <int N>
__device__ __forceinline__ void tmem_ld_wait_all(uint32_t* r) {
#pragma unroll
  for (int q = 0; q < N; q += 16) tmem_ld_wait(r + q);
}

// The issuing thread of a warp (one, always the same).
__device__ __forceinline__ bool attn_elect() {
  uint32_t p;
  asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.u32 %0, 1, 0, q;\n}\n" : "=r"(p));
  return p != 0;
}

// Shared-memory descriptors (spinq_device.cuh: umma_desc_sw128, ..._mn) by
// halves.  The high one is the same for every operand here (8-row groups 1024
// bytes apart, 128-byte swizzle); the low one holds the address, so a step within or
// between tiles is one addition of bytes / 16.
constexpr uint32_t kAttnDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t attn_desc_k(uint32_t addr) { return (addr >> 4) | (1u << 16); }              // K-major
__device__ __forceinline__ uint32_t attn_desc_mn(uint32_t addr) { return (addr >> 4) | ((16384u >> 4) << 16); }  // MN-major

// D[tmem] (+)= A[smem] * B[smem], fp16 operands.
template <bool ACC>
__device__ __forceinline__ void attn_mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n mov.b64 a, {%1, %4};\n mov.b64 b, {%2, %4};\n setp.ne.b32 p, %5, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "n"(kAttnDescHi), "n"(ACC ? 1 : 0)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: A's rows on the lanes, two values per
// 32-bit column.
template <bool ACC>
__device__ __forceinline__ void attn_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 b;\n mov.b64 b, {%2, %4};\n setp.ne.b32 p, %5, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b_lo), "r"(idesc), "n"(kAttnDescHi), "n"(ACC ? 1 : 0)
      : "memory");
}

// Instruction descriptor for kind::f16, FP16 x FP16 -> F32, A and B K-major;
// neg_a multiplies by -A.
__host__ __device__ constexpr uint32_t umma_idesc_f16_f32(int M, int N, bool neg_a) {
  return (1u << 4) | ((neg_a ? 1u : 0u) << 13) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// A tile of 128 rows of D fp16 values lies in shared memory as D / 64 atoms
// of 128 rows x 128 bytes, 128-byte swizzle; kAttnAtom bytes apart.
constexpr uint32_t kAttnAtom = 128 * 128;

// S[tmem] = Q K^T: both tiles K-major (descriptors of their starts), D / 16 K steps.
template <int D>
__device__ __forceinline__ void attn_mma_qk(uint32_t s_tmem, uint32_t q_lo, uint32_t k_lo, uint32_t idesc) {
  attn_mma_ss<false>(s_tmem, q_lo, k_lo, idesc);
#pragma unroll
  for (int ks = 1; ks < D / 16; ++ks) {
    const uint32_t off = ((ks >> 2) * kAttnAtom + (ks & 3) * 32) >> 4;
    attn_mma_ss<true>(s_tmem, q_lo + off, k_lo + off, idesc);
  }
}

// O[tmem] (+)= P V: P fp16 in tensor memory (128 tokens on 64 columns), V
// with D contiguous (MN-major), 8 K steps of 16 tokens.
template <int D>
__device__ __forceinline__ void attn_mma_pv(uint32_t o_tmem, uint32_t p_tmem, uint32_t v_lo, bool accumulate) {
  constexpr uint32_t idesc = umma_idesc_f16_f32_bmn(128, D);
  if (accumulate)
    attn_mma_ts<true>(o_tmem, p_tmem, v_lo, idesc);
  else
    attn_mma_ts<false>(o_tmem, p_tmem, v_lo, idesc);
#pragma unroll
  for (int ks = 1; ks < 8; ++ks) attn_mma_ts<true>(o_tmem, p_tmem + ks * 8, v_lo + ks * (2048 >> 4), idesc);
}

// The largest of 128 scores.
__device__ __forceinline__ float attn_row_max(const uint32_t* r) {
  float m[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) m[q] = fmaxf(__uint_as_float(r[2 * q]), __uint_as_float(r[2 * q + 1]));
#pragma unroll
  for (int i = 8; i < 128; i += 8)
#pragma unroll
    for (int q = 0; q < 4; ++q) m[q] = attn_max3(m[q], __uint_as_float(r[i + 2 * q]), __uint_as_float(r[i + 2 * q + 1]));
  return fmaxf(attn_max3(m[0], m[1], m[2]), m[3]);
}

// Two warps share a tile's 32 rows, 64 columns each.  OR of a predicate over
// the 64 threads of the pair (a barrier for both).
__device__ __forceinline__ bool attn_pair_or(bool x, int barrier) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n bar.red.or.pred q, %2, 64, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"((uint32_t)x), "r"(barrier)
      : "memory");
  return r != 0;
}
// Exchanges a value of every row between the pair's warps (half 0 and 1)
// through one slot of 32 floats.
__device__ __forceinline__ float attn_pair_swap(float* slot, float x, int half, int lane, int barrier) {
  if (half == 0) slot[lane] = x;
  named_bar_sync(barrier, 64);
  float y = slot[lane];
  named_bar_sync(barrier, 64);
  if (half == 1) slot[lane] = x;
  named_bar_sync(barrier, 64);
  if (half == 0) y = slot[lane];
  return y;
}

// Rescales this lane's row of an accumulator in tensor memory (N columns), 16
// at a time: it runs while the row's scores are held in registers.
template <int N>
__device__ __forceinline__ void attn_rescale(uint32_t o_tmem, float f) {
#pragma unroll
  for (int c = 0; c < N; c += 16) {
    uint32_t o[16];
    tmem_ld_32x32b_x16(o_tmem + c, o);
    tmem_ld_wait(o);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
    tmem_st_32x32b_x16(o_tmem + c, o);
  }
  tmem_st_wait();
}

// The same for the 32 rows of a warp in the spread layout: lane 4 g + c has the
// factors of rows g, g + 8, g + 16, g + 24.
template <int N>
__device__ __forceinline__ void attn_rescale_rows(uint32_t o_tmem, const float f[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int c = 0; c < N; c += 16) {
      uint32_t o[8];
      const uint32_t at = o_tmem + ((uint32_t)(16 * h) << 16) + c;
      tmem_ld_16x256b_x2(at, o);
#pragma unroll
      for (int x = 0; x < 8; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f[2 * h + ((x >> 1) & 1)]);
      tmem_st_16x256b_x2(at, o);
    }
  tmem_st_wait();
}

}  // namespace spinq
