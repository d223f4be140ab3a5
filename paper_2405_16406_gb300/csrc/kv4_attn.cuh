// kv4_attn.cuh -- what the attention kernels on the paged 4-bit cache share:
// value scales in the weights, codes as fp16 operands, and a warp's copies.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "spinq_device.cuh"

namespace spinq {

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

// (x & m) | c in one instruction, both constants in registers.
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t m, uint32_t c) {
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;\n" : "=r"(y) : "r"(x), "r"(m), "r"(c));
  return y;
}
// Eight codes of a word as fp16 pairs u - 8: (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ uint32_t code_pair(uint32_t x) {   // nibbles at bits 0 and 16
  const uint32_t m = and_or(x, 0x000F000Fu, 0x64006400u);     // 1024 + u
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&m), __half2half2(__ushort_as_half(0x6408)));   // 1032
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 code_pairs(uint32_t x) {
  return make_uint4(code_pair(x), code_pair(x >> 4), code_pair(x >> 8), code_pair(x >> 12));
}

// code_pairs with one shift in place of three: the codes at bits 4 and 20 are 1024 + 16 u, exact,
// and so is their sixteenth less 72.
__device__ __forceinline__ uint32_t code_pair16(uint32_t x) {
  const uint32_t m = and_or(x, 0x00F000F0u, 0x64006400u);
  const __half2 h = __hfma2(*reinterpret_cast<const __half2*>(&m), __half2half2(__ushort_as_half(0x2c00)),    // 1 / 16
                            __half2half2(__ushort_as_half(0xd480)));                                        // -72
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 code_pairs1(uint32_t x) {
  const uint32_t y = x >> 8;
  return make_uint4(code_pair(x), code_pair16(x), code_pair(y), code_pair16(y));
}

__device__ __forceinline__ uint32_t own_transpose(uint32_t x) {   // 8x8 fp16 transpose over the warp
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ void own_copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}

}  // namespace spinq
