// Loads and stores of arrays that are aligned to their elements only, and bf16.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kd {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// An address that came as a number is one of global memory (a generic pointer's loads would go through the LDS check as well).
#define KD_GLOBAL __attribute__((address_space(1)))
typedef KD_GLOBAL char* global_t;

// 16 or 8 bytes at any multiple of two: one instruction, the hardware takes any alignment of global memory.
struct __attribute__((packed, aligned(2))) Bytes16 { u32x4_t v; };
struct __attribute__((packed, aligned(2))) Bytes8 { u32x2_t v; };
__device__ __forceinline__ u32x4_t load16(const void* p) { return ((const Bytes16*)p)->v; }
__device__ __forceinline__ void store16(global_t p, const u32x4_t& v) { ((KD_GLOBAL Bytes16*)p)->v = v; }
__device__ __forceinline__ void store8(global_t p, const u32x2_t& v) { ((KD_GLOBAL Bytes8*)p)->v = v; }

__device__ __forceinline__ float bf16_float(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) { return bf16_bits(lo) | (uint32_t)bf16_bits(hi) << 16; }

}  // namespace kd
