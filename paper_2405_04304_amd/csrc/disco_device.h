// Device helpers shared by the kernel files (gfx950).
#pragma once
#include "disco_internal.h"

namespace disco {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

__device__ __forceinline__ float bf16_to_f32(bf16_t u) { return __uint_as_float(((uint32_t)u) << 16); }

__device__ __forceinline__ bf16_t f32_to_bf16(float f) {  // round to nearest even (the hardware conversion of gfx950)
  return __builtin_bit_cast(bf16_t, (__bf16)f);
}

// Two floats as bf16 in one word, the first in the low half: one instruction (two scalar conversions are put together with two more;
// in the prompt pass's attention they were a quarter of the vector instructions: 0.4 % of a pass over 3001 tokens).
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}
// ... and as bf16 hi + lo
struct HiLo { uint32_t hi, lo; };
__device__ __forceinline__ HiLo split_bf16(float a, float b) {
  HiLo r;
  r.hi = pack_bf16(a, b);
  r.lo = pack_bf16(a - __uint_as_float(r.hi << 16), b - __uint_as_float(r.hi & 0xffff0000u));
  return r;
}

// A value and its partner 16 or 32 lanes away, one half of the wavefront each way round (vector instructions; a shuffle goes through
// the LDS unit).  Lanes that are 16 and 32 apart must be active together.
struct Pair32 { float a, b; };
__device__ __forceinline__ Pair32 swap16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return Pair32{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Pair32 swap32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return Pair32{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float half_max(float v) { const Pair32 p = swap32(v); return fmaxf(p.a, p.b); }   // lanes l, l^32
__device__ __forceinline__ float half_sum(float v) { const Pair32 p = swap32(v); return p.a + p.b; }
// Across the four 16-lane rows of a wavefront (lanes l, l^16, l^32, l^48), every lane gets the result.
__device__ __forceinline__ float row4_max(float v) { const Pair32 p = swap16(v); return half_max(fmaxf(p.a, p.b)); }
__device__ __forceinline__ float row4_sum(float v) { const Pair32 p = swap16(v); return half_sum(p.a + p.b); }

// Copies from memory into LDS, 16 bytes per lane to consecutive LDS addresses from `lds` on (uniform), without registers:
// base (uniform) + lane_off, or an address per lane.  Completion is counted by vmcnt.
__device__ __forceinline__ void lds_dma_16(const void* base, const uint32_t lane_off, const uint32_t lds) {
  // m0 holds the LDS address of the wavefront's 1 KiB; the instruction has no register outputs
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds), "v"(lane_off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void lds_dma_16(const void* lane_addr, const uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds), "v"(lane_addr) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) {
  union { u32x4 u; bf16x8 b; } c; c.u = v; return c.b;
}

}  // namespace disco
