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

// (COH: for other workgroups of the same launch)
template <bool COH> __device__ __forceinline__ void st_u2(bf16_t* p, uint2 v) {
  if (COH) __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), (unsigned long long)v.x | ((unsigned long long)v.y << 32), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else *reinterpret_cast<uint2*>(p) = v;
}

// Store 4 consecutive-k activations of token m into the packed panels as bf16 hi/lo (LO false: the lo panel has no reader).
template <bool COH = false, bool LO = true>
__device__ __forceinline__ void xpack_put4(bf16_t* X, int KT, int M, int m, int k, HiLo x0, HiLo x1) {
  const int kt = k >> 5, grp = (k & 31) >> 3, e = k & 7;
  const size_t base = ((size_t)kt * 64 + grp * 16) * 8 + e;
  size_t off_hi, off_lo;
  if (M <= 8) { off_hi = base + (size_t)m * 8; off_lo = base + (size_t)(m + 8) * 8; }
  else { off_hi = base + (size_t)m * 8; off_lo = (size_t)KT * 512 + base + (size_t)m * 8; }
  st_u2<COH>(X + off_hi, make_uint2(x0.hi, x1.hi));
  if (LO) st_u2<COH>(X + off_lo, make_uint2(x0.lo, x1.lo));
}
template <bool COH = false, bool LO = true>
__device__ __forceinline__ void xpack_store4(bf16_t* X, int KT, int M, int m, int k, const float* v) {
  xpack_put4<COH, LO>(X, KT, M, m, k, split_bf16(v[0], v[1]), split_bf16(v[2], v[3]));
}

// Wavefront reductions on the DPP cross-lane network (no LDS traffic): xor-1, xor-2 inside quads,
// half-row mirror, row mirror, then row broadcasts 15 and 31; lane 63 ends up with the result, which
// is broadcast through a scalar register.  The combination order is fixed, so sums are reproducible.
#define DPP_QUAD_XOR1 0xB1
#define DPP_QUAD_XOR2 0x4E
#define DPP_ROW_HALF_MIRROR 0x141
#define DPP_ROW_MIRROR 0x140
#define DPP_ROW_ROR8 0x128
#define DPP_ROW_BCAST15 0x142
#define DPP_ROW_BCAST31 0x143

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_f(float old, float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(v), CTRL, ROW_MASK, 0xF, false));
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int dpp_i(int old, int v) {
  return __builtin_amdgcn_update_dpp(old, v, CTRL, ROW_MASK, 0xF, false);
}

__device__ __forceinline__ float wave_sum(float v) {
  v += dpp_f<DPP_QUAD_XOR1, 0xF>(0.f, v);
  v += dpp_f<DPP_QUAD_XOR2, 0xF>(0.f, v);
  v += dpp_f<DPP_ROW_HALF_MIRROR, 0xF>(0.f, v);
  v += dpp_f<DPP_ROW_MIRROR, 0xF>(0.f, v);
  v += dpp_f<DPP_ROW_BCAST15, 0xA>(0.f, v);
  v += dpp_f<DPP_ROW_BCAST31, 0xC>(0.f, v);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp_f<DPP_QUAD_XOR1, 0xF>(v, v));
  v = fmaxf(v, dpp_f<DPP_QUAD_XOR2, 0xF>(v, v));
  v = fmaxf(v, dpp_f<DPP_ROW_HALF_MIRROR, 0xF>(v, v));
  v = fmaxf(v, dpp_f<DPP_ROW_MIRROR, 0xF>(v, v));
  v = fmaxf(v, dpp_f<DPP_ROW_BCAST15, 0xA>(v, v));
  v = fmaxf(v, dpp_f<DPP_ROW_BCAST31, 0xC>(v, v));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Order-preserving map float -> uint32 (larger float <=> larger key; -inf maps above key 0, which marks
// a dropped slot) and back.
__device__ __forceinline__ uint32_t f32_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_f32(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
// Wavefront maximum of unsigned keys: the cross-lane moves fold into the max instructions (one DPP
// instruction per step; 0 is the identity, so lanes a step does not reach keep their value).
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xF, true);
  return v > o ? v : o;
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = dpp_max_u32<DPP_QUAD_XOR1, 0xF>(v);
  v = dpp_max_u32<DPP_QUAD_XOR2, 0xF>(v);
  v = dpp_max_u32<DPP_ROW_HALF_MIRROR, 0xF>(v);
  v = dpp_max_u32<DPP_ROW_MIRROR, 0xF>(v);
  v = dpp_max_u32<DPP_ROW_BCAST15, 0xA>(v);
  v = dpp_max_u32<DPP_ROW_BCAST31, 0xC>(v);
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
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
