// Device helpers shared by the kernel sources (vector types, buffer
// descriptors, wave-uniform values, bf16 / fp8 conversions).  Each translation
// unit gets its own internal copy.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rlda {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kRescaleLog2 = 8.f;          // lazy-rescale threshold of the online softmax (log2 units)
constexpr uint32_t kRsrcWord3 = 0x00020000u; // raw buffer, 32-bit data format
constexpr int kLoadNT = 2;                   // cache policy: non-temporal (KV is read once)
constexpr int kVmcnt0 = 0x0F70;             // s_waitcnt: no vector memory operation outstanding
constexpr int kPastRange = 0x40000000;       // buffer offset beyond any descriptor's records: reads 0

__device__ __forceinline__ float neg_inf() { return -__builtin_huge_valf(); }

// Workgroup barrier for data exchanged through LDS only: this wave's LDS operations
// are complete, then s_barrier.  Unlike __syncthreads it does not wait for this
// wave's global stores to complete.  The memory clobber keeps the compiler from
// moving memory accesses across it.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Values equal in every lane, moved to scalar registers so that buffer
// descriptors and loop bounds built from them stay scalar.
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uni64(int64_t x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)((uint64_t)x >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// Inclusive sum and maximum (of non-negative values) over the lanes 0 .. l of a wave,
// by DPP: shifts within rows of 16, then the rows' last lanes broadcast to the rows
// after them.  Each step is two VALU instructions where a shuffle is an LDS round trip.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_or_zero(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, true);
}
__device__ __forceinline__ int wave_scan(int x) {
  x += dpp_or_zero<0x111, 0xf>(x);   // row_shr:1, 2, 4, 8
  x += dpp_or_zero<0x112, 0xf>(x);
  x += dpp_or_zero<0x114, 0xf>(x);
  x += dpp_or_zero<0x118, 0xf>(x);
  x += dpp_or_zero<0x142, 0xa>(x);   // row_bcast:15 into rows 1 and 3
  x += dpp_or_zero<0x143, 0xc>(x);   // row_bcast:31 into rows 2 and 3
  return x;
}
__device__ __forceinline__ int wave_scan_max(int x) {
  x = max(x, dpp_or_zero<0x111, 0xf>(x));
  x = max(x, dpp_or_zero<0x112, 0xf>(x));
  x = max(x, dpp_or_zero<0x114, 0xf>(x));
  x = max(x, dpp_or_zero<0x118, 0xf>(x));
  x = max(x, dpp_or_zero<0x142, 0xa>(x));
  x = max(x, dpp_or_zero<0x143, 0xc>(x));
  return x;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes, (int)kRsrcWord3);
}

// Descriptor from wave-uniform inputs, kept in scalar registers.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc_uni(const void* base, uint32_t bytes) {
  const int64_t a = uni64((int64_t)(uintptr_t)base);
  return make_rsrc((const void*)(uintptr_t)a, (uint32_t)uni((int)bytes));
}

// Two OCP E4M3FN bytes of `w` (bytes 0,1 or, with hi_half, bytes 2,3) as floats.
__device__ __forceinline__ f32x2 fp8x2_to_f32(uint32_t w, bool hi_half) {
  return hi_half ? __builtin_amdgcn_cvt_pk_f32_fp8(w, true) : __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
}

#ifndef RLDA_FP8_DIRECT
#define RLDA_FP8_DIRECT 1
#endif
constexpr bool kFp8Direct = RLDA_FP8_DIRECT;   // fp8 -> bf16 operands in one conversion per pair

// Two e4m3 values (bytes 0, 1, or 2, 3 with hi_half), times `power`, a power of two from 2^-100
// on, to a bf16 pair, low half first.  These are bf16 values, so the conversion is exact.
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t w, bool hi_half, float power = 1.0f) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = hi_half ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, true)
                           : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, false);
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

// The largest magnitudes of bf16 values, two at a time: without their signs they order as
// integers, infinities and NaN above the others.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
template <class Words>
__device__ __forceinline__ u16x2 magnitude_max(u16x2 top, Words w) {
#pragma unroll
  for (unsigned i = 0; i < sizeof(w) / 4; ++i)
    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, (uint32_t)w[i] & 0x7FFF7FFFu));
  return top;
}
__device__ __forceinline__ bool not_finite(u16x2 top) { return top[0] >= 0x7F80 || top[1] >= 0x7F80; }

// The cap of a score, y -> cap tanh(y / cap) in log2 units (cap_log2 = cap log2(e)), for
// y = x * mul and arg = mul * 2 / cap: cap - 2 cap / (e^(2 y / cap) + 1), exact at both ends.
// Its error is 2^-22 of the cap, 1.5e-5 in a score at a cap of 64 (bf16 products of random
// signs: a few 1e-6 in the result).
// top: cap_log2, and what the caller adds to the score (at no cost).
__device__ __forceinline__ float cap_score(float x, float arg, float cap_log2, float top) {
  return __builtin_fmaf(-2.f * cap_log2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * arg) + 1.f), top);
}

// Wider caps take the odd series where |y| is below a sixteenth of the cap (the next term is
// 2e-9 of the result): their error stays 2^-18 of the score.
__host__ __device__ __forceinline__ bool wide_cap(float cap_log2) { return cap_log2 > 64.f * 1.4426950408889634f; }
__device__ __forceinline__ float cap_score_wide(float x, float mul, float arg, float cap_log2) {
  const float z = x * arg * 0.5f * 0.6931471805599453f, z2 = z * z;   // y / cap_log2
  const float small = x * mul * __builtin_fmaf(z2, __builtin_fmaf(z2, __builtin_fmaf(z2, -17.f / 315.f, 2.f / 15.f), -1.f / 3.f), 1.f);
  return __builtin_fabsf(z) < 0.0625f ? small : cap_score(x, arg, cap_log2, cap_log2);
}

}  // namespace
}  // namespace rlda
