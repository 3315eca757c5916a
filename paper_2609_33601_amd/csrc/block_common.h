// Device helpers shared by the kernels of a decoder block's other operators
// (norm, 8-bit linear, rotation with paged append, paged attention): bf16 and
// e4m3 conversions, scales, and reductions inside a wave.  Device code only.
#ifndef JQ_BLOCK_COMMON_H
#define JQ_BLOCK_COMMON_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace jq {
namespace block_detail {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Two floats rounded to bf16 (nearest even), the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2 v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ void unpack8_bf16(u32x4 u, float* f) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f[2 * j] = bf_lo(u[j]);
    f[2 * j + 1] = bf_hi(u[j]);
  }
}

__device__ __forceinline__ u32x4 pack8_bf16(const float* f) {
  return u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
}

// Eight floats rounded to e4m3 (nearest even; NaN stays NaN).
__device__ __forceinline__ u32x2 pack8_e4m3(const float* f) {
  u32x2 r;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j], f[4 * j + 1], 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * j + 2], f[4 * j + 3], v, true);
    r[j] = static_cast<uint32_t>(v);
  }
  return r;
}

// The scale of values whose largest magnitude has these bits: a (1 / 448), at
// least 2^-126 so that its reciprocal is finite; 0 where all are 0.  Bits of
// magnitudes order like the magnitudes with NaN on top, so an infinity or NaN
// among the values makes the scale one, and every product with it too.
__device__ __forceinline__ float e4m3_scale(uint32_t amax_bits) {
  float s = __uint_as_float(amax_bits) * (1.0f / 448.0f);
  if (s < 0x1p-126f) s = amax_bits == 0 ? 0.0f : 0x1p-126f;
  return s;
}
// What e4m3_quotient divides by, with its rounded reciprocal.  For a scale of 0
// (whose values are all 0) and for an infinite one both are 0: v / inf is 0 for
// a finite v and NaN for an infinite one, and so is v times 0.
struct E4m3Divisor {
  float s, inv;
};
__device__ __forceinline__ E4m3Divisor e4m3_divisor(float s) {
  const float d = __float_as_uint(s) == 0x7F800000u ? 0.0f : s;
  return {d, d == 0.0f ? 0.0f : 1.0f / d};
}

// fl32(v / s) from the rounded reciprocal of s, three operations instead of a
// division's ten: the remainder of v * inv is exact in one fma, and adding it
// times inv rounds correctly because inv is the rounded reciprocal (Markstein).
// bf16 inputs meet ties of e4m3 too often for a quotient that is an ulp off.
__device__ __forceinline__ float e4m3_quotient(float v, E4m3Divisor d) {
  const float q = v * d.inv;
  return fmaf(fmaf(-q, d.s, v), d.inv, q);
}

// The value of another lane of the same row of 16 (DPP), all lanes taking part.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xF, 0xF, true));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;

// Largest value of L neighbouring lanes (L = 2, 4, 8, 16, 32), left in each.
template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
  if constexpr (L >= 2) v = umax(v, dpp<kDppXor1>(v));
  if constexpr (L >= 4) v = umax(v, dpp<kDppXor2>(v));
  if constexpr (L >= 8) v = umax(v, dpp<kDppHalfMirror>(v));
  if constexpr (L >= 16) v = umax(v, dpp<kDppMirror>(v));
  if constexpr (L >= 32) v = umax(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), 16, 64)));
  return v;
}

// Sum over L neighbouring lanes (L = 8, 16, 32, 64), left in each, in an order
// that does not depend on the lane.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  auto f = [](uint32_t u) { return __uint_as_float(u); };
  auto u = [](float x) { return __float_as_uint(x); };
  v += f(dpp<kDppXor1>(u(v)));
  v += f(dpp<kDppXor2>(u(v)));
  v += f(dpp<kDppHalfMirror>(u(v)));
  if constexpr (L >= 16) v += f(dpp<kDppMirror>(u(v)));
  if constexpr (L == 32) v += __shfl_xor(v, 16, 64);
  if constexpr (L == 64) {
    const int i = static_cast<int>(u(v));
    v = (f(__builtin_amdgcn_readlane(i, 0)) + f(__builtin_amdgcn_readlane(i, 16))) +
        (f(__builtin_amdgcn_readlane(i, 32)) + f(__builtin_amdgcn_readlane(i, 48)));
  }
  return v;
}

// Largest of a wave, uniform.
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v) {
  const int i = static_cast<int>(lanes_max<16>(v));
  return umax(umax(static_cast<uint32_t>(__builtin_amdgcn_readlane(i, 0)), static_cast<uint32_t>(__builtin_amdgcn_readlane(i, 16))),
              umax(static_cast<uint32_t>(__builtin_amdgcn_readlane(i, 32)), static_cast<uint32_t>(__builtin_amdgcn_readlane(i, 48))));
}

// Transfers from a buffer into LDS, 16 (or 4) bytes per lane: lane i writes
// lds + 16 i (4 i).  As asm, because the compiler waits for transfers that it
// knows of before the next LDS read, whatever part of LDS that reads, and the
// whole point of several stages is not to.  A kernel waits itself (vmcnt).  The
// wait states that the compiler would put behind the writes of M0 and of
// descriptor words are in the asm; the build checks them.
constexpr int kRawBuffer = 0x00020000;             // descriptor word 3: raw bytes
constexpr uint32_t kOutsideBuffer = 0x80000000u;   // an offset past every descriptor here: reads as zero
struct Rsrc {
  u32x4 w;
};
__device__ __forceinline__ Rsrc make_rsrc(const void* base, int bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32)) & 0xFFFFu;
  const uint32_t n = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(bytes));
  return {u32x4{lo, hi, n, static_cast<uint32_t>(kRawBuffer)}};
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}
// NOPS: 4 covers a descriptor that a vector instruction has just written; 0,
// for one that lies in its registers through a loop, the write of M0 alone.
template <int NOPS = 4>
__device__ __forceinline__ void dma16(const Rsrc& r, uint32_t lds, uint32_t voffset, uint32_t soffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop %4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voffset), "s"(r.w), "s"(soffset), "n"(NOPS)
               : "memory");
}
__device__ __forceinline__ void dma4(const Rsrc& r, uint32_t lds, uint32_t voffset, uint32_t soffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voffset), "s"(r.w), "s"(soffset)
               : "memory");
}

}  // namespace block_detail
}  // namespace jq

#endif  // JQ_BLOCK_COMMON_H
