// The gated activation between a block's two linears for gfx950, written as
// bf16, as e4m3 codes with a scale for each 128 columns, or as int4 codes with
// a scale for each token.
//
//   y = act(gate) * up   (act(gate) alone where there is no up)
//   silu:      x / (1 + e^-x)
//   gelu:      x Phi(x), Phi the normal distribution
//   gelu_tanh: x / (1 + e^-2u), u = sqrt(2/pi) (x + 0.044715 x^3), which is
//              x (1 + tanh u) / 2
//   bf16: rne(y)
//   fp8:  s = max|y| (1 / 448) per 128 columns, q = e4m3(y / s)
//   int4: s = max|y| / 7 per row, q = clamp(rne(y / s), -8, 7), two a byte
//
// y stays in fp32 from the loads to the one rounding at the end.  All three are
// products of positive terms, so the left tail keeps its relative accuracy
// (1 + erf and 1 + tanh lose it by cancellation).
//
// Bound: HBM; each element is read and written once.  8192 x 12288, gated, to
// e4m3 (506 MB): 88 us, 5.7 TB/s; to bf16 103; 4608 x 12288 without an up, to
// e4m3: 38 us, 4.5 TB/s, where 20 instructions an element (quantiser and all)
// take about as long as the bytes; 2747 x 2816 to bf16: 9.4 us; one row: 2.5, a launch.
// To int4: 8192 x 12288 100 us gated (453 MB, 4.5 TB/s) and 83 without an up (252
// MB, 3.0 TB/s), where the codes' divisions count more than the bytes.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"
#include "block_internal.h"

namespace jq {

namespace {

using namespace block_detail;

constexpr float kLog2E = 1.44269504088896340736f;

// x / (1 + 2^-w).  Where 2^-w passes fp32's range the result is next to 0 (below
// |x| 2^-126) and becomes 0.
__device__ __forceinline__ float times_logistic(float x, float w) {
  return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-w));
}

// Phi(-|x|) = e^(-x^2 / 2) erfcx(z) / 2, z = |x| / sqrt(2); erfcx (e^(z^2)
// erfc z) by a polynomial in 1 / (1 + z / 2), fitted to the least relative
// error on [0, 10] (3e-8; 3e-7 in fp32), past which the power is 0.
__device__ __forceinline__ float times_normal(float x) {
  const float z = fminf(fabsf(x) * 0.70710678118654752440f, 10.0f);
  const float t = __builtin_amdgcn_rcpf(fmaf(z, 0.5f, 1.0f));
  float p = -5.504991489e-02f;
  p = fmaf(p, t, 2.638963612e-01f);
  p = fmaf(p, t, -4.414635086e-01f);
  p = fmaf(p, t, 2.211742478e-01f);
  p = fmaf(p, t, 1.708991807e-02f);
  p = fmaf(p, t, 1.812441280e-01f);
  p = fmaf(p, t, 2.497952289e-01f);
  p = fmaf(p, t, 2.810981103e-01f);
  p = fmaf(p, t, 2.822214098e-01f);
  p = fmaf(p, t, -6.012753950e-06f);
  const float tail = 0.5f * p * __builtin_amdgcn_exp2f(x * x * (-0.5f * kLog2E));
  return x * (x < 0.0f ? tail : 1.0f - tail);
}

template <Act ACT>
__device__ __forceinline__ float activate(float x) {
  constexpr float kU = 1.59576912160573071176f * kLog2E;  // 2 sqrt(2 / pi), for a power of two
  if constexpr (ACT == Act::kSilu) return times_logistic(x, x * kLog2E);
  else if constexpr (ACT == Act::kGelu) return times_normal(x);
  else return times_logistic(x, x * fmaf(x * x, 0.044715f * kU, kU));
}

// y of 8 elements.
template <Act ACT, bool GATED>
__device__ __forceinline__ void apply(u32x4 gate, u32x4 up, float* y) {
  unpack8_bf16(gate, y);
  float u[8];
  if constexpr (GATED) unpack8_bf16(up, u);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    y[j] = activate<ACT>(y[j]);
    if constexpr (GATED) y[j] *= u[j];
  }
}
__device__ __forceinline__ u32x4 load8(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }

__device__ __forceinline__ uint32_t max8(const float* y) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = umax(m, abs_bits(y[j]));
  return m;
}

// bf16 and fp8: a wave takes NC chunks of 512 columns of a row.
template <Act ACT, bool GATED, bool FP8, int NC>
__global__ __launch_bounds__(256) void gated_act_kernel(const ActArgs a) {
  const int lane = threadIdx.x & 63;
  const uint32_t per_row = (static_cast<uint32_t>(a.N) + 512 * NC - 1) / (512 * NC);
  const uint32_t units = static_cast<uint32_t>(a.M) * per_row;
  // every lane stays to the end: a block's maximum is of 16 lanes
  for (uint32_t u = blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += gridDim.x * 4) {
    const uint32_t row = u / per_row;
    const int k0 = static_cast<int>(u - row * per_row) * 512 * NC + lane * 8;
    u32x4 gate[NC], up[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int k = k0 + 512 * c;
      gate[c] = up[c] = u32x4{0, 0, 0, 0};
      if (k < a.N) {
        gate[c] = load8(a.gate + row * a.gate_stride + k);
        if constexpr (GATED) up[c] = load8(a.up + row * a.up_stride + k);
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int k = k0 + 512 * c;
      const bool in = k < a.N;
      float y[8];
      apply<ACT, GATED>(gate[c], up[c], y);
      const int64_t at = static_cast<int64_t>(row) * a.N + k;
      if constexpr (FP8) {
        const float s = e4m3_scale(lanes_max<16>(max8(y)));
        const E4m3Divisor d = e4m3_divisor(s);
        if (!in) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = e4m3_quotient(y[j], d);
        *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.y) + at) = pack8_e4m3(y);
        if (k % 128 == 0) a.scale[static_cast<int64_t>(row) * ((a.N + 127) / 128) + k / 128] = s;
      } else {
        if (in) *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + at) = pack8_bf16(y);
      }
    }
  }
}

// int4: a block takes a row, its waves NC chunks of 512 columns each.
template <Act ACT, bool GATED, int NC>
__global__ __launch_bounds__(1024) void gated_act_int4_kernel(const ActArgs a) {
  __shared__ uint32_t part[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    float y[NC][8];
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int k = (c * waves + wave) * 512 + lane * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) y[c][j] = 0.0f;
      if (k < a.N)
        apply<ACT, GATED>(load8(a.gate + row * a.gate_stride + k), GATED ? load8(a.up + row * a.up_stride + k) : u32x4{}, y[c]);
      m = umax(m, max8(y[c]));
    }
    m = wave_max_bits(m);
    if (waves > 1) {
      if (lane == 0) part[wave] = m;
      __syncthreads();
      for (int i = 0; i < waves; ++i) m = umax(m, part[i]);
    }
    const float s = __uint_as_float(m) / 7.0f;
    if (threadIdx.x == 0) a.scale[row] = s;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int k = (c * waves + wave) * 512 + lane * 8;
      if (k < a.N) *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.y) + row * (a.N / 2) + k / 2) = int4_codes(y[c], s);
    }
    if (waves > 1) __syncthreads();  // the next row writes part[] again
  }
}

template <Act ACT, bool GATED>
hipError_t launch(const ActArgs& a, NormOut out, hipStream_t st) {
  constexpr int64_t kMostBlocks = 1 << 20;
  if (out != NormOut::kInt4) {
    // With an up a wave has as much on its way with one chunk (8192 x 12288 to
    // e4m3 91 us with one and with two, 2747 x 2816 to bf16 10.8 and 11.5) as
    // without one with two (4608 x 12288 to e4m3 42 and 38.6).
    constexpr int kChunks = GATED ? 1 : 2;
    const int64_t blocks = (a.M * ((a.N + 512 * kChunks - 1) / (512 * kChunks)) + 3) / 4;
    const dim3 grid(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks));
    if (out == NormOut::kFp8) hipLaunchKernelGGL((gated_act_kernel<ACT, GATED, true, kChunks>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((gated_act_kernel<ACT, GATED, false, kChunks>), grid, dim3(256), 0, st, a);
  } else {
    const int chunks = (a.N + 511) / 512;
    const dim3 grid(static_cast<unsigned>(a.M < kMostBlocks ? a.M : kMostBlocks));
    if (chunks <= 32)
      hipLaunchKernelGGL((gated_act_int4_kernel<ACT, GATED, 2>), grid, dim3(64 * ((chunks + 1) / 2)), 0, st, a);
    else
      hipLaunchKernelGGL((gated_act_int4_kernel<ACT, GATED, 8>), grid, dim3(64 * ((chunks + 7) / 8)), 0, st, a);
  }
  return hipGetLastError();
}

template <Act ACT>
hipError_t launch(const ActArgs& a, NormOut out, hipStream_t st) {
  return a.up != nullptr ? launch<ACT, true>(a, out, st) : launch<ACT, false>(a, out, st);
}

}  // namespace

hipError_t launch_gated_act(const ActArgs& a, Act act, NormOut out, hipStream_t st) {
  switch (act) {
    case Act::kSilu: return launch<Act::kSilu>(a, out, st);
    case Act::kGelu: return launch<Act::kGelu>(a, out, st);
    default: return launch<Act::kGeluTanh>(a, out, st);
  }
}

}  // namespace jq
