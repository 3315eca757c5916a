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
// taken through e^-|.|, so the left tail keeps its relative accuracy (1 + erf
// and 1 + tanh lose it by cancellation).
//
// Bound: HBM; each element is read and written once.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"
#include "block_internal.h"

namespace jq {

namespace {

using namespace block_detail;

constexpr float kLog2E = 1.44269504088896340736f;

// 1 / (1 + e^-w) times x.
__device__ __forceinline__ float times_logistic(float x, float w) {
  const float e = __builtin_amdgcn_exp2f(-fabsf(w) * kLog2E);
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  return x * (w < 0.0f ? e * r : r);
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
  if constexpr (ACT == Act::kSilu) return times_logistic(x, x);
  else if constexpr (ACT == Act::kGelu) return times_normal(x);
  else return times_logistic(x, 1.59576912160573071176f * fmaf(0.044715f * x * x, x, x));
}

// y of 8 elements.
template <Act ACT, bool GATED>
__device__ __forceinline__ void load_y(const ActArgs& a, int64_t row, int k, float* y) {
  unpack8_bf16(*reinterpret_cast<const u32x4*>(a.gate + row * a.gate_stride + k), y);
  float u[8];
  if constexpr (GATED) unpack8_bf16(*reinterpret_cast<const u32x4*>(a.up + row * a.up_stride + k), u);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    y[j] = activate<ACT>(y[j]);
    if constexpr (GATED) y[j] *= u[j];
  }
}

__device__ __forceinline__ uint32_t max8(const float* y) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = umax(m, abs_bits(y[j]));
  return m;
}

// bf16 and fp8: a wave takes 512 columns of a row.
template <Act ACT, bool GATED, bool FP8>
__global__ __launch_bounds__(256) void gated_act_kernel(const ActArgs a) {
  const int lane = threadIdx.x & 63;
  const uint32_t per_row = (static_cast<uint32_t>(a.N) + 511) / 512;
  const uint32_t units = static_cast<uint32_t>(a.M) * per_row;
  // every lane stays to the end: a block's maximum is of 16 lanes
  for (uint32_t u = blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += gridDim.x * 4) {
    const uint32_t row = u / per_row;
    const int k = static_cast<int>(u - row * per_row) * 512 + lane * 8;
    const bool in = k < a.N;
    float y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (in) load_y<ACT, GATED>(a, row, k, y);
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
      if (k < a.N) load_y<ACT, GATED>(a, row, k, y[c]);
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
    const int64_t blocks = (a.M * ((a.N + 511) / 512) + 3) / 4;
    const dim3 grid(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks));
    if (out == NormOut::kFp8) hipLaunchKernelGGL((gated_act_kernel<ACT, GATED, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((gated_act_kernel<ACT, GATED, false>), grid, dim3(256), 0, st, a);
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
