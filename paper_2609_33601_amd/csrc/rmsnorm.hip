// RMS norm with the residual's addition for gfx950, written as bf16, as e4m3
// codes with a scale for each 128 columns, or as int4 codes with a scale for
// each token.
//
//   h  = x + residual                    (fp32; residual' = bf16(h))
//   y  = (h * r) * w,  r = 1 / sqrt(mean(h^2) + eps)
//   bf16: rne(y)
//   fp8:  s = max|y| (1 / 448) per 128 columns, q = e4m3(y / s)
//   int4: s = max|y| / 7 per row, q = clamp(rne(y / s), -8, 7), two a byte
//
// h and y stay in fp32 registers from the load to the one rounding at the
// end: a norm that wrote bf16 and a quantiser that read it back would round
// twice and move 4 bytes more for each element.
//
// Bound: HBM.  A row is read once and its codes are written once, so a row is
// held in registers by the waves of one block, 8 elements (16 bytes) per lane
// and chunk of 512.  16384 x 4096 with a residual to e4m3: 80 us from HBM, 5.9
// TB/s (71 where the last-level cache still holds a part); 2747 x 3072 to bf16:
// 7.5 us; one row: 2.5 us, a launch.  16384 x 4096 without a residual takes the
// int4 form 57 us and the e4m3 one 42 (a copy's rate: 32 and 38), for its
// divisions; with a residual both wait for memory (78 and 82).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"
#include "block_internal.h"

namespace jq {

namespace {

using namespace block_detail;

template <bool NT = false>
__device__ __forceinline__ u32x4 load8(const uint16_t* p) {
  const u32x4* q = reinterpret_cast<const u32x4*>(p);
  return NT ? __builtin_nontemporal_load(q) : *q;
}

// h = x + residual of 8 elements, and the residual's new value.
template <bool RES, bool NT>
__device__ __forceinline__ void load_h(const NormArgs& a, int64_t row, int k, float* h) {
  unpack8_bf16(load8<NT>(a.x + row * a.x_stride + k), h);
  if constexpr (RES) {
    float r[8];
    unpack8_bf16(load8<NT>(a.res + row * a.res_stride + k), r);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = h[j] + r[j];
    *reinterpret_cast<u32x4*>(a.res_out + row * a.res_out_stride + k) = pack8_bf16(h);
  }
}

__device__ __forceinline__ float sum_sq(const float* h, float acc) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc = fmaf(h[j], h[j], acc);
  return acc;
}

// y = (h * r) * w in place; the largest magnitude's bits.
__device__ __forceinline__ uint32_t apply(float* h, float r, u32x4 wv) {
  float w[8];
  unpack8_bf16(wv, w);
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    h[j] = (h[j] * r) * w[j];
    m = umax(m, abs_bits(h[j]));
  }
  return m;
}

// Eight e4m3 codes of a lane and, by the first lane of L, their block's scale.
template <int L>
__device__ __forceinline__ void store_fp8(const NormArgs& a, int64_t row, int k, const float* y, uint32_t m, bool in) {
  const float s = e4m3_scale(lanes_max<L>(m));
  const E4m3Divisor d = e4m3_divisor(s);
  if (!in) return;
  float t[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = e4m3_quotient(y[j], d);
  *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.y) + row * a.D + k) = pack8_e4m3(t);
  if (k % 128 == 0) a.scale[row * ((a.D + 127) / 128) + k / 128] = s;
}

__device__ __forceinline__ uint32_t int4_codes(const float* y, float s) {
  uint32_t out = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float t = s == 0.0f ? 0.0f : __builtin_rintf(y[j] / s);
    t = fminf(fmaxf(t, -8.0f), 7.0f);
    out |= (static_cast<uint32_t>(static_cast<int>(t)) & 0xFu) << (4 * j);
  }
  return out;
}

// Rows of up to 8 * LPR elements: LPR lanes a row, 256 / LPR rows a block.
template <int LPR, NormOut OUT, bool RES, bool NT>
__global__ __launch_bounds__(256) void rmsnorm_short_kernel(const NormArgs a) {
  constexpr int kRows = 256 / LPR;
  const int k = 8 * (threadIdx.x % LPR);
  const bool in_row = k < a.D;
  const u32x4 w = in_row ? load8(a.w + k) : u32x4{0, 0, 0, 0};
  // every lane stays to the end: the reductions read their neighbours
  for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * kRows; row0 < a.M; row0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t row = row0 + threadIdx.x / LPR;
    const bool in = in_row && row < a.M;
    float h[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (in) load_h<RES, NT>(a, row, k, h);
    const float ss = lanes_sum<LPR>(sum_sq(h, 0.0f));
    const float r = 1.0f / sqrtf(ss / static_cast<float>(a.D) + a.eps);
    const uint32_t m = apply(h, r, w);
    if constexpr (OUT == NormOut::kBf16) {
      if (in) *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + row * a.D + k) = pack8_bf16(h);
    } else if constexpr (OUT == NormOut::kFp8) {
      store_fp8<LPR < 16 ? LPR : 16>(a, row, k, h, m, in);
    } else {
      const float s = __uint_as_float(lanes_max<LPR>(m)) / 7.0f;
      if (in) {
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.y) + row * (a.D / 2) + k / 2) = int4_codes(h, s);
        if (k == 0) a.scale[row] = s;
      }
    }
  }
}

// Longer rows: a block takes a row, its waves NC chunks of 512 each; or (SOLO)
// each of its four waves a row of its own.
template <int NC, NormOut OUT, bool RES, bool NT, bool SOLO>
__global__ __launch_bounds__(SOLO ? 256 : 1024) void rmsnorm_kernel(const NormArgs a) {
  __shared__ float part[16];
  __shared__ uint32_t part_max[16];
  const int lane = threadIdx.x & 63, wave = SOLO ? 0 : threadIdx.x >> 6, waves = SOLO ? 1 : blockDim.x >> 6;
  const int rows = SOLO ? 4 : 1;
  u32x4 w[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int k = (c * waves + wave) * 512 + lane * 8;
    w[c] = k < a.D ? load8(a.w + k) : u32x4{0, 0, 0, 0};
  }
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * rows + (SOLO ? threadIdx.x >> 6 : 0); row < a.M;
       row += static_cast<int64_t>(gridDim.x) * rows) {
    float h[NC][8];
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int k = (c * waves + wave) * 512 + lane * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) h[c][j] = 0.0f;
      if (k < a.D) load_h<RES, NT>(a, row, k, h[c]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) ss = sum_sq(h[c], ss);
    ss = lanes_sum<64>(ss);
    if (waves > 1) {
      if (lane == 0) part[wave] = ss;
      __syncthreads();
      ss = part[0];
      for (int i = 1; i < waves; ++i) ss += part[i];
    }
    const float r = 1.0f / sqrtf(ss / static_cast<float>(a.D) + a.eps);
    uint32_t m[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) m[c] = apply(h[c], r, w[c]);
    float s = 0.0f;
    if constexpr (OUT == NormOut::kInt4) {
      uint32_t am = m[0];
#pragma unroll
      for (int c = 1; c < NC; ++c) am = umax(am, m[c]);
      am = wave_max_bits(am);
      if (waves > 1) {
        if (lane == 0) part_max[wave] = am;
        __syncthreads();
        am = part_max[0];
        for (int i = 1; i < waves; ++i) am = umax(am, part_max[i]);
      }
      s = __uint_as_float(am) / 7.0f;
      if (lane == 0 && wave == 0) a.scale[row] = s;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int k = (c * waves + wave) * 512 + lane * 8;
      const bool in = k < a.D;
      if constexpr (OUT == NormOut::kBf16) {
        if (in) *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.y) + row * a.D + k) = pack8_bf16(h[c]);
      } else if constexpr (OUT == NormOut::kFp8) {
        store_fp8<16>(a, row, k, h[c], m[c], in);
      } else {
        if (in) *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.y) + row * (a.D / 2) + k / 2) = int4_codes(h[c], s);
      }
    }
    if (waves > 1) __syncthreads();  // the next row writes part[] again
  }
}

template <NormOut OUT, bool RES, bool NT>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  constexpr int64_t kMostBlocks = 1 << 20;
  auto grid = [&](int64_t rows) {
    const int64_t blocks = (a.M + rows - 1) / rows;
    return dim3(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks));
  };
  if (a.D <= 64) {
    hipLaunchKernelGGL((rmsnorm_short_kernel<8, OUT, RES, NT>), grid(32), dim3(256), 0, st, a);
  } else if (a.D <= 128) {
    hipLaunchKernelGGL((rmsnorm_short_kernel<16, OUT, RES, NT>), grid(16), dim3(256), 0, st, a);
  } else if (a.D <= 256) {
    hipLaunchKernelGGL((rmsnorm_short_kernel<32, OUT, RES, NT>), grid(8), dim3(256), 0, st, a);
  } else {
    // Two chunks a wave: with one, 16384 x 4096 without a residual took 48 us
    // instead of 42, with four 45, and 4096 x 12288 66 instead of 62.
    const int chunks = (a.D + 511) / 512;
    if (chunks == 1) hipLaunchKernelGGL((rmsnorm_kernel<1, OUT, RES, NT, true>), grid(4), dim3(256), 0, st, a);
    else if (chunks == 2) hipLaunchKernelGGL((rmsnorm_kernel<2, OUT, RES, NT, true>), grid(4), dim3(256), 0, st, a);
    else if (chunks <= 32)
      hipLaunchKernelGGL((rmsnorm_kernel<2, OUT, RES, NT, false>), grid(1), dim3(64 * ((chunks + 1) / 2)), 0, st, a);
    else if (chunks <= 64)
      hipLaunchKernelGGL((rmsnorm_kernel<4, OUT, RES, NT, false>), grid(1), dim3(64 * ((chunks + 3) / 4)), 0, st, a);
    else
      hipLaunchKernelGGL((rmsnorm_kernel<8, OUT, RES, NT, false>), grid(1), dim3(64 * ((chunks + 7) / 8)), 0, st, a);
  }
  return hipGetLastError();
}

// Inputs that the caches cannot hold anyway are read past them (non-temporal
// loads: 16384 x 4096 46 -> 42 us, 2000 x 16384 with a residual 49 -> 42);
// smaller ones usually lie there, as the kernel before left them (2747 x 3072:
// 7.2 us where they do, and 8.2 past the caches).
template <NormOut OUT, bool RES>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  const bool big = a.M * a.D * (RES ? 4 : 2) > (int64_t{1} << 26);
  return big ? launch<OUT, RES, true>(a, st) : launch<OUT, RES, false>(a, st);
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs& a, NormOut out, hipStream_t st) {
  const bool res = a.res != nullptr;
  switch (out) {
    case NormOut::kBf16: return res ? launch<NormOut::kBf16, true>(a, st) : launch<NormOut::kBf16, false>(a, st);
    case NormOut::kFp8: return res ? launch<NormOut::kFp8, true>(a, st) : launch<NormOut::kFp8, false>(a, st);
    default: return res ? launch<NormOut::kInt4, true>(a, st) : launch<NormOut::kInt4, false>(a, st);
  }
}

}  // namespace jq
