// e4m3 quantisers of the 8-bit linear for gfx950.
//
//   activations: a block is 128 columns of a row (the last one may be short):
//     s = max|x| (1 / 448) (at least 2^-126; 0 for a block of zeros),
//     q = e4m3(x / s)
//   weights (once, when a model is loaded): a block is 128 rows x 128 columns.
//
// Bound: HBM, 2 bytes read and 1 written per element.  Activations: sixteen
// lanes hold a block (8 elements each), so its maximum takes four DPP steps
// and nothing passes through LDS; a wave takes 512 columns of a row.
// 16384 x 4096: 37 us, 5.4 TB/s; 77 x 12288: 2.6 us, a launch.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"
#include "block_internal.h"

namespace jq {

namespace {

using namespace block_detail;

__device__ __forceinline__ uint32_t max8(const float* f) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = umax(m, abs_bits(f[j]));
  return m;
}

__global__ __launch_bounds__(256) void quantize_fp8_kernel(const uint16_t* __restrict__ x, int64_t x_stride, int64_t M,
                                                           int K, uint8_t* __restrict__ q, float* __restrict__ scale) {
  const int lane = threadIdx.x & 63;
  const uint32_t per_row = (static_cast<uint32_t>(K) + 511) / 512;
  const uint32_t units = static_cast<uint32_t>(M) * per_row;
  for (uint32_t u = blockIdx.x * 4 + (threadIdx.x >> 6); u < units; u += gridDim.x * 4) {
    const uint32_t row = u / per_row;
    const int k = static_cast<int>(u - row * per_row) * 512 + lane * 8;
    const bool in = k < K;
    float f[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (in) unpack8_bf16(*reinterpret_cast<const u32x4*>(x + row * x_stride + k), f);
    const float s = e4m3_scale(lanes_max<16>(max8(f)));
    const E4m3Divisor d = e4m3_divisor(s);
    if (!in) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = e4m3_quotient(f[j], d);
    *reinterpret_cast<u32x2*>(q + static_cast<int64_t>(row) * K + k) = pack8_e4m3(f);
    if (k % 128 == 0) scale[static_cast<int64_t>(row) * ((K + 127) / 128) + k / 128] = s;
  }
}

__global__ __launch_bounds__(256) void pack_fp8_kernel(const uint16_t* __restrict__ w, int64_t N, int K,
                                                       uint8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t part[4];
  const int kb_count = (K + 127) / 128;
  const int64_t nb = blockIdx.x / kb_count;
  const int kb = blockIdx.x % kb_count;
  const int k = kb * 128 + 8 * (threadIdx.x & 15);
  const int r0 = threadIdx.x >> 4;
  float f[8][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t n = nb * 128 + r0 + 16 * i;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[i][j] = 0.0f;
    if (n < N && k < K) unpack8_bf16(*reinterpret_cast<const u32x4*>(w + n * K + k), f[i]);
    m = umax(m, max8(f[i]));
  }
  m = wave_max_bits(m);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  m = umax(umax(part[0], part[1]), umax(part[2], part[3]));
  const float s = e4m3_scale(m);
  const E4m3Divisor d = e4m3_divisor(s);
  if (threadIdx.x == 0) scale[blockIdx.x] = s;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t n = nb * 128 + r0 + 16 * i;
    if (n >= N || k >= K) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[i][j] = e4m3_quotient(f[i][j], d);
    *reinterpret_cast<u32x2*>(q + n * K + k) = pack8_e4m3(f[i]);
  }
}

}  // namespace

hipError_t launch_quantize_fp8(const uint16_t* x, int64_t x_stride, int64_t M, int64_t K, uint8_t* q, float* scale,
                               hipStream_t st) {
  const int64_t units = M * ((K + 511) / 512);
  const int64_t blocks = (units + 3) / 4;
  constexpr int64_t kMostBlocks = 1 << 20;
  hipLaunchKernelGGL(quantize_fp8_kernel, dim3(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks)),
                     dim3(256), 0, st, x, x_stride, M, static_cast<int>(K), q, scale);
  return hipGetLastError();
}

hipError_t launch_pack_fp8(const uint16_t* w, int64_t N, int64_t K, uint8_t* q, float* scale, hipStream_t st) {
  const int64_t blocks = ((N + 127) / 128) * ((K + 127) / 128);
  hipLaunchKernelGGL(pack_fp8_kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, w, N, static_cast<int>(K),
                     q, scale);
  return hipGetLastError();
}

}  // namespace jq
