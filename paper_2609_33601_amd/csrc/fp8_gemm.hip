// 8-bit matrix product with a scale for each block of 128, for gfx950.
//
//   y[m,n] = bf16( sum_b (sx[m,b] * sw[n/128,b]) * sum_{k in b} qx[m,k] qw[n,k]  + bias[n] )
//
// Codes are e4m3; a block's product comes out of one 16x16x128 MFMA in fp32
// and is folded into the fp32 sums with one multiply-add per output, in k
// order.  W is the MFMA's first operand, so a lane holds four consecutive
// columns n of one row m: its scale is one number per 16 rows, and its
// outputs are one 8-byte store.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"
#include "block_internal.h"
#include "gemm_common.h"

namespace jq {

namespace {

using namespace block_detail;
using gemm_detail::kBufferFlags;
using gemm_detail::kNumXcd;
using gemm_detail::kOutsideOperand;
using gemm_detail::kWaitVm0;
using gemm_detail::tile_of_block;
using gemm_detail::TileCoord;

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 join_regs(u32x4 a, u32x4 b) {
  return i32x8{static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]),
               static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]), static_cast<int>(b[3])};
}

// One block of 128 k: W rows x X rows from zero.
__device__ __forceinline__ f32x4 mfma128(i32x8 w, i32x8 x) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}

// Transfers from a buffer into LDS, 16 (or 4) bytes per lane: lane i writes
// lds + 16 i (4 i).  As asm, because the compiler waits for transfers that it
// knows of before the next LDS read, whatever part of LDS that reads, and the
// whole point of two stages is not to.  The kernel waits itself (vmcnt(0) at
// the head of a stage).  The wait states that the compiler would put behind the
// writes of M0 and of descriptor words are in the asm; the build checks them.
typedef unsigned u32x4s __attribute__((ext_vector_type(4)));
struct Rsrc {
  u32x4s w;
};
__device__ __forceinline__ Rsrc make_rsrc(const void* base, int bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32)) & 0xFFFFu;
  const uint32_t n = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(bytes));
  return {u32x4s{lo, hi, n, static_cast<uint32_t>(kBufferFlags)}};
}
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}
__device__ __forceinline__ void dma16(const Rsrc& r, uint32_t lds, uint32_t voffset, uint32_t soffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voffset), "s"(r.w), "s"(soffset)
               : "memory");
}
__device__ __forceinline__ void dma4(const Rsrc& r, uint32_t lds, uint32_t voffset, uint32_t soffset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, %3 offen lds"
               :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voffset), "s"(r.w), "s"(soffset)
               : "memory");
}

// Four columns' bias, zeros where there is none.
__device__ __forceinline__ f32x4 bias4(const uint16_t* bias, int n, int N) {
  f32x4 v = {0, 0, 0, 0};
  if (bias != nullptr) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = bf_lo(bias[min(n + r, N - 1)]);
  }
  return v;
}

__device__ __forceinline__ void store4(uint16_t* y, int64_t row, int N, int n, f32x4 v) {
  uint16_t* p = y + row * N + n;
  if (N % 4 == 0) {
    *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < N) p[r] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[r]));
  }
}

// ---------------------------------------------------------------------------
// Many output tiles.  A block takes BM x BN outputs, WM x WN waves of it
// 16 FM x 16 FN each; stages of one block of 128 k, two in LDS, both operands
// moved by buffer-to-LDS DMA.  LDS rows are 128 bytes; the 16-byte chunk c of
// row r sits at slot c ^ (r & 7), so the sixteen rows that a fragment read
// spans cover all banks.

template <int BM, int BN, int WM, int WN, int PER_CU>
__global__ __launch_bounds__(64 * WM * WN, PER_CU) void fp8_gemm_kernel(
    const uint8_t* __restrict__ qx, const float* __restrict__ sx, int M, int K, const uint8_t* __restrict__ qw,
    const float* __restrict__ sw, int N, const uint16_t* __restrict__ bias, uint16_t* __restrict__ y, int tiles_m,
    int tiles_n) {
  constexpr int kWaves = WM * WN;
  constexpr int kFM = BM / WM / 16, kFN = BN / WN / 16;
  constexpr int kXDma = BM / 8 / kWaves, kWDma = BN / 8 / kWaves;  // DMA instructions per wave and stage: 8 rows each
  constexpr int kStage = (BM + BN) * 8;                            // 16-byte slots
  static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && 128 % (BN / WN) == 0, "");
  __shared__ uint4 lds[2 * kStage];
  __shared__ float sxl[2 * BM];

  TileCoord tc;
  if (!tile_of_block(blockIdx.x, tiles_m, tiles_n, &tc)) return;
  const int m0 = tc.tm * BM, n0 = tc.tn * BN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int li = lane & 15, lg = lane >> 4;
  const int kb = (K + 127) / 128;

  // Descriptors over this tile's rows only, so operands of any size have 32-bit offsets.
  const Rsrc rx = make_rsrc(qx + static_cast<int64_t>(m0) * K, min(BM, M - m0) * K);
  const Rsrc rw = make_rsrc(qw + static_cast<int64_t>(n0) * K, min(BN, N - n0) * K);
  const Rsrc rs = make_rsrc(sx + static_cast<int64_t>(m0) * kb, min(BM, M - m0) * kb * 4);
  // Lane l of a DMA fills slot l % 8 of row l / 8.  Rows past M or N, and
  // chunks past K, have offsets outside the descriptor and read as zero.
  const int chunk = (lane & 7) ^ (lane >> 3);
  const uint32_t lds0 = lds_addr(lds), sxl0 = lds_addr(sxl);
  auto issue = [&](int stage, int ks) __attribute__((always_inline)) {
    const uint32_t buf = lds0 + stage * kStage * 16;
    const uint32_t at = ks * 128 + 16 * chunk < K ? 16 * chunk : kOutsideOperand;
#pragma unroll
    for (int j = 0; j < kXDma; ++j) {
      const int r = 8 * (wave * kXDma + j) + (lane >> 3);
      dma16(rx, buf + 1024 * (wave * kXDma + j), r * K + at, ks * 128);
    }
#pragma unroll
    for (int j = 0; j < kWDma; ++j) {
      const int r = 8 * (wave * kWDma + j) + (lane >> 3);
      dma16(rw, buf + BM * 128 + 1024 * (wave * kWDma + j), r * K + at, ks * 128);
    }
    if (wave < BM / 64) dma4(rs, sxl0 + 4 * (stage * BM + 64 * wave), (64 * wave + lane) * kb * 4, ks * 4);
  };
  const int nb = min((n0 + wn * (BN / WN)) / 128, (N - 1) / 128);
  const float* swp = sw + static_cast<int64_t>(nb) * kb;

  f32x4 acc[kFN][kFM];
#pragma unroll
  for (int a = 0; a < kFN; ++a)
#pragma unroll
    for (int b = 0; b < kFM; ++b) acc[a][b] = f32x4{0, 0, 0, 0};

  auto frag = [&](const uint4* rows, int row) __attribute__((always_inline)) -> i32x8 {
    const int s = row & 7;
    // lane group lg takes chunks lg and 4 + lg (any k order serves, the same on both sides)
    const u32x4 lo = __builtin_bit_cast(u32x4, rows[row * 8 + (lg ^ s)]);
    const u32x4 hi = __builtin_bit_cast(u32x4, rows[row * 8 + ((4 + lg) ^ s)]);
    return join_regs(lo, hi);
  };

  issue(0, 0);
  float swv = swp[0];
  for (int ks = 0; ks < kb; ++ks) {
    const int cur = ks & 1;
    __builtin_amdgcn_s_waitcnt(kWaitVm0);
    __syncthreads();
    if (ks + 1 < kb) issue(cur ^ 1, ks + 1);
    const float sw_next = swp[min(ks + 1, kb - 1)];
    const uint4* xs = lds + cur * kStage;
    const uint4* ws = xs + BM * 8;
    const int row0 = wm * (BM / WM) + li;
    i32x8 w[kFN];
#pragma unroll
    for (int a = 0; a < kFN; ++a) w[a] = frag(ws, wn * (BN / WN) + 16 * a + li);
    // Row group b multiplies while b - 1 is folded and b + 1 is read.
    i32x8 x = frag(xs, row0);
    float s = sxl[cur * BM + row0] * swv;
    float sp = 0.0f;
    f32x4 p[kFN];
#pragma unroll
    for (int b = 0; b <= kFM; ++b) {
      i32x8 xn = x;
      float sn = s;
      if (b + 1 < kFM) {
        xn = frag(xs, row0 + 16 * (b + 1));
        sn = sxl[cur * BM + row0 + 16 * (b + 1)] * swv;
      }
      f32x4 q[kFN];
#pragma unroll
      for (int a = 0; a < kFN; ++a) {
        if (b < kFM) q[a] = mfma128(w[a], x);
        if (b > 0) {
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[a][b - 1][r] = fmaf(p[a][r], sp, acc[a][b - 1][r]);
        }
      }
#pragma unroll
      for (int a = 0; a < kFN; ++a) p[a] = q[a];
      sp = s, x = xn, s = sn;
      __builtin_amdgcn_sched_barrier(0);
    }
    swv = sw_next;
  }

#pragma unroll
  for (int a = 0; a < kFN; ++a) {
    const int n = n0 + wn * (BN / WN) + 16 * a + 4 * lg;
    if (n >= N) continue;
    const f32x4 bv = bias4(bias, n, N);
#pragma unroll
    for (int b = 0; b < kFM; ++b) {
      const int m = m0 + wm * (BM / WM) + 16 * b + li;
      if (m < M) store4(y, m, N, n, acc[a][b] + bv);
    }
  }
}

// ---------------------------------------------------------------------------
// Few output tiles.  A block takes 16 MB rows x 16 NB columns and its W waves
// split K: wave w takes blocks of 128 k number w, w + W, ..., straight into
// registers, no LDS or barrier in the loop.  The partial sums meet once, in
// LDS, in wave order.

template <int MB, int NB, int W>
__global__ __launch_bounds__(64 * W) void fp8_few_kernel(
    const uint8_t* __restrict__ qx, const float* __restrict__ sx, int M, int K, const uint8_t* __restrict__ qw,
    const float* __restrict__ sw, int N, const uint16_t* __restrict__ bias, uint16_t* __restrict__ y, int tiles_m,
    int tiles_n) {
  __shared__ f32x4 red[W * 64];
  TileCoord tc;
  if (!tile_of_block(blockIdx.x, tiles_m, tiles_n, &tc)) return;
  const int m0 = 16 * MB * tc.tm, n0 = 16 * NB * tc.tn;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int kb = (K + 127) / 128;
  const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(qx) + static_cast<int64_t>(m0) * K, 0, min(16 * MB, M - m0) * K, kBufferFlags);
  const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(qw) + static_cast<int64_t>(n0) * K, 0, min(16 * NB, N - n0) * K, kBufferFlags);
  // Lane group lg takes chunks lg and 4 + lg of a row's eight (any k order
  // serves, the same on both sides): an instruction reads 64 consecutive
  // bytes of each of 16 rows.
  auto load = [&](__amdgpu_buffer_rsrc_t rs, int f, int h, int ks) __attribute__((always_inline)) -> u32x4 {
    const int at = ks * 128 + 64 * h + 16 * lg;
    return __builtin_bit_cast(
        u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, at < K ? (16 * f + li) * K + at : kOutsideOperand, 0, 0));
  };
  f32x4 acc[NB][MB];
#pragma unroll
  for (int a = 0; a < NB; ++a)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[a][b] = f32x4{0, 0, 0, 0};
  for (int ks = wave; ks < kb; ks += W) {
    i32x8 w[NB], x[MB];
    float sxv[MB], swv[NB];
#pragma unroll
    for (int a = 0; a < NB; ++a) {
      w[a] = join_regs(load(rw, a, 0, ks), load(rw, a, 1, ks));
      swv[a] = sw[static_cast<int64_t>(min(n0 + 16 * a, N - 1) / 128) * kb + ks];
    }
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      x[b] = join_regs(load(rx, b, 0, ks), load(rx, b, 1, ks));
      sxv[b] = sx[static_cast<int64_t>(min(m0 + 16 * b + li, M - 1)) * kb + ks];
    }
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        const f32x4 p = mfma128(w[a], x[b]);
        const float s = sxv[b] * swv[a];
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[a][b][r] = fmaf(p[r], s, acc[a][b][r]);
      }
  }
#pragma unroll
  for (int a = 0; a < NB; ++a)
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      if (a + b) __syncthreads();
      red[wave * 64 + lane] = acc[a][b];
      __syncthreads();
      if (wave == 0) {
        f32x4 v = red[lane];
#pragma unroll
        for (int k = 1; k < W; ++k) v += red[k * 64 + lane];
        const int m = m0 + 16 * b + li, n = n0 + 16 * a + 4 * lg;
        if (m < M && n < N) store4(y, m, N, n, v + bias4(bias, n, N));
      }
    }
}

}  // namespace

hipError_t launch_fp8_gemm(const uint8_t* qx, const float* sx, int64_t M, int64_t K, const uint8_t* qw,
                           const float* sw, int64_t N, const uint16_t* bias, uint16_t* y, hipStream_t st) {
  const int Mi = static_cast<int>(M), Ki = static_cast<int>(K), Ni = static_cast<int>(N);
  auto tiles = [&](int bm, int bn, int* tm, int* tn) {
    *tm = static_cast<int>((M + bm - 1) / bm);
    *tn = static_cast<int>((N + bn - 1) / bn);
    return static_cast<unsigned>((static_cast<int64_t>(*tm) * *tn + kNumXcd - 1) / kNumXcd * kNumXcd);
  };
  int tm, tn;
  if (M <= 128) {
    if (M <= 16) {
      const unsigned blocks = tiles(16, 16, &tm, &tn);
      hipLaunchKernelGGL((fp8_few_kernel<1, 1, 8>), dim3(blocks), dim3(512), 0, st, qx, sx, Mi, Ki, qw, sw, Ni, bias, y, tm, tn);
    } else {
      const unsigned blocks = tiles(32, 32, &tm, &tn);
      hipLaunchKernelGGL((fp8_few_kernel<2, 2, 4>), dim3(blocks), dim3(256), 0, st, qx, sx, Mi, Ki, qw, sw, Ni, bias, y, tm, tn);
    }
  } else if (M * N <= 256 * 256 * 256) {
    const unsigned blocks = tiles(128, 128, &tm, &tn);
    hipLaunchKernelGGL((fp8_gemm_kernel<128, 128, 2, 2, 2>), dim3(blocks), dim3(256), 0, st, qx, sx, Mi, Ki, qw, sw, Ni, bias, y, tm, tn);
  } else {
    const unsigned blocks = tiles(256, 256, &tm, &tn);
    hipLaunchKernelGGL((fp8_gemm_kernel<256, 256, 2, 4, 2>), dim3(blocks), dim3(512), 0, st, qx, sx, Mi, Ki, qw, sw, Ni, bias, y, tm, tn);
  }
  return hipGetLastError();
}

}  // namespace jq
