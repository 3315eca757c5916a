// 8-bit matrix product with a scale for each block of 128, for gfx950.
//
//   y[m,n] = bf16( sum_b (sx[m,b] * sw[n/128,b]) * sum_{k in b} qx[m,k] qw[n,k]  + bias[n] )
//
// Codes are e4m3; a block's product comes out of one 16x16x128 MFMA in fp32 (of
// eight neighbouring k it cuts products at 2^-14 of the largest, as the other fp8
// MFMAs do; outputs' errors against 64 bits stay at their rounding, 0.0017) and is
// folded into the fp32 sums with one multiply-add per output, in k
// order.  W is the MFMA's first operand, so a lane holds four consecutive
// columns n of one row m: its scale is one number per 16 rows, and its
// outputs are one 8-byte store.
//
// Bound: the weights' bytes for few rows (1 x 12288 -> 4096: 9.3 us, 5.4 TB/s,
// where the last-level cache of 256 MB holds them, 14 us from HBM), their transfers
// for some dozens, the chain of a wave alone on its SIMD for some hundreds, the
// matrix cores for many.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "block_common.h"
#include "block_internal.h"
#include "gemm_common.h"
#include "jq_internal.h"

namespace jq {

namespace {

using namespace block_detail;
using gemm_detail::kNumXcd;
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

// Tile t in the grouped order of tile_of_block: 8 tiles of m per sweep of n.
__device__ __forceinline__ TileCoord tile_at(int t, int tiles_m, int tiles_n) {
  constexpr int kGroup = gemm_detail::kGroupM;
  const int group = t / (kGroup * tiles_n), first_m = group * kGroup;
  const int gm = min(tiles_m - first_m, kGroup), r = t - group * kGroup * tiles_n;
  return {first_m + r % gm, r / gm};
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

// A row of Y may start at any even address: these stores take any alignment
// (4691 x 304 -> 3273: 23 us, element by element 38).
template <typename T>
__device__ __forceinline__ void store_any(uint16_t* p, T v) {
  __builtin_memcpy(p, &v, sizeof(T));
}

__device__ __forceinline__ void store4(uint16_t* y, int64_t row, int N, int n, f32x4 v) {
  uint16_t* p = y + row * N + n;
  if (n + 4 <= N) {
    store_any(p, u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])});
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < N) p[r] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[r]));
  }
}

// ---------------------------------------------------------------------------
// Many output tiles.  A block takes BM x BN outputs, WM x WN waves of it
// 16 FM x 16 FN each, and walks a sequence of tiles as one sequence of stages
// of 128 k.  Both operands come by buffer-to-LDS transfers, two stages in LDS.
// LDS rows are 128 bytes; the 16-byte chunk c of row r sits at slot
// c ^ (r & 7), so that the sixteen rows a fragment read spans cover all banks.
//
// The one barrier of a stage stands before its last two row groups, whose
// operands are in registers by then: behind it the stage's buffer is free for
// the transfers of the stage after next, and the next stage's weights and first
// row group are read while the two groups multiply.  Between stages, and
// between tiles, the matrix pipe sees no gap but the stores.
//
// 8192 x 4096 -> 12288: 395 to 410 us among other calls, 2.0 to 2.1 PFLOP/s (406
// to 463 in traces of a dozen launches).  Power holds the clock: the same instructions on operands that do not change from stage to
// stage take 280 us, and the stores 20 to 40 of the 395.

template <int BM, int BN, int WM, int WN, int WPS>
__global__ __launch_bounds__(64 * WM * WN, WPS) void fp8_gemm_kernel(
    const uint8_t* __restrict__ qx, const float* __restrict__ sx, int M, int K, const uint8_t* __restrict__ qw,
    const float* __restrict__ sw, int N, const uint16_t* __restrict__ bias, uint16_t* __restrict__ y, int tiles_m,
    int tiles_n) {
  constexpr int kWaves = WM * WN;
  constexpr int kFM = BM / WM / 16, kFN = BN / WN / 16;
  constexpr int kXDma = BM / 8 / kWaves, kWDma = BN / 8 / kWaves;  // transfers per wave and stage: 8 rows each
  constexpr int kXSlots = BM * 8, kWSlots = BN * 8;                // of 16 bytes, per stage
  static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0 && 128 % (BN / WN) == 0, "");
  static_assert(kFN == 4 && kFM >= 4 && BM / 64 <= kWaves, "");
  __shared__ uint4 lds[2 * kXSlots + 2 * kWSlots];  // two stages of X, then of W: both within one offset's reach
  __shared__ float sxl[2 * BM];

  // XCD x takes a contiguous range of tiles, its blocks in turn.
  const int T = tiles_m * tiles_n, per_xcd = (T + kNumXcd - 1) / kNumXcd;
  const int step = gridDim.x / kNumXcd, xcd = blockIdx.x % kNumXcd;
  const int first = xcd * per_xcd + blockIdx.x / kNumXcd, end = min((xcd + 1) * per_xcd, T);
  if (first >= end) return;
  const int kb = (K + 127) / 128;
  const int stages = ((end - 1 - first) / step + 1) * kb;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int li = lane & 15, lg = lane >> 4;
  const uint32_t lds0 = lds_addr(lds), sxl0 = lds_addr(sxl);

  // Transfers run two stages ahead of the products: their own tile and stage.
  // Descriptors cover a tile's rows only, so operands of any size have 32-bit
  // offsets; rows past M or N, and chunks past K, have offsets outside the
  // descriptor and read as zero.  Lane l of a transfer fills slot l % 8 of row l / 8.
  const int chunk = (lane & 7) ^ (lane >> 3);
  int to = first, ks_to = 0, left = stages;
  Rsrc rx, rw, rs;
  auto aim = [&]() __attribute__((always_inline)) {
    const TileCoord tc = tile_at(to, tiles_m, tiles_n);
    const int m0 = tc.tm * BM, n0 = tc.tn * BN;
    rx = make_rsrc(qx + static_cast<int64_t>(m0) * K, min(BM, M - m0) * K);
    rw = make_rsrc(qw + static_cast<int64_t>(n0) * K, min(BN, N - n0) * K);
    rs = make_rsrc(sx + static_cast<int64_t>(m0) * kb, min(BM, M - m0) * kb * 4);
  };
  // A stage's transfers, a third at a time: a wave that issues all of them in
  // a row stands still for them.
  static_assert(kXDma == 4 && kWDma == 4, "");
  constexpr bool kSpread = kFM >= 8;  // a short stage has no time to lose
  auto issue = [&](int buf, auto part) __attribute__((always_inline)) {
    if (left == 0) return;
    const uint32_t at = ks_to * 128 + 16 * chunk < K ? 16 * chunk + (lane >> 3) * K : kOutsideBuffer;
    auto pair = [&](const Rsrc& r, uint32_t dst, int i) __attribute__((always_inline)) {
      const int row = 8 * (4 * wave + i);
      dma16(r, dst + 128 * row, row * K + at, ks_to * 128);
      dma16(r, dst + 128 * row + 1024, (row + 8) * K + at, ks_to * 128);
    };
    const uint32_t xd = lds0 + 16 * kXSlots * buf, wd = lds0 + 16 * (2 * kXSlots + kWSlots * buf);
    if constexpr (decltype(part)::value == 0) {
      pair(rx, xd, 0);
    } else if constexpr (decltype(part)::value == 1) {
      pair(rx, xd, 2), pair(rw, wd, 0);
    } else {
      pair(rw, wd, 2);
      if (wave < BM / 64) dma4(rs, sxl0 + 4 * (buf * BM + 64 * wave), (64 * wave + lane) * kb * 4, ks_to * 4);
    }
    if (decltype(part)::value == 2) {
      --left;
      if (++ks_to == kb) {
        ks_to = 0;
        to += step;
        if (left > 0) aim();
      }
    }
  };
  const std::integral_constant<int, 0> c0{};
  const std::integral_constant<int, 1> c1{};
  const std::integral_constant<int, 2> c2{};

  f32x4 acc[kFN][kFM];
  auto frag = [&](const uint4* rows, int row) __attribute__((always_inline)) -> i32x8 {
    // lane group lg takes chunks lg and 4 + lg (any k order serves, the same on both sides)
    const int s = row & 7;
    const u32x4 lo = __builtin_bit_cast(u32x4, rows[row * 8 + (lg ^ s)]);
    const u32x4 hi = __builtin_bit_cast(u32x4, rows[row * 8 + ((4 + lg) ^ s)]);
    return join_regs(lo, hi);
  };
  const int xrow = wm * (BM / WM) + li, wrow = wn * (BN / WN) + li;
  auto x_at = [&](int buf, int b) __attribute__((always_inline)) { return frag(lds + buf * kXSlots, xrow + 16 * b); };
  auto w_at = [&](int buf, int a) __attribute__((always_inline)) { return frag(lds + 2 * kXSlots + buf * kWSlots, wrow + 16 * a); };
  auto s_at = [&](int buf, int b) __attribute__((always_inline)) { return sxl[buf * BM + xrow + 16 * b]; };

  // The tile being multiplied, and its weights' scales.
  int at = first, ks = 0;
  TileCoord tc = tile_at(at, tiles_m, tiles_n);
  auto scales = [&]() __attribute__((always_inline)) {
    const float* p = sw + static_cast<int64_t>(min((tc.tn * BN + wn * (BN / WN)) / 128, (N - 1) / 128)) * kb;
    return (const __attribute__((address_space(4))) float*)p;
  };
  // read with scalar loads: a vector load's wait would take in the transfers under way
  typedef const __attribute__((address_space(4))) float* uniform_f32;
  uniform_f32 swp = scales();

  // The sums start from the bias.
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int a = 0; a < kFN; ++a) {
      const f32x4 v = bias4(bias, min(tc.tn * BN + wn * (BN / WN) + 16 * a + 4 * lg, N - 1), N);
#pragma unroll
      for (int b = 0; b < kFM; ++b) acc[a][b] = v;
    }
  };
  // Row group b of the tile.
  auto store = [&](int b) __attribute__((always_inline)) {
    const int m = tc.tm * BM + xrow + 16 * b, n0 = tc.tn * BN + wn * (BN / WN);
    if (n0 + 64 <= N) {
      // Lane group lg holds columns 16 a + 4 lg ..; swapping registers between
      // groups gives it 8 consecutive ones of each 32, so that a store covers
      // 64 consecutive bytes of each of 16 rows instead of 32.
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 v0 = acc[2 * h][b], v1 = acc[2 * h + 1][b];
        u32x4 out;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const auto r = __builtin_amdgcn_permlane32_swap(pack_bf16(v0[2 * i], v0[2 * i + 1]),
                                                          pack_bf16(v1[2 * i], v1[2 * i + 1]), false, false);
          const auto q = __builtin_amdgcn_permlane16_swap(r[0], r[1], false, false);
          out[i] = q[0], out[2 + i] = q[1];
        }
        if (m < M) store_any(y + static_cast<int64_t>(m) * N + n0 + 32 * h + 8 * lg, out);
      }
    } else if (m < M) {
#pragma unroll
      for (int a = 0; a < kFN; ++a)
        if (n0 + 16 * a + 4 * lg < N) store4(y, m, N, n0 + 16 * a + 4 * lg, acc[a][b]);
    }
  };

  i32x8 w[2][kFN], x0;  // this stage's weights and the next one's; a stage's first row group
  float s0, swv = swp[0];
  auto stage = [&](auto B_) __attribute__((always_inline)) {
    constexpr int B = decltype(B_)::value;
    const int next_ks = ks + 1 == kb ? 0 : ks + 1;
    i32x8 x[kFM];
    float s[kFM];
    x[0] = x0, s[0] = s0 * swv;
    i32x8 xn;
    float sn = 0.0f;
    f32x4 p[4];  // products in flight; each is folded three products later
    auto fold = [&](int t) __attribute__((always_inline)) {
      const int a = t % kFN, b = t / kFN;
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[a][b][r] = fmaf(p[t % 4][r], s[b], acc[a][b][r]);
    };
    const bool last = next_ks == 0;  // of a tile: its row groups are stored as they are done
    if (kSpread) issue(1 - B, c2);
#pragma unroll
    for (int b = 0; b < kFM; ++b) {
      if (b < kFM - 3) {
        x[b + 1] = x_at(B, b + 1), s[b + 1] = s_at(B, b + 1) * swv;
      } else if (b == kFM - 3) {
#pragma unroll
        for (int i = 1; i <= 2; ++i) x[b + i] = x_at(B, b + i), s[b + i] = s_at(B, b + i) * swv;
      } else if (b == kFM - 2) {
        __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) and lgkmcnt(0): the next stage is here, this one is read
        __syncthreads();
        issue(B, c0);
        if (!kSpread) issue(B, c1), issue(B, c2);
        w[1 - B][0] = w_at(1 - B, 0), w[1 - B][1] = w_at(1 - B, 1);
      } else {
        if (kSpread) issue(B, c1);
        w[1 - B][2] = w_at(1 - B, 2), w[1 - B][3] = w_at(1 - B, 3);
        xn = x_at(1 - B, 0), sn = s_at(1 - B, 0);
      }
#pragma unroll
      for (int a = 0; a < kFN; ++a) {
        const int t = b * kFN + a;
        p[t % 4] = mfma128(w[B][a], x[b]);
        if (t >= 3) fold(t - 3);
        __builtin_amdgcn_sched_barrier(0);  // one product, one fold: the compiler would group them
        if (a == kFN - 2 && b > 0 && last) {
          store(b - 1);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
#pragma unroll
    for (int t = kFM * kFN - 3; t < kFM * kFN; ++t) fold(t);
    x0 = xn, s0 = sn;
    ks = next_ks;
    if (last) {
      store(kFM - 1);
      at += step;
      if (at < end) {
        tc = tile_at(at, tiles_m, tiles_n);
        swp = scales();
        clear();
      }
    }
    swv = swp[ks];
  };

  aim();
  issue(0, c0), issue(0, c1), issue(0, c2);
  issue(1, c0), issue(1, c1);
  if (!kSpread) issue(1, c2);  // else at the head of the first stage
  clear();
  __builtin_amdgcn_s_waitcnt(kWaitVm0);
  __syncthreads();
#pragma unroll
  for (int a = 0; a < kFN; ++a) w[0][a] = w_at(0, a);
  x0 = x_at(0, 0), s0 = s_at(0, 0);
  for (int i = 0; i < stages; i += 2) {
    stage(c0);
    if (i + 1 == stages) break;
    stage(c1);
  }
}

// ---------------------------------------------------------------------------
// Few output tiles.  A block takes 16 MB rows x 16 NB columns and its W waves
// split K: wave w takes the blocks of 128 k number w, w + W, ...  Each wave
// moves its operands into an LDS ring of its own, S - 1 blocks ahead, and waits
// for nobody; the partial sums meet once, at the end, in wave order.
// Through LDS, because eight neighbouring lanes of a transfer read one row's
// 128 bytes: a CU takes in 123 B/ns that way.  Straight into registers,
// neighbouring lanes are the rows of an MFMA operand, 16 bytes of each, and
// that reaches a third of it (77 x 12288 -> 4096: 55 us).  Waiting for transfers
// bounds it: 77 x 12288 -> 4096 takes 15.8 us in 48 x 32 blocks, and 21.5 with the
// weights from HBM instead of the last-level cache.  With transfers in a row it
// took 18.2: 10.9 of them with nothing moved, 15.8 with nothing multiplied.  The
// blocks' tiles of X and W, 252 MB in all, would take 8 us at a CU's rate into LDS
// and the weights' 50 MB 9.5 at a copy's: the rest is latency that two blocks of k
// on their way to each wave do not cover.

template <int MB, int NB, int W, int S>
__global__ __launch_bounds__(64 * W) void fp8_few_kernel(
    const uint8_t* __restrict__ qx, const float* __restrict__ sx, int M, int K, const uint8_t* __restrict__ qw,
    const float* __restrict__ sw, int N, const uint16_t* __restrict__ bias, uint16_t* __restrict__ y, int tiles_m,
    int tiles_n) {
  constexpr int kFrags = MB + NB;                   // 16 rows x 128 bytes each
  constexpr int kOps = 2 * kFrags + 1;              // transfers of a block of k
  constexpr int kSlots = kFrags * 128 + 16;         // 16-byte slots: the fragments, then 64 scales
  static_assert(8 % NB == 0 && S >= 2 && (S - 2) * kOps < 64 && MB <= 4, "");
  constexpr int kRedSlots = W * 64 * NB;  // the sums of one row group
  __shared__ uint4 lds[W * S * kSlots > kRedSlots ? W * S * kSlots : kRedSlots];
  TileCoord tc;
  if (!tile_of_block(blockIdx.x, tiles_m, tiles_n, &tc)) return;
  const int m0 = 16 * MB * tc.tm, n0 = 16 * NB * tc.tn;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int kb = (K + 127) / 128;
  const Rsrc rx = make_rsrc(qx + static_cast<int64_t>(m0) * K, min(16 * MB, M - m0) * K);
  const Rsrc rw = make_rsrc(qw + static_cast<int64_t>(n0) * K, min(16 * NB, N - n0) * K);
  const Rsrc rs = make_rsrc(sx + static_cast<int64_t>(m0) * kb, min(16 * MB, M - m0) * kb * 4);
  const uint4* ring = lds + wave * S * kSlots;
  const uint32_t ring_at = lds_addr(ring);

  // Lane l of a transfer fills slot l % 8 of row l / 8 with chunk slot ^ row, as
  // in the kernel above.  Blocks past the last read as zeros, so that every
  // step has the same number of transfers under way.
  const int chunk = (lane & 7) ^ (lane >> 3);
  const uint32_t row_at = (lane >> 3) * K + 16 * chunk;
  // Transfer i of a block of k: two of each fragment, then the scales.
  auto issue = [&](int slot, int u, int i) __attribute__((always_inline)) {
    const uint32_t dst = ring_at + slot * kSlots * 16;
    if (i < 2 * kFrags) {
      const int f = i / 2, h = i % 2;
      const uint32_t at = u * 128 + 16 * chunk < K ? row_at : kOutsideBuffer;
      dma16<0>(f < NB ? rw : rx, dst + 1024 * i, at + (16 * (f < NB ? f : f - NB) + 8 * h) * K, u < kb ? u * 128 : 0);
    } else if (i == 2 * kFrags) {
      dma4(rs, dst + 2048 * kFrags, u < kb && lane < 16 * MB ? lane * kb * 4 + u * 4 : kOutsideBuffer, 0);
    }
  };
  auto frag = [&](const uint4* rows) __attribute__((always_inline)) -> i32x8 {
    const int s = li & 7;
    return join_regs(__builtin_bit_cast(u32x4, rows[li * 8 + (lg ^ s)]),
                     __builtin_bit_cast(u32x4, rows[li * 8 + ((4 + lg) ^ s)]));
  };

  f32x4 acc[NB][MB];
#pragma unroll
  for (int a = 0; a < NB; ++a)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[a][b] = f32x4{0, 0, 0, 0};
  typedef const __attribute__((address_space(4))) float* uniform_f32;
  const uniform_f32 swp = (uniform_f32)(sw + static_cast<int64_t>(n0 / 128) * kb);
#pragma unroll
  for (int i = 0; i < S - 1; ++i)
#pragma unroll
    for (int k = 0; k < kOps; ++k) issue(i, wave + W * i, k);
  float swv = swp[min(wave, kb - 1)];
  int slot = 0;
  // The transfers of the block S - 1 ahead are dealt out between the products: a
  // CU's waves share the path that takes them, and a wave that issues a block's
  // worth in a row stands in its queue (333 x 4096 -> 4096: 16.9 us, dealt 14.9).
  constexpr int kPer = (kOps + MB * NB) / (MB * NB + 1);
  for (int u = wave; u < kb; u += W) {
    const float sw_next = swp[min(u + W, kb - 1)];
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((S - 2) * kOps) : "memory");
    const uint4* at = ring + slot * kSlots;
    const int into = slot == 0 ? S - 1 : slot - 1, ahead = u + W * (S - 1);  // the slot before this one has been read
    auto deal = [&](int step) __attribute__((always_inline)) {
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (kPer * step + k < kOps) issue(into, ahead, kPer * step + k);
    };
    i32x8 w[NB];
#pragma unroll
    for (int a = 0; a < NB; ++a) w[a] = frag(at + 128 * a);
    deal(0);
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      const i32x8 x = frag(at + 128 * (NB + b));
      const float s = reinterpret_cast<const float*>(at + 128 * kFrags)[16 * b + li] * swv;
#pragma unroll
      for (int a = 0; a < NB; ++a) {
        const f32x4 p = mfma128(w[a], x);
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[a][b][r] = fmaf(p[r], s, acc[a][b][r]);
        deal(1 + b * NB + a);
      }
    }
    swv = sw_next;
    slot = slot + 1 == S ? 0 : slot + 1;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // no transfer lands in what follows
  f32x4* red = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    __syncthreads();
#pragma unroll
    for (int a = 0; a < NB; ++a) red[(a * W + wave) * 64 + lane] = acc[a][b];
    __syncthreads();
    for (int a = wave; a < NB; a += W) {
      f32x4 v = red[a * W * 64 + lane];
#pragma unroll
      for (int k = 1; k < W; ++k) v += red[(a * W + k) * 64 + lane];
      const int m = m0 + 16 * b + li, n = n0 + 16 * a + 4 * lg;
      if (m < M && n < N) store4(y, m, N, n, v + bias4(bias, n, N));
    }
  }
}

}  // namespace

namespace {

// The kernels that a product may take, with what estimates their time in ns:
// a launch, each round of resident blocks, and each block of 128 k that a
// wave walks, once per round and once per block that the busiest CU has.
// Fitted to 259 shapes (M 1 .. 8192, K 256 .. 16384, N 64 .. 16384, over their
// logarithms) to 10 to 16% each; the kernel with the lowest estimate was 0.6%
// slower than the best one on average, 16% at worst; on 68 other shapes (M 1 ..
// 4096, weights from HBM) 0.8 and 17%.
// 96 x 4096 -> 4096 takes 9.8 us with 48 x 32 blocks, 18 with 16 x 16 ones and 32
// with 128 x 128; 1 x 4096 -> 4096 6.1 with 16 x 16 blocks and 13 with 64 x 64;
// 4096 x 4096 -> 4096 68 with 256 x 256 and 90 with 128 x 128.
struct Fp8Kernel {
  int mb, nb, waves, per_cu;            // of 16 rows and columns; waves that split K; blocks on a CU
  float launch, round, round_k, each_k;
};
constexpr int kFp8Few = 8;  // those of fp8_few_kernel come first, then the two of fp8_gemm_kernel
constexpr Fp8Kernel kFp8Kernels[kFp8Few + 2] = {
    {1, 1, 8, 2, 1713, 696, 0, 425},    {1, 2, 4, 3, 1779, 551, 31, 330},  {1, 2, 4, 2, 1628, 928, 0, 318},
    {2, 2, 4, 1, 1124, 1500, 438, 0},   {3, 2, 4, 1, 1097, 1713, 600, 0},  {2, 4, 4, 1, 1209, 1730, 713, 0},
    {3, 4, 2, 2, 1124, 2203, 406, 227}, {4, 4, 4, 1, 1065, 2098, 1078, 0}, {8, 8, 1, 2, 1429, 1896, 205, 554},
    {16, 16, 1, 1, 0, 4787, 1796, 0},
};

}  // namespace

int fp8_gemm_route(int64_t M, int64_t N, int64_t K, int64_t cus) {
  const int64_t kb = (K + 127) / 128;
  int best = -1;
  float best_ns = 0;
  for (int i = 0; i < kFp8Few + 2; ++i) {
    const Fp8Kernel& k = kFp8Kernels[i];
    const int64_t tiles = (M + 16 * k.mb - 1) / (16 * k.mb) * ((N + 16 * k.nb - 1) / (16 * k.nb));
    const int64_t each = (tiles + cus - 1) / cus, rounds = (each + k.per_cu - 1) / k.per_cu;
    const int64_t steps = (kb + k.waves - 1) / k.waves;
    if (tiles >= (1 << 22) && i < kFp8Few) continue;  // a grid holds fewer than 2^32 threads
    const float ns = k.launch + rounds * k.round + static_cast<float>(steps) * (rounds * k.round_k + each * k.each_k);
    if (best < 0 || ns < best_ns) best = i, best_ns = ns;
  }
  return best;
}

hipError_t launch_fp8_gemm(const uint8_t* qx, const float* sx, int64_t M, int64_t K, const uint8_t* qw,
                           const float* sw, int64_t N, const uint16_t* bias, uint16_t* y, hipStream_t st) {
  int64_t cus;
  const hipError_t e = device_route_cus(&cus);
  if (e != hipSuccess) return e;
  const int r = fp8_gemm_route(M, N, K, cus);
  const int tm = static_cast<int>((M + 16 * kFp8Kernels[r].mb - 1) / (16 * kFp8Kernels[r].mb));
  const int tn = static_cast<int>((N + 16 * kFp8Kernels[r].nb - 1) / (16 * kFp8Kernels[r].nb));
  const int64_t tiles = (static_cast<int64_t>(tm) * tn + kNumXcd - 1) / kNumXcd * kNumXcd;
#define JQ_FP8(KERNEL, BLOCKS, THREADS)                                                                          \
  hipLaunchKernelGGL((KERNEL), dim3(static_cast<unsigned>(BLOCKS)), dim3(THREADS), 0, st, qx, sx,                \
                     static_cast<int>(M), static_cast<int>(K), qw, sw, static_cast<int>(N), bias, y, tm, tn)
#define JQ_FEW(MB, NB, W, S) JQ_FP8((fp8_few_kernel<MB, NB, W, S>), tiles, 64 * W)
  switch (r) {
    case 0: JQ_FEW(1, 1, 8, 2); break;
    case 1: JQ_FEW(1, 2, 4, 2); break;
    case 2: JQ_FEW(1, 2, 4, 3); break;
    case 3: JQ_FEW(2, 2, 4, 3); break;
    case 4: JQ_FEW(3, 2, 4, 3); break;
    case 5: JQ_FEW(2, 4, 4, 3); break;
    case 6: JQ_FEW(3, 4, 2, 2); break;
    case 7: JQ_FEW(4, 4, 4, 2); break;
    // these walk tiles of their own accord: as many blocks as fit the device
    case 8: JQ_FP8((fp8_gemm_kernel<128, 128, 2, 2, 2>), std::min(tiles, 2 * cus), 256); break;
    default: JQ_FP8((fp8_gemm_kernel<256, 256, 2, 4, 2>), std::min(tiles, cus), 512); break;
  }
#undef JQ_FEW
#undef JQ_FP8
  return hipGetLastError();
}

}  // namespace jq
