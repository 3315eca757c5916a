// Rotation of the new tokens' queries and keys by their positions, and their
// keys and values written into a paged cache, for gfx950.
//
//   (a, b) -> (a c - b s, a s + b c),  c = cos[position, i], s = sin[position, i]
//   on the pairs (i, i + R/2), or (2i, 2i + 1) if interleaved, i < R/2; the
//   other D - R elements of a head pass unchanged.  Values are not rotated.
//   Cache: [pages, Hk, page, D]; slot = page number * page + place in the page.
//   bf16, or e4m3 codes with s = max|.| (1 / 448) of each token and head.
//
// Bound: HBM; each element is read and written once.  A lane holds both
// halves of eight pairs (two 16-byte loads), so the rotation is lane-local,
// and D / 16 lanes hold a head, so the 8-bit cache's maximum is a few DPP
// steps.  One launch does queries, keys and values.  8191 tokens of 32 + 8 + 8
// heads of 128 to an 8-bit cache: 36 us, 5.2 TB/s, as plain copies run (0.25 GB
// 5.4, 4 GB 4.9), and 39 us a call from HBM, 31 from the last-level cache; two, four or eight heads a lane took 41, 43 and 46 us.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"
#include "block_internal.h"

namespace jq {

namespace {

using namespace block_detail;

// LPH lanes a head: D / 16 rounded up to a power of two.
template <int LPH, bool FP8, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_append_kernel(const AppendArgs a) {
  const int per_token = a.Hq + 2 * a.Hk;
  const int64_t heads = a.T * per_token;
  const int c = threadIdx.x % LPH;  // 16 elements: 8 pairs, or 16 in a row
  constexpr int kHeads = 256 / LPH;
  const int half = a.R / 2;
  for (int64_t h0 = static_cast<int64_t>(blockIdx.x) * kHeads; h0 < heads; h0 += static_cast<int64_t>(gridDim.x) * kHeads) {
    const int64_t at = h0 + threadIdx.x / LPH;
    const bool live = at < heads && 16 * c < a.D;
    // h0 < 2^31 by the caller's check, so 32-bit division
    const uint32_t t = live ? static_cast<uint32_t>(at) / static_cast<uint32_t>(per_token) : 0;
    const int h = live ? static_cast<int>(static_cast<uint32_t>(at) - t * per_token) : 0;
    const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hk;
    const int hk = is_q ? h : is_v ? h - a.Hq - a.Hk : h - a.Hq;
    const uint16_t* src = is_q ? a.q + t * a.q_stride : is_v ? a.v + t * a.v_stride : a.k + t * a.k_stride;
    src += static_cast<int64_t>(hk) * a.D;
    // Where the two runs of eight elements lie in the head.
    const bool turned = !is_v && 16 * c < a.R;
    const int i0 = turned && !INTERLEAVED ? 8 * c : 16 * c;
    const int i1 = turned && !INTERLEAVED ? half + 8 * c : 16 * c + 8;
    const int64_t pos = live ? a.positions[t] : 0;
    const int64_t slot = live && !is_q ? a.slots[t] : 0;
    const bool pos_ok = pos >= 0 && pos < a.P;
    float f[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) f[j] = 0.0f;
    if (live) {
      unpack8_bf16(*reinterpret_cast<const u32x4*>(src + i0), f);
      unpack8_bf16(*reinterpret_cast<const u32x4*>(src + i1), f + 8);
      if (turned) {
        // a position outside the tables has no rotation: NaN
        const int64_t row = (pos_ok ? pos : 0) * half + 8 * c;
        float cs[8], sn[8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          *reinterpret_cast<f32x4*>(cs + 4 * j) = *reinterpret_cast<const f32x4*>(a.cos + row + 4 * j);
          *reinterpret_cast<f32x4*>(sn + 4 * j) = *reinterpret_cast<const f32x4*>(a.sin + row + 4 * j);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int ia = INTERLEAVED ? 2 * j : j, ib = INTERLEAVED ? 2 * j + 1 : 8 + j;
          const float x = f[ia], y = f[ib];
          const float cj = pos_ok ? cs[j] : __builtin_nanf(""), sj = pos_ok ? sn[j] : __builtin_nanf("");
          f[ia] = x * cj - y * sj;
          f[ib] = x * sj + y * cj;
        }
      }
    }
    if (is_q) {
      if (live) {
        uint16_t* dst = a.q_out + t * a.q_out_stride + static_cast<int64_t>(hk) * a.D;
        *reinterpret_cast<u32x4*>(dst + i0) = pack8_bf16(f);
        *reinterpret_cast<u32x4*>(dst + i1) = pack8_bf16(f + 8);
      }
    }
    float s = 0.0f;
    if constexpr (FP8) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) m = umax(m, abs_bits(f[j]));
      s = e4m3_scale(lanes_max<LPH>(m));  // all lanes of the wave: before any leaves
    }
    if (!live || is_q || slot < 0 || slot >= a.num_slots) continue;
    const int64_t page = slot >> a.page_shift;
    const int64_t line = ((page * a.Hk + hk) << a.page_shift) + (slot & (a.page - 1));
    if constexpr (FP8) {
      const E4m3Divisor d = e4m3_divisor(s);
#pragma unroll
      for (int j = 0; j < 16; ++j) f[j] = e4m3_quotient(f[j], d);
      uint8_t* dst = static_cast<uint8_t*>(is_v ? a.v_cache : a.k_cache) + line * a.D;
      *reinterpret_cast<u32x2*>(dst + i0) = pack8_e4m3(f);
      *reinterpret_cast<u32x2*>(dst + i1) = pack8_e4m3(f + 8);
      if (c == 0) (is_v ? a.v_scale : a.k_scale)[line] = s;
    } else {
      uint16_t* dst = static_cast<uint16_t*>(is_v ? a.v_cache : a.k_cache) + line * a.D;
      *reinterpret_cast<u32x4*>(dst + i0) = pack8_bf16(f);
      *reinterpret_cast<u32x4*>(dst + i1) = pack8_bf16(f + 8);
    }
  }
}

template <int LPH>
hipError_t launch(const AppendArgs& a, hipStream_t st) {
  const int64_t heads = a.T * (a.Hq + 2 * a.Hk);
  const int64_t blocks = (heads + 256 / LPH - 1) / (256 / LPH);
  constexpr int64_t kMostBlocks = 1 << 20;
  const dim3 grid(static_cast<unsigned>(blocks < kMostBlocks ? blocks : kMostBlocks)), block(256);
  if (a.fp8) {
    if (a.interleaved) hipLaunchKernelGGL((rope_append_kernel<LPH, true, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rope_append_kernel<LPH, true, false>), grid, block, 0, st, a);
  } else {
    if (a.interleaved) hipLaunchKernelGGL((rope_append_kernel<LPH, false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rope_append_kernel<LPH, false, false>), grid, block, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_append(const AppendArgs& a, hipStream_t st) {
  switch ((a.D + 15) / 16) {
    case 1: return launch<1>(a, st);
    case 2: return launch<2>(a, st);
    case 3: case 4: return launch<4>(a, st);
    case 5: case 6: case 7: case 8: return launch<8>(a, st);
    default: return launch<16>(a, st);
  }
}

}  // namespace jq
