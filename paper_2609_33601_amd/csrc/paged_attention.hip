// Attention of a sequence's newest tokens over its paged key-value cache, for
// gfx950: one new token a sequence, or the block of tokens that block
// diffusion decodes at once.
//
//   p = softmax over visible t of scale * (q . k_t),  o = sum_t p_t v_t
//   visible: t < len, and for causal calls t <= len - Tq + i for new token i.
//   A query that sees nothing gives zeros (and lse = -inf).
//
// What bounds it: reading the cache once.  Everything else follows from that.
//  * Columns.  The query heads of one key head, times the new tokens, are the
//    columns of a matrix product, 16 (or 32, 64) of them at a time, so a
//    cached row is read once for all of them.
//  * S^T = K Q^T and O^T = V^T P^T on 16x16x32 MFMAs.  With S transposed, the
//    lane that holds a column's scores holds the same column's row of P as
//    the next product's operand, for the same tokens: lane group g has tokens
//    4g..4g+3 of each of two 16-token halves, and since a product may take
//    its k in any order, that is the order V is read in.  P never leaves its
//    registers, and the running maximum, sum and rescaling are per lane.
//  * V arrives row-major, 8 tokens x D/16 consecutive values per lane; pairs
//    of tokens are zipped with one v_perm_b32 per two values.
//  * The key axis is cut into parts of `chunk` tokens, a block each, whose
//    four waves take 32-token tiles in turn, each with its own running
//    softmax, and join in LDS.  With more than one part the parts' sums go to
//    the workspace and a second kernel joins them.
// Scores, statistics and sums are fp32; P is rounded to bf16 for its product
// (its sum is of the unrounded values), which is the precision of V itself.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "block_common.h"
#include "block_internal.h"

namespace jq {

namespace {

using namespace block_detail;

constexpr int kWaves = 4;
constexpr int kTile = 32;  // tokens of a wave's step
constexpr float kNegInf = -__builtin_inff();

// Largest over the lanes that differ in the upper two lane bits.
__device__ __forceinline__ float max_groups(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_groups(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// Two e4m3 values (one half of u) to bf16, exactly.
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_pair_to_bf16(uint32_t u) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HI));
}

// BYTES (4 .. 32) from p into dst's dwords.
template <int BYTES>
__device__ __forceinline__ void load_bytes(const uint8_t* p, uint32_t* dst) {
  if constexpr (BYTES == 4) {
    dst[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (BYTES == 8) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(p);
    dst[0] = v[0], dst[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p + 16 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) dst[4 * i + j] = v[j];
    }
  }
}

// The partial results of a part: [b][hk][part][column] of D sums, then of the
// maximum (in powers of two) and the sum.
struct PartView {
  float* o;
  float* ml;
};
__host__ __device__ __forceinline__ PartView part_view(float* ws, int64_t rows, int D) { return {ws, ws + rows * D}; }

// NG groups of 16 columns per wave.
template <int D, bool FP8, int NG, int WPS>
__global__ __launch_bounds__(64 * kWaves, WPS) void paged_attention_kernel(const AttnArgs a, int chunk, int parts,
                                                                           int col_blocks) {
  constexpr int kB = FP8 ? 1 : 2;   // bytes of a cached value
  constexpr int kDV = D / 16;       // values of a V row per lane
  constexpr int kKS = D / 32;       // k-steps of the first product
  __shared__ float red_o[kWaves * 16 * (D + 4)];
  __shared__ float red_m[kWaves * 16], red_l[kWaves * 16];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  // Blocks that share a part's keys lie next to each other; parts of one head follow.
  int id = blockIdx.x;
  const int cb = id % col_blocks;
  id /= col_blocks;
  const int part = id % parts;
  id /= parts;
  const int hk = id % a.Hk;
  const int b = id / a.Hk;

  const int G = a.Hq / a.Hk;
  const int cols = a.Tq * G;
  const int page = 1 << a.page_shift;
  int len = a.lens[b];
  len = min(len, a.max_len);
  const int t0 = part * chunk;
  const int t1 = min(len, t0 + chunk);
  const bool direct = parts == 1;
  if (t0 >= t1 && !direct) return;  // the joining kernel counts parts by len, too

  // Queries: column -> (new token, head of the group).  Columns past the last repeat it.
  int qi[NG];        // new token of this lane's column
  int64_t qrow[NG];  // its row in [B, Tq, Hq]
  bf16x8 qf[NG][kKS];
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    const int col = min((cb * NG + n) * 16 + li, cols - 1);
    qi[n] = col / G;
    qrow[n] = (static_cast<int64_t>(b) * a.Tq + qi[n]) * a.Hq + hk * G + (col - qi[n] * G);
    const uint16_t* qp = a.q + qrow[n] * D;
#pragma unroll
    for (int c = 0; c < kKS; ++c) {
      // which eight of a head a lane feeds to step c: with bytes, sixteen consecutive values serve two steps
      const int d = FP8 ? 64 * (c / 2) + 16 * lg + 8 * (c % 2) : 32 * c + 8 * lg;
      qf[n][c] = *reinterpret_cast<const bf16x8*>(qp + d);
    }
  }

  f32x4 o[NG][kDV];
  float m[NG], l[NG];
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    m[n] = kNegInf, l[n] = 0.0f;
#pragma unroll
    for (int j = 0; j < kDV; ++j) o[n][j] = f32x4{0, 0, 0, 0};
  }
  const float scale2 = a.scale * 1.44269504088896340736f;  // exponentials are powers of two
  const int32_t* table = a.table + static_cast<int64_t>(b) * a.table_cols;
  const uint8_t* kbase = static_cast<const uint8_t*>(a.k_cache);
  const uint8_t* vbase = static_cast<const uint8_t*>(a.v_cache);
  bool bad = false;  // a page number outside the cache was met

  for (int tile = t0 + wave * kTile; tile < t1; tile += kWaves * kTile) {
    // Pages hold 16 tokens or more, so each half of a tile lies in one page.
    // Tokens past the end read the last one (finite numbers that count for nothing).
    int64_t line[2];  // first cached row of the half
    int last[2];      // its last readable place
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int h0 = tile + 16 * s < len ? tile + 16 * s : tile;
      const int pi = h0 >> a.page_shift;
      int pg = table[pi];
      if (pg < 0 || pg >= a.num_pages) bad = true, pg = 0;
      line[s] = ((static_cast<int64_t>(pg) * a.Hk + hk) << a.page_shift) + (h0 & (page - 1));
      last[s] = min(len - 1 - h0, 15);
    }

    uint32_t kf[2][kKS * 4 * kB / 2];
    float ks[2][4], vs[2][4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint8_t* kp = kbase + (line[s] + min(li, last[s])) * (D * kB);
#pragma unroll
      for (int c = 0; c < kKS * kB / 2; ++c) load_bytes<16>(kp + 64 * c + 16 * lg, kf[s] + 4 * c);
      if constexpr (FP8) {
        *reinterpret_cast<f32x4*>(ks[s]) = *reinterpret_cast<const f32x4*>(a.k_scale + line[s] + 4 * lg);
        *reinterpret_cast<f32x4*>(vs[s]) = *reinterpret_cast<const f32x4*>(a.v_scale + line[s] + 4 * lg);
      }
    }
    uint32_t vf[8][kDV * kB / 4];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int s = e / 4;
      const uint8_t* vp = vbase + (line[s] + min(4 * lg + e % 4, last[s])) * (D * kB);
      load_bytes<kDV * kB>(vp + li * (kDV * kB), vf[e]);
    }

    // scores
    f32x4 sc[NG][2];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int c = 0; c < kKS; ++c) {
        bf16x8 kv;
        if constexpr (FP8) {
          const uint32_t w0 = kf[s][2 * c], w1 = kf[s][2 * c + 1];
          kv = __builtin_bit_cast(bf16x8, u32x4{e4m3_pair_to_bf16<false>(w0), e4m3_pair_to_bf16<true>(w0),
                                                e4m3_pair_to_bf16<false>(w1), e4m3_pair_to_bf16<true>(w1)});
        } else {
          kv = __builtin_bit_cast(bf16x8, u32x4{kf[s][4 * c], kf[s][4 * c + 1], kf[s][4 * c + 2], kf[s][4 * c + 3]});
        }
#pragma unroll
        for (int n = 0; n < NG; ++n)
          sc[n][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, qf[n][c], c ? sc[n][s] : f32x4{0, 0, 0, 0}, 0, 0, 0);
      }

    // softmax: this lane's column, tokens tile + 16 s + 4 lg + r
    bf16x8 p[NG];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      const int end = a.causal ? min(len, len - a.Tq + 1 + qi[n]) : len;
      float v[8];
      float top = kNegInf;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = tile + 16 * (e / 4) + 4 * lg + e % 4;
        float x = sc[n][e / 4][e % 4] * scale2;
        if constexpr (FP8) x *= ks[e / 4][e % 4];
        v[e] = t < end ? x : kNegInf;
        top = fmaxf(top, v[e]);
      }
      top = fmaxf(max_groups(top), m[n]);
      const float base = top == kNegInf ? 0.0f : top;  // nothing seen yet: every power below is 0
      if (__any(top != m[n])) {
        const float keep = __builtin_amdgcn_exp2f(m[n] - base);
        l[n] *= keep;
#pragma unroll
        for (int j = 0; j < kDV; ++j) o[n][j] *= keep;
        m[n] = top;
      }
      float pe[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        pe[e] = __builtin_amdgcn_exp2f(v[e] - base);
        l[n] += pe[e];
        if constexpr (FP8) pe[e] = v[e] == kNegInf ? 0.0f : pe[e] * vs[e / 4][e % 4];
      }
      p[n] = __builtin_bit_cast(bf16x8, pack8_bf16(pe));
    }

    // O^T += V^T P^T, one MFMA per value of a lane's V rows
    auto vt = [&](int j) __attribute__((always_inline)) -> bf16x8 {
      u32x4 r;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        uint32_t x, y;  // the dwords of tokens 2h and 2h + 1 that hold value j
        if constexpr (FP8) {
          const uint32_t wx = vf[2 * h][j / 4], wy = vf[2 * h + 1][j / 4];
          x = (j & 2) ? e4m3_pair_to_bf16<true>(wx) : e4m3_pair_to_bf16<false>(wx);
          y = (j & 2) ? e4m3_pair_to_bf16<true>(wy) : e4m3_pair_to_bf16<false>(wy);
        } else {
          x = vf[2 * h][j / 2];
          y = vf[2 * h + 1][j / 2];
        }
        r[h] = __builtin_amdgcn_perm(y, x, (j & 1) ? 0x07060302u : 0x05040100u);
      }
      return __builtin_bit_cast(bf16x8, r);
    };
#pragma unroll
    for (int j = 0; j < kDV; ++j) {
      const bf16x8 v = vt(j);
#pragma unroll
      for (int n = 0; n < NG; ++n) o[n][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[n], o[n][j], 0, 0, 0);
    }
  }

  if (__any(bad)) {
#pragma unroll
    for (int n = 0; n < NG; ++n) l[n] = __builtin_nanf(""), m[n] = 0.0f;
  }

  // Join the waves.  A lane holds, of column li, values d = kDV (4 lg + r) + j:
  // kDV * 4 in a row, from kDV * 4 * lg.
  const PartView pv = part_view(a.ws, static_cast<int64_t>(a.B) * a.Hk * parts * cols, D);
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    if (n) __syncthreads();
    const float ln = sum_groups(l[n]);
    float* mine = red_o + (wave * 16 + li) * (D + 4) + kDV * 4 * lg;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < kDV; j += 4)
        *reinterpret_cast<f32x4*>(mine + r * kDV + j) = f32x4{o[n][j][r], o[n][j + 1][r], o[n][j + 2][r], o[n][j + 3][r]};
    if (lg == 0) red_m[wave * 16 + li] = m[n], red_l[wave * 16 + li] = ln;
    __syncthreads();
    // thread -> (column, D / 16 values)
    const int c = threadIdx.x / 16, d0 = (threadIdx.x % 16) * kDV;
    const int col = (cb * NG + n) * 16 + c;
    if (col >= cols) continue;
    float top = red_m[c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, red_m[w * 16 + c]);
    const float base = top == kNegInf ? 0.0f : top;
    float sum = 0.0f, acc[kDV];
#pragma unroll
    for (int j = 0; j < kDV; ++j) acc[j] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(red_m[w * 16 + c] - base);
      sum += f * red_l[w * 16 + c];
#pragma unroll
      for (int j = 0; j < kDV; ++j) acc[j] += f * red_o[(w * 16 + c) * (D + 4) + d0 + j];
    }
    if (direct) {
      const int tq = col / G;
      const int64_t row = (static_cast<int64_t>(b) * a.Tq + tq) * a.Hq + hk * G + (col - tq * G);
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      uint32_t y[kDV / 2];
#pragma unroll
      for (int j = 0; j < kDV / 2; ++j) y[j] = pack_bf16(acc[2 * j] * inv, acc[2 * j + 1] * inv);
      uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + row * D + d0);
#pragma unroll
      for (int j = 0; j < kDV / 2; ++j) dst[j] = y[j];
      if (a.lse != nullptr && d0 == 0) a.lse[row] = sum == 0.0f ? kNegInf : (top + __builtin_log2f(sum)) * 0.69314718055994530942f;
    } else {
      const int64_t row = ((static_cast<int64_t>(b) * a.Hk + hk) * parts + part) * cols + col;
#pragma unroll
      for (int j = 0; j < kDV; j += 4)
        *reinterpret_cast<f32x4*>(pv.o + row * D + d0 + j) = f32x4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
      if (d0 == 0) *reinterpret_cast<float2*>(pv.ml + 2 * row) = make_float2(top, sum);
    }
  }
}

// Joins the parts of each query column: a block per column, D / 4 lanes of
// four values, the rest of its 256 threads over the parts.
template <int D>
__global__ __launch_bounds__(256) void paged_attention_join_kernel(const AttnArgs a, int chunk, int parts) {
  constexpr int kLanes = D / 4, kSets = 256 / kLanes;
  __shared__ f32x4 red[kSets * kLanes];
  __shared__ float red_s[kSets];
  const int G = a.Hq / a.Hk, cols = a.Tq * G;
  int id = blockIdx.x;
  const int col = id % cols;
  id /= cols;
  const int hk = id % a.Hk, b = id / a.Hk;
  const int len = min(a.lens[b], a.max_len);
  const int live = len > 0 ? (len + chunk - 1) / chunk : 0;
  const PartView pv = part_view(a.ws, static_cast<int64_t>(a.B) * a.Hk * parts * cols, D);
  const int64_t row0 = (static_cast<int64_t>(b) * a.Hk + hk) * parts * cols + col;
  const int set = threadIdx.x / kLanes, ln = threadIdx.x % kLanes;

  float top = kNegInf;
  for (int i = 0; i < live; ++i) top = fmaxf(top, pv.ml[2 * (row0 + static_cast<int64_t>(i) * cols)]);
  const float base = top == kNegInf ? 0.0f : top;
  f32x4 acc = {0, 0, 0, 0};
  float sum = 0.0f;
  for (int i = set; i < live; i += kSets) {
    const int64_t row = row0 + static_cast<int64_t>(i) * cols;
    const float2 ml = *reinterpret_cast<const float2*>(pv.ml + 2 * row);
    const float f = __builtin_amdgcn_exp2f(ml.x - base);
    sum += f * ml.y;
    acc += f * *reinterpret_cast<const f32x4*>(pv.o + row * D + 4 * ln);
  }
  red[threadIdx.x] = acc;
  if (ln == 0) red_s[set] = sum;
  __syncthreads();
  if (set) return;
  sum = red_s[0];
  for (int s = 1; s < kSets; ++s) {
    acc += red[s * kLanes + ln];
    sum += red_s[s];
  }
  const int tq = col / G;
  const int64_t row = (static_cast<int64_t>(b) * a.Tq + tq) * a.Hq + hk * G + (col - tq * G);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<u32x2*>(a.out + row * D + 4 * ln) = u32x2{pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)};
  if (a.lse != nullptr && ln == 0) a.lse[row] = sum == 0.0f ? kNegInf : (top + __builtin_log2f(sum)) * 0.69314718055994530942f;
}

template <int D, bool FP8, int NG, int WPS>
hipError_t launch_ng(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const int cols = a.Tq * (a.Hq / a.Hk);
  const int col_blocks = (cols + 16 * NG - 1) / (16 * NG);
  const int64_t blocks = static_cast<int64_t>(a.B) * a.Hk * p.parts * col_blocks;
  hipLaunchKernelGGL((paged_attention_kernel<D, FP8, NG, WPS>), dim3(static_cast<unsigned>(blocks)), dim3(64 * kWaves), 0,
                     st, a, p.chunk, p.parts, col_blocks);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  const int64_t rows = static_cast<int64_t>(a.B) * a.Hk * cols;
  hipLaunchKernelGGL((paged_attention_join_kernel<D>), dim3(static_cast<unsigned>(rows)), dim3(256), 0, st, a, p.chunk,
                     p.parts);
  return hipGetLastError();
}

template <int D, bool FP8>
hipError_t launch_d(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  constexpr int kWps = D == 256 ? 1 : 2;
  switch (p.cols) {
    case 16: return launch_ng<D, FP8, 1, kWps>(a, p, st);
    case 32: return launch_ng<D, FP8, 2, kWps>(a, p, st);
    default: return launch_ng<D, FP8, D == 256 ? 2 : 4, 1>(a, p, st);
  }
}

}  // namespace

AttnPlan attention_plan(int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D, int64_t max_len) {
  const int64_t cols = Tq * (Hq / Hk);
  AttnPlan p;
  p.cols = cols <= 16 ? 16 : cols <= 32 || D == 256 ? 32 : 64;
  const int64_t heads = B * Hk * ((cols + p.cols - 1) / p.cols);
  constexpr int64_t kStep = kWaves * kTile;  // a block's tokens per round
  constexpr int64_t kBlocks = 1024;          // four blocks for each CU
  const int64_t most = (max_len + kStep - 1) / kStep;
  const int64_t want = std::max<int64_t>(1, std::min(most, (kBlocks + heads - 1) / heads));
  const int64_t steps = (most + want - 1) / want;  // of a part
  p.chunk = static_cast<int>(steps * kStep);
  p.parts = static_cast<int>((most + steps - 1) / steps);
  return p;
}

hipError_t launch_paged_attention(const AttnArgs& a, hipStream_t st) {
  const AttnPlan p = attention_plan(a.B, a.Tq, a.Hq, a.Hk, a.D, a.max_len);
  if (a.fp8) {
    switch (a.D) {
      case 64: return launch_d<64, true>(a, p, st);
      case 128: return launch_d<128, true>(a, p, st);
      default: return launch_d<256, true>(a, p, st);
    }
  }
  switch (a.D) {
    case 64: return launch_d<64, false>(a, p, st);
    case 128: return launch_d<128, false>(a, p, st);
    default: return launch_d<256, false>(a, p, st);
  }
}

}  // namespace jq
