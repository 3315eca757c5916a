// Attention of many new tokens for gfx950: packed prompts of different lengths
// over their own keys and values, or chunks of new tokens, packed too, over a
// paged cache.
//
//   p = softmax over visible t of scale * (q . k_t),  o = sum_t p_t v_t
//   visible: t < n_k, and for causal calls t <= n_k - n_q + i for new token i.
//   A query that sees nothing gives zeros (and lse = -inf).
//
// Two products of 2 D operations for each query and key that it sees, so the
// matrix cores bound it where there are many columns (new tokens times the
// heads that share a key head).
//  * S^T = K Q^T and O^T = V^T P^T on 32x32x16 MFMAs.  With S transposed a lane
//    holds a column's scores, which are, packed, the column's operand of the
//    second product for the same keys: a product may take its k in any order, so
//    V is read in that one (transposed out of LDS, 4 keys x 16 values at a time).
//    P never leaves its registers; maximum, sum and rescaling are per lane.
//  * A block has four waves of 32 columns and takes 64 keys a step; transfers
//    bring the next step's rows into the other half of LDS meanwhile.  Two blocks
//    a CU.  Waves of 64 columns, which read LDS half as often, need a SIMD each:
//    955 TFLOP/s at 8192 tokens, 32 heads of 128; with the next step's scores
//    between this one's exponentials and products 1074; two waves a SIMD 1088.
//    At D = 64 two of 64 columns fit a SIMD.
//  * Tiles of columns are found on the device from the starts, so a call needs no
//    lengths on the host; heads run fastest, so that blocks with the same keys
//    share an XCD's cache.
//  * With few blocks the key axis is cut into parts, whose sums go to the
//    workspace and a second kernel joins.
// Scores, statistics and sums are fp32.  The weights take part in their product
// as one bf16 each, half of a step relative: outputs are 0.0023 (rms) from 64
// bits where their own rounding is 0.0017.  Both parts of a weight, as for few
// columns, would be half as many products again.
//
// What bounds it: a step's 32 MFMAs of a wave take 1024 cycles, its 117 vector
// instructions and 32 exponentials 725, and two waves' step takes 3570 for the 3500
// that these sum to, so the two kinds hardly overlap: the matrix cores are busy for
// 57% of a step, and by the counters for 51 to 57% of whole calls, at 1.75 to 1.9
// GHz.  (One wave a SIMD, which issues less, clocked at 2.3 GHz and took as long,
// and a fifth of the vector instructions taken out gave 1 to 2%, which points to
// power; the power itself was not read.)  A large library product runs at 1450
// TFLOP/s on this card.  4608 tokens, 24 heads of 128, all of them seen: 271 to 280
// us from card to card, 930 to 960 TFLOP/s (864 equal blocks for 512 places); 8192
// causal, 32 on 8 heads: 509, 1080; 2048 over 32768 cached: 965 to 1024, 1050 to
// 1110, and from e4m3 1160 to 1180 us, whose scales and widening are 130 more
// instructions a step.  Three prompts of up to 77 tokens: 6.0 us, a launch and two
// steps' chain; 16 tokens over 2080: 12.6, two launches.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "block_common.h"
#include "block_internal.h"

namespace jq {

namespace {

using namespace block_detail;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(4))) int32_t* uniform_i32;
typedef __attribute__((address_space(3))) bf16x4* lds_bf16x4;

constexpr float kNegInf = -__builtin_inff();
constexpr int kThreads = 256;

__device__ __forceinline__ float max_halves(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// What a product is multiplied with to be a power of two; 0 as next to nothing,
// for the masked ones' sake.
__device__ __forceinline__ float power_scale(float scale) {
  return scale == 0.0f ? 0x1p-126f : fabsf(scale) * 1.44269504088896340736f;
}
__device__ __forceinline__ float log_sum(float m, float l) {
  return l == 0.0f ? kNegInf : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

// A block's place: a sequence, its rows in the packed tensors, its tile of
// columns, and its keys.
struct Place {
  int seq, row0, rows, tile;
  int key0, keys;  // rows of its own keys, or cached tokens
};

// The rows of sequence b.  Starts outside [0, T] are brought into it, so
// whatever they are, the rows lie in the tensors.
__device__ __forceinline__ void rows_of(const int32_t* starts, int64_t T, int b, int* row0, int* rows) {
  const int t = static_cast<int>(T);
  const int s0 = min(max(starts[b], 0), t), s1 = min(max(starts[b + 1], 0), t);
  *row0 = s0;
  *rows = max(s1 - s0, 0);
}

// The place of the `index`-th of `tiles` tiles of `per` columns, counted from the
// last one of the last sequence, so that the longest of a causal sequence come
// first; seq = -1 where there are fewer.  All lanes of a wave take part.
template <bool PAGED>
__device__ __forceinline__ Place find_tile(const PromptArgs& a, int G, int per, int index, int tiles) {
  const int lane = threadIdx.x & 63;
  const int shift = __builtin_ctz(per);
  const bool many = a.B > 64;
  int first = 0;  // of 64 sequences, a lane each
  int slot = tiles - 1 - index;
  if (many) {
    // Sequence b has the places from starts[b] G / per + min(b, starts[b]) on, as
    // many as it needs or more, so a search finds it (4096 sequences of one token
    // over up to 64, 8 key heads: 350 us, by a walk along all sequences 960).
    static_assert(kPromptMaxSequences <= 64 * 4096);
    for (int step = a.B > 4096 ? 4096 : 64; step > 1; step /= 64) {
      const int b = first + lane * step;
      const int start = b < a.B ? min(max(a.starts[b], 0), static_cast<int>(a.T)) : 0;
      const int from = b < a.B ? (start * G >> shift) + min(b, start) : slot + 1;
      const uint64_t hit = __ballot(from <= slot);
      if (hit == 0) break;  // and below
      first += (63 - __builtin_clzll(hit)) * step;
    }
  }
  // a lane's sequence; its keys are asked for with the rows, not after them
  const int b = first + lane;
  int row0 = 0, rows = 0, key0 = 0, keys = 0;
  if (b < a.B) {
    rows_of(a.starts, a.T, b, &row0, &rows);
    if constexpr (PAGED) keys = min(max(a.lens[b], 0), a.max_len);
    else rows_of(a.k_starts, a.Tk, b, &key0, &keys);
  }
  const int n = (rows * G + per - 1) >> shift;
  int tile, l;
  if (many) {
    tile = slot - ((row0 * G >> shift) + min(b, row0));
    const uint64_t hit = __ballot(b < a.B && tile >= 0);
    l = hit == 0 ? 0 : 63 - __builtin_clzll(hit);
  } else {
    // fewer tiles than places where sequences are empty or fill their last
    // tile, so without gaps: the sum over the sequences behind
    int upto = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int v = __shfl_down(upto, d, 64);
      upto += lane + d < 64 ? v : 0;
    }
    tile = upto - 1 - index;
    const uint64_t hit = __ballot(tile >= 0 && tile < n);
    l = hit == 0 ? 0 : __builtin_ctzll(hit);
  }
  Place p;
  p.tile = __builtin_amdgcn_readlane(tile, l);
  p.seq = p.tile >= 0 && p.tile < __builtin_amdgcn_readlane(n, l) ? first + l : -1;
  p.row0 = __builtin_amdgcn_readlane(row0, l);
  p.rows = __builtin_amdgcn_readlane(rows, l);
  p.key0 = __builtin_amdgcn_readlane(key0, l);
  p.keys = __builtin_amdgcn_readlane(keys, l);
  return p;
}

// Which 16-byte chunk of a row in LDS holds chunk c.  Keys are read a row a
// lane, 16 bytes each; values transposed, 64 bytes of each of eight rows: both
// touch every bank evenly this way.
template <int D>
__device__ __forceinline__ int key_slot(int row, int c) {
  constexpr int kMask = D / 8 < 16 ? D / 8 - 1 : 15;
  return c ^ (row & kMask);
}
template <int D>
__device__ __forceinline__ int value_slot(int row, int c) {
  return D == 64 ? c ^ ((row >> 1 & 1) << 2) : c ^ ((row & 3) << 2);
}

template <int D, int QG, PromptKv KV>
struct Sizes {
  static constexpr int kKeys = 64;                  // keys of a step
  static constexpr int kRow = 2 * D;                // bytes of a row in LDS
  static constexpr int kHalf = kKeys * kRow;        // a step's keys, or its values
  static constexpr int kStage = 2 * kHalf + (KV == PromptKv::kPagedFp8 ? 8 * kKeys : 0);
  static constexpr int kLane = QG * (D / 2 + 2);    // floats of a lane's result: outputs, maxima, sums
  static constexpr int kJoin = 2 * 64 * 4 * kLane;  // two waves' results, where halves of the keys are joined
  static constexpr int kLds = 2 * kStage > kJoin ? 2 * kStage : kJoin;
  static constexpr int kPerSimd = D <= 128 ? 2 : 1;
  // Two steps at a time, with their buffers at constant places, where registers
  // allow (8192 tokens, 32 heads of 128: 1050 -> 1036 us; 4096, 16 heads of 256,
  // causal: 198 -> 187).
  static constexpr bool kUnroll = QG == 1 && !(D == 256 && KV == PromptKv::kPagedFp8);
};

// The place of a key's (or value's) row: its first element, and the index of its scale.
template <int D, PromptKv KV>
__device__ __forceinline__ int64_t row_place(const PromptArgs& a, int seq, int hk, int key0, int t, int64_t stride,
                                             int64_t* line) {
  if constexpr (KV == PromptKv::kDense) {
    return static_cast<int64_t>(key0 + t) * stride + static_cast<int64_t>(hk) * D;
  } else {
    const uint32_t pg = static_cast<uint32_t>(a.table[static_cast<int64_t>(seq) * a.table_cols + (t >> a.page_shift)]);
    const int64_t page = pg < static_cast<uint32_t>(a.num_pages) ? pg : 0;
    *line = ((page * a.Hk + hk) << a.page_shift) + (t & ((1 << a.page_shift) - 1));
    return *line * D;
  }
}
// Elements i .. i + 7 of a row, and one of them, as bf16.
template <PromptKv KV>
__device__ __forceinline__ u32x4 eight_of(const void* p, int64_t i) {
  if constexpr (KV == PromptKv::kPagedFp8) {
    const u32x2 u = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(p) + i);
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      w[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[j], 1.0f, false));
      w[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u[j], 1.0f, true));
    }
    return w;
  } else {
    return *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i);
  }
}
template <PromptKv KV>
__device__ __forceinline__ uint32_t one_of(const void* p, int64_t i) {
  if constexpr (KV == PromptKv::kPagedFp8) {
    const uint32_t u = static_cast<const uint8_t*>(p)[i];
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, false)) & 0xFFFFu;
  } else {
    return static_cast<const uint16_t*>(p)[i];
  }
}
__device__ __forceinline__ bool odd_bf16(uint32_t u) { return (u & 0x7F80u) == 0x7F80u; }

// Calls f(t) for the tokens [t0, t1) that have an infinity or NaN among their
// values, until it returns false; for one wave, eight values a lane.
template <int D, PromptKv KV, class F>
__device__ __forceinline__ void for_odd_values(const PromptArgs& a, int seq, int hk, int key0, int t0, int t1, F f) {
  constexpr int kPieces = D / 8, kRows = 64 / kPieces;
  const int lane = threadIdx.x & 63;
  for (int t = t0; t < t1; t += kRows) {
    bool odd = false;
    if (t + lane / kPieces < t1) {
      int64_t line;
      const int64_t at = row_place<D, KV>(a, seq, hk, key0, t + lane / kPieces, a.v_stride, &line);
      const u32x4 w = eight_of<KV>(a.v, at + 8 * (lane % kPieces));
#pragma unroll
      for (int j = 0; j < 4; ++j) odd |= odd_bf16(w[j]) || odd_bf16(w[j] >> 16);
    }
    const uint64_t hit = __ballot(odd);
#pragma unroll 1
    for (int r = 0; r < kRows; ++r)
      if ((hit >> (r * kPieces) & ((1ull << kPieces) - 1)) != 0 && !f(t + r)) return;
  }
}

// A wave's 32 columns over the keys [t0, t1), straight from memory: for columns
// beside which a product met an infinity or NaN among the values of tokens that
// only some of them see, which such a value's weight of 0 does not take away.
// Values of the tokens from `all` on, which some columns do not see, are read as
// 0 where they are not finite, and those tokens are put in afterwards, for the
// columns that see them.  Nothing of the fast path is alive here, so it costs
// that path no registers (masks inside its product took 70 more).
//
// Bound by the latency of its loads, 4 us for 32 keys: 2048 tokens over 32768
// with all new tokens' values NaN take 6.3 ms instead of 1.0, 512 over 2048 91
// us instead of 24 (one column after the other, a key a lane: 3700).
template <int D, PromptKv KV>
__device__ __forceinline__ void wave_columns(const PromptArgs& a, int seq, int hk, int key0, int t0, int t1, int all,
                                             const uint16_t* q_row, int lim, f32x16* o, float* m, float* l) {
  constexpr bool kFp8 = KV == PromptKv::kPagedFp8;
  constexpr int kSteps = D / 16, kOut = D / 32;
  const int li = threadIdx.x & 31, lh = threadIdx.x >> 5 & 1;
  auto place = [&](int t, int64_t stride, int64_t* line) { return row_place<D, KV>(a, seq, hk, key0, t, stride, line); };
  const float scale2 = power_scale(a.scale);
  const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
  lim = min(lim, t1);
#pragma unroll
  for (int n = 0; n < kOut; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = 0.0f;
  float top = kNegInf, sum = 0.0f;
#pragma unroll 1
  for (int t = t0; t < t1; t += 32) {
    int64_t line = 0;
    const int64_t k_row = place(min(t + li, t1 - 1), a.k_stride, &line);
    float k_scale = 1.0f, v_scale = 1.0f;  // of key li
    if constexpr (kFp8) k_scale = a.k_scale[line], v_scale = a.v_scale[line];
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(q_row + 16 * c) ^ flip;
      const bf16x8 k = __builtin_bit_cast(bf16x8, eight_of<KV>(a.k, k_row + 16 * c + 8 * lh));
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, __builtin_bit_cast(bf16x8, x), s, 0, 0, 0);
    }
    float next = top;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = 8 * (i / 4) + 4 * lh + i % 4;
      if constexpr (kFp8) s[i] *= __shfl(k_scale, j, 64);
      s[i] = t + j < lim ? s[i] * scale2 : kNegInf;
      next = fmaxf(next, s[i]);
    }
    next = max_halves(next);
    const float base = next == kNegInf ? 0.0f : next, keep = __builtin_amdgcn_exp2f(top - base);
    top = next;
    sum *= keep;
#pragma unroll
    for (int n = 0; n < kOut; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[n][i] *= keep;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - base);
      sum += s[i];
      if constexpr (kFp8) {
        const int j = 8 * (i / 4) + 4 * lh + i % 4;
        const float f = __shfl(v_scale, j, 64);
        s[i] = t + j < lim ? s[i] * f : 0.0f;
      }
    }
#pragma unroll
    for (int k16 = 0; k16 < 2; ++k16) {
      // sixteen keys from a multiple of sixteen on lie in one page
      const int first = min(t + 16 * k16, t1 - 1), stride = KV == PromptKv::kDense ? static_cast<int>(a.v_stride) : D;
      const int64_t at = place(first, a.v_stride, &line) + li;
      float e[8];
      int off[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        e[j] = s[8 * k16 + j];
        off[j] = min(8 * (j / 4) + 4 * lh + j % 4, t1 - 1 - first) * stride;
      }
      const bf16x8 p = __builtin_bit_cast(bf16x8, pack8_bf16(e));
#pragma unroll
      for (int n = 0; n < kOut; ++n) {
        __builtin_amdgcn_sched_barrier(0);  // eight loads at a time: registers are short
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = one_of<KV>(a.v, at + off[j] + 32 * n);
          if (odd_bf16(x[j]) && t + 16 * k16 + 8 * (j / 4) + 4 * lh + j % 4 >= all) x[j] = 0;
        }
        const u32x4 v = {x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16};
        o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), p, o[n], 0, 0, 0);
      }
    }
  }
  *m = top, *l = sum_halves(sum);
  for_odd_values<D, KV>(a, seq, hk, key0, max(all, t0), t1, [&](int t) {
    int64_t line = 0;
    const int64_t k_row = place(t, a.k_stride, &line) + 8 * lh, v_row = place(t, a.v_stride, &line) + 4 * lh;
    float dot = 0.0f;
#pragma unroll 1
    for (int c = 0; c < kSteps; ++c) {
      float x[8], k[8];
      unpack8_bf16(*reinterpret_cast<const u32x4*>(q_row + 16 * c) ^ flip, x);
      unpack8_bf16(eight_of<KV>(a.k, k_row + 16 * c), k);
#pragma unroll
      for (int j = 0; j < 8; ++j) dot = fmaf(x[j], k[j], dot);
    }
    dot = sum_halves(dot);
    if constexpr (kFp8) dot *= a.k_scale[line];
    float w = __builtin_amdgcn_exp2f(dot * scale2 - (top == kNegInf ? 0.0f : top));
    if constexpr (kFp8) w *= a.v_scale[line];
    if (t < lim) {
#pragma unroll
      for (int n = 0; n < kOut; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t v = one_of<KV>(a.v, v_row + 32 * n + 8 * (i / 4) + i % 4);
          if (odd_bf16(v)) o[n][i] = fmaf(w, bf_lo(v), o[n][i]);
        }
    }
    return true;
  });
}

template <int D, int QG, PromptKv KV>
__global__ __launch_bounds__(kThreads, (Sizes<D, QG, KV>::kPerSimd)) void prompt_attention_kernel(
    const PromptArgs a, int tiles, int per, int parts, int least) {
  using Z = Sizes<D, QG, KV>;
  constexpr bool kFp8 = KV == PromptKv::kPagedFp8, kPaged = KV != PromptKv::kDense;
  constexpr int kKeys = Z::kKeys, kSteps = D / 16, kOut = D / 32, kWaveRows = kKeys / 4;
  constexpr int kBytes = kFp8 ? 1 : 2;                 // of a cached value
  constexpr int kPerRow = D * kBytes / 16;             // 16-byte pieces of a cached row
  constexpr int kLoads = kWaveRows * kPerRow / 64;     // transfers of a wave for a step's keys (and its values)
  __shared__ __attribute__((aligned(16))) uint8_t lds[Z::kLds];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 31, lh = lane >> 5;
  const int G = a.Hq / a.Hk;
  const int hk = blockIdx.x % a.Hk, rest = blockIdx.x / a.Hk;
  const int part = rest / tiles;
  const int index = rest % tiles;
  const Place at = find_tile<kPaged>(a, G, per, index, tiles);
  if (at.seq < 0) return;

  const int key0 = at.key0, nk = at.keys;
  const int cols = at.rows * G, col0 = at.tile * per, last_col = min(col0 + per, cols) - 1;
  // A wave has 32 QG columns; where two waves have all of the tile's, the other
  // two have the same ones, and each pair takes half of every step's keys.
  const bool halves = last_col - col0 < 64 * QG;
  const int wcol = col0 + (halves ? wave & 1 : wave) * 32 * QG;
  const bool busy = wcol < cols;
  auto limit = [&](int col) { return a.causal ? min(max(nk - at.rows + col / G + 1, 0), nk) : nk; };
  const int block_end = limit(last_col);
  const int wave_end = limit(min(wcol + 32 * QG, cols) - 1), wave_all = limit(min(wcol, cols - 1));
  // Its part of the keys: every sequence is cut by its own length, so the bound
  // that the host knows decides only how many parts there may be.  The bounds go
  // to scalar registers by hand: left to itself the compiler works out a step's
  // rows in vector ones (2048 tokens over 32768, in turn on one card: 983 us
  // instead of 965).
  const int chunk = parts == 1 ? nk : max(((nk - 1) / parts / 64 + 1) * 64, least);
  const int t_begin = __builtin_amdgcn_readfirstlane(min(static_cast<int64_t>(part) * chunk, static_cast<int64_t>(block_end)));
  const int t_end = __builtin_amdgcn_readfirstlane(min(block_end - t_begin, chunk) + t_begin);
  const int steps = (t_end - t_begin + kKeys - 1) / kKeys;

  // queries
  int row[QG], lim[QG];
  bf16x8 q[QG][kSteps];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    const int col = min(wcol + 32 * g + li, cols - 1), token = col / G, head = hk * G + col - token * G;
    lim[g] = limit(col);
    row[g] = (at.row0 + token) * a.Hq + head;
    const uint16_t* src = a.q + static_cast<int64_t>(at.row0 + token) * a.q_stride + static_cast<int64_t>(head) * D + 8 * lh;
#pragma unroll
    for (int c = 0; c < kSteps; ++c) {
      u32x4 v = *reinterpret_cast<const u32x4*>(src + 16 * c);
      if (a.scale < 0.0f) v ^= 0x80008000u;  // so that scores grow with their products
      q[g][c] = __builtin_bit_cast(bf16x8, v);
    }
  }
  f32x16 o[kOut][QG];
  float m[QG], l[QG];
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    m[g] = kNegInf, l[g] = 0.0f;
#pragma unroll
    for (int t = 0; t < kOut; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][g][i] = 0.0f;
  }
  const float scale2 = power_scale(a.scale);

  // Transfers: wave w brings rows [w kWaveRows, (w + 1) kWaveRows) of a step.
  const uint32_t lds0 = lds_addr(lds);
  const int64_t k_row_bytes = kPaged ? D * kBytes : a.k_stride * 2, v_row_bytes = kPaged ? D * kBytes : a.v_stride * 2;
  uint32_t k_off[kLoads], v_off[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int r = i * (64 / kPerRow) + lane / kPerRow, c = lane % kPerRow, rr = wave * kWaveRows + r;
    if constexpr (kFp8) {
      k_off[i] = v_off[i] = r * D + 16 * c;
    } else {
      k_off[i] = static_cast<uint32_t>(r * k_row_bytes) + 16 * key_slot<D>(rr, c);
      v_off[i] = static_cast<uint32_t>(r * v_row_bytes) + 16 * value_slot<D>(rr, c);
    }
  }
  const uniform_i32 table = (uniform_i32)(a.table + static_cast<int64_t>(at.seq) * a.table_cols);
  bool bad = false;
  auto page_of = [&](int t) __attribute__((always_inline)) { return t < t_end ? table[t >> a.page_shift] : 0; };
  int page_next = 0;
  if constexpr (kPaged) page_next = page_of(t_begin + wave * kWaveRows);
  struct Src {
    const uint8_t *k, *v;
    int64_t line;  // paged: index of the first row
    int rows;
  };
  auto source = [&](int t0) __attribute__((always_inline)) {
    Src s;
    const int t = t0 + wave * kWaveRows;
    s.rows = min(max(t_end - t, 0), kWaveRows);
    s.line = 0;
    if constexpr (kPaged) {
      int pg = page_next;
      page_next = page_of(t + kKeys);
      if (s.rows > 0 && static_cast<uint32_t>(pg) >= static_cast<uint32_t>(a.num_pages)) bad = true, s.rows = 0;
      if (s.rows == 0) pg = 0;
      s.line = ((static_cast<int64_t>(pg) * a.Hk + hk) << a.page_shift) + (s.rows ? t & ((1 << a.page_shift) - 1) : 0);
      s.k = static_cast<const uint8_t*>(a.k) + s.line * (D * kBytes);
      s.v = static_cast<const uint8_t*>(a.v) + s.line * (D * kBytes);
    } else {
      const int64_t r = key0 + (s.rows ? t : 0);
      s.k = static_cast<const uint8_t*>(a.k) + r * k_row_bytes + static_cast<int64_t>(hk) * D * 2;
      s.v = static_cast<const uint8_t*>(a.v) + r * v_row_bytes + static_cast<int64_t>(hk) * D * 2;
    }
    return s;
  };
  auto span = [&](const Src& s, int64_t row_bytes) __attribute__((always_inline)) {
    return s.rows == 0 ? 0 : static_cast<int>((s.rows - 1) * row_bytes + D * kBytes);
  };
  // bf16: straight into LDS
  auto issue = [&](int buf, int t0) __attribute__((always_inline)) {
    const Src s = source(t0);
    const Rsrc rk = make_rsrc(s.k, span(s, k_row_bytes)), rv = make_rsrc(s.v, span(s, v_row_bytes));
    const uint32_t dst = lds0 + buf * Z::kStage + wave * kWaveRows * Z::kRow;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) dma16(rk, dst + 1024 * i, k_off[i], 0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) dma16(rv, dst + Z::kHalf + 1024 * i, v_off[i], 0);
  };
  // e4m3: through registers, widened to bf16 (exactly) on the way.  At D = 256,
  // where registers are short, keys and values have the same ones in turn: keys
  // are put after a step's scores, values after its sums, each asked for half a
  // step before (2048 tokens over 16384, 16 heads of 256: 681 us; with both at
  // once, and 65 registers in memory, 1192; at D = 128 that way 1199 instead of
  // 1170 for 2048 over 32768, and 154 instead of 145 for a ragged batch).
  constexpr bool kTurns = kFp8 && D == 256;
  u32x4 kr[kFp8 ? kLoads : 1], vr[kFp8 && !kTurns ? kLoads : 1];
  float sr = 0.0f;
  Src held{};
  auto load_rows = [&](u32x4* r, const uint8_t* p) __attribute__((always_inline)) {
    if constexpr (kFp8) {
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, span(held, D), kRawBuffer);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) r[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, k_off[i], 0, 0));
    }
  };
  auto fetch = [&](int t0) __attribute__((always_inline)) {
    if constexpr (kFp8) {
      held = source(t0);
      load_rows(kr, held.k);
      if constexpr (!kTurns) load_rows(vr, held.v);
      // lanes 0 .. 31 a scale of a key each, 32 .. 63 of a value
      sr = li < held.rows ? (lh ? a.v_scale : a.k_scale)[held.line + li] : 0.0f;
    }
  };
  auto put_rows = [&](int buf, const u32x4* r, bool values) __attribute__((always_inline)) {
    if constexpr (kFp8) {
      uint8_t* base = lds + buf * Z::kStage;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int rr = wave * kWaveRows + i * (64 / kPerRow) + lane / kPerRow, c = 2 * (lane % kPerRow);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 w;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            w[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r[i][2 * h + j], 1.0f, false));
            w[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r[i][2 * h + j], 1.0f, true));
          }
          uint8_t* dst = base + rr * Z::kRow + (values ? Z::kHalf + 16 * value_slot<D>(rr, c + h) : 16 * key_slot<D>(rr, c + h));
          *reinterpret_cast<u32x4*>(dst) = w;
        }
      }
    }
  };
  auto put_keys = [&](int buf) __attribute__((always_inline)) {
    if constexpr (kFp8) {
      put_rows(buf, kr, false);
      if (li < kWaveRows)
        *reinterpret_cast<float*>(lds + buf * Z::kStage + 2 * Z::kHalf + 4 * (lh * kKeys + wave * kWaveRows + li)) = sr;
    }
  };
  // what is between step i's scores and its sums, and after them, at D = 256
  auto keys_turn = [&](int i) __attribute__((always_inline)) {
    if constexpr (kTurns) {
      if (i + 1 >= steps) return;
      put_keys((i + 1) & 1);
      load_rows(kr, held.v);
    }
  };
  auto values_turn = [&](int i) __attribute__((always_inline)) {
    if constexpr (kTurns) {
      if (i + 1 >= steps) return;
      put_rows((i + 1) & 1, kr, true);
      if (i + 2 < steps) fetch(t_begin + (i + 2) * kKeys);
    }
  };

  // Where a lane reads: key rows li (+ 32), 16-byte chunk 2 step + lh; of the
  // values, for the transposing read, four rows 4 lh + li / 4 % 4 of 16 and of
  // these the 8 bytes li % 4 of the 16 columns li / 16.
  uint32_t k_at[kSteps], v_at[kOut];
#pragma unroll
  for (int c = 0; c < kSteps; ++c) k_at[c] = li * Z::kRow + 16 * key_slot<D>(li, 2 * c + lh);
#pragma unroll
  for (int t = 0; t < kOut; ++t) {
    const int r = 4 * lh + (lane & 15) / 4;
    v_at[t] = Z::kHalf + r * Z::kRow + 16 * value_slot<D>(r, 4 * t + 2 * (li / 16) + (lane & 3) / 2) + 8 * (lane & 1);
  }
  auto value_frag = [&](const uint8_t* base, int t, int k16) __attribute__((always_inline)) {
    const uint8_t* p = base + v_at[t] + k16 * 16 * Z::kRow;
    const bf16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(p));
    const bf16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(p + 8 * Z::kRow));
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  // The keys t0 .. of a stage: all of them, or half `part` of them.
  auto step = [&](const uint8_t* stage, int t0, int index, int part, auto count, auto mask) __attribute__((always_inline)) {
    constexpr int kSub = decltype(count)::value;
    constexpr bool kMask = decltype(mask)::value;
    const uint8_t* base = stage + part * 32 * Z::kRow;
    const float* scales = reinterpret_cast<const float*>(stage + 2 * Z::kHalf) + 32 * part;
    t0 += 32 * part;
    f32x16 s[kSub][QG];
#pragma unroll
    for (int n = 0; n < kSub; ++n) {
#pragma unroll
      for (int g = 0; g < QG; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][g][i] = 0.0f;
#pragma unroll
      for (int c = 0; c < kSteps; ++c) {
        const bf16x8 k = *reinterpret_cast<const bf16x8*>(base + k_at[c] + n * 32 * Z::kRow);
#pragma unroll
        for (int g = 0; g < QG; ++g) s[n][g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[g][c], s[n][g], 0, 0, 0);
      }
    }
    keys_turn(index);
    if constexpr (kFp8) {
#pragma unroll
      for (int n = 0; n < kSub; ++n)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f32x4 f = *reinterpret_cast<const f32x4*>(scales + 32 * n + 2 * i + 4 * lh);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int g = 0; g < QG; ++g) s[n][g][i + j] *= f[j];
        }
    }
    if constexpr (kMask) {
#pragma unroll
      for (int g = 0; g < QG; ++g) {
        const int rel = lim[g] - t0 - 4 * lh;
#pragma unroll
        for (int n = 0; n < kSub; ++n)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (32 * n + 8 * (i / 4) + i % 4 >= rel) s[n][g][i] = kNegInf;
      }
    }
    bf16x8 p[2 * kSub][QG];
#pragma unroll
    for (int g = 0; g < QG; ++g) {
      float top = s[0][g][0];
#pragma unroll
      for (int n = 0; n < kSub; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][g][i]);
      top = max_halves(top) * scale2;
      // the maximum follows only when left more than 2^8 behind: weights stay
      // below that, and fp32 sums of them are as exact
      const bool more = top > m[g] + 8.0f;
      if (__any(more)) {
        const float keep = more ? __builtin_amdgcn_exp2f(m[g] - top) : 1.0f;
        m[g] = more ? top : m[g];
        l[g] *= keep;
#pragma unroll
        for (int t = 0; t < kOut; ++t) {
#pragma unroll
          for (int i = 0; i < 16; ++i) o[t][g][i] *= keep;
        }
      }
      const float base_m = m[g] == kNegInf ? 0.0f : m[g];
#pragma unroll
      for (int n = 0; n < kSub; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[n][g][i], scale2, -base_m));
          l[g] += e;
          s[n][g][i] = e;
        }
    }
    if constexpr (kFp8) {
#pragma unroll
      for (int n = 0; n < kSub; ++n)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f32x4 f = *reinterpret_cast<const f32x4*>(scales + kKeys + 32 * n + 2 * i + 4 * lh);
#pragma unroll
          for (int g = 0; g < QG; ++g) {
            const int rel = kMask ? lim[g] - t0 - 4 * lh : kKeys;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              s[n][g][i + j] = 32 * n + 2 * i + j < rel ? s[n][g][i + j] * f[j] : 0.0f;
          }
        }
    }
#pragma unroll
    for (int k16 = 0; k16 < 2 * kSub; ++k16)
#pragma unroll
      for (int g = 0; g < QG; ++g) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = s[k16 / 2][g][8 * (k16 & 1) + j];
        p[k16][g] = __builtin_bit_cast(bf16x8, pack8_bf16(e));
      }
#pragma unroll
    for (int k16 = 0; k16 < 2 * kSub; ++k16)
#pragma unroll
      for (int t = 0; t < kOut; ++t) {
        const bf16x8 v = value_frag(base, t, k16);
#pragma unroll
        for (int g = 0; g < QG; ++g) o[t][g] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[k16][g], o[t][g], 0, 0, 0);
      }
    values_turn(index);
  };

  if (steps > 0) {
    if constexpr (kFp8) {
      fetch(t_begin);
      put_keys(0);
      if constexpr (kTurns) load_rows(kr, held.v);
      put_rows(0, kTurns ? kr : vr, true);
      if (steps > 1) fetch(t_begin + kKeys);
    } else {
      issue(0, t_begin);
      if (steps > 1) issue(1, t_begin + kKeys);
    }
  }
  auto arrive = [&](int i) __attribute__((always_inline)) {
    if constexpr (kFp8) {
      __syncthreads();
      if (kTurns || i + 1 >= steps) return;
      put_keys((i + 1) & 1);
      put_rows((i + 1) & 1, vr, true);
      if (i + 2 < steps) fetch(t_begin + (i + 2) * kKeys);
    } else if (i == 0 && steps > 1) {
      // both buffers' transfers are on their way
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kLoads) : "memory");
      __syncthreads();
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (i + 1 < steps) issue((i + 1) & 1, t_begin + (i + 1) * kKeys);
    }
  };
  auto run = [&](int part, auto count) __attribute__((always_inline)) {
    // steps that every column sees whole; those that some see in part; the rest
    const int first = t_begin + 32 * part;
    const int plain = busy ? max(min(wave_all, t_end) - first + 64 - 32 * decltype(count)::value, 0) / kKeys : 0;
    const int seen = busy ? max(min(wave_end, t_end) - first + kKeys - 1, 0) / kKeys : 0;
    int i = 0;
    if constexpr (Z::kUnroll) {
      for (; i + 1 < plain; i += 2) {
        arrive(i);
        step(lds, t_begin + i * kKeys, i, part, count, std::false_type());
        arrive(i + 1);
        step(lds + Z::kStage, t_begin + (i + 1) * kKeys, i + 1, part, count, std::false_type());
      }
    } else {
      for (; i < plain; ++i) {
        arrive(i);
        step(lds + (i & 1) * Z::kStage, t_begin + i * kKeys, i, part, count, std::false_type());
      }
    }
    for (; i < seen; ++i) {
      arrive(i);
      step(lds + (i & 1) * Z::kStage, t_begin + i * kKeys, i, part, count, std::true_type());
    }
    for (; i < steps; ++i) {
      arrive(i);
      keys_turn(i);
      values_turn(i);
    }
  };
  if (halves) run(wave >> 1, std::integral_constant<int, 1>());
  else run(0, std::integral_constant<int, 2>());
  if constexpr (kPaged) bad = __syncthreads_or(bad);
#pragma unroll
  for (int g = 0; g < QG; ++g) l[g] = sum_halves(l[g]);
  if (halves) {
    // the second pair's results through LDS to the first
    __syncthreads();
    float* mine = reinterpret_cast<float*>(lds) + (wave & 1) * 64 * Z::kLane;
    if (wave >= 2) {
#pragma unroll
      for (int g = 0; g < QG; ++g) {
#pragma unroll
        for (int t = 0; t < kOut; ++t)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<f32x4*>(mine + ((g * kOut + t) * 4 + i / 4) * 256 + 4 * lane) =
                f32x4{o[t][g][i], o[t][g][i + 1], o[t][g][i + 2], o[t][g][i + 3]};
        mine[QG * kOut * 1024 + 128 * g + lane] = m[g];
        mine[QG * kOut * 1024 + 128 * g + 64 + lane] = l[g];
      }
    }
    __syncthreads();
    if (wave >= 2) return;
#pragma unroll
    for (int g = 0; g < QG; ++g) {
      const float m1 = mine[QG * kOut * 1024 + 128 * g + lane], l1 = mine[QG * kOut * 1024 + 128 * g + 64 + lane];
      const float top = fmaxf(m[g], m1), base = top == kNegInf ? 0.0f : top;
      const float f0 = __builtin_amdgcn_exp2f(m[g] - base), f1 = __builtin_amdgcn_exp2f(m1 - base);
      m[g] = top;
      l[g] = l[g] * f0 + l1 * f1;
#pragma unroll
      for (int t = 0; t < kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(mine + ((g * kOut + t) * 4 + i / 4) * 256 + 4 * lane);
#pragma unroll
          for (int j = 0; j < 4; ++j) o[t][g][i + j] = o[t][g][i + j] * f0 + v[j] * f1;
        }
    }
  }
  if (!busy) return;
  // An infinity or NaN among the values of tokens that only some of the columns
  // see reaches the others through a weight of 0.  Seldom enough to look for
  // such values only where there is such a result.
  bool leaked = false;
  if (a.causal) {
    float sum = 0.0f;
#pragma unroll
    for (int g = 0; g < QG; ++g)
#pragma unroll
      for (int t = 0; t < kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(o[t][g][i], 0.0f, sum);
    if (__builtin_expect(__any(sum != 0.0f), 0))
      for_odd_values<D, KV>(a, at.seq, hk, key0, max(wave_all, t_begin), t_end, [&](int) {
        leaked = true;
        return false;
      });
  }
  if (__builtin_expect(leaked, 0)) {
#pragma unroll
    for (int g = 0; g < QG; ++g) {
      const int col = min(wcol + 32 * g + li, cols - 1), token = col / G, head = hk * G + col - token * G;
      const uint16_t* src = a.q + static_cast<int64_t>(at.row0 + token) * a.q_stride + static_cast<int64_t>(head) * D + 8 * lh;
      f32x16 acc[kOut];
      wave_columns<D, KV>(a, at.seq, hk, key0, t_begin, min(t_end, wave_end), wave_all, src, lim[g], acc, &m[g], &l[g]);
#pragma unroll
      for (int t = 0; t < kOut; ++t) o[t][g] = acc[t];
    }
  }

  // results: lane (li, lh) has values 32 t + 8 (i / 4) + 4 lh + i % 4 of its columns
#pragma unroll
  for (int g = 0; g < QG; ++g) {
    if (bad) l[g] = __builtin_nanf("");
    if (wcol + 32 * g + li >= cols) continue;
    if (parts > 1) {
      const int64_t all = a.T * a.Hq, r = part * all + row[g];
      if (lh == 0) *reinterpret_cast<float2*>(a.ws + parts * all * D + 2 * r) = float2{m[g], l[g]};
      if (steps <= 0) continue;
#pragma unroll
      for (int t = 0; t < kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(a.ws + r * D + 32 * t + 2 * i + 4 * lh) =
              f32x4{o[t][g][i], o[t][g][i + 1], o[t][g][i + 2], o[t][g][i + 3]};
    } else {
      const float inv = l[g] == 0.0f ? 0.0f : 1.0f / l[g];
      if (a.lse != nullptr && lh == 0) a.lse[row[g]] = log_sum(m[g], l[g]);
#pragma unroll
      for (int t = 0; t < kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<u32x2*>(a.out + static_cast<int64_t>(row[g]) * D + 32 * t + 2 * i + 4 * lh) =
              u32x2{pack_bf16(o[t][g][i] * inv, o[t][g][i + 1] * inv), pack_bf16(o[t][g][i + 2] * inv, o[t][g][i + 3] * inv)};
    }
  }
}

// Joins the parts of the key axis: D / 4 lanes a row of the packed queries, and
// SETS such groups that take the row's parts in turn.  A part that a row's
// block did not reach has a sum of 0 and no outputs.
template <int D, int SETS>
__global__ __launch_bounds__(kThreads) void prompt_join_kernel(const PromptArgs a, int parts) {
  constexpr int kLanes = D / 4, kRows = kThreads / (kLanes * SETS), kBatch = 4;
  __shared__ f32x4 red[SETS > 1 ? kThreads : 1];
  __shared__ float2 red_ml[SETS > 1 ? kRows * SETS : 1];
  const int64_t all = a.T * a.Hq;
  const int set = threadIdx.x / kLanes % SETS, r = threadIdx.x / (kLanes * SETS);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + r;
  const int d = 4 * (threadIdx.x % kLanes);
  const float2* ml = reinterpret_cast<const float2*>(a.ws + parts * all * D);
  float top = kNegInf, sum = 0.0f;
  f32x4 acc = {0, 0, 0, 0};
  if (row < all) {
    for (int i = set; i < parts; i += SETS * kBatch) {
      // All loads of a batch on their way at once; where there are many rows, only
      // those that a block wrote (1038 rows of 32 heads: 10.6 -> 8.5 us).
      float2 w[kBatch];
      f32x4 v[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int64_t at = static_cast<int64_t>(min(i + j * SETS, parts - 1)) * all + row;
        w[j] = ml[at];
        if (SETS > 1) v[j] = *reinterpret_cast<const f32x4*>(a.ws + at * D + d);
      }
      if constexpr (SETS == 1) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int64_t at = static_cast<int64_t>(min(i + j * SETS, parts - 1)) * all + row;
          if (w[j].y != 0.0f) v[j] = *reinterpret_cast<const f32x4*>(a.ws + at * D + d);
        }
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (i + j * SETS >= parts || w[j].y == 0.0f) continue;
        const float next = fmaxf(top, w[j].x), base = next == kNegInf ? 0.0f : next;
        const float keep = __builtin_amdgcn_exp2f(top - base), f = __builtin_amdgcn_exp2f(w[j].x - base);
        sum = sum * keep + f * w[j].y;
        acc = acc * keep + f * v[j];
        top = next;
      }
    }
  }
  if constexpr (SETS > 1) {
    red[threadIdx.x] = acc;
    if (d == 0) red_ml[r * SETS + set] = float2{top, sum};
    __syncthreads();
    if (set) return;
    for (int i = 1; i < SETS; ++i) top = fmaxf(top, red_ml[r * SETS + i].x);
    const float base = top == kNegInf ? 0.0f : top;
    sum = 0.0f;
    acc = f32x4{0, 0, 0, 0};
    for (int i = 0; i < SETS; ++i) {
      const float f = __builtin_amdgcn_exp2f(red_ml[r * SETS + i].x - base);
      sum += f * red_ml[r * SETS + i].y;
      acc += f * red[(r * SETS + i) * kLanes + d / 4];
    }
  }
  // rows that no sequence has stay as they are
  const int64_t first = static_cast<int64_t>(max(a.starts[0], 0)) * a.Hq, last = static_cast<int64_t>(a.starts[a.B]) * a.Hq;
  if (row >= all || row < first || row >= last) return;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<u32x2*>(a.out + row * D + d) = u32x2{pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)};
  if (a.lse != nullptr && d == 0) a.lse[row] = log_sum(top, sum);
}

template <int D>
void launch_join(const PromptArgs& a, const PromptPlan& p, hipStream_t st) {
  const int64_t rows = a.T * a.Hq;
  constexpr int kSets = 1024 / D;
  const int64_t per = 1024 / D;  // rows of a block of one set
  if (p.parts > 4 && rows < 8192) {
    hipLaunchKernelGGL((prompt_join_kernel<D, kSets>), dim3(static_cast<unsigned>(rows)), dim3(kThreads), 0, st, a, p.parts);
  } else {
    hipLaunchKernelGGL((prompt_join_kernel<D, 1>), dim3(static_cast<unsigned>((rows + per - 1) / per)), dim3(kThreads), 0, st,
                       a, p.parts);
  }
}

template <int D, int QG, PromptKv KV>
void launch_tiles(const PromptArgs& a, const PromptPlan& p, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(p.tiles * a.Hk * p.parts));
  hipLaunchKernelGGL((prompt_attention_kernel<D, QG, KV>), grid, dim3(kThreads), 0, st, a, static_cast<int>(p.tiles),
                     p.cols, p.parts, p.least);
}

template <int D, PromptKv KV>
hipError_t launch_d(const PromptArgs& a, const PromptPlan& p, hipStream_t st) {
  if constexpr (D == 64 && KV != PromptKv::kPagedFp8) {
    if (p.cols == 256) launch_tiles<D, 2, KV>(a, p, st);
    else launch_tiles<D, 1, KV>(a, p, st);
  } else {
    launch_tiles<D, 1, KV>(a, p, st);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  launch_join<D>(a, p, st);
  return hipGetLastError();
}

template <PromptKv KV>
hipError_t launch_kv(const PromptArgs& a, const PromptPlan& p, hipStream_t st) {
  switch (a.D) {
    case 64: return launch_d<64, KV>(a, p, st);
    case 128: return launch_d<128, KV>(a, p, st);
    default: return launch_d<256, KV>(a, p, st);
  }
}

}  // namespace

// What a call takes, in us, from what its blocks' steps took over 71 chunked
// shapes (1 to 64 sequences, 1 to 1024 new tokens, 600 to 32768 cached, equal
// and ragged, both caches, every choice of columns and parts timed): a step of
// 64 keys, alone on a CU or in pairs, for 128 columns and for up to 64, and the
// join.  On 220 shapes drawn at random the choice by this is 2.9% from the best
// one on average and 39% at most; a fixed number of blocks a CU was 21% on
// average of the 71.
static float prompt_cost(int64_t cols, int64_t blocks, int64_t steps, int64_t parts, int64_t rows, int64_t D, bool half) {
  constexpr float kAlone[2] = {1.15f, 0.85f}, kPair[2] = {1.84f, 1.11f}, kWhole = 0.6f;
  const float n = static_cast<float>(blocks);
  auto rounds = [&](int64_t slots) {
    return kWhole * static_cast<float>((blocks + slots - 1) / slots) + (1.0f - kWhole) * n / static_cast<float>(slots);
  };
  float us;  // of a step, with what waits for a place
  if (D == 256) us = 2.09f * kAlone[half] * std::max(1.0f, rounds(256));
  else us = (D == 64 ? 0.77f : 1.0f) * (blocks <= 256 ? kAlone[half] : kPair[half] * std::max(1.0f, rounds(512)));
  us *= static_cast<float>(steps);
  if (parts > 1) us += 4.0f + static_cast<float>(rows * parts * (D + 2)) * (8.0f / 5.0e6f);
  return us;
}

// The most tiles that B sequences of T tokens have.
static int64_t prompt_tiles(int64_t T, int64_t B, int64_t G, int64_t cols) { return T * G / cols + std::min(B, T); }

PromptPlan prompt_plan(int64_t T, int64_t B, int64_t Hq, int64_t Hk, int64_t D, int64_t max_len, bool paged) {
  const int64_t G = Hq / Hk, expect = paged ? max_len : (max_len + B - 1) / B;  // keys of a sequence
  // a tile a sequence, or, of longer ones, the last tile half full
  auto blocks_of = [&](int64_t cols) {
    const int64_t n = std::min(B, T);
    return (T * G <= cols * n ? n : (T * G + cols - 1) / cols + n / 2) * Hk;
  };
  PromptPlan p;
  p.parts = 1, p.least = 0;
  if (D == 64 && T * G / 256 * Hk >= 512) {
    // columns enough for blocks of 256, whose waves read a key for 64 columns
    // instead of 32 (4096 tokens, 32 heads: 167 us with 128, 146 with 256)
    p.cols = 256;
  } else {
    // A prompt over its own keys is not cut: half its parts would see nothing
    // (1024 tokens, 32 heads on 8 key heads of 128: 21 us, in two parts 35).
    const bool cut = paged ? max_len >= 256 : expect >= 4096 || (expect >= 512 && max_len >= 4 * T);
    float best = 0.0f;
    for (const int cols : {128, 64}) {
      const int64_t blocks = blocks_of(cols);
      const bool half = cols == 64 || T * G <= 64 * std::min(B, T);
      for (int64_t parts = 1; parts <= 256; parts += (parts + 3) / 4) {
        const int64_t chunk = ((expect + parts - 1) / parts + 63) / 64;  // steps
        if (parts > 1 && (!cut || chunk < 2 || blocks * parts >= 1 << 20)) break;
        const int64_t used = (expect + 64 * chunk - 1) / (64 * chunk);
        const float us = prompt_cost(cols, blocks * used, chunk, used, T * Hq, D, half);
        if (best == 0.0f || us < best) {
          best = us;
          p.cols = cols;
          p.parts = static_cast<int>(used);
          // A shorter sequence has as many parts, but none below this: with 128 keys
          // at least, a ragged batch of chunks and single tokens takes 153 us
          // instead of 145, 8 x 64 tokens over 2000 under a limit of 131072 77 and 54.
          p.least = static_cast<int>(std::min<int64_t>(64 * chunk, 512));
        }
      }
    }
  }
  p.tiles = prompt_tiles(T, B, G, p.cols);
  return p;
}

PromptPlan prompt_plan_of(PromptPlan p, int64_t T, int64_t B, int64_t G, PromptKv kv) {
  if (kv == PromptKv::kPagedFp8 && p.cols == 256) p.cols = 128, p.tiles = prompt_tiles(T, B, G, 128);
  return p;
}

hipError_t launch_prompt_attention(const PromptArgs& a, PromptPlan p, hipStream_t st) {
  p = prompt_plan_of(p, a.T, a.B, a.Hq / a.Hk, a.kv);
  switch (a.kv) {
    case PromptKv::kDense: return launch_kv<PromptKv::kDense>(a, p, st);
    case PromptKv::kPagedBf16: return launch_kv<PromptKv::kPagedBf16>(a, p, st);
    default: return launch_kv<PromptKv::kPagedFp8>(a, p, st);
  }
}

}  // namespace jq
