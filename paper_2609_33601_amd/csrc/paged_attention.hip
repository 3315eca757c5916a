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
//    columns of a matrix product, 16 (or 64) of them at a time, so a
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
// Scores, statistics and sums are fp32; P takes part in its product as the sum
// of two bf16, so that the outputs' rounding is the only one that shows.
// One sequence of 131072 tokens, 8 key heads of 128: 96 us, 5.6 TB/s of cache;
// 64 sequences of 1 .. 8192, 8-bit: 110 us, 4.8 TB/s; 4 blocks of 64 new tokens
// over up to 2080, 32 key heads: 31 us, 3.3 TB/s (36 with the cache from HBM).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "block_common.h"
#include "block_internal.h"

namespace jq {

namespace {

using namespace block_detail;

constexpr int kWaves = 4;
constexpr int kTile = 32;  // tokens of a wave's step
typedef const __attribute__((address_space(4))) int32_t* uniform_i32;
constexpr float kNegInf = -__builtin_inff();

// Largest over the lanes that differ in the upper two lane bits.
__device__ __forceinline__ float max_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
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

// Where a block is: heads run fastest, so that with the usual numbers of heads
// an XCD (every eighth block) has its share of every sequence, however their
// lengths differ, and blocks with the same keys share its cache; the last
// parts, which most sequences do not have, come last.
struct BlockPlace {
  int hk, b, cb, part;
};
__device__ __forceinline__ BlockPlace block_place(const AttnArgs& a, int col_blocks) {
  const int id = blockIdx.x, bh = id / a.Hk;
  return {id % a.Hk, bh % a.B, bh / a.B % col_blocks, bh / a.B / col_blocks};
}

// The queries of column `col` (new token, head of the key head's group): the
// new token, the row in [B, Tq, Hq] and the operand of the first product.
template <int D, bool FP8>
struct Query {
  int token;
  int64_t row;
  bf16x8 f[D / 32];
  __device__ __forceinline__ void load(const AttnArgs& a, int b, int hk, int col, int lg) {
    const int G = a.Hq / a.Hk;
    token = col / G;
    row = (static_cast<int64_t>(b) * a.Tq + token) * a.Hq + hk * G + (col - token * G);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      // which eight of a head a lane feeds to step c: with bytes, sixteen consecutive values serve two steps
      const int d = FP8 ? 64 * (c / 2) + 16 * lg + 8 * (c % 2) : 32 * c + 8 * lg;
      u32x4 v = *reinterpret_cast<const u32x4*>(a.q + row * D + d);
      if (a.scale < 0.0f) v ^= 0x80008000u;  // so that scores grow with their products
      f[c] = __builtin_bit_cast(bf16x8, v);
    }
  }
};

// What a product is multiplied with to be a power of two; 0 as next to nothing,
// for the masked ones' sake.
__device__ __forceinline__ float power_scale(float scale) {
  return scale == 0.0f ? 0x1p-126f : fabsf(scale) * 1.44269504088896340736f;
}

// S^T of 16 tokens: their rows' 16-byte chunks 4 c + lg, times the queries.
template <int D, bool FP8>
__device__ __forceinline__ f32x4 scores(const uint32_t* k, const Query<D, FP8>& q) {
  f32x4 s = {0, 0, 0, 0};
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    u32x4 kv;
    if constexpr (FP8) {
      const uint32_t w0 = k[2 * c], w1 = k[2 * c + 1];
      kv = u32x4{e4m3_pair_to_bf16<false>(w0), e4m3_pair_to_bf16<true>(w0), e4m3_pair_to_bf16<false>(w1),
                 e4m3_pair_to_bf16<true>(w1)};
    } else {
      kv = u32x4{k[4 * c], k[4 * c + 1], k[4 * c + 2], k[4 * c + 3]};
    }
    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kv), q.f[c], s, 0, 0, 0);
  }
  return s;
}

// N more products of a lane's column (-inf: not seen): the powers of two of
// their scores over m, with the sum l and the output brought along.  m follows
// the largest score only where that has grown by more than 2^8, which seldom
// comes after a column's first tokens (16 columns would otherwise be brought
// along in two steps of five for a thousand tokens of random scores): powers
// then reach 2^8 and their rounding stays relative.
template <int N, int DV>
__device__ __forceinline__ void online_softmax(float (&v)[N], float scale2, float& m, float& l, f32x4 (&o)[DV]) {
  float top = v[0];
#pragma unroll
  for (int e = 1; e < N; ++e) top = fmaxf(top, v[e]);
  top = max_groups(top) * scale2;
  const bool grown = top > m + 8.0f;
  if (__any(grown)) {
    const float next = grown ? top : m;
    const float keep = __builtin_amdgcn_exp2f(m - (next == kNegInf ? 0.0f : next));
    l *= keep;
#pragma unroll
    for (int j = 0; j < DV; ++j) o[j] *= keep;
    m = next;
  }
  const float base = m == kNegInf ? 0.0f : m;  // nothing seen yet: every power below is 0
#pragma unroll
  for (int e = 0; e < N; ++e) {
    v[e] = __builtin_amdgcn_exp2f(fmaf(v[e], scale2, -base));
    l += v[e];
  }
}

// A lane's eight weights as the sum of two bf16, 16 bits in all: rounded to one
// of them, weights cost the outputs as much again as their own rounding does
// (rms error 0.0024 instead of 0.0017).  Both parts of a weight have its sign, and
// the second, taken of the weight and a millionth more, is 0 only where the weight
// is, so that an infinite value stays one.
struct Weights {
  bf16x8 high, low;
};
__device__ __forceinline__ Weights split_weights(const float (&v)[8]) {
  constexpr float kMore = 1.0f + 0x1p-20f;
  u32x4 high, low;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t a = __float_as_uint(v[2 * j]), b = __float_as_uint(v[2 * j + 1]);
    high[j] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    low[j] = pack_bf16(fmaf(v[2 * j], kMore, -bf_hi(a)), fmaf(v[2 * j + 1], kMore, -bf_hi(b)));
  }
  return {__builtin_bit_cast(bf16x8, high), __builtin_bit_cast(bf16x8, low)};
}

// O^T += V^T P^T of 32 tokens, two MFMAs per value of a lane's V rows: v[e] are
// D / 16 consecutive values of tokens 4 lg + e % 4 of both groups of 16.  The
// operand of value j, for each token of a lane.
template <bool FP8, int ROW>
__device__ __forceinline__ bf16x8 value_operand(const uint32_t (*v)[ROW], int j) {
  u32x4 r;
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    uint32_t x, y;  // the dwords of tokens 2h and 2h + 1 that hold value j
    if constexpr (FP8) {
      const uint32_t wx = v[2 * h][j / 4], wy = v[2 * h + 1][j / 4];
      x = (j & 2) ? e4m3_pair_to_bf16<true>(wx) : e4m3_pair_to_bf16<false>(wx);
      y = (j & 2) ? e4m3_pair_to_bf16<true>(wy) : e4m3_pair_to_bf16<false>(wy);
    } else {
      x = v[2 * h][j / 2];
      y = v[2 * h + 1][j / 2];
    }
    r[h] = __builtin_amdgcn_perm(y, x, (j & 1) ? 0x07060302u : 0x05040100u);
  }
  return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ f32x4 mfma32(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
template <int D, bool FP8, int ROW>
__device__ __forceinline__ void add_values(const uint32_t (*v)[ROW], const Weights& p, f32x4 (&o)[D / 16]) {
  // Two values at a time, so that no product waits for the one before it; the
  // compiler, left to itself, puts a value's two products next to each other.
  constexpr int kAllButMfma = 0x496;
#pragma unroll
  for (int j = 0; j < D / 16; j += 2) {
    const bf16x8 a = value_operand<FP8>(v, j), b = value_operand<FP8>(v, j + 1);
    o[j] = mfma32(a, p.low, o[j]);
    __builtin_amdgcn_sched_barrier(kAllButMfma);
    o[j + 1] = mfma32(b, p.low, o[j + 1]);
    __builtin_amdgcn_sched_barrier(kAllButMfma);
    o[j] = mfma32(a, p.high, o[j]);
    __builtin_amdgcn_sched_barrier(kAllButMfma);
    o[j + 1] = mfma32(b, p.high, o[j + 1]);
    __builtin_amdgcn_sched_barrier(kAllButMfma);
  }
}

// Whether any of a step's values is an infinity or NaN: adding one unit to an
// exponent (bf16) or code (e4m3) that is all ones carries into its sign bit.
template <bool FP8, int ROW>
__device__ __forceinline__ bool any_not_finite(const uint32_t (*v)[ROW]) {
  constexpr uint32_t kBits = FP8 ? 0x7F7F7F7Fu : 0x7F807F80u, kUnit = FP8 ? 0x01010101u : 0x00800080u;
  uint32_t all = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int i = 0; i < ROW; ++i) all |= (v[e][i] & kBits) + kUnit;
  return __any((all & ~kBits & (FP8 ? 0x80808080u : 0x80008000u)) != 0);
}

// The same step where columns see different numbers of its tokens (`seen` of
// the lane's column) and a value is an infinity or NaN, which a weight of 0
// would carry into columns that do not see it: once for each number of tokens,
// the rows from there on zeroed, and only its columns take the result.  Leaves
// nothing for the usual product (a branch around that took 46 registers more).
template <int D, bool FP8, int ROW>
__device__ __forceinline__ void add_values_apart(uint32_t (*v)[ROW], Weights& p, int seen, int lg, f32x4 (&o)[D / 16]) {
#pragma unroll 1
  for (int n = kTile; n > 0; --n) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = 16 * (e / 4) + 4 * lg + e % 4 < n;
#pragma unroll
      for (int i = 0; i < ROW; ++i) v[e][i] = in ? v[e][i] : 0u;
    }
    const bool mine = min(seen, kTile) == n;
    if (!__any(mine)) continue;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      const bf16x8 a = value_operand<FP8>(v, j);
      const f32x4 sum = mfma32(a, p.high, mfma32(a, p.low, o[j]));
#pragma unroll
      for (int r = 0; r < 4; ++r) o[j][r] = mine ? sum[r] : o[j][r];
      __builtin_amdgcn_sched_barrier(0);  // seldom run: registers matter more than speed
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int i = 0; i < ROW; ++i) v[e][i] = 0u;
  p.high = p.low = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
}

__device__ __forceinline__ float log_sum(float top, float sum) {
  return sum == 0.0f ? kNegInf : (top + __builtin_log2f(sum)) * 0.69314718055994530942f;
}

// Up to 16 columns: the waves of a block take steps of 32 tokens in turn.
template <int D, bool FP8, int WPS>
__global__ __launch_bounds__(64 * kWaves, WPS) void paged_attention_kernel(const AttnArgs a, int chunk, int parts) {
  constexpr int kB = FP8 ? 1 : 2;   // bytes of a cached value
  constexpr int kDV = D / 16;       // values of a V row per lane
  constexpr int kVRow = kDV * kB / 4;
  __shared__ float red_o[kWaves * 16 * (D + 4)];
  __shared__ float red_m[kWaves * 16], red_l[kWaves * 16];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const BlockPlace at = block_place(a, 1);
  const int b = at.b, hk = at.hk, part = at.part;
  const int G = a.Hq / a.Hk, cols = a.Tq * G;
  const int page = 1 << a.page_shift;
  const int len = min(a.lens[b], a.max_len);
  const int t0 = part * chunk, t1 = min(len, t0 + chunk);
  const bool direct = parts == 1;
  if (t0 >= t1 && !direct) return;  // the joining kernel counts parts by len, too

  Query<D, FP8> q;
  q.load(a, b, hk, min(li, cols - 1), lg);  // columns past the last repeat it
  const int end = a.causal ? min(len, len - a.Tq + 1 + q.token) : len;

  f32x4 o[kDV];
#pragma unroll
  for (int j = 0; j < kDV; ++j) o[j] = f32x4{0, 0, 0, 0};
  float m = kNegInf, l = 0.0f;
  const float scale2 = power_scale(a.scale);
  const int seen_by_all = a.causal ? min(len, len - a.Tq + 1) : len;  // tokens before it are, by every column
  const bool apart = a.causal && a.Tq > 1;  // columns may see different numbers of tokens
  // read with scalar loads: uniform, and nobody writes it meanwhile
  const uniform_i32 table = (uniform_i32)(a.table + static_cast<int64_t>(b) * a.table_cols);
  const uint8_t* kbase = static_cast<const uint8_t*>(a.k_cache);
  const uint8_t* vbase = static_cast<const uint8_t*>(a.v_cache);
  const uint32_t num_pages = static_cast<uint32_t>(a.num_pages);  // below 2^31
  bool bad = false;  // a page number outside the cache was met

  // A step's place: the first cached row of each group of 16 tokens, and the
  // group's last readable one.  Pages hold 16 tokens or more, so a group lies in
  // one page.  Tokens past the end read the last one of their group, groups past
  // the end the first group.
  struct Place {
    int64_t line[2];
    int last[2];
  };
  auto locate = [&](int tile) __attribute__((always_inline)) -> Place {
    Place p;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int h0 = tile + 16 * s < len ? tile + 16 * s : tile;
      int pg = table[h0 >> a.page_shift];
      if (static_cast<uint32_t>(pg) >= num_pages) bad = true, pg = 0;
      p.line[s] = ((static_cast<int64_t>(pg) * a.Hk + hk) << a.page_shift) + (h0 & (page - 1));
      p.last[s] = min(len - 1 - h0, 15);
    }
    return p;
  };
  uint32_t kf[2][D * kB / 16], vf[8][kVRow];
  float ks[2][4], vs[2][4];
  auto load_k = [&](const Place& p) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint8_t* kp = kbase + (p.line[s] + min(li, p.last[s])) * (D * kB) + 16 * lg;
#pragma unroll
      for (int c = 0; c < D * kB / 64; ++c) load_bytes<16>(kp + 64 * c, kf[s] + 4 * c);
      if constexpr (FP8) *reinterpret_cast<f32x4*>(ks[s]) = *reinterpret_cast<const f32x4*>(a.k_scale + p.line[s] + 4 * lg);
    }
  };
  auto load_v = [&](const Place& p) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if constexpr (FP8) *reinterpret_cast<f32x4*>(vs[s]) = *reinterpret_cast<const f32x4*>(a.v_scale + p.line[s] + 4 * lg);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        load_bytes<kDV * kB>(vbase + (p.line[s] + min(4 * lg + e, p.last[s])) * (D * kB) + li * (kDV * kB), vf[4 * s + e]);
    }
  };

  // The next step's keys are requested when this one's have been multiplied,
  // and its values when this one's have: the registers are free by then, and
  // a wave always has a step on its way.
  auto step = [&](int tile, auto more) __attribute__((always_inline)) {
    Place next;
    if constexpr (more) next = locate(tile + kWaves * kTile);

    // this lane's column, tokens tile + 16 s + 4 lg + r
    float v[8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const f32x4 sc = scores<D, FP8>(kf[s], q);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[4 * s + r] = FP8 ? sc[r] * ks[s][r] : sc[r];
    }
    if constexpr (more) load_k(next);
    // Columns of at most 16 new tokens differ in a sequence's last two tiles
    // alone, and those are the last steps of two waves (or parts).
    const bool mask = !decltype(more)::value && tile + kTile > seen_by_all;
    const int left = end - tile - 4 * lg, in_len = len - tile - 4 * lg;  // from the lane's first token on
    if (mask) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 16 * (e / 4) + e % 4 < left ? v[e] : kNegInf;
    }
    online_softmax(v, scale2, m, l, o);
    if constexpr (FP8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= vs[e / 4][e % 4];
      if (mask) {  // an unseen token's scale may be anything
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 16 * (e / 4) + e % 4 < left ? v[e] : 0.0f;
      }
    }
    // Only a wave's last step may reach past the end.  The rows read there count
    // for nothing, which an infinity times 0 would not do.
    if constexpr (!more) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = 16 * (e / 4) + e % 4 < in_len;
#pragma unroll
        for (int i = 0; i < kVRow; ++i) vf[e][i] = in ? vf[e][i] : 0u;
      }
    }
    Weights p = split_weights(v);
    if (mask && apart && any_not_finite<FP8>(vf)) add_values_apart<D, FP8>(vf, p, end - tile, lg, o);
    add_values<D, FP8>(vf, p, o);
    if constexpr (more) load_v(next);
  };
  int tile = t0 + wave * kTile;
  if (tile < t1) {
    const Place first = locate(tile);
    load_k(first);
    load_v(first);
    for (; tile + kWaves * kTile < t1; tile += kWaves * kTile) step(tile, std::true_type{});
    step(tile, std::false_type{});
  }
  if (__any(bad)) l = __builtin_nanf(""), m = 0.0f;

  // Join the waves.  A lane holds, of column li, values d = kDV (4 lg + r) + j:
  // 4 kDV in a row, from 4 kDV lg.
  l = sum_groups(l);
  float* mine = red_o + (wave * 16 + li) * (D + 4) + kDV * 4 * lg;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < kDV; j += 4)
      *reinterpret_cast<f32x4*>(mine + r * kDV + j) = f32x4{o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]};
  if (lg == 0) red_m[wave * 16 + li] = m, red_l[wave * 16 + li] = l;
  __syncthreads();
  // thread -> (column, D / 16 values)
  const int c = threadIdx.x / 16, d0 = (threadIdx.x % 16) * kDV;
  if (c >= cols) return;
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
    const int tq = c / G;
    const int64_t row = (static_cast<int64_t>(b) * a.Tq + tq) * a.Hq + hk * G + (c - tq * G);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint32_t* dst = reinterpret_cast<uint32_t*>(a.out + row * D + d0);
#pragma unroll
    for (int j = 0; j < kDV / 2; ++j) dst[j] = pack_bf16(acc[2 * j] * inv, acc[2 * j + 1] * inv);
    if (a.lse != nullptr && d0 == 0) a.lse[row] = log_sum(top, sum);
  } else {
    const PartView pv = part_view(a.ws, static_cast<int64_t>(a.B) * a.Hk * parts * cols, D);
    const int64_t row = ((static_cast<int64_t>(b) * a.Hk + hk) * parts + part) * cols + c;
#pragma unroll
    for (int j = 0; j < kDV; j += 4)
      *reinterpret_cast<f32x4*>(pv.o + row * D + d0 + j) = f32x4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
    if (d0 == 0) *reinterpret_cast<float2*>(pv.ml + 2 * row) = make_float2(top, sum);
  }
}

// More columns: a block takes 64 of them, and 64 tokens at a time, which
// transfers bring into LDS once for all its eight waves, one stage ahead of the
// products: wave w has columns 16 (w % 4) .. and half w / 4 of the tokens.  A
// row's 16-byte chunk c sits at chunk c ^ (row & 15) of its place in LDS (as far
// as the row has chunks), so that the sixteen rows an operand spans cover all
// banks.  What bounds it is the chain from a stage's rows to its outputs (0.9 us
// without the transfers); two blocks a CU run theirs side by side, and the
// transfers alone would take about as long.  V read transposed out of LDS
// instead of zipped took as long (29 us of 29), eight waves' stores of a part
// instead of four's too.  A causal block walks all stages of its part, also those
// that none of its columns see: a prompt takes about twice the stages that it
// needs (2048 new tokens, 32 query heads on 8 key heads of 128: 146 us).
constexpr int kWideWaves = 8, kWideTile = 64;

template <int D, bool FP8, bool CAUSAL, int WPS>
__global__ __launch_bounds__(64 * kWideWaves, WPS) void paged_attention_wide_kernel(const AttnArgs a, int chunk,
                                                                                    int parts, int col_blocks) {
  constexpr int kB = FP8 ? 1 : 2;
  constexpr int kDV = D / 16, kVRow = kDV * kB / 4;
  constexpr int kRow = D * kB;                     // bytes of a cached row
  constexpr int kChunks = kRow / 16;
  constexpr int kMask = (kChunks < 16 ? kChunks : 16) - 1;
  constexpr int kGroup = 16 * kRow;                // bytes of a group of 16 tokens
  constexpr int kKeys = 4 * kGroup, kStage = 2 * kKeys + 512;  // keys, values, their scales
  constexpr int kRedRow = 4 * kDV + 2;             // floats of a lane at the end: its outputs, maximum and sum
  constexpr int kRed = 4 * 64 * kRedRow * 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * kStage > kRed ? 2 * kStage : kRed];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = wave / 4;
  const int li = lane & 15, lg = lane >> 4;
  // Which of the sixteenths of a value row a lane takes, and where it finds them in
  // its outputs: 4 r + lg are side by side over the lane groups where they are
  // stored (diffusion block 33.5 -> 32.5 us, 38 sequences of up to 67, e4m3, D = 256
  // 55 -> 53), 4 lg + r do not collide in LDS where a lane's are two chunks (39 -> 36
  // at D = 256, bf16), and spare the registers that the causal form lacks (37 -> 35).
  constexpr bool kSide = !CAUSAL && kRow <= 256;
  const int vi = kSide ? 4 * (li % 4) + li / 4 : li;
  auto sixteenth = [&](int r) __attribute__((always_inline)) { return kSide ? 4 * r + lg : 4 * lg + r; };
  const BlockPlace at = block_place(a, col_blocks);
  const int b = at.b, hk = at.hk, part = at.part;
  const int G = a.Hq / a.Hk, cols = a.Tq * G;
  const int page = 1 << a.page_shift;
  const int len = min(a.lens[b], a.max_len);
  const int t0 = part * chunk, t1 = min(len, t0 + chunk);
  const bool direct = parts == 1;
  if (t0 >= t1 && !direct) return;

  const int col0 = 64 * at.cb + 16 * (wave % 4);
  const bool busy = col0 < cols;  // else this wave only moves data
  Query<D, FP8> q;
  q.load(a, b, hk, min(col0 + li, cols - 1), lg);
  const int end = CAUSAL ? min(len, len - a.Tq + 1 + q.token) : len;
  f32x4 o[kDV];
#pragma unroll
  for (int j = 0; j < kDV; ++j) o[j] = f32x4{0, 0, 0, 0};
  float m = kNegInf, l = 0.0f;
  const float scale2 = power_scale(a.scale);
  const int seen_by_all = CAUSAL ? min(len, len - a.Tq + 1 + col0 / G) : len;  // tokens before it are, by every column
  const uniform_i32 table = (uniform_i32)(a.table + static_cast<int64_t>(b) * a.table_cols);
  const uint32_t num_pages = static_cast<uint32_t>(a.num_pages);  // below 2^31
  bool bad = false;
  const uint32_t lds0 = lds_addr(lds);

  // A stage's group that this wave moves: waves 0..3 the keys, 4..7 the values
  // of 16 rows that lie in one page.  A group past the end reads the stage's
  // first one; what lies past the end counts for nothing.
  auto first_row = [&](int tile) __attribute__((always_inline)) {
    return tile + 16 * (wave % 4) < len ? tile + 16 * (wave % 4) : tile;
  };
  int pg_next = t0 < t1 ? table[first_row(t0) >> a.page_shift] : 0;
  auto issue = [&](int buf, int tile) __attribute__((always_inline)) {
    const int g = wave % 4;
    const int h0 = first_row(tile);
    int pg = pg_next;
    pg_next = table[first_row(min(tile + kWideTile, len - 1)) >> a.page_shift];
    if (static_cast<uint32_t>(pg) >= num_pages) bad = true, pg = 0;
    const int64_t line = ((static_cast<int64_t>(pg) * a.Hk + hk) << a.page_shift) + (h0 & (page - 1));
    const Rsrc r = make_rsrc(static_cast<const uint8_t*>(half ? a.v_cache : a.k_cache) + line * kRow, kGroup);
    const uint32_t dst = lds0 + buf * kStage + half * kKeys + g * kGroup;
#pragma unroll
    for (int i = 0; i < kGroup / 1024; ++i) {
      const int row = 1024 / kRow * i + lane / kChunks, c = lane % kChunks;
      dma16(r, dst + 1024 * i, row * kRow + 16 * (c ^ (row & kMask)), 0);
    }
    if constexpr (FP8) {
      const Rsrc rs = make_rsrc((half ? a.v_scale : a.k_scale) + line, 64);
      if (lane < 16) dma4(rs, lds0 + buf * kStage + 2 * kKeys + 256 * half + 64 * g, 4 * lane, 0);
    }
  };

  if (t0 < t1) issue(0, t0);
  int buf = 0;
  for (int tile = t0; tile < t1; tile += kWideTile, buf ^= 1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tile + kWideTile < t1) issue(buf ^ 1, tile + kWideTile);
    const int first = tile + 32 * half;  // of this wave's tokens
    if (!busy || first >= t1) continue;
    const uint8_t* keys = lds + buf * kStage + 2 * half * kGroup;
    const uint8_t* values = keys + kKeys;
    const float* ks = reinterpret_cast<const float*>(lds + buf * kStage + 2 * kKeys) + 32 * half;
    float v[8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint32_t kf[kRow / 16];
#pragma unroll
      for (int c = 0; c < kRow / 64; ++c)
        load_bytes<16>(keys + s * kGroup + li * kRow + 16 * ((4 * c + lg) ^ (li & kMask)), kf + 4 * c);
      const f32x4 sc = scores<D, FP8>(kf, q);
      f32x4 f = {1, 1, 1, 1};
      if constexpr (FP8) f = *reinterpret_cast<const f32x4*>(ks + 16 * s + 4 * lg);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[4 * s + r] = FP8 ? sc[r] * f[r] : sc[r];
    }
    const bool mask = first + 32 > seen_by_all;
    const int left = end - first - 4 * lg, in_len = len - first - 4 * lg;  // from the lane's first token on
    if (mask) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 16 * (e / 4) + e % 4 < left ? v[e] : kNegInf;
    }
    online_softmax(v, scale2, m, l, o);
    if constexpr (FP8) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const f32x4 f = *reinterpret_cast<const f32x4*>(ks + 64 + 16 * s + 4 * lg);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[4 * s + r] *= f[r];
      }
      if (mask) {  // an unseen token's scale may be anything
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 16 * (e / 4) + e % 4 < left ? v[e] : 0.0f;
      }
    }
    uint32_t vf[8][kVRow];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int row = 4 * lg + e % 4, at_byte = vi * (kDV * kB);
      const uint8_t* src = values + (e / 4) * kGroup + row * kRow;
      if constexpr (kDV * kB <= 16) {
        load_bytes<kDV * kB>(src + 16 * ((at_byte / 16) ^ (row & kMask)) + at_byte % 16, vf[e]);
      } else {
        load_bytes<16>(src + 16 * ((at_byte / 16) ^ (row & kMask)), vf[e]);
        load_bytes<16>(src + 16 * ((at_byte / 16 + 1) ^ (row & kMask)), vf[e] + 4);
      }
    }
    // Rows past the end count for nothing, which an infinity times 0 would not do.
    if (first + 32 > len) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool in = 16 * (e / 4) + e % 4 < in_len;
#pragma unroll
        for (int i = 0; i < kVRow; ++i) vf[e][i] = in ? vf[e][i] : 0u;
      }
    }
    Weights p = split_weights(v);
    if constexpr (CAUSAL) {  // columns may see different numbers of tokens
      if (mask && any_not_finite<FP8>(vf)) add_values_apart<D, FP8>(vf, p, end - first, lg, o);
    }
    add_values<D, FP8>(vf, p, o);
  }
  // a wave sees the pages of its own groups alone
  bad = __syncthreads_or(bad);
  // the second half of the tokens joins the first
  float* red = reinterpret_cast<float*>(lds) + ((wave % 4) * kRedRow) * 64 + lane;
  if (half) {
#pragma unroll
    for (int j = 0; j < kDV; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[64 * (4 * j + r)] = o[j][r];
    red[64 * 4 * kDV] = m;
    red[64 * (4 * kDV + 1)] = l;
  }
  __syncthreads();
  if (half || !busy) return;
  {
    const float m2 = red[64 * 4 * kDV], l2 = red[64 * (4 * kDV + 1)];
    const float top = fmaxf(m, m2), base = top == kNegInf ? 0.0f : top;
    const float f1 = __builtin_amdgcn_exp2f(m - base), f2 = __builtin_amdgcn_exp2f(m2 - base);
    l = l * f1 + l2 * f2;
    m = top;
#pragma unroll
    for (int j = 0; j < kDV; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[j][r] = o[j][r] * f1 + red[64 * (4 * j + r)] * f2;
  }
  if (bad) l = __builtin_nanf(""), m = 0.0f;
  l = sum_groups(l);
  if (col0 + li >= cols) return;
  if (direct) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      uint16_t* dst = a.out + q.row * D + kDV * sixteenth(r);
#pragma unroll
      for (int j = 0; j < kDV; j += 4)
        *reinterpret_cast<u32x2*>(dst + j) =
            u32x2{pack_bf16(o[j][r] * inv, o[j + 1][r] * inv), pack_bf16(o[j + 2][r] * inv, o[j + 3][r] * inv)};
    }
    if (a.lse != nullptr && lg == 0) a.lse[q.row] = log_sum(m, l);
  } else {
    const PartView pv = part_view(a.ws, static_cast<int64_t>(a.B) * a.Hk * parts * cols, D);
    const int64_t row = ((static_cast<int64_t>(b) * a.Hk + hk) * parts + part) * cols + col0 + li;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < kDV; j += 4)
        *reinterpret_cast<f32x4*>(pv.o + row * D + kDV * sixteenth(r) + j) =
            f32x4{o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]};
    if (lg == 0) *reinterpret_cast<float2*>(pv.ml + 2 * row) = make_float2(m, l);
  }
}

// Joins the parts of the query columns.  A column's DC values (D of them, or
// a piece of them where there are few columns) are taken by DC / 4 lanes, and
// its parts by SETS such groups in turn; 256 threads hold 1024 / (DC * SETS)
// columns.
template <int D, int DC, int SETS>
__global__ __launch_bounds__(256) void paged_attention_join_kernel(const AttnArgs a, int chunk, int parts, int rows) {
  constexpr int kLanes = DC / 4, kCols = 256 / (kLanes * SETS), kPieces = D / DC;
  __shared__ f32x4 red[SETS > 1 ? 256 : 1];
  __shared__ float red_m[SETS > 1 ? kCols * SETS : 1], red_s[SETS > 1 ? kCols * SETS : 1];
  const int ln = threadIdx.x % kLanes, set = threadIdx.x / kLanes % SETS, c = threadIdx.x / (kLanes * SETS);
  const int piece = blockIdx.x % kPieces, at = blockIdx.x / kPieces * kCols + c;  // [b][hk][column]
  const int G = a.Hq / a.Hk, cols = a.Tq * G;
  const int row_in = min(at, rows - 1);
  const int col = row_in % cols, bh = row_in / cols, hk = bh % a.Hk, b = bh / a.Hk;
  const int len = min(a.lens[b], a.max_len);
  const int live = len > 0 ? (len + chunk - 1) / chunk : 0;
  const PartView pv = part_view(a.ws, static_cast<int64_t>(rows) * parts, D);
  const int64_t row0 = static_cast<int64_t>(bh) * parts * cols + col;
  const int d = piece * DC + 4 * ln;

  // this group's parts, with a running maximum like the tokens themselves
  float top = kNegInf, sum = 0.0f;
  f32x4 acc = {0, 0, 0, 0};
#pragma unroll 4
  for (int i = set; i < live; i += SETS) {
    const int64_t row = row0 + static_cast<int64_t>(i) * cols;
    const float2 ml = *reinterpret_cast<const float2*>(pv.ml + 2 * row);
    const f32x4 v = *reinterpret_cast<const f32x4*>(pv.o + row * D + d);
    const float next = fmaxf(top, ml.x);
    const float base = next == kNegInf ? 0.0f : next;
    const float keep = __builtin_amdgcn_exp2f(top - base), f = __builtin_amdgcn_exp2f(ml.x - base);
    sum = sum * keep + f * ml.y;
    acc = acc * keep + f * v;
    top = next;
  }
  if constexpr (SETS > 1) {
    red[threadIdx.x] = acc;
    if (ln == 0) red_m[c * SETS + set] = top, red_s[c * SETS + set] = sum;
    __syncthreads();
    if (set) return;
    const float* m = red_m + c * SETS;
    for (int s = 1; s < SETS; ++s) top = fmaxf(top, m[s]);
    const float base = top == kNegInf ? 0.0f : top;
    sum = 0.0f;
    acc = f32x4{0, 0, 0, 0};
    for (int s = 0; s < SETS; ++s) {
      const float f = __builtin_amdgcn_exp2f(m[s] - base);
      sum += f * red_s[c * SETS + s];
      acc += f * red[(c * SETS + s) * kLanes + ln];
    }
  }
  if (at >= rows) return;
  const int tq = col / G;
  const int64_t row = (static_cast<int64_t>(b) * a.Tq + tq) * a.Hq + hk * G + (col - tq * G);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<u32x2*>(a.out + row * D + d) = u32x2{pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv)};
  if (a.lse != nullptr && d == 0) a.lse[row] = log_sum(top, sum);
}

template <int D>
hipError_t launch_join(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const int rows = a.B * a.Tq * a.Hq;
#define JQ_JOIN(DC, SETS)                                                                                           \
  {                                                                                                                 \
    constexpr int kCols = 1024 / (DC * SETS);                                                                       \
    hipLaunchKernelGGL((paged_attention_join_kernel<D, DC, SETS>), dim3((rows + kCols - 1) / kCols * (D / DC)),     \
                       dim3(256), 0, st, a, p.chunk, p.parts, rows);                                                \
  }
  // Few columns of many parts: more threads on each, and its values over several
  // blocks.  Whole calls, D = 128, 32 x 32 against 256 / D groups against one: 256
  // parts of 16 columns 21.5, 35 and 49 us, 128 of 16 14, 21 and 27, 64 of 16 20.4,
  // 22 and 26; 32 parts are even (of 32 columns 10.9, 10.3 and 12.6, of 512 29, 28
  // and 29).  16 parts of 64 columns: 256 / D 9.7, one 11.1; 8 of 4096 34.7, 34.6.
  if (p.parts >= 32) JQ_JOIN(32, 32)
  else if (p.parts >= 8 && rows < 4096) JQ_JOIN(D, (256 / D))
  else JQ_JOIN(D, 1)
#undef JQ_JOIN
  return hipGetLastError();
}

template <int D, bool FP8>
hipError_t launch_d(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const int cols = a.Tq * (a.Hq / a.Hk);
  const int col_blocks = (cols + p.cols - 1) / p.cols;
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(a.B) * a.Hk * p.parts * col_blocks));
  if (p.cols == 16) {
    hipLaunchKernelGGL((paged_attention_kernel<D, FP8, D == 256 ? 1 : 2>), grid, dim3(64 * kWaves), 0, st, a, p.chunk,
                       p.parts);
  } else {
    constexpr int kWps = D == 256 ? 2 : 4;
    if (a.causal) {
      hipLaunchKernelGGL((paged_attention_wide_kernel<D, FP8, true, kWps>), grid, dim3(64 * kWideWaves), 0, st, a,
                         p.chunk, p.parts, col_blocks);
    } else {
      hipLaunchKernelGGL((paged_attention_wide_kernel<D, FP8, false, kWps>), grid, dim3(64 * kWideWaves), 0, st, a,
                         p.chunk, p.parts, col_blocks);
    }
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  return launch_join<D>(a, p, st);
}

}  // namespace

// Parts of the key axis.  One part needs no second kernel, which costs 2.7 us;
// a block of one part takes 1.1 us per 128 tokens, so up to three such rounds
// stay whole.  Beyond that, enough parts to have a block for each CU (more only
// add to what every block spends outside its loop: 1 x 131072 tokens, 8 key
// heads: 256 blocks 96 us, 1024 99, 4096 106), and with several sequences, whose
// lengths may differ, up to four of at least 2^18 / D tokens each (64 sequences
// of 1 .. 8192 tokens: one part 134 us, two 122, four 115, eight 114; 64 of 4096
// each: 101, 105, 109, 115), and no more than 2048 blocks for it (256 sequences of
// up to 2048, 2048 blocks a part: one part 190 us, two 196, four 196, and 356, 374
// and 388 where all are as long; 128 of up to 4096, 1024 a part: 192, 193, 188).  Of the wide kernel a CU holds two blocks up to
// D = 128, and several sequences get as many of four rounds or more (6 of up to
// 12047 tokens, 96 blocks a part: three parts 90 us, six 56; 3 of up to 3922,
// 96: 50 and 39; 16 of 2085 each, 128: two parts 34, four 35).
// The lengths are on the device, so max_len decides: a sequence of 4096 tokens (8
// key heads of 128) takes 11 us under its own length and 43 under 131072, whose
// parts are longer.  Four rounds are about even with and without parts, more are
// not (8 sequences of 512: one part 9.1 us, four 9.4; of 1024: 16.6 and 12.7).
AttnPlan attention_plan(int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D, int64_t max_len) {
  const int64_t cols = Tq * (Hq / Hk);
  AttnPlan p;
  p.cols = cols <= 16 ? 16 : 64;
  const int64_t heads = B * Hk * ((cols + p.cols - 1) / p.cols);
  constexpr int64_t kRound = kWaves * kTile;  // tokens of a block's round; two stages of the wide kernel
  constexpr int64_t kCus = 256;
  const int64_t rounds = (max_len + kRound - 1) / kRound;
  int64_t parts = 1;
  if (rounds > 3) {
    parts = (kCus + heads - 1) / heads;
    if (B > 1) {
      parts = std::max(parts, p.cols > 16 && D <= 128 ? std::min((2 * kCus + heads - 1) / heads, rounds / 4)
                                                      : std::min({int64_t{4}, max_len * D >> 18, 2048 / heads}));
    }
    parts = std::min(parts, rounds);
  }
  const int64_t each = (rounds + parts - 1) / parts;
  p.chunk = static_cast<int>(each * kRound);
  p.parts = static_cast<int>((rounds + each - 1) / each);
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
