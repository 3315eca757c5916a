// C ABI of the decoder block's other operators (include/jq_block.h): argument
// checks, workspace layout and kernel launches.  Every check runs before any
// launch, so a rejected call writes nothing.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_internal.h"
#include "jq_block.h"

namespace {

constexpr size_t kWsAlign = 256;
constexpr int64_t kMaxRows = int64_t(1) << 30;
constexpr int64_t kMaxK = 65536;
constexpr int64_t kMaxPage = 65536;
constexpr int64_t kMaxStride = int64_t(1) << 32;

size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
jq_status from_hip(hipError_t e) { return e == hipSuccess ? JQ_OK : JQ_ERR_HIP; }
hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }
const uint16_t* u16(const void* p) { return static_cast<const uint16_t*>(p); }

// The distance between rows of `width` elements that are read 8 at a time.
jq_status check_stride(int64_t stride, int64_t width) {
  if (stride < width || stride > kMaxStride) return JQ_ERR_INVALID_ARG;
  return stride % 8 == 0 ? JQ_OK : JQ_ERR_MISALIGNED;
}

jq_status check_fp8_shape(int64_t rows, int64_t K) {
  if (rows <= 0 || K <= 0) return JQ_ERR_INVALID_ARG;
  if (rows > kMaxRows || K < 16 || K % 16 != 0 || K > kMaxK) return JQ_ERR_UNSUPPORTED_SHAPE;
  return JQ_OK;
}

jq_status check_act(const void* x, int64_t x_stride, int64_t M, int64_t K) {
  if (x == nullptr) return JQ_ERR_INVALID_ARG;
  jq_status st = check_fp8_shape(M, K);
  if (st != JQ_OK) return st;
  if (M * ((K + 511) / 512) >= (int64_t(1) << 31)) return JQ_ERR_UNSUPPORTED_SHAPE;
  st = check_stride(x_stride, K);
  if (st != JQ_OK) return st;
  return aligned(x, 16) ? JQ_OK : JQ_ERR_MISALIGNED;
}

jq_status check_fp8_gemm(const void* q, const float* sx, int64_t M, int64_t K, const void* wq, const float* sw,
                         int64_t N, const void* bias, const void* y) {
  if (q == nullptr || sx == nullptr || wq == nullptr || sw == nullptr || y == nullptr) return JQ_ERR_INVALID_ARG;
  jq_status st = check_fp8_shape(M, K);
  if (st != JQ_OK) return st;
  st = check_fp8_shape(N, K);
  if (st != JQ_OK) return st;
  // a grid holds fewer than 2^32 threads: 2^18 blocks of 512 for few rows, M * N / 2^16 of 512 for many
  if (N > (int64_t(1) << 22) || M * N >= (int64_t(1) << 38)) return JQ_ERR_UNSUPPORTED_SHAPE;
  if (!aligned(q, 16) || !aligned(wq, 16) || !aligned(y, 16)) return JQ_ERR_MISALIGNED;
  if (!aligned(sx, 4) || !aligned(sw, 4) || (bias != nullptr && !aligned(bias, 2))) return JQ_ERR_MISALIGNED;
  return JQ_OK;
}

size_t fp8_workspace_bytes(int64_t M, int64_t K) {
  if (check_fp8_shape(M, K) != JQ_OK) return 0;
  return round_up(static_cast<size_t>(M) * static_cast<size_t>(K), kWsAlign) +
         round_up(static_cast<size_t>(M) * static_cast<size_t>((K + 127) / 128) * sizeof(float), kWsAlign);
}

// log2 of a page size, or -1 for one that is not supported.
int page_shift(int64_t page) {
  if (page < 16 || page > kMaxPage || (page & (page - 1)) != 0) return -1;
  int s = 0;
  while ((int64_t(1) << s) < page) ++s;
  return s;
}

// Heads, head length and the cache of jq_rope_append and jq_paged_attention.
jq_status check_cache(int64_t Hk, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                      int64_t num_pages, int64_t page, jq_cache_type type) {
  if (k_cache == nullptr || v_cache == nullptr || num_pages <= 0 || Hk <= 0) return JQ_ERR_INVALID_ARG;
  if (type != JQ_CACHE_BF16 && type != JQ_CACHE_FP8) return JQ_ERR_INVALID_ARG;
  const bool fp8 = type == JQ_CACHE_FP8;
  if (fp8 != (k_scale != nullptr) || fp8 != (v_scale != nullptr)) return JQ_ERR_INVALID_ARG;
  if (page_shift(page) < 0 || num_pages > (int64_t(1) << 31) - 1 || Hk > 65536) return JQ_ERR_UNSUPPORTED_SHAPE;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16)) return JQ_ERR_MISALIGNED;
  if (fp8 && (!aligned(k_scale, 16) || !aligned(v_scale, 16))) return JQ_ERR_MISALIGNED;
  return JQ_OK;
}

constexpr int64_t kMaxAxis = int64_t(1) << 30;
constexpr int64_t kMaxBlocks = int64_t(1) << 24;

jq_status check_attention(int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D, int64_t max_len) {
  if (B <= 0 || Tq <= 0 || Hq <= 0 || Hk <= 0 || max_len <= 0) return JQ_ERR_INVALID_ARG;
  if (Hq % Hk != 0 || (D != 64 && D != 128 && D != 256)) return JQ_ERR_UNSUPPORTED_SHAPE;
  if (B > (1 << 20) || Tq > (1 << 20) || Hq > 65536 || max_len > kMaxAxis) return JQ_ERR_UNSUPPORTED_SHAPE;
  const int64_t cols = Tq * (Hq / Hk);
  // both kernels' grids: fewer than 2^24 blocks of 256 threads
  if (B * Hk >= kMaxBlocks || B * Hk * cols >= kMaxBlocks) return JQ_ERR_UNSUPPORTED_SHAPE;
  const jq::AttnPlan p = jq::attention_plan(B, Tq, Hq, Hk, D, max_len);
  if (B * Hk * ((cols + p.cols - 1) / p.cols) * p.parts >= kMaxBlocks) return JQ_ERR_UNSUPPORTED_SHAPE;
  return JQ_OK;
}

size_t attention_workspace_bytes(int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D, int64_t max_len) {
  if (check_attention(B, Tq, Hq, Hk, D, max_len) != JQ_OK) return 0;
  const jq::AttnPlan p = jq::attention_plan(B, Tq, Hq, Hk, D, max_len);
  if (p.parts == 1) return 0;
  const size_t rows = static_cast<size_t>(B) * static_cast<size_t>(Tq) * static_cast<size_t>(Hq) * p.parts;
  return round_up(rows * (static_cast<size_t>(D) + 2) * sizeof(float), kWsAlign);
}

}  // namespace

extern "C" {

jq_status jq_rmsnorm(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                     const void* weight, int64_t M, int64_t D, float eps, jq_norm_out out, void* y, float* scale,
                     void* residual_out, int64_t residual_out_stride, void* stream) {
  if (x == nullptr || weight == nullptr || y == nullptr || M <= 0 || D <= 0) return JQ_ERR_INVALID_ARG;
  if (out != JQ_NORM_BF16 && out != JQ_NORM_FP8 && out != JQ_NORM_INT4) return JQ_ERR_INVALID_ARG;
  if ((residual != nullptr) != (residual_out != nullptr)) return JQ_ERR_INVALID_ARG;
  if ((out != JQ_NORM_BF16) != (scale != nullptr)) return JQ_ERR_INVALID_ARG;
  if (!(eps >= 0.0f)) return JQ_ERR_INVALID_ARG;
  if (M > kMaxRows || D % 8 != 0 || D > jq::kNormMaxD) return JQ_ERR_UNSUPPORTED_SHAPE;
  if (out == JQ_NORM_INT4 && D % 64 != 0) return JQ_ERR_UNSUPPORTED_SHAPE;
  jq_status st = check_stride(x_stride, D);
  if (st == JQ_OK && residual != nullptr) st = check_stride(residual_stride, D);
  if (st == JQ_OK && residual != nullptr) st = check_stride(residual_out_stride, D);
  if (st != JQ_OK) return st;
  if (!aligned(x, 16) || !aligned(residual, 16) || !aligned(weight, 16) || !aligned(y, 16) ||
      !aligned(residual_out, 16) || !aligned(scale, 4))
    return JQ_ERR_MISALIGNED;
  jq::NormArgs a;
  a.x = u16(x), a.res = u16(residual), a.w = u16(weight);
  a.res_out = static_cast<uint16_t*>(residual_out), a.y = y, a.scale = scale;
  a.M = M, a.x_stride = x_stride, a.res_stride = residual_stride, a.res_out_stride = residual_out_stride;
  a.D = static_cast<int>(D), a.eps = eps;
  return from_hip(jq::launch_rmsnorm(a, static_cast<jq::NormOut>(out), as_stream(stream)));
}

jq_status jq_quantize_act_fp8(const void* x_bf16, int64_t x_stride, int64_t M, int64_t K, void* q, float* scale,
                              void* stream) {
  if (q == nullptr || scale == nullptr) return JQ_ERR_INVALID_ARG;
  const jq_status st = check_act(x_bf16, x_stride, M, K);
  if (st != JQ_OK) return st;
  if (!aligned(q, 16) || !aligned(scale, 4)) return JQ_ERR_MISALIGNED;
  return from_hip(jq::launch_quantize_fp8(u16(x_bf16), x_stride, M, K, static_cast<uint8_t*>(q), scale, as_stream(stream)));
}

jq_status jq_pack_weight_fp8(const void* w_bf16, int64_t N, int64_t K, void* wq, float* w_scale, void* stream) {
  if (w_bf16 == nullptr || wq == nullptr || w_scale == nullptr) return JQ_ERR_INVALID_ARG;
  const jq_status st = check_fp8_shape(N, K);
  if (st != JQ_OK) return st;
  // a grid of 2^24 blocks or more would not fit its 32-bit count of threads
  if (((N + 127) / 128) * ((K + 127) / 128) >= (int64_t(1) << 24)) return JQ_ERR_UNSUPPORTED_SHAPE;
  if (!aligned(w_bf16, 16) || !aligned(wq, 16) || !aligned(w_scale, 4)) return JQ_ERR_MISALIGNED;
  return from_hip(jq::launch_pack_fp8(u16(w_bf16), N, K, static_cast<uint8_t*>(wq), w_scale, as_stream(stream)));
}

size_t jq_fp8_workspace_bytes(int64_t M, int64_t K) { return fp8_workspace_bytes(M, K); }

jq_status jq_fp8_gemm(const void* q, const float* scale, int64_t M, int64_t K, const void* wq, const float* w_scale,
                      int64_t N, const void* bias_bf16, void* y_bf16, void* stream) {
  const jq_status st = check_fp8_gemm(q, scale, M, K, wq, w_scale, N, bias_bf16, y_bf16);
  if (st != JQ_OK) return st;
  return from_hip(jq::launch_fp8_gemm(static_cast<const uint8_t*>(q), scale, M, K, static_cast<const uint8_t*>(wq),
                                      w_scale, N, u16(bias_bf16), static_cast<uint16_t*>(y_bf16), as_stream(stream)));
}

int jq_internal_fp8_route(int64_t M, int64_t N, int64_t K, int64_t cus) { return jq::fp8_gemm_route(M, N, K, cus); }

jq_status jq_fp8_linear(const void* x_bf16, int64_t x_stride, int64_t M, int64_t K, const void* wq,
                        const float* w_scale, int64_t N, const void* bias_bf16, void* y_bf16, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (workspace == nullptr) return JQ_ERR_INVALID_ARG;
  jq_status st = check_act(x_bf16, x_stride, M, K);
  if (st != JQ_OK) return st;
  // the activation operands live in the workspace; check the rest with stand-ins
  st = check_fp8_gemm(x_bf16, w_scale, M, K, wq, w_scale, N, bias_bf16, y_bf16);
  if (st != JQ_OK) return st;
  if (!aligned(workspace, kWsAlign)) return JQ_ERR_MISALIGNED;
  if (workspace_bytes < fp8_workspace_bytes(M, K)) return JQ_ERR_WORKSPACE_TOO_SMALL;
  uint8_t* q = static_cast<uint8_t*>(workspace);
  float* s = reinterpret_cast<float*>(q + round_up(static_cast<size_t>(M) * static_cast<size_t>(K), kWsAlign));
  const hipError_t e = jq::launch_quantize_fp8(u16(x_bf16), x_stride, M, K, q, s, as_stream(stream));
  if (e != hipSuccess) return JQ_ERR_HIP;
  return from_hip(jq::launch_fp8_gemm(q, s, M, K, static_cast<const uint8_t*>(wq), w_scale, N, u16(bias_bf16),
                                      static_cast<uint16_t*>(y_bf16), as_stream(stream)));
}

jq_status jq_rope_append(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                         int64_t v_stride, int64_t T, int64_t Hq, int64_t Hk, int64_t D, const int32_t* positions,
                         const float* cos, const float* sin, int64_t P, int64_t R, int interleaved,
                         const int64_t* slots, void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache,
                         float* k_scale, float* v_scale, int64_t num_pages, int64_t page_size, jq_cache_type type,
                         void* stream) {
  if (k == nullptr || v == nullptr || positions == nullptr || slots == nullptr) return JQ_ERR_INVALID_ARG;
  if (T <= 0 || D <= 0 || Hq < 0 || R < 0 || P < 0) return JQ_ERR_INVALID_ARG;
  if ((Hq > 0) != (q != nullptr) || (Hq > 0) != (q_out != nullptr)) return JQ_ERR_INVALID_ARG;
  if (R > 0 && (cos == nullptr || sin == nullptr || P == 0)) return JQ_ERR_INVALID_ARG;
  jq_status st = check_cache(Hk, k_cache, v_cache, k_scale, v_scale, num_pages, page_size, type);
  if (st != JQ_OK) return st;
  if (D % 16 != 0 || D > 256 || R % 16 != 0 || R > D || Hq > 65536) return JQ_ERR_UNSUPPORTED_SHAPE;
  if (T > kMaxRows || T * (Hq + 2 * Hk) >= (int64_t(1) << 31)) return JQ_ERR_UNSUPPORTED_SHAPE;
  st = check_stride(k_stride, Hk * D);
  if (st == JQ_OK) st = check_stride(v_stride, Hk * D);
  if (st == JQ_OK && Hq > 0) st = check_stride(q_stride, Hq * D);
  if (st == JQ_OK && Hq > 0) st = check_stride(q_out_stride, Hq * D);
  if (st != JQ_OK) return st;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(cos, 16) ||
      !aligned(sin, 16) || !aligned(positions, 4) || !aligned(slots, 8))
    return JQ_ERR_MISALIGNED;
  jq::AppendArgs a;
  a.q = u16(q), a.k = u16(k), a.v = u16(v), a.q_out = static_cast<uint16_t*>(q_out);
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.q_out_stride = q_out_stride;
  a.positions = positions, a.cos = cos, a.sin = sin, a.slots = slots;
  a.k_cache = k_cache, a.v_cache = v_cache, a.k_scale = k_scale, a.v_scale = v_scale;
  a.T = T, a.P = P, a.num_slots = num_pages * page_size;
  a.Hq = static_cast<int>(Hq), a.Hk = static_cast<int>(Hk), a.D = static_cast<int>(D), a.R = static_cast<int>(R);
  a.page = static_cast<int>(page_size), a.page_shift = page_shift(page_size);
  a.interleaved = interleaved != 0, a.fp8 = type == JQ_CACHE_FP8;
  return from_hip(jq::launch_rope_append(a, as_stream(stream)));
}

size_t jq_paged_attention_workspace_bytes(int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D, int64_t max_len) {
  return attention_workspace_bytes(B, Tq, Hq, Hk, D, max_len);
}

jq_status jq_paged_attention(const void* q, const void* k_cache, const void* v_cache, const float* k_scale,
                             const float* v_scale, const int32_t* page_table, int64_t table_cols,
                             const int32_t* lens, int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D,
                             int64_t num_pages, int64_t page_size, int64_t max_len, float sm_scale, int causal,
                             jq_cache_type type, void* out, float* lse, void* workspace, size_t workspace_bytes,
                             void* stream) {
  if (q == nullptr || page_table == nullptr || lens == nullptr || out == nullptr || table_cols <= 0)
    return JQ_ERR_INVALID_ARG;
  jq_status st = check_cache(Hk, k_cache, v_cache, k_scale, v_scale, num_pages, page_size, type);
  if (st != JQ_OK) return st;
  st = check_attention(B, Tq, Hq, Hk, D, max_len);
  if (st != JQ_OK) return st;
  if (table_cols > kMaxAxis) return JQ_ERR_UNSUPPORTED_SHAPE;
  if (max_len > table_cols * page_size) return JQ_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(page_table, 4) || !aligned(lens, 4) || !aligned(lse, 4))
    return JQ_ERR_MISALIGNED;
  const size_t need = attention_workspace_bytes(B, Tq, Hq, Hk, D, max_len);
  if (need > 0) {
    if (workspace == nullptr) return JQ_ERR_INVALID_ARG;
    if (!aligned(workspace, kWsAlign)) return JQ_ERR_MISALIGNED;
    if (workspace_bytes < need) return JQ_ERR_WORKSPACE_TOO_SMALL;
  }
  jq::AttnArgs a;
  a.q = u16(q), a.k_cache = k_cache, a.v_cache = v_cache, a.k_scale = k_scale, a.v_scale = v_scale;
  a.table = page_table, a.lens = lens, a.out = static_cast<uint16_t*>(out), a.lse = lse;
  a.ws = static_cast<float*>(workspace), a.num_pages = num_pages;
  a.B = static_cast<int>(B), a.Tq = static_cast<int>(Tq), a.Hq = static_cast<int>(Hq), a.Hk = static_cast<int>(Hk);
  a.D = static_cast<int>(D), a.page_shift = page_shift(page_size), a.table_cols = static_cast<int>(table_cols);
  a.max_len = static_cast<int>(max_len), a.scale = sm_scale, a.causal = causal != 0, a.fp8 = type == JQ_CACHE_FP8;
  return from_hip(jq::launch_paged_attention(a, as_stream(stream)));
}

}  // extern "C"
