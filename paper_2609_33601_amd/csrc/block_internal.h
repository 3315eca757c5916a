// Internal launch interface between the C ABI of the decoder block's other
// operators (include/jq_block.h) and their gfx950 kernels.
#ifndef JQ_BLOCK_INTERNAL_H
#define JQ_BLOCK_INTERNAL_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace jq {

enum class NormOut { kBf16 = 0, kFp8 = 1, kInt4 = 2 };

struct NormArgs {
  const uint16_t* x;
  const uint16_t* res;   // nullptr: no residual
  const uint16_t* w;
  uint16_t* res_out;
  void* y;
  float* scale;
  int64_t M;
  int64_t x_stride, res_stride, res_out_stride;  // elements between rows
  int D;
  float eps;
};
constexpr int64_t kNormMaxD = 65536;
hipError_t launch_rmsnorm(const NormArgs& a, NormOut out, hipStream_t st);

// bf16 [M,K] (rows x_stride apart) -> e4m3 codes [M,K] and scales [M, ceil(K/128)].
hipError_t launch_quantize_fp8(const uint16_t* x, int64_t x_stride, int64_t M, int64_t K, uint8_t* q, float* scale,
                               hipStream_t st);
// bf16 [N,K] -> e4m3 codes [N,K] and scales [ceil(N/128), ceil(K/128)].
hipError_t launch_pack_fp8(const uint16_t* w, int64_t N, int64_t K, uint8_t* q, float* scale, hipStream_t st);

// y = bf16(sum over blocks of 128 k of sx * sw * (codes' product) + bias).
hipError_t launch_fp8_gemm(const uint8_t* qx, const float* sx, int64_t M, int64_t K, const uint8_t* qw,
                           const float* sw, int64_t N, const uint16_t* bias, uint16_t* y, hipStream_t st);
// Which of its kernels an M x K by K x N product takes on `cus` CUs.
int fp8_gemm_route(int64_t M, int64_t N, int64_t K, int64_t cus);

struct AppendArgs {
  const uint16_t *q, *k, *v;
  uint16_t* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;  // elements between tokens
  const int32_t* positions;
  const float *cos, *sin;  // [P, R/2]
  const int64_t* slots;
  void *k_cache, *v_cache;
  float *k_scale, *v_scale;
  int64_t T, P, num_slots;
  int Hq, Hk, D, R, page, page_shift;
  bool interleaved, fp8;
};
hipError_t launch_rope_append(const AppendArgs& a, hipStream_t st);

struct AttnArgs {
  const uint16_t* q;  // [B, Tq, Hq, D]
  const void *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  const int32_t* table;  // [B, table_cols]
  const int32_t* lens;   // [B]
  uint16_t* out;
  float* lse;            // [B, Tq, Hq] or nullptr
  float* ws;
  int64_t num_pages;
  int B, Tq, Hq, Hk, D, page_shift, table_cols, max_len;
  float scale;
  bool causal, fp8;
};
// How the key axis of a call is cut: tokens of a part, the parts of the
// longest sequence, and the query columns (new tokens times heads that share
// a key head) that a block takes.
struct AttnPlan {
  int chunk, parts, cols;
};
AttnPlan attention_plan(int64_t B, int64_t Tq, int64_t Hq, int64_t Hk, int64_t D, int64_t max_len);
hipError_t launch_paged_attention(const AttnArgs& a, hipStream_t st);

}  // namespace jq

// For the tests only (no part of the C ABI): the kernel that a product takes.
extern "C" int jq_internal_fp8_route(int64_t M, int64_t N, int64_t K, int64_t cus);

#endif  // JQ_BLOCK_INTERNAL_H
