// Internal launchers of the 8-bit serving kernels (host side).  Not part of
// the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "moe.h"

namespace moe {

// ---- int8 rows (i8_quant.hip)
// q, scale of `rows` bf16 rows; with n_valid (device) rows from *n_valid on
// are left alone.
hipError_t launch_i8_quant_rows(const bf16_t* x, int64_t ldx, int rows, int K, const int32_t* n_valid, int8_t* q,
                                float* scale, hipStream_t s);
// The same from the SwiGLU activation as the gate/up product leaves it: a
// [rows, F], a_top [rows, F / kI8Cols].
hipError_t launch_i8_requant(const float* a, const float* a_top, int rows, int F, const int32_t* n_valid, int8_t* q,
                             float* scale, hipStream_t s);
// w [E, K, N] bf16 -> q [E, N, K], scale [E, N].
hipError_t launch_i8_quant_weight(const bf16_t* w, int E, int K, int N, int8_t* q, float* scale, hipStream_t s);

// ---- products of int8 rows (i8_gemm.hip)
// out[m][n] = sa[m] sb[n] <a[m], b[n]>, bf16 or fp32.
hipError_t launch_i8_matmul(const int8_t* a, const float* sa, const int8_t* b, const float* sb, int M, int N, int K,
                            void* out, int64_t ldo, bool f32, hipStream_t s);

// The same from a few bf16 rows, rounded to int8 on the way; false (and
// nothing launched) where there are more than that takes.
bool launch_i8_linear_fused(const bf16_t* x, int64_t ldx, const int8_t* b, const float* sb, int M, int N, int K,
                            void* out, int64_t ldo, bool f32, hipStream_t s);

// Rows grouped by expert: expert e's are offsets[e] .. offsets[e + 1].
struct I8Rows {
  int rows_cap, E;
  const int32_t* offsets;
};
// Columns of one partial of the SwiGLU activation.
constexpr int kI8Cols = 32;
// A = silu(G) U of each routed row (x row rows[r], or r where rows is null),
// and the largest magnitude among each kI8Cols columns (a_top).
hipError_t launch_i8_gateup(const I8Rows& r, const int8_t* x, const float* sx, const int32_t* rows,
                            const moe_i8_experts& w, int H, int F, float* a, float* a_top, hipStream_t s);
// O = A W_down.
hipError_t launch_i8_down(const I8Rows& r, const int8_t* a, const float* sa, const moe_i8_experts& w, int H, int F,
                          bf16_t* o, hipStream_t s);

// ---- the paged cache (kv_cache.hip)
hipError_t launch_kv_plan(const moe_kv_plan_dims& d, const int32_t* old_len, const int32_t* new_len,
                          int32_t* block_table, const int32_t* free_ids, const int32_t* n_free, int32_t* row_start,
                          int32_t* kv_len, int32_t* positions, int32_t* slots, int32_t* seq, int32_t* state,
                          hipStream_t s);
hipError_t launch_kv_append(const moe_kv_cache& c, const moe_kv_batch& b, const bf16_t* k, const bf16_t* v, int64_t ld,
                            hipStream_t s);
hipError_t launch_kv_read(const moe_kv_cache& c, int B, int W, const int32_t* block_table, const int32_t* kv_start,
                          int total, bf16_t* k_out, bf16_t* v_out, hipStream_t s);

// ---- attention over it (kv_attention.hip)
size_t kv_attention_ws(const moe_kv_cache& c, const moe_kv_batch& b, const moe_kv_attn& a);
hipError_t launch_kv_attention(const moe_kv_cache& c, const moe_kv_batch& b, const moe_kv_attn& a, const bf16_t* q,
                               int64_t ldq, bf16_t* out, int64_t ldo, void* ws, hipStream_t s);

}  // namespace moe
