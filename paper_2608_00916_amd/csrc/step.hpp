// Internal launchers of a decoding step's kernels around attention and the
// products: norms, the expert layer for a few tokens, token sampling (host
// side).  Not part of the C ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"
#include "moe.h"

namespace moe {

// ---- residual sum and root-mean-square norm (norm.hip)
struct NormFwd {
  const bf16_t *x, *r;  // r null: no residual
  int64_t ldx, ldr;
  const bf16_t* w;
  bf16_t *h, *y;  // either may be null
  int8_t* q;      // may be null
  float* scale;
  int T, H;
  float eps;
};
hipError_t launch_norm_fwd(const NormFwd& a, hipStream_t s);

struct NormBwd {
  const bf16_t *h, *dy, *dh;  // dh null: no gradient of the sum from elsewhere
  int64_t ldh, lddy, lddh;
  const bf16_t* w;
  bf16_t* dx;
  void* dw;  // fp32 or bf16
  bool dw_fp32;
  float* part;  // norm_bwd_parts(T, H) rows of H
  int T, H;
  float eps;
};
int norm_bwd_parts(int T, int H);
hipError_t launch_norm_bwd(const NormBwd& a, hipStream_t s);

// ---- the expert layer for a few tokens (decode.hip)
constexpr int kDecodeMaxT = MOE_DECODE_MAX_T;
constexpr int kDecodeParts = 3;  // bf16 summands of a value of the activation

// A routed row is named by its slot t k + j.
struct DecodeRows {
  const uint8_t* mask;  // may be null
  float* part;          // [splits, T, E] the router's sums over its ranges of K
  int32_t* topk_idx;    // [T, k]
  float* gates;         // [T, k]
  int32_t* counts;      // [E]
  int T, H, E, F, k;
};
// part, counts = 0 and, with q, the tokens' int8 rows.
hipError_t launch_decode_router(const DecodeRows& r, const bf16_t* x, const bf16_t* w_r, int8_t* q, float* sx,
                                hipStream_t s);
// Whether the gate/up product makes the selection (topk_idx, gates, counts)
// from part; else it is there before.
constexpr int kDecodeFusedT = 8;
inline bool decode_fused(int T) { return T <= kDecodeFusedT; }
// SwiGLU of the slots' tokens through their experts: a [kDecodeParts, T k, F] as
// summands, or with decode_ranges(..) > 1 each range's G and U, gu [ranges, 2, T k, F].
int decode_ranges(int T, int E, int F, int k);
hipError_t launch_decode_gateup(const DecodeRows& r, const bf16_t* x, const bf16_t* w_gate, const bf16_t* w_up,
                                bf16_t* a, float* gu, hipStream_t s);
// a [T k, F], top [T k, F / 16] the largest magnitudes of 16 columns each.
hipError_t launch_decode_gateup_i8(const DecodeRows& r, const int8_t* x, const float* sx, const moe_i8_experts& w,
                                   float* a, float* top, hipStream_t s);
// o [T k, H] = the activation through W_down (a8, sa: room for its int8 rows).
hipError_t launch_decode_down(const DecodeRows& r, const bf16_t* a, const float* gu, const bf16_t* w_down, float* o,
                              hipStream_t s);
hipError_t launch_decode_down_i8(const DecodeRows& r, const float* a, const float* top, int8_t* a8, float* sa,
                                 const moe_i8_experts& w, float* o, hipStream_t s);
// y [T, H] = sum_j gates o.
hipError_t launch_decode_combine(const DecodeRows& r, const float* o, bf16_t* y, hipStream_t s);

// ---- token sampling (sample.hip)
struct SampleArgs {
  const void* logits;
  int64_t ld;
  bool fp32;
  int B, V;
  const float *temperature, *top_p, *min_p;  // any may be null: off
  const int32_t* top_k;
  const float* u;
  int32_t* token;
  float* logprob;  // may be null
};
size_t sample_ws(int B, int V);
hipError_t launch_sample(const SampleArgs& a, void* ws, hipStream_t s);

}  // namespace moe
