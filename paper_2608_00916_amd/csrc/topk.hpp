// Selection of a token's top-k experts by one wave (device side), shared by
// the router and the expert layer for a few tokens.
#pragma once

#include <math.h>

#include "common.hpp"
#include "moe.h"

namespace moe {

// K ranges of the router's product.  One count for every T: it is the order in
// which a token's logits are summed, and a passage must select the same
// experts alone and inside a batch.  16 ranges up to T = 1024, where few
// tokens leave most of the chip idle, took 8.8 us against 12.9 at T = 64 (the
// top-k 1 us more), but a token's logits then differed in their last bits on
// either side of that T.
constexpr int kRouterSplits = 4;
// The k of one range: whole 64-deep steps.
__host__ __device__ constexpr int router_range(int H) { return cdiv(cdiv(H, kRouterSplits), 64) * 64; }

// Order-preserving key of an fp32 value: a > b  <=>  key(a) > key(b), and
// -0 == +0 share a key.
__device__ __forceinline__ uint32_t order_key(float v) {
  uint32_t u = __float_as_uint(v);
  if (v == 0.0f) u = 0u;
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key >> 31) ? (key & 0x7fffffffu) : ~key);
}

__device__ __forceinline__ int ballot_count(bool p) { return __popcll(__ballot(p)); }

// Top-k of one token, held by a wave: lane l holds the logits of experts
// e = l + 64 m, m < PL (key 0 and value 0 where e >= E).  Selection: the k
// largest logits, ties to the lower expert, in slot order (descending logit,
// then ascending expert).  Exact: a radix search for the k-th largest order
// key (each wave-wide count is a ballot and a popcount), then the keys equal
// to it are taken by lower expert index; an entry's slot counts the selected
// keys that beat it, broadcast one by one.  Gates
// g_j = exp(z_j - z_0) / sum_j' exp(z_j' - z_0).  Keys of absent experts are
// 0, below every logit's key, so they never count.  Returns the largest logit.
template <int PL>
__device__ __forceinline__ float topk_select(const float (&val)[PL], const uint32_t (&key)[PL], int k, int lane,
                                             int32_t* __restrict__ idx_row, float* __restrict__ g_row,
                                             int32_t* __restrict__ cnt_row) {
  uint32_t kth = 0u;  // largest P with #{key >= P} >= k, or the first found with k
  for (int b = 31; b >= 0; --b) {
    const uint32_t cand = kth | (1u << b);
    int cnt = 0;
#pragma unroll
    for (int m = 0; m < PL; ++m) cnt += ballot_count(key[m] >= cand);
    kth = cnt >= k ? cand : kth;
    if (cnt == k) break;  // exactly the k largest reach it: no lower bit changes the selection
  }
  int above = 0;
#pragma unroll
  for (int m = 0; m < PL; ++m) above += ballot_count(key[m] > kth);
  const int need = k - above;  // entries equal to the k-th key, by lower expert index
  const unsigned long long below = (1ull << lane) - 1ull;
  bool sel[PL];
  unsigned long long selmask[PL];
  int eq_before = 0;
#pragma unroll
  for (int m = 0; m < PL; ++m) {
    const unsigned long long eq = __ballot(key[m] == kth);
    const int rank_eq = eq_before + __popcll(eq & below);
    eq_before += __popcll(eq);
    sel[m] = key[m] > kth || (key[m] == kth && rank_eq < need);
    selmask[m] = __ballot(sel[m]);
  }
  int slot[PL];
#pragma unroll
  for (int m = 0; m < PL; ++m) slot[m] = 0;
  uint32_t kmax = 0u;
#pragma unroll
  for (int mj = 0; mj < PL; ++mj) {
    unsigned long long msk = selmask[mj];
    while (msk != 0ull) {
      const int lj = __builtin_ctzll(msk);
      msk &= msk - 1ull;
      const uint32_t kj = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(key[mj]), lj));
      const int ej = lj + kWave * mj;
      kmax = kj > kmax ? kj : kmax;
#pragma unroll
      for (int m = 0; m < PL; ++m) {
        const int e = lane + kWave * m;
        slot[m] += (sel[m] && (kj > key[m] || (kj == key[m] && ej < e))) ? 1 : 0;
      }
    }
  }
  const float top = key_value(kmax);
  float w = 0.0f;
  float wm[PL];
#pragma unroll
  for (int m = 0; m < PL; ++m) {
    wm[m] = sel[m] ? expf(val[m] - top) : 0.0f;
    w += wm[m];
  }
  const float sum = wave_sum(w);
#pragma unroll
  for (int m = 0; m < PL; ++m)
    if (sel[m]) {
      idx_row[slot[m]] = lane + kWave * m;
      g_row[slot[m]] = wm[m] / sum;
      atomicAdd(cnt_row + lane + kWave * m, 1);
    }
  return top;
}

}  // namespace moe
