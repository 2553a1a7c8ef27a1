// The expert layer for a few tokens.  Reading the weights of the experts that
// the tokens picked bounds it: at one token and top-8 of a 30B-A3B model 75 MB
// in bf16 for 75 MFLOP.  So every weight goes from memory straight into the
// registers of the one wave that multiplies it, in whole 128-byte lines and
// with as many of them in flight as registers hold, and the K axis is split
// over a workgroup's waves until the (expert, columns) tiles fill the chip.
//
// A workgroup takes one used expert and a tile of columns, finds the expert's
// rows (at most one per token) from the selection by itself, and multiplies
// them 16 at a time on the matrix cores: 16 rows are the least that an
// instruction takes, and the weights have to be read for one as for 16.
#include <algorithm>
#include <type_traits>

#include "i8_core.hpp"
#include "i8_round.hpp"
#include "step.hpp"
#include "topk.hpp"
#include "trace.hpp"

namespace moe {

namespace {

// An address as a wave's base and a lane's 32-bit offset, the form that leaves
// the address arithmetic to the scalar unit.
template <class T>
__device__ __forceinline__ const char* at_bytes(const T* base, uint32_t offset) {
  return reinterpret_cast<const char*>(base) + offset;
}
__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// ---- router
// Logits in the router's own order of summation, so that the selection is
// moe_infer's bit for bit: range s of K goes through the same instructions in
// the same order into plane s of part [kRouterSplits, T, E].  A workgroup of
// one wave takes one range, 32 experts and 16 tokens, its loads all issued ahead
// of the products: what one compute unit can fetch bounds it.  Further
// workgroups round the tokens to int8 rows (q null: none), work that needs no
// launch of its own.
constexpr int kRouterCols = 32;
__global__ __launch_bounds__(kWave, 1) void k_decode_router(const bf16_t* __restrict__ x,
                                                                        const bf16_t* __restrict__ w_r, int T, int H,
                                                                        int E, float* __restrict__ part,
                                                                        int32_t* __restrict__ counts,
                                                                        int8_t* __restrict__ q, float* __restrict__ sx) {
  const int lane = threadIdx.x;
  const int cols = cdiv(E, kRouterCols), tiles = cols * cdiv(T, 16);
  if (static_cast<int>(blockIdx.x) >= tiles * kRouterSplits) {  // a token's int8 row
    const int t = blockIdx.x - tiles * kRouterSplits;
    const bf16_t* src = x + static_cast<int64_t>(t) * H;
    uint32_t m = 0;
    for (int c = lane * 8; c < H; c += 512) m = max(m, top8(*reinterpret_cast<const uint4*>(src + c)));
    const Rounder r(wave_umax(m));
    for (int c = lane * 8; c < H; c += 512)
      *reinterpret_cast<uint2*>(q + static_cast<int64_t>(t) * H + c) = quant8(*reinterpret_cast<const uint4*>(src + c), r);
    if (lane == 0) sx[t] = r.scale;
    return;
  }
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < E; i += blockDim.x) counts[i] = 0;
  const int split = blockIdx.x / tiles, tile = blockIdx.x % tiles;
  const int e0 = tile % cols * kRouterCols + (lane & 15) * 2, t = tile / cols * 16 + (lane & 15);
  const int quad = (lane >> 4) * 8;
  const int range = router_range(H), k0 = min(H, split * range), k1 = min(H, k0 + range);
  const bool in_e = e0 < E, in_t = t < T;  // E is even
  f32x4 acc[2] = {};
  constexpr int U = 16;  // a range of H = 2048 at once: the latency of one access bounds it
  // lanes past the experts or the tokens read the first ones; what they hold is not stored
  const uint32_t w_at = static_cast<uint32_t>(quad * E + (in_e ? e0 : 0)) * 2, x_at = static_cast<uint32_t>(quad) * 2;
  const bf16_t* const x_row = x + static_cast<int64_t>(in_t ? t : 0) * H;
  for (int k = k0; k < k1; k += U * 32) {
    uint32_t w[U][8];
    uint4 xv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k + u * 32 >= k1) break;
      xv[u] = *reinterpret_cast<const uint4*>(at_bytes(x_row + k + u * 32, x_at));
#pragma unroll
      for (int r = 0; r < 8; ++r)
        w[u][r] = *reinterpret_cast<const uint32_t*>(at_bytes(w_r + static_cast<int64_t>(k + u * 32 + r) * E, w_at));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k + u * 32 >= k1) break;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        uint32_t c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          c[i] = __builtin_amdgcn_perm(w[u][2 * i + 1], w[u][2 * i], p ? 0x07060302u : 0x05040100u);
        acc[p] = mfma16x16x32(make_uint4(c[0], c[1], c[2], c[3]), xv[u], acc[p]);
      }
    }
  }
  // lane l holds experts 2 (4 (l / 16) + i) + p of the tile for token l % 16
  if (!in_t) return;
  float* out = part + (static_cast<int64_t>(split) * T + t) * E;
  const int first = tile % cols * kRouterCols + 8 * (lane >> 4);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (first + 2 * i < E) *reinterpret_cast<float2*>(out + first + 2 * i) = make_float2(acc[0][i], acc[1][i]);
}

// ---- which rows a workgroup has
struct Rows {
  int32_t slot[kDecodeMaxT];  // of the expert, in token order
  int expert, n;
};
// The blockIdx.y-th used expert and its slots; one wave finds them.
__device__ __forceinline__ void find_rows(const DecodeRows& r, const int32_t* counts, const int32_t* topk_idx, Rows& rows) {
  const int lane = threadIdx.x;
  if (r.T == 1) {  // the slots are the experts
    if (lane == 0) {
      rows.slot[0] = blockIdx.y;
      rows.expert = topk_idx[blockIdx.y];
      rows.n = 1;
    }
    return;
  }
  int e = -1, before = 0;
  const int want = blockIdx.y;
  for (int m = 0; m < r.E; m += kWave) {
    const unsigned long long used = __ballot(m + lane < r.E && counts[min(m + lane, r.E - 1)] > 0);
    const int n = __popcll(used);
    if (e < 0 && want < before + n) {
      unsigned long long u = used;
      for (int i = before; i < want; ++i) u &= u - 1ull;
      e = m + __builtin_ctzll(u);
    }
    before += n;
  }
  int slot = -1;
  if (e >= 0 && lane < r.T)
    for (int j = 0; j < r.k; ++j)
      if (topk_idx[lane * r.k + j] == e) slot = lane * r.k + j;
  const unsigned long long has = __ballot(slot >= 0);
  if (slot >= 0) rows.slot[__popcll(has & ((1ull << lane) - 1ull))] = slot;
  if (lane == 0) {
    rows.expert = e;
    rows.n = __popcll(has);
  }
}
__device__ __forceinline__ bool read_rows(const DecodeRows& r, Rows& rows) {
  if (threadIdx.x < kWave) find_rows(r, r.counts, r.topk_idx, rows);
  __syncthreads();
  return rows.expert >= 0;
}

// Selection of up to kFusedT tokens by every workgroup of the gate/up product
// for itself, a wave per token, instead of a launch between the router and it;
// the first workgroup leaves it for the launches after.
constexpr int kFusedT = kDecodeFusedT;
struct Selection {
  int32_t idx[kFusedT * MOE_MAX_TOPK];
  float gates[kFusedT * MOE_MAX_TOPK];
  int32_t counts[MOE_MAX_EXPERTS];
};
template <int PL>
__device__ __forceinline__ void select_token(const DecodeRows& r, int t, Selection& sel) {
  const int lane = threadIdx.x & 63;
  float val[PL];
  uint32_t key[PL];
#pragma unroll
  for (int m = 0; m < PL; ++m) {
    const int e = lane + kWave * m;
    float v[kRouterSplits];
#pragma unroll
    for (int s = 0; s < kRouterSplits; ++s) v[s] = e < r.E ? r.part[(static_cast<int64_t>(s) * r.T + t) * r.E + e] : 0.0f;
    val[m] = v[0];
#pragma unroll
    for (int s = 1; s < kRouterSplits; ++s) val[m] += v[s];
    key[m] = e < r.E ? max(order_key(val[m]), 1u) : 0u;
  }
  topk_select<PL>(val, key, r.k, lane, sel.idx + t * r.k, sel.gates + t * r.k, sel.counts);
}
__device__ __forceinline__ bool select_rows(const DecodeRows& r, Selection& sel, Rows& rows) {
  const int tid = threadIdx.x, wave = tid >> 6;
  for (int i = tid; i < r.E; i += blockDim.x) sel.counts[i] = 0;
  __syncthreads();
  for (int t = wave; t < r.T; t += blockDim.x / kWave) {
    if (r.mask != nullptr && r.mask[t] == 0) {
      if ((tid & 63) < r.k) {
        sel.idx[t * r.k + (tid & 63)] = -1;
        sel.gates[t * r.k + (tid & 63)] = 0.0f;
      }
    } else if (r.E <= kWave) {
      select_token<1>(r, t, sel);
    } else if (r.E <= 2 * kWave) {
      select_token<2>(r, t, sel);
    } else {
      select_token<4>(r, t, sel);
    }
  }
  __syncthreads();
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) {
    for (int i = tid; i < r.T * r.k; i += blockDim.x) {
      r.topk_idx[i] = sel.idx[i];
      r.gates[i] = sel.gates[i];
    }
    for (int i = tid; i < r.E; i += blockDim.x) r.counts[i] = sel.counts[i];
  }
  if (tid < kWave) find_rows(r, sel.counts, sel.idx, rows);
  __syncthreads();
  return rows.expert >= 0;
}

// ---- bf16 products
// Eight K rows of a lane's four columns -> the matrix instruction's operand
// for column p of each lane: eight K values of one column.
__device__ __forceinline__ uint4 column(const uint2 (&v)[8], int p) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = p < 2 ? v[2 * i].x : v[2 * i].y, b = p < 2 ? v[2 * i + 1].x : v[2 * i + 1].y;
    w[i] = __builtin_amdgcn_perm(b, a, p & 1 ? 0x07060302u : 0x05040100u);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint2 stream8(const char* p) {
  typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p)));
}

// Columns of a tile: lane l holds columns 4 (l % 16) + p, so a load of 8 bytes
// a lane brings four rows of a whole 128-byte line.  Two columns a lane, half
// lines, reached 3.2 TB/s where these reach 5.6 (16 tokens).
constexpr int kCols = 64;

// Products of 16 NT rows with NB column-contiguous matrices [K, N] at their
// pointers' columns, steps s0, s0 + stride, ... < s1 of 32 k, U of them in
// flight.  get(t, k, parts) gives the PARTS summands of row tile t's operand;
// begin() comes after the first weights' loads and before the first get.
template <int NT, int NB, int PARTS, int U, class Begin, class Get>
__device__ __forceinline__ void few_rows(const bf16_t* const (&b)[NB], int N, int s0, int s1, int stride, Begin& begin,
                                         const Get& get, f32x4 (&acc)[NT][NB][4]) {
  const int lane = threadIdx.x & 63;
  const int quad = (lane >> 4) * 8;
  const uint32_t at = (static_cast<uint32_t>(quad) * N + (lane & 15) * 4) * 2;  // N <= 2^24
  auto batch = [&](int s, auto count) {
    constexpr int n = decltype(count)::value;
    uint2 v[n][NB][8];
    uint4 xv[n][NT][PARTS];
#pragma unroll
    for (int u = 0; u < n; ++u) {
      const int k = (s + u * stride) * 32;
#pragma unroll
      for (int m = 0; m < NB; ++m)
#pragma unroll
        for (int r = 0; r < 8; ++r) v[u][m][r] = stream8(at_bytes(b[m] + static_cast<int64_t>(k + r) * N, at));
    }
    begin();
#pragma unroll
    for (int u = 0; u < n; ++u)
#pragma unroll
      for (int t = 0; t < NT; ++t) get(t, (s + u * stride) * 32 + quad, xv[u][t]);
#pragma unroll
    for (int u = 0; u < n; ++u)
#pragma unroll
      for (int m = 0; m < NB; ++m)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const uint4 w = column(v[u][m], p);
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < PARTS; ++i) acc[t][m][p] = mfma16x16x32(xv[u][t][i], w, acc[t][m][p]);
        }
  };
  int s = s0;
  for (; s + (U - 1) * stride < s1; s += U * stride) batch(s, std::integral_constant<int, U>{});
  for (; s < s1; s += stride) batch(s, std::integral_constant<int, 1>{});
}

// Sum over the waves of one row tile's products, which each holds per lane as
// f32x4 (or i32x4): element i of lane l, fragment f.  `red` has
// WAVES * FRAGS * 256 entries.
template <int FRAGS, class V4, class S>
__device__ __forceinline__ void put_parts(const V4 (&part)[FRAGS], S* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int f = 0; f < FRAGS; ++f) *reinterpret_cast<V4*>(red + ((wave * FRAGS + f) * kWave + lane) * 4) = part[f];
}
template <int WAVES, int FRAGS, class S>
__device__ __forceinline__ S sum_parts(const S* red, int f, int at) {
  S t = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) t += red[(w * FRAGS + f) * 256 + at];
  return t;
}
// Row and column (of 64, or of 16) of entry `at` of fragment p.
__device__ __forceinline__ int entry_row(int at) { return 4 * (at >> 6) + (at & 3); }
__device__ __forceinline__ int entry_lane(int at) { return (at >> 2) & 15; }

// The activation as three bf16, each the upper half of what those before it
// leave: 3 x 8 bits are all of an fp32, so A enters the down product as it is, at
// the price of two more matrix instructions under the same weights.  Two, rounded
// (2^-17 of A), moved the output by 2.4e-6 of its norm before its rounding to bf16,
// where fp32 sums move it by 4e-7.
//
// All three have A's sign and none is zero where A is not, so that an infinite
// weight meets them as it meets A (a zero would make NaN of it): where nothing is
// left a summand is 2^-26 of A's power of two (2^-126 where that is less), below
// the last bit of an fp32.  All three are infinite, or NaN, where A is; a NaN comes
// from arithmetic, quiet, so its upper half is one.
struct Split {
  bf16_t part[kDecodeParts];
  __device__ __forceinline__ explicit Split(float v) {
    const uint32_t all = __float_as_uint(v), exponent = all >> 23 & 0xff;
    const bool some = (all & 0x7fff0000u) != 0;
    const bf16_t least = some ? (all >> 16 & 0x8000u) | (exponent > 27 ? exponent - 26 : 1) << 7 : 0;
#pragma unroll
    for (int i = 0; i < kDecodeParts; ++i) {
      const uint32_t bits = __float_as_uint(v);
      part[i] = i == 0 || exponent == 0xff ? all >> 16 : (bits & 0x7fff0000u) != 0 ? bits >> 16 : least;
      v -= __uint_as_float(bits & 0xffff0000u);
    }
  }
};

// Waves per workgroup: the gate/up product splits a long K (H), the down
// product a shorter one (F).
constexpr int kUpWaves = 8, kDownWaves = 4;

// gridDim.z ranges of K: 1 where the tiles fill the chip, and the activation
// is written; else a range's G and U are, and the down product adds them up.
template <int NT, int U>
__device__ __forceinline__ void gateup_tiles(const DecodeRows& r, const Rows& rows, int first, const bf16_t* __restrict__ x,
                                             const bf16_t* const (&b)[2], bf16_t* __restrict__ a, float* __restrict__ gu,
                                             float* red) {
  const int lane = threadIdx.x & 63, wave = wave_index(), n = rows.n;
  const bf16_t* xr[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int i = first + t * 16 + (lane & 15);
    xr[t] = i < n ? x + static_cast<int64_t>(rows.slot[i] / r.k) * r.H : nullptr;
  }
  auto get = [&](int t, int k, uint4 (&v)[1]) {
    v[0] = xr[t] != nullptr ? *reinterpret_cast<const uint4*>(xr[t] + k) : make_uint4(0, 0, 0, 0);
  };
  f32x4 acc[NT][2][4] = {};
  auto begin = [] {};
  few_rows<NT, 2, 1, U>(b, r.F, blockIdx.z * kUpWaves + wave, r.H / 32, gridDim.z * kUpWaves, begin, get, acc);
  const int64_t R = static_cast<int64_t>(r.T) * r.k;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (first + t * 16 >= n) break;
    __syncthreads();  // the last tile has been read
    f32x4 part[8];
#pragma unroll
    for (int f = 0; f < 8; ++f) part[f] = acc[t][f / 4][f % 4];
    put_parts(part, red);
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * 256; i += kUpWaves * kWave) {
      const int p = i >> 8, at = i & 255, m = first + t * 16 + entry_row(at);
      if (m >= n) continue;
      const float g = sum_parts<kUpWaves, 8>(red, p, at), u = sum_parts<kUpWaves, 8>(red, 4 + p, at);
      const int64_t to = static_cast<int64_t>(rows.slot[m]) * r.F + blockIdx.x * kCols + entry_lane(at) * 4 + p;
      if (gridDim.z == 1) {
        const Split s(silu_f(g) * u);
#pragma unroll
        for (int j = 0; j < kDecodeParts; ++j) a[to + j * R * r.F] = s.part[j];
      } else {
        gu[to + 2 * blockIdx.z * R * r.F] = g;
        gu[to + (2 * blockIdx.z + 1) * R * r.F] = u;
      }
    }
  }
}

// With ranges of K there is at most one workgroup per compute unit: four steps'
// weights in flight a wave instead of two workgroups.
template <bool FUSED, bool RANGES>
__global__ __launch_bounds__(kUpWaves* kWave, RANGES ? 2 : 4) void k_decode_gateup(DecodeRows r, const bf16_t* __restrict__ x,
                                                                   const bf16_t* __restrict__ w_gate,
                                                                   const bf16_t* __restrict__ w_up,
                                                                   bf16_t* __restrict__ a, float* __restrict__ gu) {
  __shared__ Rows rows;
  __shared__ __attribute__((aligned(16))) float red[kUpWaves * 8 * 256];
  if constexpr (FUSED) {
    __shared__ Selection sel;
    if (!select_rows(r, sel, rows)) return;
  } else {
    if (!read_rows(r, rows)) return;
  }
  const int64_t base = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(rows.expert)) * r.H * r.F + blockIdx.x * kCols;
  const bf16_t* const b[2] = {w_gate + base, w_up + base};
  // more than 16 rows in pairs of tiles: what comes in again then is few experts' weights
  if (FUSED || rows.n <= 16) {
    gateup_tiles<1, RANGES ? 4 : 2>(r, rows, 0, x, b, a, gu, red);
  } else {
    for (int t = 0; t < rows.n; t += 32) gateup_tiles<2, 1>(r, rows, t, x, b, a, gu, red);
  }
}

// The activation comes from a, or (RANGES) from LDS, act [rows][kDecodeParts][F].
template <int NT, bool RANGES>
__device__ __forceinline__ void down_tiles(const DecodeRows& r, const Rows& rows, int first, const bf16_t* __restrict__ a,
                                           const float* __restrict__ gu, const bf16_t* const (&b)[1],
                                           float* __restrict__ o, bf16_t* act, float* red) {
  const int lane = threadIdx.x & 63, wave = wave_index(), n = rows.n;
  const int64_t RF = static_cast<int64_t>(r.T) * r.k * r.F;
  int64_t row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int i = first + t * 16 + (lane & 15);
    row[t] = i >= n ? -1 : RANGES ? kDecodeParts * i * r.F : static_cast<int64_t>(rows.slot[i]) * r.F;
  }
  auto get = [&](int t, int k, uint4 (&v)[kDecodeParts]) {
    const bf16_t* src = (RANGES ? act : a) + row[t] + k;
#pragma unroll
    for (int i = 0; i < kDecodeParts; ++i)
      v[i] = row[t] >= 0 ? *reinterpret_cast<const uint4*>(src + i * (RANGES ? r.F : RF)) : make_uint4(0, 0, 0, 0);
  };
  // the ranges' sums and SwiGLU, under the first weights' way here
  bool begun = false;
  auto begin = [&] {
    if (!RANGES || begun) return;
    begun = true;
    for (int i = threadIdx.x; i < n * r.F; i += kDownWaves * kWave) {
      const int m = i / r.F, c = i % r.F;
      const float* src = gu + static_cast<int64_t>(rows.slot[m]) * r.F + c;
      const float g = src[0] + src[2 * RF], u = src[RF] + src[3 * RF];
      const Split s(silu_f(g) * u);
#pragma unroll
      for (int j = 0; j < kDecodeParts; ++j) act[(kDecodeParts * m + j) * r.F + c] = s.part[j];
    }
    __syncthreads();
  };
  f32x4 acc[NT][1][4] = {};
  few_rows<NT, 1, kDecodeParts, RANGES ? 6 : NT == 1 ? 2 : 1>(b, r.H, wave, r.F / 32, kDownWaves, begin, get, acc);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (first + t * 16 >= n) break;
    __syncthreads();  // the last tile has been read
    put_parts(acc[t][0], red);
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * 256; i += kDownWaves * kWave) {
      const int p = i >> 8, at = i & 255, m = first + t * 16 + entry_row(at);
      if (m < n)
        o[static_cast<int64_t>(rows.slot[m]) * r.H + blockIdx.x * kCols + entry_lane(at) * 4 + p] =
            sum_parts<kDownWaves, 4>(red, p, at);
    }
  }
}

// Four waves per SIMD hold a pair of tiles in registers; five spilled 68 bytes a
// lane (64 tokens: 223 us, 227 with them).
template <bool RANGES>
__global__ __launch_bounds__(kDownWaves* kWave, RANGES ? 2 : 4) void k_decode_down(DecodeRows r, const bf16_t* __restrict__ a,
                                                                   const float* __restrict__ gu,
                                                                   const bf16_t* __restrict__ w_down,
                                                                   float* __restrict__ o) {
  __shared__ Rows rows;
  __shared__ __attribute__((aligned(16))) float red[kDownWaves * 4 * 256];
  if (!read_rows(r, rows)) return;
  const bf16_t* const b[1] = {w_down + static_cast<int64_t>(__builtin_amdgcn_readfirstlane(rows.expert)) * r.H * r.F + blockIdx.x * kCols};
  extern __shared__ __attribute__((aligned(16))) bf16_t act[];  // [rows][kDecodeParts][F]
  if (RANGES || rows.n <= 16) {
    down_tiles<1, RANGES>(r, rows, 0, a, gu, b, o, act, red);
  } else {
    for (int t = 0; t < rows.n; t += 32) down_tiles<2, RANGES>(r, rows, t, a, gu, b, o, act, red);
  }
}

// ---- int8 weights.  They are K-contiguous, and the instruction takes 16
// bytes of channel l % 16 per lane, half a line of each of 16 channels: the down
// product (rows of F) loads them so.  The gate/up product (rows of H, longer
// than a wave's share) brings whole 128-byte lines of 8 channels by a load, lane
// l the bytes 16 c of channel l % 8, c = l / 16 and 4 more in the upper half of
// 16 lanes; two such loads, of channels 0 .. 7 and 8 .. 15, become two operands by
// an exchange between the halves.  With that its loads can pass the caches: 77 ->
// 66 us at 64 tokens (6.0 TB/s), where half lines lose their other half.  The down
// product lost by it (48 -> 53 us).
__device__ __forceinline__ uint32_t line_at(int K) {  // K <= 2^17
  const int lane = threadIdx.x & 63;
  return static_cast<uint32_t>(lane & 7) * K + ((lane >> 4) + 4 * ((lane >> 3) & 1)) * 16;
}
__device__ __forceinline__ uint32_t with_upper(uint32_t a, uint32_t b) {  // lanes 8 .. 15 of 16: b of 8 lanes below
  return __builtin_amdgcn_update_dpp(a, b, 0x128, 0xf, 0xc, false);
}
__device__ __forceinline__ uint32_t with_lower(uint32_t b, uint32_t a) {  // lanes 0 .. 7 of 16: a of 8 lanes above
  return __builtin_amdgcn_update_dpp(b, a, 0x128, 0xf, 0x3, false);
}
__device__ __forceinline__ void to_operands(uint4& a, uint4& b) {
  const uint4 u = a, v = b;
  a = make_uint4(with_upper(u.x, v.x), with_upper(u.y, v.y), with_upper(u.z, v.z), with_upper(u.w, v.w));
  b = make_uint4(with_lower(v.x, u.x), with_lower(v.y, u.y), with_lower(v.z, u.z), with_lower(v.w, u.w));
}

// Products of 16 NT int8 rows (pointers at the lane's row and quarter) with 16
// channels of NB matrices of pitch K (pointers at the first), units u0, u0 + stride, ... < u1 of 128 k, U of
// them in flight; begin() as in few_rows.
template <int NT, int NB, int U, bool LINES, class Begin>
__device__ __forceinline__ void few_rows_i8(const int8_t* const (&b)[NB], int K, const int8_t* const (&x)[NT], int u0,
                                            int u1, int stride, Begin& begin, i32x4 (&acc)[NT][NB]) {
  const int lane = threadIdx.x & 63;
  const uint32_t at = LINES ? line_at(K) : static_cast<uint32_t>(lane & 15) * K + (lane >> 4) * 16;
  auto batch = [&](int unit, auto count) {
    constexpr int n = decltype(count)::value;
    uint4 w[n][2][NB], v[n][2][NT];
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int m = 0; m < NB; ++m) {
          const int8_t* const from = b[m] + (unit + i * stride) * 128;
          if constexpr (LINES) w[i][h][m] = load_nt(at_bytes(from + static_cast<int64_t>(8 * h) * K, at));
          else w[i][h][m] = *reinterpret_cast<const uint4*>(at_bytes(from + 64 * h, at));
        }
    begin();
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          v[i][h][t] = x[t] != nullptr ? *reinterpret_cast<const uint4*>(x[t] + (unit + i * stride) * 128 + h * 64)
                                       : make_uint4(0, 0, 0, 0);
    if constexpr (LINES)
#pragma unroll
      for (int i = 0; i < n; ++i)
#pragma unroll
        for (int m = 0; m < NB; ++m) to_operands(w[i][0][m], w[i][1][m]);
#pragma unroll
    for (int i = 0; i < n; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int m = 0; m < NB; ++m) acc[t][m] = mfma_i8(v[i][h][t], w[i][h][m], acc[t][m]);
  };
  int unit = u0;
  for (; unit + (U - 1) * stride < u1; unit += U * stride) batch(unit, std::integral_constant<int, U>{});
  for (; unit < u1; unit += stride) batch(unit, std::integral_constant<int, 1>{});
}

// Where the tiles are many, short workgroups of which many fit a compute unit:
// two waves and one unit of k in flight in each (eight waves took 1.3 times as
// long at 16 tokens).  Where they are so few that a compute unit has four at
// most, eight waves with all of K in flight at once.
constexpr int kUpWaves8 = 2, kUpWaves8Few = 8, kDownWaves8 = 4;

template <int NT, int WAVES, int U>
__device__ __forceinline__ void gateup_tiles_i8(const DecodeRows& r, const Rows& rows, int first,
                                                const int8_t* __restrict__ x, const float* __restrict__ sx,
                                                const moe_i8_experts& w, float* __restrict__ a, float* __restrict__ top,
                                                int* red) {
  const int lane = threadIdx.x & 63, wave = wave_index(), n = rows.n, H = r.H;
  const int64_t channel = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(rows.expert)) * r.F + blockIdx.x * 16;
  const int quad = (lane >> 4) * 16;
  const int8_t* const b[2] = {w.w_gate + channel * H, w.w_up + channel * H};
  const int8_t* xr[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int i = first + t * 16 + (lane & 15);
    xr[t] = i < n ? x + static_cast<int64_t>(rows.slot[i] / r.k) * H + quad : nullptr;
  }
  i32x4 acc[NT][2] = {};
  auto begin = [] {};
  few_rows_i8<NT, 2, U, true>(b, H, xr, wave, H / 128, WAVES, begin, acc);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (first + t * 16 >= n) break;
    __syncthreads();  // the last tile has been read
    put_parts(acc[t], red);
    __syncthreads();
    for (int i = threadIdx.x; i < 256; i += WAVES * kWave) {
      const int m = first + t * 16 + entry_row(i), c = entry_lane(i), slot = rows.slot[min(m, n - 1)];
      const float s = sx[slot / r.k];
      const float g = static_cast<float>(unwrap(sum_parts<WAVES, 2>(red, 0, i))) * s * w.s_gate[channel + c];
      const float u = static_cast<float>(unwrap(sum_parts<WAVES, 2>(red, 1, i))) * s * w.s_up[channel + c];
      const float v = silu_f(g) * u;
      // the row's largest of these 16 channels, in lanes 4, 8, 16 and 32 apart
      uint32_t most = __float_as_uint(v) & 0x7fffffffu;
#pragma unroll
      for (int d = 4; d <= 32; d <<= 1) most = max(most, static_cast<uint32_t>(shfl_xor(static_cast<int>(most), d)));
      if (m >= n) continue;
      a[static_cast<int64_t>(slot) * r.F + blockIdx.x * 16 + c] = v;
      if (c == 0) top[static_cast<int64_t>(slot) * (r.F / 16) + blockIdx.x] = __uint_as_float(most);
    }
  }
}

template <bool FUSED, int WAVES>
__global__ __launch_bounds__(WAVES* kWave, WAVES == kUpWaves8 ? 6 : 2) void k_decode_gateup_i8(DecodeRows r, const int8_t* __restrict__ x,
                                                                       const float* __restrict__ sx, moe_i8_experts w,
                                                                       float* __restrict__ a, float* __restrict__ top) {
  __shared__ Rows rows;
  __shared__ __attribute__((aligned(16))) int red[WAVES * 2 * 256];
  if constexpr (FUSED) {
    __shared__ Selection sel;
    if (!select_rows(r, sel, rows)) return;
  } else {
    if (!read_rows(r, rows)) return;
  }
  if (FUSED || rows.n <= 16) {
    gateup_tiles_i8<1, WAVES, WAVES == kUpWaves8 ? 1 : 2>(r, rows, 0, x, sx, w, a, top, red);
  } else {
    for (int t = 0; t < rows.n; t += 32) gateup_tiles_i8<2, WAVES, 1>(r, rows, t, x, sx, w, a, top, red);
  }
}

// A slot's row of the activation as an int8 row, by one wave; its scale.
__device__ __forceinline__ float round_row(const DecodeRows& r, int slot, const float* __restrict__ a,
                                           const float* __restrict__ top, int8_t* q) {
  const int lane = threadIdx.x & 63, parts = r.F / 16;
  const float* const tops = top + static_cast<int64_t>(slot) * parts;
  const float* const src = a + static_cast<int64_t>(slot) * r.F;
  uint32_t m = 0;
  for (int i = lane; i < parts; i += kWave) m = max(m, __float_as_uint(tops[i]));
  const Rounder rd(wave_umax(m));
#pragma unroll 4
  for (int c = lane * 4; c < r.F; c += 256) {
    const float4 v = *reinterpret_cast<const float4*>(src + c);
    *reinterpret_cast<uint32_t*>(q + c) = pack4(rd(v.x), rd(v.y), rd(v.z), rd(v.w));
  }
  return rd.scale;
}

// The activation's rows as int8 rows, a wave per slot: where every workgroup of
// the down product would otherwise round many rows for itself.
__global__ __launch_bounds__(256) void k_decode_requant(DecodeRows r, const float* __restrict__ a,
                                                        const float* __restrict__ top, int8_t* __restrict__ q,
                                                        float* __restrict__ scale) {
  const int slot = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (slot >= r.T * r.k || r.topk_idx[slot] < 0) return;
  const float s = round_row(r, slot, a, top, q + static_cast<int64_t>(slot) * r.F);
  if ((threadIdx.x & 63) == 0) scale[slot] = s;
}

// O = A W_down: 16 channels per wave, all of F, so no sum over waves.  The
// rows' int8 values and scales are the slots', in a and sa, or (ROUND) rows 0, 1,
// .. of LDS, rounded by begin() under the first weights' way here.
template <int NT, int U, bool ROUND, class Begin>
__device__ __forceinline__ void down_tiles_i8(const DecodeRows& r, const Rows& rows, int first, const int8_t* a,
                                              const float* sa, const moe_i8_experts& w, float* __restrict__ o,
                                              Begin& begin) {
  const int lane = threadIdx.x & 63, wave = wave_index(), n = rows.n, F = r.F;
  const int first_column = (blockIdx.x * kDownWaves8 + wave) * 16, column = first_column + (lane & 15);
  const int64_t channel = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(rows.expert)) * r.H + first_column;
  const int quad = (lane >> 4) * 16;
  const int8_t* const b[1] = {w.w_down + channel * F};
  const int8_t* ar[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int i = first + t * 16 + (lane & 15);
    ar[t] = i < n ? a + static_cast<int64_t>(ROUND ? i : rows.slot[i]) * F + quad : nullptr;
  }
  i32x4 acc[NT][1] = {};
  few_rows_i8<NT, 1, U, false>(b, F, ar, 0, F / 128, 1, begin, acc);
  const float sd = w.s_down[channel + (lane & 15)];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = first + t * 16 + 4 * (lane >> 4) + i;
      if (m < n)
        o[static_cast<int64_t>(rows.slot[m]) * r.H + column] = static_cast<float>(unwrap(acc[t][0][i])) * sa[ROUND ? m : rows.slot[m]] * sd;
    }
}

__global__ __launch_bounds__(kDownWaves8* kWave, 6) void k_decode_down_i8(DecodeRows r, const int8_t* __restrict__ a,
                                                                       const float* __restrict__ sa, moe_i8_experts w,
                                                                       float* __restrict__ o) {
  __shared__ Rows rows;
  if (!read_rows(r, rows)) return;
  auto begin = [] {};
  if (rows.n <= 16) {
    down_tiles_i8<1, 2, false>(r, rows, 0, a, sa, w, o, begin);
  } else {
    for (int t = 0; t < rows.n; t += 32) down_tiles_i8<2, 2, false>(r, rows, t, a, sa, w, o, begin);
  }
}

// The same from the activation itself, for up to kFusedT tokens.
__global__ __launch_bounds__(kDownWaves8* kWave) void k_decode_down_i8_few(DecodeRows r, const float* __restrict__ a,
                                                                          const float* __restrict__ top,
                                                                          moe_i8_experts w, float* __restrict__ o) {
  __shared__ Rows rows;
  __shared__ float sa[kFusedT];
  extern __shared__ __attribute__((aligned(16))) int8_t a8[];  // [rows, F]
  if (!read_rows(r, rows)) return;
  bool begun = false;
  auto begin = [&] {
    if (begun) return;
    begun = true;
    for (int i = threadIdx.x >> 6; i < rows.n; i += kDownWaves8) {
      const float s = round_row(r, rows.slot[i], a, top, a8 + i * r.F);
      if ((threadIdx.x & 63) == 0) sa[i] = s;
    }
    __syncthreads();
  };
  down_tiles_i8<1, 6, true>(r, rows, 0, a8, sa, w, o, begin);
}

// y[t] = sum_j gates o, in slot order; 0 for a token without rows.  Eight
// slots' values are on their way at once.
__global__ __launch_bounds__(256) void k_decode_combine(DecodeRows r, const float* __restrict__ o, bf16_t* __restrict__ y) {
  const int t = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= r.H) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (uniform_load(r.topk_idx + t * r.k) >= 0)
    for (int j0 = 0; j0 < r.k; j0 += 8) {
      float4 v[8];
      float g[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = j0 + j < r.k;
        const int slot = t * r.k + min(j0 + j, r.k - 1);
        v[j] = *reinterpret_cast<const float4*>(o + static_cast<int64_t>(slot) * r.H + c);
        g[j] = uniform_load(r.gates + slot);
        v[j] = make_float4(in ? v[j].x : 0.f, in ? v[j].y : 0.f, in ? v[j].z : 0.f, in ? v[j].w : 0.f);
        g[j] = in ? g[j] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s.x = fmaf(g[j], v[j].x, s.x), s.y = fmaf(g[j], v[j].y, s.y);
        s.z = fmaf(g[j], v[j].z, s.z), s.w = fmaf(g[j], v[j].w, s.w);
      }
    }
  *reinterpret_cast<uint2*>(y + static_cast<int64_t>(t) * r.H + c) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
}

// Experts that the tokens may use, the grid's second axis.
int slots(const DecodeRows& r) { return std::min(r.E, r.T * r.k); }

}  // namespace

// Ranges of K of the bf16 gate/up product: two where few tokens leave its
// tiles fewer than half of the chip's 256 compute units.  The down product then
// holds the rows of an expert in LDS, at most 48 KB: with T k < E they are at
// most the grid's slots, hence slots F <= 128 kCols values of three bf16, and else
// E >= 8 slots leave F <= 16 kCols for at most kFusedT rows.
int decode_ranges(int T, int E, int F, int k) {
  return decode_fused(T) && F / kCols * std::min(E, T * k) <= 128 ? 2 : 1;
}

hipError_t launch_decode_router(const DecodeRows& r, const bf16_t* x, const bf16_t* w_r, int8_t* q, float* sx,
                                hipStream_t s) {
  TraceScope trace_scope(K_DECODE_ROUTER, s);
  const int tiles = cdiv(r.E, kRouterCols) * cdiv(r.T, 16) * kRouterSplits, more = q != nullptr ? r.T : 0;
  hipLaunchKernelGGL(k_decode_router, dim3(tiles + more), dim3(kWave), 0, s, x, w_r, r.T, r.H, r.E, r.part, r.counts, q, sx);
  return hipGetLastError();
}

hipError_t launch_decode_gateup(const DecodeRows& r, const bf16_t* x, const bf16_t* w_gate, const bf16_t* w_up,
                                bf16_t* a, float* gu, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_GATEUP, s);
  const dim3 grid(r.F / kCols, slots(r), decode_ranges(r.T, r.E, r.F, r.k));
  if (grid.z > 1)
    hipLaunchKernelGGL((k_decode_gateup<true, true>), grid, dim3(kUpWaves * kWave), 0, s, r, x, w_gate, w_up, a, gu);
  else if (decode_fused(r.T))
    hipLaunchKernelGGL((k_decode_gateup<true, false>), grid, dim3(kUpWaves * kWave), 0, s, r, x, w_gate, w_up, a, gu);
  else
    hipLaunchKernelGGL((k_decode_gateup<false, false>), grid, dim3(kUpWaves * kWave), 0, s, r, x, w_gate, w_up, a, gu);
  return hipGetLastError();
}

hipError_t launch_decode_down(const DecodeRows& r, const bf16_t* a, const float* gu, const bf16_t* w_down, float* o,
                              hipStream_t s) {
  TraceScope trace_scope(K_DECODE_DOWN, s);
  const dim3 grid(r.H / kCols, slots(r));
  if (decode_ranges(r.T, r.E, r.F, r.k) > 1)
    hipLaunchKernelGGL(k_decode_down<true>, grid, dim3(kDownWaves * kWave), kDecodeParts * r.T * r.F * sizeof(bf16_t), s, r, a, gu, w_down, o);
  else
    hipLaunchKernelGGL(k_decode_down<false>, grid, dim3(kDownWaves * kWave), 0, s, r, a, gu, w_down, o);
  return hipGetLastError();
}

hipError_t launch_decode_gateup_i8(const DecodeRows& r, const int8_t* x, const float* sx, const moe_i8_experts& w,
                                   float* a, float* top, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_GATEUP, s);
  const dim3 grid(r.F / 16, slots(r));
  if (decode_fused(r.T) && grid.x * grid.y <= 1024)
    hipLaunchKernelGGL((k_decode_gateup_i8<true, kUpWaves8Few>), grid, dim3(kUpWaves8Few * kWave), 0, s, r, x, sx, w, a, top);
  else if (decode_fused(r.T))
    hipLaunchKernelGGL((k_decode_gateup_i8<true, kUpWaves8>), grid, dim3(kUpWaves8 * kWave), 0, s, r, x, sx, w, a, top);
  else
    hipLaunchKernelGGL((k_decode_gateup_i8<false, kUpWaves8>), grid, dim3(kUpWaves8 * kWave), 0, s, r, x, sx, w, a, top);
  return hipGetLastError();
}

hipError_t launch_decode_down_i8(const DecodeRows& r, const float* a, const float* top, int8_t* a8, float* sa,
                                 const moe_i8_experts& w, float* o, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_DOWN, s);
  const dim3 grid(r.H / (16 * kDownWaves8), slots(r)), block(kDownWaves8 * kWave);
  // rows in LDS: an expert has at most T
  if (decode_fused(r.T) && r.T * r.F <= 65536) {
    hipLaunchKernelGGL(k_decode_down_i8_few, grid, block, r.T * r.F, s, r, a, top, w, o);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(k_decode_requant, dim3(cdiv(r.T * r.k, 4)), dim3(256), 0, s, r, a, top, a8, sa);
  hipLaunchKernelGGL(k_decode_down_i8, grid, block, 0, s, r, a8, sa, w, o);
  return hipGetLastError();
}

hipError_t launch_decode_combine(const DecodeRows& r, const float* o, bf16_t* y, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_COMBINE, s);
  hipLaunchKernelGGL(k_decode_combine, dim3(cdiv(r.H, 1024), r.T), dim3(256), 0, s, r, o, y);
  return hipGetLastError();
}

}  // namespace moe
