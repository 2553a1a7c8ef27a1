// The expert layer for a few tokens.  Reading the weights of the experts that
// the tokens picked bounds it: at one token and top-8 of a 30B-A3B model 75 MB
// in bf16 for 75 MFLOP.  So every weight goes from memory straight into the
// registers of the one wave that multiplies it, in wide loads with many of
// them in flight, and the K axis is split over a workgroup's waves until the
// few (expert, columns) tiles fill the chip.
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
#include "trace.hpp"

namespace moe {

namespace {

// The slots of the blockIdx.y-th used expert in token order; false where there
// are fewer used experts.  One wave finds them; ends with a barrier.
struct Rows {
  int32_t slot[kDecodeMaxT];
  int expert, n;
};
__device__ __forceinline__ bool find_rows(const DecodeRows& r, Rows& rows) {
  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x;
    int e = -1, before = 0;
    const int want = blockIdx.y;
    for (int m = 0; m < r.E; m += kWave) {
      const unsigned long long used = __ballot(m + lane < r.E && r.counts[min(m + lane, r.E - 1)] > 0);
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
        if (r.topk_idx[lane * r.k + j] == e) slot = lane * r.k + j;
    const unsigned long long has = __ballot(slot >= 0);
    if (slot >= 0) rows.slot[__popcll(has & ((1ull << lane) - 1ull))] = slot;
    if (lane == 0) {
      rows.expert = e;
      rows.n = __popcll(has);
    }
  }
  __syncthreads();
  return rows.expert >= 0;
}

// CW neighbouring bf16 of a weight row.
template <int CW>
struct Vec;
template <>
struct Vec<2> {
  using T = uint32_t;
};
template <>
struct Vec<4> {
  using T = uint2;
};
__device__ __forceinline__ uint32_t word(uint32_t v, int) { return v; }
__device__ __forceinline__ uint32_t word(const uint2& v, int i) { return i == 0 ? v.x : v.y; }

// Two rows' bf16 at the same column (the low or the high half of a word) side by side.
__device__ __forceinline__ uint32_t lows(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t highs(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Eight consecutive K rows of a lane's CW columns -> the matrix instruction's
// operand for column p of each lane: eight K values of one column.
template <int CW>
__device__ __forceinline__ uint4 column(const typename Vec<CW>::T (&v)[8], int p) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = word(v[2 * i], p >> 1), b = word(v[2 * i + 1], p >> 1);
    w[i] = p & 1 ? highs(a, b) : lows(a, b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Products of up to 16 NT rows (bf16, K-contiguous, row pitch K, row id
// row_of[i]) with NB column-contiguous matrices [K, N] at columns c0 .. c0 +
// 16 CW, the K axis split over the workgroup's WAVES waves, 32 at a time.
// Lane l holds columns c0 + CW (l % 16) + p: a load of CW columns per lane
// brings four rows of 32 CW bytes each.
template <int NT, int CW, int NB, int WAVES, int U>
__device__ __forceinline__ void few_rows(const bf16_t* __restrict__ x, const int (&row)[NT], const bf16_t* const (&b)[NB],
                                         int K, int N, f32x4 (&acc)[NT][NB][CW]) {
  using V = typename Vec<CW>::T;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int quad = (lane >> 4) * 8;
  const int steps = K / 32;
  const int64_t col = (lane & 15) * CW;
  auto batch = [&](int s0, auto count) {
    constexpr int n = decltype(count)::value;
    V v[n][NB][8];
    uint4 xv[n][NT];
#pragma unroll
    for (int u = 0; u < n; ++u) {
      const int k = (s0 + u * WAVES) * 32 + quad;
#pragma unroll
      for (int m = 0; m < NB; ++m)
#pragma unroll
        for (int r = 0; r < 8; ++r)
          v[u][m][r] = *reinterpret_cast<const V*>(b[m] + static_cast<int64_t>(k + r) * N + col);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        xv[u][t] = row[t] >= 0 ? *reinterpret_cast<const uint4*>(x + static_cast<int64_t>(row[t]) * K + k) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < n; ++u)
#pragma unroll
      for (int m = 0; m < NB; ++m)
#pragma unroll
        for (int p = 0; p < CW; ++p) {
          const uint4 w = column<CW>(v[u][m], p);
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[t][m][p] = mfma16x16x32(xv[u][t], w, acc[t][m][p]);
        }
  };
  int s = wave;
  for (; s + (U - 1) * WAVES < steps; s += U * WAVES) batch(s, std::integral_constant<int, U>{});
  for (; s < steps; s += WAVES) batch(s, std::integral_constant<int, 1>{});
}

// Sum over the waves of one row tile's products, which each holds per lane as
// f32x4 (or i32x4): element i of lane l, fragment f.  `red` has
// WAVES * FRAGS * 256 entries.
template <int WAVES, int FRAGS, class V4, class S>
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

// Waves per workgroup: the gate/up product splits a long K (H), the down
// product a shorter one (F).
constexpr int kUpWaves = 8, kDownWaves = 4;

template <int NT, int CW>
__global__ __launch_bounds__(kUpWaves* kWave) void k_decode_gateup(DecodeRows r, const bf16_t* __restrict__ x,
                                                                   const bf16_t* __restrict__ w_gate,
                                                                   const bf16_t* __restrict__ w_up,
                                                                   bf16_t* __restrict__ a) {
  __shared__ Rows rows;
  __shared__ float red[kUpWaves * 2 * CW * 256];
  if (!find_rows(r, rows)) return;
  const int lane = threadIdx.x & 63, n = rows.n;
  int token[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int i = t * 16 + (lane & 15);
    token[t] = i < n ? rows.slot[i] / r.k : -1;
  }
  const int64_t base = static_cast<int64_t>(rows.expert) * r.H * r.F + blockIdx.x * (16 * CW);
  const bf16_t* const b[2] = {w_gate + base, w_up + base};
  f32x4 acc[NT][2][CW] = {};
  few_rows<NT, CW, 2, kUpWaves, NT == 1 ? 4 / (CW / 2) : 2>(x, token, b, r.H, r.F, acc);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t * 16 >= n) break;
    if (t > 0) __syncthreads();
    f32x4 part[2 * CW];
#pragma unroll
    for (int f = 0; f < 2 * CW; ++f) part[f] = acc[t][f / CW][f % CW];
    put_parts<kUpWaves, 2 * CW>(part, red);
    __syncthreads();
    for (int i = threadIdx.x; i < CW * 256; i += kUpWaves * kWave) {
      const int p = i >> 8, at = i & 255, l = at >> 2, m = t * 16 + 4 * (l >> 4) + (at & 3);
      if (m >= n) continue;
      const float g = sum_parts<kUpWaves, 2 * CW>(red, p, at), u = sum_parts<kUpWaves, 2 * CW>(red, CW + p, at);
      // the one rounding between the products: the down product's operand is bf16
      a[static_cast<int64_t>(rows.slot[m]) * r.F + blockIdx.x * (16 * CW) + (l & 15) * CW + p] = f2bf(silu_f(g) * u);
    }
  }
}

template <int NT, int CW>
__global__ __launch_bounds__(kDownWaves* kWave) void k_decode_down(DecodeRows r, const bf16_t* __restrict__ a,
                                                                   const bf16_t* __restrict__ w_down,
                                                                   float* __restrict__ o) {
  __shared__ Rows rows;
  __shared__ float red[kDownWaves * CW * 256];
  if (!find_rows(r, rows)) return;
  const int lane = threadIdx.x & 63, n = rows.n;
  int row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int i = t * 16 + (lane & 15);
    row[t] = i < n ? rows.slot[i] : -1;
  }
  const bf16_t* const b[1] = {w_down + static_cast<int64_t>(rows.expert) * r.H * r.F + blockIdx.x * (16 * CW)};
  f32x4 acc[NT][1][CW] = {};
  few_rows<NT, CW, 1, kDownWaves, NT == 1 ? 6 / (CW / 2) : 2>(a, row, b, r.F, r.H, acc);
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t * 16 >= n) break;
    if (t > 0) __syncthreads();
    put_parts<kDownWaves, CW>(acc[t][0], red);
    __syncthreads();
    for (int i = threadIdx.x; i < CW * 256; i += kDownWaves * kWave) {
      const int p = i >> 8, at = i & 255, l = at >> 2, m = t * 16 + 4 * (l >> 4) + (at & 3);
      if (m < n)
        o[static_cast<int64_t>(rows.slot[m]) * r.H + blockIdx.x * (16 * CW) + (l & 15) * CW + p] =
            sum_parts<kDownWaves, CW>(red, p, at);
    }
  }
}

// ---- int8 weights.  They are K-contiguous: lane l reads 16 bytes of channel
// l % 16, the instruction's operand as it is, and two loads a whole 128-byte line.
template <int NT>
__global__ __launch_bounds__(kUpWaves* kWave) void k_decode_gateup_i8(DecodeRows r, const int8_t* __restrict__ x,
                                                                      const float* __restrict__ sx, moe_i8_experts w,
                                                                      float* __restrict__ a) {
  __shared__ Rows rows;
  __shared__ int red[kUpWaves * 2 * 256];
  if (!find_rows(r, rows)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = rows.n, H = r.H;
  const int64_t channel = static_cast<int64_t>(rows.expert) * r.F + blockIdx.x * 16;
  const int quad = (lane >> 4) * 16;
  const int8_t* const wg = w.w_gate + (channel + (lane & 15)) * H + quad;
  const int8_t* const wu = w.w_up + (channel + (lane & 15)) * H + quad;
  const int8_t* xr[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int i = t * 16 + (lane & 15);
    xr[t] = i < n ? x + static_cast<int64_t>(rows.slot[i] / r.k) * H + quad : nullptr;
  }
  i32x4 acc[NT][2] = {};
  auto batch = [&](int unit, auto count) {  // units of 128 k, kUpWaves apart
    constexpr int m = decltype(count)::value;
    uint4 g[m][2], u[m][2], v[m][2][NT];
#pragma unroll
    for (int i = 0; i < m; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = (unit + i * kUpWaves) * 128 + h * 64;
        g[i][h] = *reinterpret_cast<const uint4*>(wg + k);
        u[i][h] = *reinterpret_cast<const uint4*>(wu + k);
#pragma unroll
        for (int t = 0; t < NT; ++t)
          v[i][h][t] = xr[t] != nullptr ? *reinterpret_cast<const uint4*>(xr[t] + k) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
    for (int i = 0; i < m; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[t][0] = mfma_i8(v[i][h][t], g[i][h], acc[t][0]);
          acc[t][1] = mfma_i8(v[i][h][t], u[i][h], acc[t][1]);
        }
  };
  const int units = H / 128;
  int unit = wave;
  for (; unit + kUpWaves < units; unit += 2 * kUpWaves) batch(unit, std::integral_constant<int, 2>{});
  if (unit < units) batch(unit, std::integral_constant<int, 1>{});
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t * 16 >= n) break;
    if (t > 0) __syncthreads();
    put_parts<kUpWaves, 2>(acc[t], red);
    __syncthreads();
    const int at = threadIdx.x, l = at >> 2, m = t * 16 + 4 * (l >> 4) + (at & 3), c = l & 15;
    if (at < 256 && m < n) {
      const float s = sx[rows.slot[m] / r.k];
      const float g = static_cast<float>(unwrap(sum_parts<kUpWaves, 2>(red, 0, at))) * s * w.s_gate[channel + c];
      const float u = static_cast<float>(unwrap(sum_parts<kUpWaves, 2>(red, 1, at))) * s * w.s_up[channel + c];
      a[static_cast<int64_t>(rows.slot[m]) * r.F + blockIdx.x * 16 + c] = silu_f(g) * u;
    }
  }
}

// O = A W_down, 64 channels per workgroup, 16 per wave.  The activation's rows
// are rounded to int8 by every workgroup for itself (from L2): their largest
// magnitudes first, then kChunk columns at a time into LDS, while the chunk's
// weights are on their way into registers.
constexpr int kDownChunk = 1024, kDownUnits = kDownChunk / 128;
constexpr int kDownPitch = kDownChunk + 16;  // 16 rows of one fragment read in distinct banks

__global__ __launch_bounds__(kDownWaves* kWave) void k_decode_down_i8(DecodeRows r, const float* __restrict__ a,
                                                                      moe_i8_experts w, float* __restrict__ o) {
  __shared__ Rows rows;
  __shared__ uint32_t tops[kDecodeMaxT];
  __shared__ __attribute__((aligned(16))) int8_t a8[16 * kDownPitch];
  if (!find_rows(r, rows)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = rows.n, F = r.F;
  for (int i = wave; i < n; i += kDownWaves) {
    const float* src = a + static_cast<int64_t>(rows.slot[i]) * F;
    uint32_t m = 0;
    for (int c = lane * 2; c < F; c += 128) {
      const float2 v = *reinterpret_cast<const float2*>(src + c);
      m = max(m, max(__float_as_uint(v.x) & 0x7fffffffu, __float_as_uint(v.y) & 0x7fffffffu));
    }
    m = wave_umax(m);
    if (lane == 0) tops[i] = m;
  }
  const int64_t channel = static_cast<int64_t>(rows.expert) * r.H + blockIdx.x * 64 + wave * 16;
  const int quad = (lane >> 4) * 16;
  const int8_t* const wd = w.w_down + (channel + (lane & 15)) * F + quad;
  constexpr int kTiles = kDecodeMaxT / 16;
  i32x4 acc[kTiles] = {};
  for (int k0 = 0; k0 < F; k0 += kDownChunk) {
    uint4 v[kDownUnits][2];
#pragma unroll
    for (int i = 0; i < kDownUnits; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + i * 128 + h * 64;
        v[i][h] = k < F ? *reinterpret_cast<const uint4*>(wd + k) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      if (t * 16 >= n) break;
      __syncthreads();  // the tops are there, the last tile has been read
      for (int i = wave; i < 16; i += kDownWaves) {
        const int m = t * 16 + i;
        const Rounder rd(m < n ? tops[m] : 0u);
        const float* src = m < n ? a + static_cast<int64_t>(rows.slot[m]) * F : nullptr;
        for (int c = lane * 4; c < kDownChunk; c += 256) {
          float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
          if (src != nullptr && k0 + c < F) f = *reinterpret_cast<const float4*>(src + k0 + c);
          *reinterpret_cast<uint32_t*>(a8 + i * kDownPitch + c) = pack4(rd(f.x), rd(f.y), rd(f.z), rd(f.w));
        }
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kDownUnits; ++i) {
        if (k0 + i * 128 >= F) break;
#pragma unroll
        for (int h = 0; h < 2; ++h)
          acc[t] = mfma_i8(*reinterpret_cast<const uint4*>(a8 + (lane & 15) * kDownPitch + i * 128 + h * 64 + quad),
                           v[i][h], acc[t]);
      }
    }
  }
  const float sd = w.s_down[channel + (lane & 15)];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    if (t * 16 >= n) break;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = t * 16 + 4 * (lane >> 4) + i;
      if (m < n)
        o[static_cast<int64_t>(rows.slot[m]) * r.H + blockIdx.x * 64 + wave * 16 + (lane & 15)] =
            static_cast<float>(unwrap(acc[t][i])) * Rounder(tops[m]).scale * sd;
    }
  }
}

// y[t] = sum_j g o, in slot order; 0 for a token without rows.
__global__ __launch_bounds__(256) void k_decode_combine(DecodeRows r, const float* __restrict__ gates,
                                                        const float* __restrict__ o, bf16_t* __restrict__ y) {
  const int t = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= r.H) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (r.topk_idx[t * r.k] >= 0)
    for (int j = 0; j < r.k; ++j) {
      const float g = gates[t * r.k + j];
      const float4 v = *reinterpret_cast<const float4*>(o + static_cast<int64_t>(t * r.k + j) * r.H + c);
      s.x = fmaf(g, v.x, s.x), s.y = fmaf(g, v.y, s.y), s.z = fmaf(g, v.z, s.z), s.w = fmaf(g, v.w, s.w);
    }
  *reinterpret_cast<uint2*>(y + static_cast<int64_t>(t) * r.H + c) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
}

// Experts that the tokens may use, the grid's second axis.
int slots(const DecodeRows& r) { return std::min(r.E, r.T * r.k); }

}  // namespace

// Row tiles of 16 that one expert may have: 1, 2 or 4.
#define MOE_DECODE_TILES(T, CALL) \
  do {                            \
    if ((T) <= 16) CALL(1);       \
    else if ((T) <= 32) CALL(2);  \
    else CALL(4);                 \
  } while (0)

hipError_t launch_decode_gateup(const DecodeRows& r, const bf16_t* x, const bf16_t* w_gate, const bf16_t* w_up,
                                bf16_t* a, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_GATEUP, s);
#define MOE_CALL(NT) \
  hipLaunchKernelGGL((k_decode_gateup<NT, 2>), dim3(r.F / 32, slots(r)), dim3(kUpWaves * kWave), 0, s, r, x, w_gate, w_up, a)
  MOE_DECODE_TILES(r.T, MOE_CALL);
#undef MOE_CALL
  return hipGetLastError();
}

hipError_t launch_decode_down(const DecodeRows& r, const bf16_t* a, const bf16_t* w_down, float* o, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_DOWN, s);
#define MOE_CALL(NT) \
  hipLaunchKernelGGL((k_decode_down<NT, 2>), dim3(r.H / 32, slots(r)), dim3(kDownWaves * kWave), 0, s, r, a, w_down, o)
  MOE_DECODE_TILES(r.T, MOE_CALL);
#undef MOE_CALL
  return hipGetLastError();
}

hipError_t launch_decode_gateup_i8(const DecodeRows& r, const int8_t* x, const float* sx, const moe_i8_experts& w,
                                   float* a, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_GATEUP, s);
#define MOE_CALL(NT) \
  hipLaunchKernelGGL((k_decode_gateup_i8<NT>), dim3(r.F / 16, slots(r)), dim3(kUpWaves * kWave), 0, s, r, x, sx, w, a)
  MOE_DECODE_TILES(r.T, MOE_CALL);
#undef MOE_CALL
  return hipGetLastError();
}

hipError_t launch_decode_down_i8(const DecodeRows& r, const float* a, const moe_i8_experts& w, float* o, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_DOWN, s);
  hipLaunchKernelGGL(k_decode_down_i8, dim3(r.H / 64, slots(r)), dim3(kDownWaves * kWave), 0, s, r, a, w, o);
  return hipGetLastError();
}

hipError_t launch_decode_combine(const DecodeRows& r, const float* gates, const float* o, bf16_t* y, hipStream_t s) {
  TraceScope trace_scope(K_DECODE_COMBINE, s);
  hipLaunchKernelGGL(k_decode_combine, dim3(cdiv(r.H, 1024), r.T), dim3(256), 0, s, r, gates, o, y);
  return hipGetLastError();
}

}  // namespace moe
