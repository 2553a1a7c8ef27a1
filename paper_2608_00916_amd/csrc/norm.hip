// Sum of a row with the residual, its root-mean-square norm in bf16 and in
// int8 rows, and the backward.  Memory bounds all of it: every value is read
// once into registers, reduced there, and written once.
//
//   h = bf16(x + r),  s = (mean h^2 + eps)^(-1/2),  y = h s w
//
// The norm is that of the sum as it is stored, so that the backward, which has
// the stored one, differentiates exactly what the forward computed.  Sums,
// statistics and products are fp32; the int8 rows are those of the fp32
// product, which meets no bf16 on its way.
#include <algorithm>

#include "i8_round.hpp"
#include "step.hpp"
#include "trace.hpp"

namespace moe {

namespace {

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  f[0] = lo_bf(v.x), f[1] = hi_bf(v.x), f[2] = lo_bf(v.y), f[3] = hi_bf(v.y);
  f[4] = lo_bf(v.z), f[5] = hi_bf(v.z), f[6] = lo_bf(v.w), f[7] = hi_bf(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// A row belongs to WAVES waves, VEC 16-byte vectors per lane: in the forward a
// row of up to 2048 columns is one wave's (no barrier), one of up to 8192 four
// waves' and the longest, 32768, sixteen waves'.
template <int WAVES>
constexpr int kRowThreads = WAVES * kWave;
// Waves of a workgroup: several rows where a row is one wave's.
template <int WAVES>
constexpr int kFwdRows = WAVES == 1 ? 4 : 1;
template <int WAVES>
constexpr int kBwdRows = WAVES == 1 ? 8 : WAVES == 4 ? 2 : 1;

// Sum (or largest) over a row's waves; every lane gets it.  `red` is this
// row's and this call's own, so no barrier follows the read.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* red, int wave) {
  v = wave_sum(v);
  if constexpr (WAVES == 1) return v;
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) t += red[i];
  return t;
}
template <int WAVES>
__device__ __forceinline__ uint32_t row_umax(uint32_t v, uint32_t* red, int wave) {
  v = wave_umax(v);
  if constexpr (WAVES == 1) return v;
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) t = max(t, red[i]);
  return t;
}

template <int WAVES, int VEC>
__global__ __launch_bounds__(kRowThreads<WAVES>* kFwdRows<WAVES>) void k_norm_fwd(NormFwd a) {
  __shared__ float sums[WAVES];
  __shared__ uint32_t tops[WAVES];
  const int in_row = threadIdx.x % kRowThreads<WAVES>, wave = in_row >> 6;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kFwdRows<WAVES> + threadIdx.x / kRowThreads<WAVES>;
  if (row >= a.T) return;  // whole waves, and only where a row is one wave's
  const int H = a.H;
  uint4 held[VEC];
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const int c = (i * kRowThreads<WAVES> + in_row) * 8;
    held[i] = c < H ? *reinterpret_cast<const uint4*>(a.x + row * a.ldx + c) : make_uint4(0, 0, 0, 0);
  }
  if (a.r != nullptr) {
    uint4 res[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int c = (i * kRowThreads<WAVES> + in_row) * 8;
      res[i] = c < H ? *reinterpret_cast<const uint4*>(a.r + row * a.ldr + c) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      float f[8], g[8];
      unpack8(held[i], f);
      unpack8(res[i], g);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] += g[j];
      held[i] = pack8(f);
      const int c = (i * kRowThreads<WAVES> + in_row) * 8;
      if (a.h != nullptr && c < H) *reinterpret_cast<uint4*>(a.h + row * H + c) = held[i];
    }
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    float f[8];
    unpack8(held[i], f);
#pragma unroll
    for (int j = 0; j < 8; ++j) sq = fmaf(f[j], f[j], sq);
  }
  uint4 wv[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const int c = (i * kRowThreads<WAVES> + in_row) * 8;
    wv[i] = c < H ? *reinterpret_cast<const uint4*>(a.w + c) : make_uint4(0, 0, 0, 0);
  }
  const float s = 1.0f / sqrtf(row_sum<WAVES>(sq, sums, wave) / static_cast<float>(H) + a.eps);
  float v[VEC][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    float f[8], w[8];
    unpack8(held[i], f);
    unpack8(wv[i], w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[i][j] = f[j] * s * w[j];
      top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
    }
    const int c = (i * kRowThreads<WAVES> + in_row) * 8;
    if (a.y != nullptr && c < H) *reinterpret_cast<uint4*>(a.y + row * H + c) = pack8(v[i]);
  }
  if (a.q == nullptr) return;
  const Rounder r(row_umax<WAVES>(top, tops, wave));
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const int c = (i * kRowThreads<WAVES> + in_row) * 8;
    if (c < H)
      *reinterpret_cast<uint2*>(a.q + row * H + c) =
          make_uint2(pack4(r(v[i][0]), r(v[i][1]), r(v[i][2]), r(v[i][3])),
                     pack4(r(v[i][4]), r(v[i][5]), r(v[i][6]), r(v[i][7])));
  }
  if (in_row == 0) a.scale[row] = r.scale;
}

// Backward.  With n = h s and g = dy w,
//   dx = s (g - n mean(g n)) + dh,   dw = sum_t dy n.
// Both means of a row come from one pass over its registers.  A workgroup
// takes rows blockIdx.x, + gridDim.x, ... (times its rows at a time) and keeps
// its share of dw in registers, or in LDS for rows of over 16384, whose
// registers are full; the shares are added in a fixed order by k_norm_dw, so
// dw does not depend on timing.  Few registers per lane are what counts:
// rows of 2048 by one wave of four vectors a lane (210 registers, two waves per
// SIMD) took 36 us at 8192 x 2048, the adding of the shares included, four
// waves of one vector 25 (5.3 TB/s of what is read and written; a copy reaches
// 5.4, the forward 6.5), both in a row of calls on the same tensors, a part of
// which the last-level cache serves; from HBM the call takes 30.
template <int WAVES, int VEC>
__global__ __launch_bounds__(kRowThreads<WAVES>* kBwdRows<WAVES>) void k_norm_bwd(NormBwd a) {
  constexpr int ROWS = kBwdRows<WAVES>, RT = kRowThreads<WAVES>;
  __shared__ float2 sums[2][ROWS][WAVES];
  constexpr bool kInLds = VEC > 2;
  extern __shared__ __attribute__((aligned(16))) float dws[];  // ROWS H floats where there are rows at a time, or kInLds
  const int in_row = threadIdx.x % RT, wave = in_row >> 6, slot = threadIdx.x / RT;
  const int H = a.H;
  const float inv_h = 1.0f / static_cast<float>(H);
  float acc[kInLds ? 1 : VEC][8];
  uint4 wv[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    const int c = (i * RT + in_row) * 8;
    wv[i] = c < H ? *reinterpret_cast<const uint4*>(a.w + c) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {  // LDS: a lane's own entries, side by side with its neighbours': no barrier
      if constexpr (!kInLds) acc[i][j] = 0.0f;
      else dws[(i * 8 + j) * RT + in_row] = 0.0f;
    }
  }
  int turn = 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * ROWS;
  // Where registers allow, a row's loads go out before the sums of the one
  // before it: 31.5 -> 30.3 us at 8192 x 2048 from HBM, the
  // adding of the shares included.
  constexpr bool kAhead = VEC == 1;
  uint4 hv[VEC], dv[VEC], uv[VEC], hn[VEC], dn[VEC], un[VEC];
  auto load = [&](int64_t row, uint4(&h)[VEC], uint4(&d)[VEC], uint4(&u)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int c = (i * RT + in_row) * 8;
      const bool in = row < a.T && c < H;
      h[i] = in ? *reinterpret_cast<const uint4*>(a.h + row * a.ldh + c) : make_uint4(0, 0, 0, 0);
      d[i] = in ? *reinterpret_cast<const uint4*>(a.dy + row * a.lddy + c) : make_uint4(0, 0, 0, 0);
      if constexpr (!kInLds) u[i] = in && a.dh != nullptr ? *reinterpret_cast<const uint4*>(a.dh + row * a.lddh + c) : make_uint4(0, 0, 0, 0);
    }
  };
  if constexpr (kAhead) load(static_cast<int64_t>(blockIdx.x) * ROWS + slot, hn, dn, un);
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * ROWS; base < a.T; base += step) {
    const int64_t row = base + slot;
    const bool on = row < a.T;  // the loop's trips are the workgroup's, its barrier is met by all
    if constexpr (kAhead) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) hv[i] = hn[i], dv[i] = dn[i], uv[i] = un[i];
      load(row + step, hn, dn, un);
    } else {
      load(row, hv, dv, uv);
    }
    float sq = 0.0f, gh = 0.0f;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      float h[8], d[8], w[8];
      unpack8(hv[i], h);
      unpack8(dv[i], d);
      unpack8(wv[i], w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sq = fmaf(h[j], h[j], sq);
        gh = fmaf(d[j] * w[j], h[j], gh);
      }
    }
    sq = wave_sum(sq);
    gh = wave_sum(gh);
    if constexpr (WAVES > 1) {
      // two sets of sums in turn: a set is written again only after the other's barrier
      if ((threadIdx.x & 63) == 0) sums[turn][slot][wave] = make_float2(sq, gh);
      __syncthreads();
      sq = gh = 0.0f;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) {
        sq += sums[turn][slot][i].x;
        gh += sums[turn][slot][i].y;
      }
      turn ^= 1;
    }
    const float s = 1.0f / sqrtf(sq * inv_h + a.eps);
    const float c1 = gh * inv_h * s * s;  // mean(g n) s: what a unit of h takes off g
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int c = (i * RT + in_row) * 8;
      if (!on || c >= H) continue;
      float h[8], d[8], w[8], u[8];
      unpack8(hv[i], h);
      unpack8(dv[i], d);
      unpack8(wv[i], w);
      if constexpr (kInLds)  // no registers to hold it meanwhile
        uv[i] = a.dh != nullptr ? *reinterpret_cast<const uint4*>(a.dh + row * a.lddh + c) : make_uint4(0, 0, 0, 0);
      unpack8(uv[i], u);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float& sum = kInLds ? dws[(i * 8 + j) * RT + in_row] : acc[kInLds ? 0 : i][j];
        sum = fmaf(d[j], h[j] * s, sum);
        u[j] = fmaf(s, fmaf(-h[j], c1, d[j] * w[j]), u[j]);
      }
      *reinterpret_cast<uint4*>(a.dx + row * H + c) = pack8(u);
    }
  }
  float* part = a.part + static_cast<int64_t>(blockIdx.x) * H;
  if constexpr (ROWS > 1) {  // the rows' shares side by side in LDS, then added in their order
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int c = (i * RT + in_row) * 8;
      if (c >= H) continue;
      float* const at = dws + slot * H + c;
      *reinterpret_cast<float4*>(at) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
      *reinterpret_cast<float4*>(at + 4) = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < H; c += RT * ROWS) {
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < ROWS; ++k) t += dws[k * H + c];
      part[c] = t;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const int c = (i * RT + in_row) * 8;
      if (c >= H) continue;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = kInLds ? dws[(i * 8 + j) * RT + in_row] : acc[kInLds ? 0 : i][j];
      *reinterpret_cast<float4*>(part + c) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(part + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
}

// dw[c] = sum of the workgroups' shares: 16 runs of them, each in order, then
// the runs in order.
__global__ __launch_bounds__(1024) void k_norm_dw(const float* __restrict__ part, int n, int H, void* __restrict__ dw,
                                                  bool fp32) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, run = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  const int per = cdiv(n, 16), first = run * per, last = min(n, first + per);
  float t = 0.0f;
  if (c < H) {
#pragma unroll 16
    for (int i = first; i < last; ++i) t += part[static_cast<int64_t>(i) * H + c];
  }
  red[run][lane] = t;
  __syncthreads();
  if (run != 0 || c >= H) return;
  t = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) t += red[i][lane];
  if (fp32) static_cast<float*>(dw)[c] = t;
  else static_cast<bf16_t*>(dw)[c] = f2bf(t);
}

// Waves of a row by its length: forward and backward.
int fwd_waves(int H) { return H <= 2048 ? 1 : H <= 8192 ? 4 : 16; }
int bwd_waves(int H) { return H <= 1024 ? 1 : H <= 4096 ? 4 : 16; }

template <int WAVES, int VEC>
void start_fwd(const NormFwd& a, hipStream_t s) {
  constexpr int rows = kFwdRows<WAVES>;
  hipLaunchKernelGGL((k_norm_fwd<WAVES, VEC>), dim3(cdiv(a.T, rows)), dim3(kRowThreads<WAVES> * rows), 0, s, a);
}
template <int WAVES, int VEC>
void start_bwd(const NormBwd& a, hipStream_t s) {
  constexpr int rows = kBwdRows<WAVES>;
  hipLaunchKernelGGL((k_norm_bwd<WAVES, VEC>), dim3(norm_bwd_parts(a.T, a.H)), dim3(kRowThreads<WAVES> * rows),
                     (VEC > 2 ? VEC * 8 * kRowThreads<WAVES> : rows > 1 ? rows * a.H : 0) * sizeof(float), s, a);
}

}  // namespace

// A grid dimension holds fewer than 2^32 threads: rows in slices.
constexpr int kSlice = 1 << 21;

hipError_t launch_norm_fwd(const NormFwd& all, hipStream_t s) {
  TraceScope trace_scope(K_NORM_FWD, s);
  const int waves = fwd_waves(all.H), vec = cdiv(all.H, waves * 512);
  for (int64_t t = 0; t < all.T; t += kSlice) {
    NormFwd a = all;
    const int64_t out = t * a.H;
    a.T = static_cast<int>(std::min<int64_t>(kSlice, all.T - t));
    a.x += t * a.ldx;
    if (a.r != nullptr) a.r += t * a.ldr;
    if (a.h != nullptr) a.h += out;
    if (a.y != nullptr) a.y += out;
    if (a.q != nullptr) a.q += out, a.scale += t;
    if (waves == 1) {
      if (vec == 1) start_fwd<1, 1>(a, s);
      else if (vec == 2) start_fwd<1, 2>(a, s);
      else if (vec == 3) start_fwd<1, 3>(a, s);
      else start_fwd<1, 4>(a, s);
    } else if (waves == 4) {
      if (vec == 2) start_fwd<4, 2>(a, s);
      else if (vec == 3) start_fwd<4, 3>(a, s);
      else start_fwd<4, 4>(a, s);
    } else {
      if (vec == 2) start_fwd<16, 2>(a, s);
      else if (vec == 3) start_fwd<16, 3>(a, s);
      else start_fwd<16, 4>(a, s);
    }
  }
  return hipGetLastError();
}

// Workgroups of the backward, hence shares of dw: enough to fill the chip, few
// enough that adding them costs little (a share is written and read again in
// fp32: 256 of rows of 5120 are 8% of what 3001 rows move, 512 are 17%).
int norm_bwd_parts(int T, int H) {
  const int waves = bwd_waves(H), rows = waves == 1 ? kBwdRows<1> : waves == 4 ? kBwdRows<4> : kBwdRows<16>;
  return std::min((T - 1) / rows + 1, waves == 16 ? 256 : 512);  // no sum that T near 2^31 overflows
}

hipError_t launch_norm_bwd(const NormBwd& a, hipStream_t s) {
  TraceScope trace_scope(K_NORM_BWD, s);
  const int waves = bwd_waves(a.H), vec = cdiv(a.H, waves * 512);
  if (waves == 1) {
    if (vec == 1) start_bwd<1, 1>(a, s);
    else start_bwd<1, 2>(a, s);
  } else if (waves == 4) {
    if (vec == 1) start_bwd<4, 1>(a, s);
    else start_bwd<4, 2>(a, s);
  } else {
    if (vec == 1) start_bwd<16, 1>(a, s);
    else if (vec == 2) start_bwd<16, 2>(a, s);
    else if (vec == 3) start_bwd<16, 3>(a, s);
    else start_bwd<16, 4>(a, s);
  }
  hipLaunchKernelGGL(k_norm_dw, dim3(cdiv(a.H, 64)), dim3(1024), 0, s, a.part, norm_bwd_parts(a.T, a.H), a.H, a.dw,
                     a.dw_fp32);
  return hipGetLastError();
}

}  // namespace moe
