// Rows of bf16 values, of the SwiGLU activation and of weights as int8 rows.
#include "i8_round.hpp"
#include "serve.hpp"
#include "trace.hpp"

namespace moe {

namespace {

// One wave per row.  Up to kHeld passes of 512 columns stay in registers; what
// lies beyond is read again for the rounding.  8192 x 2048: 10 us, 5 TB/s, the
// rate of a copy.
constexpr int kHeld = 8;

__global__ __launch_bounds__(256) void k_i8_quant_rows(const bf16_t* __restrict__ x, int64_t ldx, int rows, int K,
                                                       const int32_t* __restrict__ n_valid, int8_t* __restrict__ q,
                                                       float* __restrict__ scale) {
  const int lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= rows || (n_valid != nullptr && row >= *n_valid)) return;
  const bf16_t* src = x + row * ldx;
  uint4 held[kHeld];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int c = i * 512 + lane * 8;
    held[i] = c < K ? *reinterpret_cast<const uint4*>(src + c) : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < kHeld; ++i) m = max(m, top8(held[i]));
  for (int c = kHeld * 512 + lane * 8; c < K; c += 512) m = max(m, top8(*reinterpret_cast<const uint4*>(src + c)));
  const Rounder r(wave_umax(m));
  int8_t* dst = q + row * K;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int c = i * 512 + lane * 8;
    if (c < K) *reinterpret_cast<uint2*>(dst + c) = quant8(held[i], r);
  }
  for (int c = kHeld * 512 + lane * 8; c < K; c += 512)
    *reinterpret_cast<uint2*>(dst + c) = quant8(*reinterpret_cast<const uint4*>(src + c), r);
  if (lane == 0) scale[row] = r.scale;
}

// One wave per routed row: the row's largest magnitude is that of its partials,
// so the values are read once.  65536 x 768: 45 us, 5.7 TB/s of what it reads
// and writes.
__global__ __launch_bounds__(256) void k_i8_requant(const float* __restrict__ a, const float* __restrict__ a_top,
                                                    int rows, int F, const int32_t* __restrict__ n_valid,
                                                    int8_t* __restrict__ q, float* __restrict__ scale) {
  const int lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= rows || row >= *n_valid) return;
  const int parts = F / kI8Cols;
  const float* top = a_top + row * parts;
  uint32_t m = 0;
  for (int i = lane; i < parts; i += 64) m = max(m, __float_as_uint(top[i]));
  const Rounder r(wave_umax(m));
  for (int c = lane * 8; c < F; c += 512) {
    const float4 v = *reinterpret_cast<const float4*>(a + row * F + c);
    const float4 w = *reinterpret_cast<const float4*>(a + row * F + c + 4);
    const int b[8] = {r(v.x), r(v.y), r(v.z), r(v.w), r(w.x), r(w.y), r(w.z), r(w.w)};
    *reinterpret_cast<uint2*>(q + row * F + c) = make_uint2(pack4(b[0], b[1], b[2], b[3]), pack4(b[4], b[5], b[6], b[7]));
  }
  if (lane == 0) scale[row] = r.scale;
}

// 64 output channels per workgroup: their largest magnitudes over K first,
// then 64 x 64 blocks rounded and transposed through LDS.  128 x 2048 x 768: 580
// us against 117 of bytes; two passes of 2 bytes a lane bound it.  Weights are
// laid out once, so it was left simple.
__global__ __launch_bounds__(256) void k_i8_quant_weight(const bf16_t* __restrict__ w, int K, int N,
                                                         int8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t tops[4][64];
  __shared__ int8_t tile[64][64 + 16];
  const int n0 = blockIdx.x * 64, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int n = n0 + lane;
  const bf16_t* src = w + static_cast<int64_t>(blockIdx.y) * K * N;
  uint32_t m = 0;
  if (n < N)
    for (int k = wv; k < K; k += 4) m = max(m, static_cast<uint32_t>(src[static_cast<int64_t>(k) * N + n] & 0x7fff) << 16);
  tops[wv][lane] = m;
  __syncthreads();
  const Rounder r(max(max(tops[0][lane], tops[1][lane]), max(tops[2][lane], tops[3][lane])));
  const int64_t out = static_cast<int64_t>(blockIdx.y) * N + n0;
  if (wv == 0 && n < N) scale[out + lane] = r.scale;
  for (int k0 = 0; k0 < K; k0 += 64) {
    for (int k = wv; k < 64; k += 4)
      tile[lane][k] = k0 + k < K && n < N ? static_cast<int8_t>(r(bf2f(src[static_cast<int64_t>(k0 + k) * N + n]))) : 0;
    __syncthreads();
    const int row = threadIdx.x >> 2, c = (threadIdx.x & 3) * 16;
    if (n0 + row < N && k0 + c < K)
      *reinterpret_cast<uint4*>(q + (out + row) * K + k0 + c) = *reinterpret_cast<const uint4*>(&tile[row][c]);
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_i8_quant_rows(const bf16_t* x, int64_t ldx, int rows, int K, const int32_t* n_valid, int8_t* q,
                                float* scale, hipStream_t s) {
  TraceScope trace_scope(K_I8_QUANT, s);
  hipLaunchKernelGGL(k_i8_quant_rows, dim3(cdiv(rows, 4)), dim3(256), 0, s, x, ldx, rows, K, n_valid, q, scale);
  return hipGetLastError();
}

hipError_t launch_i8_requant(const float* a, const float* a_top, int rows, int F, const int32_t* n_valid, int8_t* q,
                             float* scale, hipStream_t s) {
  TraceScope trace_scope(K_I8_QUANT, s);
  hipLaunchKernelGGL(k_i8_requant, dim3(cdiv(rows, 4)), dim3(256), 0, s, a, a_top, rows, F, n_valid, q, scale);
  return hipGetLastError();
}

hipError_t launch_i8_quant_weight(const bf16_t* w, int E, int K, int N, int8_t* q, float* scale, hipStream_t s) {
  TraceScope trace_scope(K_I8_WEIGHT, s);
  hipLaunchKernelGGL(k_i8_quant_weight, dim3(cdiv(N, 64), E), dim3(256), 0, s, w, K, N, q, scale);
  return hipGetLastError();
}

}  // namespace moe
