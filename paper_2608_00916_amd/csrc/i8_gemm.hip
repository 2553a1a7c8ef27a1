// Products of int8 rows on the gfx950 matrix cores: C[m][n] = sum_k A[m][k]
// B[n][k], exact in int32, scaled by one factor per row of A and of B.
//
// Both operands are K-contiguous, so a tile step is KB bytes of each of its
// BM + BN rows.  They go straight from global memory into LDS (16 bytes per
// lane); v_mfma_i32_16x16x64_i8 takes 16 consecutive k per lane, one
// ds_read_b128.  A row's 16-byte chunks are XOR-swizzled so that the 16 rows
// of one fragment read lie in distinct banks; the copy into LDS is linear in
// the lanes, so the swizzle is applied to the global address instead.
//
// Rows past the last one read that row again (their results are not stored),
// and chunks past K are cleared in the A fragments of the last step, so no
// load leaves its operand.
//
// The B fragment is fed first: lane l then holds C[m = l % 16][n = 4 (l / 16)
// + i], four consecutive columns of one row.
#include "serve.hpp"
#include "trace.hpp"

namespace moe {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4 mfma_i8(const uint4& p, const uint4& q, i32x4 acc) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, p), __builtin_bit_cast(i32x4, q), acc, 0, 0,
                                               0);
}

// 16 bytes per lane from global memory to LDS at base + 16 lane.
__device__ __forceinline__ void copy_to_lds(const int8_t* src, int8_t* lds_base) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src),
                                   (__attribute__((address_space(3))) void*)(lds_base), 16, 0, 0);
}

// Every wave's copies into LDS have landed (a wave's own count as vector loads).
__device__ __forceinline__ void copies_landed() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// BM x BN tile over WM x WN waves in K steps of KB bytes.
template <int BM_, int BN_, int WM_, int WN_, int KB_>
struct I8Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KB = KB_;
  static constexpr int kWaves = WM * WN;
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  static constexpr int kStage = (BM + BN) * KB;
  static constexpr int kChunks = KB / 16;               // 16-byte chunks of a row
  static constexpr int kRowsPer = 64 / kChunks;         // rows one wave-wide copy covers
  static constexpr int kCopies = (BM + BN) / kRowsPer / kWaves;  // copies per wave and step
  static_assert(kCopies * kRowsPer * kWaves == BM + BN, "a step's rows must split evenly over the waves");
  static_assert(BM % (kRowsPer * kWaves) == 0, "a copy must not straddle A and B");
};

// Chunk position of chunk c of row r.  LDS has 64 banks (256 bytes): rows of
// 128 bytes repeat every 2, rows of 64 bytes every 4.
template <int KB>
__device__ __forceinline__ int swizzle(int r, int c) {
  return KB == 128 ? c ^ ((r >> 1) & 7) : c ^ ((r >> 2) & 3);
}

// One tile: a_row(r) and b_row(r) give the first byte of tile row r of either
// operand (any r below BM, BN; rows without data repeat another).
template <class C, class ARow, class BRow>
__device__ __forceinline__ void i8_tile(int K, ARow a_row, BRow b_row, int8_t* st0, int8_t* st1,
                                        i32x4 (&acc)[C::FM][C::FN]) {
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wv / C::WN, wn = wv % C::WN;
  const int8_t* src[C::kCopies];
  int chunk[C::kCopies];
#pragma unroll
  for (int i = 0; i < C::kCopies; ++i) {
    const int r = (i * C::kWaves + wv) * C::kRowsPer + lane / C::kChunks;
    chunk[i] = swizzle<C::KB>(r, lane % C::kChunks);
    src[i] = (r < C::BM ? a_row(r) : b_row(r - C::BM));
  }
  const int steps = cdiv(K, C::KB);
  auto load = [&](int kt, int8_t* st) {
    const bool last = (kt + 1) * C::KB > K;
#pragma unroll
    for (int i = 0; i < C::kCopies; ++i) {
      int off = kt * C::KB + chunk[i] * 16;
      if (last && off >= K) off = 0;
      copy_to_lds(src[i] + off, st + (i * C::kWaves + wv) * 1024);
    }
  };
#pragma unroll
  for (int m = 0; m < C::FM; ++m)
#pragma unroll
    for (int n = 0; n < C::FN; ++n) acc[m][n] = i32x4{0, 0, 0, 0};
  const int g = lane >> 4, row = lane & 15;
  auto compute = [&](int kt, const int8_t* st) {
    const int8_t* at = st + (wm * C::FM * 16 + row) * C::KB;
    const int8_t* bt = st + (C::BM + wn * C::FN * 16 + row) * C::KB;
#pragma unroll
    for (int s = 0; s < C::KB / 64; ++s) {
      uint4 a[C::FM], b[C::FN];
      const int c = swizzle<C::KB>(row, s * 4 + g) * 16;
#pragma unroll
      for (int n = 0; n < C::FN; ++n) b[n] = *reinterpret_cast<const uint4*>(bt + n * 16 * C::KB + c);
#pragma unroll
      for (int m = 0; m < C::FM; ++m) a[m] = *reinterpret_cast<const uint4*>(at + m * 16 * C::KB + c);
      if ((kt + 1) * C::KB > K && kt * C::KB + s * 64 + g * 16 >= K)
#pragma unroll
        for (int m = 0; m < C::FM; ++m) a[m] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int m = 0; m < C::FM; ++m)
#pragma unroll
        for (int n = 0; n < C::FN; ++n) acc[m][n] = mfma_i8(b[n], a[m], acc[m][n]);
    }
  };
  load(0, st0);
  for (int kt = 0; kt < steps; kt += 2) {
    copies_landed();
    if (kt + 1 < steps) load(kt + 1, st1);
    compute(kt, st0);
    if (kt + 1 >= steps) break;
    copies_landed();
    if (kt + 2 < steps) load(kt + 2, st0);
    compute(kt + 1, st1);
  }
}

// Tile coordinates of a 1-D grid: the grid's workgroups go to the 8 XCDs in
// turn; each XCD takes a contiguous run of tiles.
__device__ __forceinline__ int xcd_order(int i, int n) {
  const int x = i & 7, per = n >> 3, rest = n & 7;
  return x * per + min(x, rest) + (i >> 3);
}

using Dense = I8Tile<128, 128, 2, 2, 128>;

template <bool F32>
__global__ __launch_bounds__(Dense::kThreads) void k_i8_matmul(const int8_t* __restrict__ a,
                                                               const float* __restrict__ sa,
                                                               const int8_t* __restrict__ b,
                                                               const float* __restrict__ sb, int M, int N, int K,
                                                               void* __restrict__ out, int64_t ldo) {
  using C = Dense;
  __shared__ __attribute__((aligned(16))) int8_t st0[C::kStage];
  __shared__ __attribute__((aligned(16))) int8_t st1[C::kStage];
  const int nt = cdiv(N, C::BN);
  const int t = xcd_order(blockIdx.x, gridDim.x);
  const int m0 = t / nt * C::BM, n0 = t % nt * C::BN;
  i32x4 acc[C::FM][C::FN];
  i8_tile<C>(
      K, [&](int r) { return a + static_cast<int64_t>(min(m0 + r, M - 1)) * K; },
      [&](int r) { return b + static_cast<int64_t>(min(n0 + r, N - 1)) * K; }, st0, st1, acc);
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int mb = m0 + wv / C::WN * C::FM * 16 + (lane & 15), nb = n0 + wv % C::WN * C::FN * 16 + (lane >> 4) * 4;
#pragma unroll
  for (int m = 0; m < C::FM; ++m) {
    const int row = mb + m * 16;
    if (row >= M) continue;
    const float s = sa[row];
#pragma unroll
    for (int n = 0; n < C::FN; ++n) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = nb + n * 16 + i;
        if (col >= N) continue;
        const float v = static_cast<float>(acc[m][n][i]) * s * sb[col];
        if (F32) static_cast<float*>(out)[row * ldo + col] = v;
        else static_cast<bf16_t*>(out)[row * ldo + col] = f2bf(v);
      }
    }
  }
}

// The tile of the row-tile table that workgroup column `t` takes, or rows = 0.
struct RowTile {
  int first, e, rows;
};
__device__ __forceinline__ RowTile row_tile(const int2* desc, int t) {
  const int32_t* d = reinterpret_cast<const int32_t*>(desc + t);
  const int first = uniform_load(d), y = uniform_load(d + 1);
  return {first, y & 255, y >> 8};
}

// Gate and up columns side by side: each wave takes matching halves.
using GateUp = I8Tile<128, 256, 2, 4, 128>;

__global__ __launch_bounds__(GateUp::kThreads) void k_i8_gateup(I8Rows rt, const int8_t* __restrict__ x,
                                                                const float* __restrict__ sx,
                                                                const int32_t* __restrict__ rows, moe_i8_experts w,
                                                                int H, int F, int16_t* __restrict__ a,
                                                                float* __restrict__ a_top) {
  using C = GateUp;
  __shared__ __attribute__((aligned(16))) int8_t st0[C::kStage];
  __shared__ __attribute__((aligned(16))) int8_t st1[C::kStage];
  __shared__ uint32_t tops[C::BM];
  constexpr int kHalf = C::FN / 2;  // fragments of gate, then of up, per wave
  const int parts = F / kI8Cols;
  const int tiles = uniform_load(rt.tile_start + rt.E) * parts;
  for (int i = blockIdx.x; i < tiles; i += gridDim.x) {
    const int t = xcd_order(i, tiles);
    const int p = t % parts;
    const RowTile tile = row_tile(rt.tile_desc, t / parts);
    const int64_t col0 = static_cast<int64_t>(tile.e) * F + p * kI8Cols;
    i32x4 acc[C::FM][C::FN];
    __syncthreads();  // the stages and `tops` are free
    if (threadIdx.x < C::BM) tops[threadIdx.x] = 0;
    i8_tile<C>(
        H,
        [&](int r) {
          const int64_t row = tile.first + min(r, tile.rows - 1);
          return x + (rows != nullptr ? rows[row] : row) * static_cast<int64_t>(H);
        },
        [&](int r) {  // wave wn's 64 columns: 32 of gate, the same 32 of up
          const int8_t* m = (r & 32) ? w.w_up : w.w_gate;
          return m + (col0 + (r >> 6) * 32 + (r & 31)) * H;
        },
        st0, st1, acc);
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int mb = wv / C::WN * C::FM * 16 + (lane & 15), nb = wv % C::WN * 32 + (lane >> 4) * 4;
    float4 sg[kHalf], su[kHalf];
#pragma unroll
    for (int n = 0; n < kHalf; ++n) {
      sg[n] = *reinterpret_cast<const float4*>(w.s_gate + col0 + nb + n * 16);
      su[n] = *reinterpret_cast<const float4*>(w.s_up + col0 + nb + n * 16);
    }
    float act[C::FM][kHalf][4];
#pragma unroll
    for (int m = 0; m < C::FM; ++m) {
      const int r = mb + m * 16;
      const int64_t row = tile.first + min(r, tile.rows - 1);
      const float s = sx[rows != nullptr ? rows[row] : row];
      uint32_t top = 0;
#pragma unroll
      for (int n = 0; n < kHalf; ++n) {
        const float g4[4] = {sg[n].x, sg[n].y, sg[n].z, sg[n].w}, u4[4] = {su[n].x, su[n].y, su[n].z, su[n].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float gate = static_cast<float>(acc[m][n][i]) * s * g4[i];
          const float up = static_cast<float>(acc[m][n + kHalf][i]) * s * u4[i];
          act[m][n][i] = silu_f(gate) * up;
          top = max(top, __float_as_uint(act[m][n][i]) & 0x7fffffffu);
        }
      }
      // the row's other columns: lanes 16 apart, then the waves beside this one
      top = max(top, static_cast<uint32_t>(shfl_xor(static_cast<int>(top), 16)));
      top = max(top, static_cast<uint32_t>(shfl_xor(static_cast<int>(top), 32)));
      if (lane < 16) atomicMax(&tops[r], top);
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < C::FM; ++m) {
      const int r = mb + m * 16;
      if (r >= tile.rows) continue;
      const int64_t row = tile.first + r;
      const uint32_t tb = tops[r];
      const float top = __uint_as_float(tb);
      const float inv = tb == 0 || tb >= 0x7f800000u ? 0.0f : 32767.0f / top;
#pragma unroll
      for (int n = 0; n < kHalf; ++n) {
        int v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = tb >= 0x7f800000u ? 0 : static_cast<int>(__builtin_rintf(act[m][n][i] * inv));
        *reinterpret_cast<uint2*>(a + row * F + p * kI8Cols + nb + n * 16) =
            make_uint2((v[0] & 0xffff) | (static_cast<uint32_t>(v[1]) << 16),
                       (v[2] & 0xffff) | (static_cast<uint32_t>(v[3]) << 16));
      }
      if (wv % C::WN == 0 && lane < 16) a_top[row * parts + p] = top;
    }
  }
}

using Down = I8Tile<128, 128, 2, 2, 128>;

__global__ __launch_bounds__(Down::kThreads) void k_i8_down(I8Rows rt, const int8_t* __restrict__ a,
                                                            const float* __restrict__ sa, moe_i8_experts w, int H,
                                                            int F, bf16_t* __restrict__ o) {
  using C = Down;
  __shared__ __attribute__((aligned(16))) int8_t st0[C::kStage];
  __shared__ __attribute__((aligned(16))) int8_t st1[C::kStage];
  const int nt = H / C::BN;
  const int tiles = uniform_load(rt.tile_start + rt.E) * nt;
  for (int i = blockIdx.x; i < tiles; i += gridDim.x) {
    const int t = xcd_order(i, tiles);
    const RowTile tile = row_tile(rt.tile_desc, t / nt);
    const int n0 = t % nt * C::BN;
    const int64_t col0 = static_cast<int64_t>(tile.e) * H + n0;
    i32x4 acc[C::FM][C::FN];
    __syncthreads();  // the stages are free
    i8_tile<C>(
        F, [&](int r) { return a + static_cast<int64_t>(tile.first + min(r, tile.rows - 1)) * F; },
        [&](int r) { return w.w_down + (col0 + r) * F; }, st0, st1, acc);
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int mb = wv / C::WN * C::FM * 16 + (lane & 15), nb = wv % C::WN * C::FN * 16 + (lane >> 4) * 4;
#pragma unroll
    for (int m = 0; m < C::FM; ++m) {
      const int r = mb + m * 16;
      if (r >= tile.rows) continue;
      const int64_t row = tile.first + r;
      const float s = sa[row];
#pragma unroll
      for (int n = 0; n < C::FN; ++n) {
        const float4 sc = *reinterpret_cast<const float4*>(w.s_down + col0 + nb + n * 16);
        *reinterpret_cast<uint2*>(o + row * H + n0 + nb + n * 16) =
            make_uint2(pack_bf16x2(static_cast<float>(acc[m][n][0]) * s * sc.x, static_cast<float>(acc[m][n][1]) * s * sc.y),
                       pack_bf16x2(static_cast<float>(acc[m][n][2]) * s * sc.z, static_cast<float>(acc[m][n][3]) * s * sc.w));
      }
    }
  }
}

constexpr int kMaxGrid = 4096;

int max_tiles(const I8Rows& r) { return cdiv(r.rows_cap, 128) + r.E; }

}  // namespace

hipError_t launch_i8_matmul(const int8_t* a, const float* sa, const int8_t* b, const float* sb, int M, int N, int K,
                            void* out, int64_t ldo, bool f32, hipStream_t s) {
  TraceScope trace_scope(K_I8_MATMUL, s);
  const dim3 grid(cdiv(M, Dense::BM) * cdiv(N, Dense::BN));
  if (f32) hipLaunchKernelGGL(k_i8_matmul<true>, grid, dim3(Dense::kThreads), 0, s, a, sa, b, sb, M, N, K, out, ldo);
  else hipLaunchKernelGGL(k_i8_matmul<false>, grid, dim3(Dense::kThreads), 0, s, a, sa, b, sb, M, N, K, out, ldo);
  return hipGetLastError();
}

hipError_t launch_i8_gateup(const I8Rows& r, const int8_t* x, const float* sx, const int32_t* rows,
                            const moe_i8_experts& w, int H, int F, int16_t* a, float* a_top, hipStream_t s) {
  TraceScope trace_scope(K_I8_GATEUP, s);
  const int64_t tiles = static_cast<int64_t>(max_tiles(r)) * (F / kI8Cols);
  const int grid = static_cast<int>(tiles < kMaxGrid ? tiles : kMaxGrid);
  hipLaunchKernelGGL(k_i8_gateup, dim3(grid), dim3(GateUp::kThreads), 0, s, r, x, sx, rows, w, H, F, a, a_top);
  return hipGetLastError();
}

hipError_t launch_i8_down(const I8Rows& r, const int8_t* a, const float* sa, const moe_i8_experts& w, int H, int F,
                          bf16_t* o, hipStream_t s) {
  TraceScope trace_scope(K_I8_DOWN, s);
  const int64_t tiles = static_cast<int64_t>(max_tiles(r)) * (H / Down::BN);
  const int grid = static_cast<int>(tiles < kMaxGrid ? tiles : kMaxGrid);
  hipLaunchKernelGGL(k_i8_down, dim3(grid), dim3(Down::kThreads), 0, s, r, a, sa, w, H, F, o);
  return hipGetLastError();
}

}  // namespace moe
