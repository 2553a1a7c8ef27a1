// Products of int8 rows: dense, few rows (each weight read once, straight into
// registers), and grouped over the experts.
#include "i8_core.hpp"
#include "i8_round.hpp"
#include "serve.hpp"
#include "trace.hpp"

namespace moe {

namespace {

// ---------------------------------------------------------------- dense
struct DenseArgs {
  const int8_t* a;
  const float* sa;
  const int8_t* b;
  const float* sb;
  int M, N, K;
  void* out;
  int64_t ldo;
};

// Tiles in bands of kBand row tiles, down the rows first: the tiles that run
// at once on an XCD share their rows of A and of B in its L2.
// kWide: N and the output's pitch allow 16-byte stores.
template <class C, bool F32, bool kWide>
struct DenseJob {
  static constexpr int kBand = C::BM == 256 ? 4 : 8;
  struct Tile {
    int m0, n0, rows;
  };
  DenseArgs p;
  Items items;
  float* swap;  // !kWide: 16 rows of this wave's 64 columns, float4s XOR-swizzled by row
  float sa[C::FM];
  float4 sb[C::FN];

  __device__ __forceinline__ Tile tile(int i) const {
    const int mt = cdiv(p.M, C::BM), nt = cdiv(p.N, C::BN);
    int t, half;
    items.at(i, &t, &half);
    t = xcd_order(t, mt * nt);
    const int band = t / (kBand * nt), in = t % (kBand * nt);
    const int h = min(kBand, mt - band * kBand);
    const int m0 = (band * kBand + in % h) * C::BM + (half > 0 ? C::BM / 2 : 0);
    return {m0, in / h * C::BN, min(half < 0 ? C::BM : C::BM / 2, p.M - m0)};
  }
  static constexpr int kParts = 1;
  static constexpr bool kSkip = C::WM > 1, kAnyInt8 = true;
  __device__ __forceinline__ I8Source a(const Tile& t) const {
    return {p.a + static_cast<int64_t>(t.m0) * p.K, t.rows};
  }
  __device__ __forceinline__ I8Source b(const Tile& t, int) const {
    return {p.b + static_cast<int64_t>(t.n0) * p.K, min(C::BN, p.N - t.n0)};
  }
  static __device__ __forceinline__ int b_part(int) { return 0; }
  static __device__ __forceinline__ int b_row(int q) { return q; }
  __device__ __forceinline__ int row0() const { return (threadIdx.x >> 6) / C::WN * C::FM * 16 + (threadIdx.x & 15); }
  __device__ __forceinline__ int col0() const {
    return (threadIdx.x >> 6) % C::WN * C::FN * 16 + ((threadIdx.x & 63) >> 4) * 8;
  }
  __device__ __forceinline__ void prefetch(const Tile& t) {
#pragma unroll
    for (int m = 0; m < C::FM; ++m) sa[m] = p.sa[min(t.m0 + row0() + m * 16, p.M - 1)];
    const int c = t.n0 + col0();
#pragma unroll
    for (int n = 0; n < C::FN; ++n) {
      const int cn = c + C::col(n);
      if (kWide) sb[n] = *reinterpret_cast<const float4*>(p.sb + min(cn, p.N - 4));
      else sb[n] = make_float4(p.sb[min(cn, p.N - 1)], p.sb[min(cn + 1, p.N - 1)], p.sb[min(cn + 2, p.N - 1)],
                               p.sb[min(cn + 3, p.N - 1)]);
    }
  }
  __device__ __forceinline__ void finish(const Tile& t, const i32x4 (&acc)[C::FM][C::FN]) const {
    const int c = t.n0 + col0(), r0 = t.m0 + row0();
    constexpr int kSize = F32 ? 4 : 2;
    char* dst = static_cast<char*>(p.out) + (r0 * p.ldo + c) * kSize;
#pragma unroll
    for (int m = 0; m < C::FM; ++m, dst += p.ldo * (16 * kSize)) {
      float v[4 * C::FN];
#pragma unroll
      for (int n = 0; n < C::FN; ++n) {
        v[4 * n] = static_cast<float>(acc[m][n][0]) * sa[m] * sb[n].x;
        v[4 * n + 1] = static_cast<float>(acc[m][n][1]) * sa[m] * sb[n].y;
        v[4 * n + 2] = static_cast<float>(acc[m][n][2]) * sa[m] * sb[n].z;
        v[4 * n + 3] = static_cast<float>(acc[m][n][3]) * sa[m] * sb[n].w;
      }
      if constexpr (!kWide) {
        // rows of odd pitch: 64 consecutive columns of a row per store
        const int lane = threadIdx.x & 63, rows = p.M - (r0 + m * 16 - (lane & 15));
        const int col = c - (lane >> 4) * 8 + lane;
#pragma unroll
        for (int n = 0; n < C::FN; ++n)
          *reinterpret_cast<float4*>(swap + (lane & 15) * 64 + 4 * ((2 * (lane >> 4) + C::col(n) / 4) ^ (lane & 15))) =
              make_float4(v[4 * n], v[4 * n + 1], v[4 * n + 2], v[4 * n + 3]);
        char* line = static_cast<char*>(p.out) + ((r0 + m * 16 - (lane & 15)) * p.ldo + col) * kSize;
#pragma unroll
        for (int h = 0; h < 16; h += 8) {  // eight reads under way at once
          float x[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) x[r] = swap[(h + r) * 64 + (4 * ((lane >> 2) ^ (h + r)) | (lane & 3))];
#pragma unroll
          for (int r = 0; r < 8; ++r, line += p.ldo * kSize) {
            if (h + r >= rows || col >= p.N) continue;
            if (F32) *reinterpret_cast<float*>(line) = x[r];
            else *reinterpret_cast<bf16_t*>(line) = f2bf(x[r]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);  // one row of fragments at a time: registers
        continue;
      }
      if (r0 + m * 16 >= p.M) continue;
#pragma unroll
      for (int i = 0; i < 4 * C::FN; i += 16 / kSize) {
        if (c + C::col(i / 4) >= p.N) continue;
        uint4 w;
        if (F32) w = __builtin_bit_cast(uint4, make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]));
        else w = make_uint4(pack_bf16x2(v[i], v[i + 1]), pack_bf16x2(v[i + 2], v[i + 3]),
                            pack_bf16x2(v[i + 4], v[i + 5]), pack_bf16x2(v[i + 6], v[i + 7]));
        *reinterpret_cast<uint4*>(dst + C::col(i / 4) * kSize) = w;
      }
    }
  }
};

template <class C, bool kTail, bool F32, bool kWide>
__global__ __launch_bounds__(C::kThreads) void k_i8_matmul(DenseArgs p) {
  __shared__ __attribute__((aligned(16))) int8_t st[2 * C::kStage];
  using Job = DenseJob<C, F32, kWide>;
  __shared__ __attribute__((aligned(16))) float swap[kWide ? 4 : C::kWaves * 16 * 64];
  const Items items(C::WM > 1, cdiv(p.M, C::BM) * cdiv(p.N, C::BN));
  Job job{p, items, swap + (kWide ? 0 : (threadIdx.x >> 6) * 16 * 64)};
  i8_stream<C, kTail, false>(p.K, items.count(), job, st);
}

// ---------------------------------------------------------------- few rows
// Tiles of 16 MT x 16 NT whose 8 waves take the 64-byte slices of k in turn:
// every wave has operands of its own, so they go straight into registers, with
// several slices of each wave in flight at once; the waves' sums meet in LDS.
// Where tiles are few this beats the streamed tiles, whose steps follow each
// other (512 x 1024 x 8192: 64 steps of 0.6 us).  With kFused the rows of A are
// bf16, and every workgroup rounds them to int8 in LDS itself: one launch, no
// trip through memory.
constexpr int kFewWaves = 8;
constexpr int kFusedRows = 16, kFusedBytes = 49152;

template <int MT, int NT, bool kFused, bool F32>
__global__ __launch_bounds__(64 * kFewWaves) void k_i8_few(DenseArgs p, const bf16_t* __restrict__ x, int64_t ldx) {
  extern __shared__ __attribute__((aligned(16))) int8_t a8[];  // kFused: [M][K + 16]
  __shared__ i32x4 sums[kFewWaves][MT][NT][64];
  __shared__ float scales[kFusedRows];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, g = lane >> 4, i16 = lane & 15;
  const int nt = cdiv(p.N, 16 * NT);
  const int m0 = blockIdx.x / nt * (16 * MT), n0 = blockIdx.x % nt * (16 * NT);
  const int8_t *arow[MT], *brow[NT];
#pragma unroll
  for (int m = 0; m < MT; ++m) arow[m] = p.a + static_cast<int64_t>(min(m0 + m * 16 + i16, p.M - 1)) * p.K;
#pragma unroll
  for (int n = 0; n < NT; ++n) brow[n] = p.b + static_cast<int64_t>(min(n0 + n * 16 + i16, p.N - 1)) * p.K;
  constexpr int kAhead = NT == 1 ? 4 : 2;  // slices in flight per wave
  const int slices = cdiv(p.K, 64);
  uint4 b[kAhead][NT], a[kFused ? 1 : kAhead][MT];
  // chunks past K are read from K's last one and cleared in A
  auto load = [&](int s, int i) {
    const int k = min(s, slices - 1) * 64 + g * 16, kk = min(k, p.K - 16);
#pragma unroll
    for (int n = 0; n < NT; ++n) b[i][n] = *reinterpret_cast<const uint4*>(brow[n] + kk);
    if constexpr (!kFused) {
#pragma unroll
      for (int m = 0; m < MT; ++m) a[i][m] = *reinterpret_cast<const uint4*>(arow[m] + kk);
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) load(wv + i * kFewWaves, i);
  if constexpr (kFused) {
    for (int r = wv; r < p.M; r += kFewWaves) {
      const bf16_t* src = x + r * ldx;
      uint32_t m = 0;
      for (int c = lane * 8; c < p.K; c += 512) m = max(m, top8(*reinterpret_cast<const uint4*>(src + c)));
      const Rounder f(wave_umax(m));
      for (int c = lane * 8; c < p.K; c += 512)
        *reinterpret_cast<uint2*>(a8 + r * (p.K + 16) + c) = quant8(*reinterpret_cast<const uint4*>(src + c), f);
      if (lane == 0) scales[r] = f.scale;
    }
    __syncthreads();
  }
  i32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = i32x4{0, 0, 0, 0};
  for (int s0 = wv; s0 < slices; s0 += kAhead * kFewWaves) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int s = s0 + i * kFewWaves;
      const int k = s * 64 + g * 16;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        uint4 x8 = make_uint4(0, 0, 0, 0);
        if constexpr (kFused) {
          if (i16 < p.M && k < p.K) x8 = *reinterpret_cast<const uint4*>(a8 + i16 * (p.K + 16) + k);
        } else {
          if (k < p.K) x8 = a[i][m];
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = mfma_i8(b[i][n], x8, acc[m][n]);
      }
      load(s + kAhead * kFewWaves, i);
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) sums[wv][m][n][lane] = acc[m][n];
  __syncthreads();
  for (int i = threadIdx.x; i < MT * NT * 256; i += 64 * kFewWaves) {
    const int c = i % (16 * NT), r = i / (16 * NT), row = m0 + r, col = n0 + c;
    if (row >= p.M || col >= p.N) continue;
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) sum += sums[w][r >> 4][c >> 4][(c >> 2 & 3) * 16 + (r & 15)][c & 3];
    const float v = static_cast<float>(unwrap(static_cast<int>(sum))) * (kFused ? scales[row] : p.sa[row]) * p.sb[col];
    if (F32) static_cast<float*>(p.out)[row * p.ldo + col] = v;
    else static_cast<bf16_t*>(p.out)[row * p.ldo + col] = f2bf(v);
  }
}

// ---------------------------------------------------------------- grouped
// Row tiles of the experts, BM rows each: the running count of tiles per expert, in LDS.
template <class C>
struct RowTiles {
  const int32_t* offsets;
  const int* first;  // [E + 1]
  int E;
  __device__ __forceinline__ void find(int i, int half, int* e, int* row, int* rows) const {
    int lo = 0, hi = E;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= i) lo = mid;
      else hi = mid;
    }
    *e = __builtin_amdgcn_readfirstlane(lo);
    const int off = uniform_load(offsets + *e), end = uniform_load(offsets + *e + 1);
    *row = off + (i - __builtin_amdgcn_readfirstlane(first[*e])) * C::BM + (half > 0 ? C::BM / 2 : 0);
    *rows = min(half < 0 ? C::BM : C::BM / 2, end - *row);
  }
};

// first[0 .. E]: every thread calls it.
template <class C>
__device__ __forceinline__ void count_row_tiles(const int32_t* offsets, int E, int* first) {
  const int e = threadIdx.x;
  if (e < 64) {  // one wave, up to 4 experts a lane (E <= 256)
    int n[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int x = e * 4 + i;
      n[i] = x < E ? cdiv(offsets[x + 1] - offsets[x], C::BM) : 0;
      sum += n[i];
    }
    int incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int u = __shfl_up(incl, off, 64);
      incl += e >= off ? u : 0;
    }
    int run = incl - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (e * 4 + i <= E) first[e * 4 + i] = run;
      run += n[i];
    }
    if (e == 63 && E == 256) first[256] = run;
  }
  __syncthreads();
}

struct GroupedArgs {
  const int32_t* offsets;
  int E;
  const int8_t* x;      // rows of A
  const float* sx;      // their scales
  const int32_t* rows;  // gate/up: row of x of each routed row, or null
  moe_i8_experts w;
  int H, F;
  float* act;  // gate/up out
  float* top;
  bf16_t* o;  // down out
};

// Gate and up columns side by side: a lane's first run of 8 columns is of
// gate, the other the same columns of up.  A tile is BN / 2 columns of both;
// a wave's 32 columns of one row are one partial of the activation.
template <class C, bool kGather>
struct GateUpJob {
  static constexpr int kHalf = 8, kPart = kI8Cols, kCols = C::BN / 2;
  struct Tile {
    int e, row, rows, col;
  };
  GroupedArgs p;
  RowTiles<C> rt;
  Items items;
  float s[C::FM];
  float4 sg[C::FN / 2], su[C::FN / 2];

  // the column tiles of a row tile in turn: they share its rows of x
  __device__ __forceinline__ Tile tile(int i) const {
    const int nt = p.F / kCols;
    int t, half;
    items.at(i, &t, &half);
    t = xcd_order(t, items.tiles);
    Tile x;
    rt.find(t / nt, half, &x.e, &x.row, &x.rows);
    x.col = t % nt * kCols;
    return x;
  }
  static constexpr int kParts = 2;  // gate, up
  static constexpr bool kSkip = C::WM > 1, kAnyInt8 = false;  // rows rounded here
  __device__ __forceinline__ int64_t source(int row) const { return kGather ? p.rows[row] : row; }
  __device__ __forceinline__ I8Source a(const Tile& t) const {
    if (kGather) return {p.x, t.rows, p.rows + t.row};
    return {p.x + static_cast<int64_t>(t.row) * p.H, t.rows};
  }
  __device__ __forceinline__ I8Source b(const Tile& t, int part) const {
    return {(part ? p.w.w_up : p.w.w_gate) + (static_cast<int64_t>(t.e) * p.F + t.col) * p.H, kCols};
  }
  static __device__ __forceinline__ int b_part(int q) { return q / kPart & 1; }
  static __device__ __forceinline__ int b_row(int q) { return q / (2 * kPart) * kPart + q % kPart; }
  __device__ __forceinline__ int row0() const { return (threadIdx.x >> 6) / C::WN * C::FM * 16 + (threadIdx.x & 15); }
  __device__ __forceinline__ int col0() const {
    return (threadIdx.x >> 6) % C::WN * kPart + ((threadIdx.x & 63) >> 4) * kHalf;
  }
  __device__ __forceinline__ void prefetch(const Tile& t) {
#pragma unroll
    for (int m = 0; m < C::FM; ++m) s[m] = p.sx[source(t.row + min(row0() + m * 16, t.rows - 1))];
    const int64_t c = static_cast<int64_t>(t.e) * p.F + t.col + col0();
#pragma unroll
    for (int n = 0; n < C::FN / 2; ++n) {
      sg[n] = *reinterpret_cast<const float4*>(p.w.s_gate + c + n * 4);
      su[n] = *reinterpret_cast<const float4*>(p.w.s_up + c + n * 4);
    }
  }
  // With G = s g, U = s u (s the row's scale): silu(G) U = s g / (1 + e^-G) s u,
  // the gate closed first: G U may pass fp32 where silu(G) is 0.
  // It is left in fp32: in 16 bits, each with its partial's scale, one value in
  // 1000 came out a step of its 8 bits away, which rows of few columns show
  // (0.004 of the output against 0.0017; 3 percent faster at 65536 rows).
  __device__ __forceinline__ void finish(const Tile& t, const i32x4 (&acc)[C::FM][C::FN]) const {
    static_assert(kHalf == 8, "two 16-byte stores a row");
    const int parts = p.F / kPart;
#pragma unroll
    for (int m = 0; m < C::FM; ++m) {
      const int r = row0() + m * 16;
      const float e = s[m] * -1.4426950408889634f;
      float v[kHalf];
      uint32_t top = 0;
#pragma unroll
      for (int n = 0; n < C::FN / 2; ++n) {
        const float g4[4] = {sg[n].x, sg[n].y, sg[n].z, sg[n].w}, u4[4] = {su[n].x, su[n].y, su[n].z, su[n].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float gate = static_cast<float>(acc[m][n][i]) * g4[i];
          const float up = static_cast<float>(acc[m][n + C::FN / 2][i]) * u4[i];
          const float sig = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(gate * e));
          v[4 * n + i] = gate * s[m] * sig * (up * s[m]);
          top = max(top, __float_as_uint(v[4 * n + i]) & 0x7fffffffu);
        }
      }
      top = max(top, static_cast<uint32_t>(shfl_xor(static_cast<int>(top), 16)));
      top = max(top, static_cast<uint32_t>(shfl_xor(static_cast<int>(top), 32)));
      if (r >= t.rows) continue;
      const int64_t row = t.row + r;
      float* dst = p.act + row * p.F + t.col + col0();
      *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(dst + 4) = make_float4(v[4], v[5], v[6], v[7]);
      if ((threadIdx.x & 63) < 16) p.top[row * parts + (t.col + col0()) / kPart] = __uint_as_float(top);
    }
  }
};

template <class C, bool>
struct DownJob {
  struct Tile {
    int e, row, rows, col;
  };
  GroupedArgs p;
  RowTiles<C> rt;
  Items items;
  float s[C::FM];
  float4 sw[C::FN];

  __device__ __forceinline__ Tile tile(int i) const {
    const int nt = cdiv(p.H, C::BN);
    int t, half;
    items.at(i, &t, &half);
    t = xcd_order(t, items.tiles);
    Tile x;
    rt.find(t / nt, half, &x.e, &x.row, &x.rows);
    x.col = t % nt * C::BN;
    return x;
  }
  static constexpr int kParts = 1;
  static constexpr bool kSkip = C::WM > 1, kAnyInt8 = false;  // rows rounded here
  __device__ __forceinline__ I8Source a(const Tile& t) const {
    return {p.x + static_cast<int64_t>(t.row) * p.F, t.rows};
  }
  __device__ __forceinline__ I8Source b(const Tile& t, int) const {
    return {p.w.w_down + (static_cast<int64_t>(t.e) * p.H + t.col) * p.F, min(C::BN, p.H - t.col)};
  }
  static __device__ __forceinline__ int b_part(int) { return 0; }
  static __device__ __forceinline__ int b_row(int q) { return q; }
  __device__ __forceinline__ int row0() const { return (threadIdx.x >> 6) / C::WN * C::FM * 16 + (threadIdx.x & 15); }
  __device__ __forceinline__ int col0() const {
    return (threadIdx.x >> 6) % C::WN * C::FN * 16 + ((threadIdx.x & 63) >> 4) * 8;
  }
  __device__ __forceinline__ void prefetch(const Tile& t) {
#pragma unroll
    for (int m = 0; m < C::FM; ++m) s[m] = p.sx[t.row + min(row0() + m * 16, t.rows - 1)];
#pragma unroll
    for (int n = 0; n < C::FN; ++n)
      sw[n] = *reinterpret_cast<const float4*>(p.w.s_down + static_cast<int64_t>(t.e) * p.H +
                                               min(t.col + col0() + C::col(n), p.H - 4));
  }
  __device__ __forceinline__ void finish(const Tile& t, const i32x4 (&acc)[C::FM][C::FN]) const {
    const int c = t.col + col0();
    // H is a multiple of 128: of a wave's 64 columns all are there or none is
    if (c >= p.H) return;
#pragma unroll
    for (int m = 0; m < C::FM; ++m) {
      const int r = row0() + m * 16;
      if (r >= t.rows) continue;
      bf16_t* dst = p.o + static_cast<int64_t>(t.row + r) * p.H + c;
#pragma unroll
      for (int n = 0; n < C::FN; n += 2) {
        const auto f = [&](int nn, int i, float w) { return static_cast<float>(acc[m][nn][i]) * s[m] * w; };
        *reinterpret_cast<uint4*>(dst + C::col(n)) =
            make_uint4(pack_bf16x2(f(n, 0, sw[n].x), f(n, 1, sw[n].y)), pack_bf16x2(f(n, 2, sw[n].z), f(n, 3, sw[n].w)),
                       pack_bf16x2(f(n + 1, 0, sw[n + 1].x), f(n + 1, 1, sw[n + 1].y)),
                       pack_bf16x2(f(n + 1, 2, sw[n + 1].z), f(n + 1, 3, sw[n + 1].w)));
      }
    }
  }
};

template <class C, template <class, bool> class Job, bool kGather>
__global__ __launch_bounds__(C::kThreads) void k_i8_grouped(GroupedArgs p, int K, int col_tiles) {
  __shared__ __attribute__((aligned(16))) int8_t st[2 * C::kStage];
  __shared__ int first[MOE_MAX_EXPERTS + 1];
  count_row_tiles<C>(p.offsets, p.E, first);
  const Items items(C::WM > 1, __builtin_amdgcn_readfirstlane(first[p.E]) * col_tiles);
  Job<C, kGather> job{p, {p.offsets, first, p.E}, items};
  i8_stream<C, false, kGather>(K, items.count(), job, st);
}

constexpr int kCus = 256;

using Tall = I8Tile<256, 256, 2, 4>;   // 128 KB of LDS: one workgroup per CU
using Small = I8Tile<128, 128, 2, 2>;  // 64 KB: two
using Low = I8Tile<32, 256, 1, 4>;     // 72 KB: two

int grid_of(int64_t items, int per_cu) { return static_cast<int>(items < kCus * per_cu ? items : kCus * per_cu); }

template <class C, bool kTail, bool F32>
void launch_dense(const DenseArgs& p, int per_cu, hipStream_t s) {
  const int64_t tiles = static_cast<int64_t>(cdiv(p.M, C::BM)) * cdiv(p.N, C::BN);
  const dim3 grid(grid_of(2 * tiles, per_cu)), block(C::kThreads);
  if (p.N % 8 == 0 && p.ldo % 8 == 0) hipLaunchKernelGGL((k_i8_matmul<C, kTail, F32, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((k_i8_matmul<C, kTail, F32, false>), grid, block, 0, s, p);
}

template <class C>
void launch_dense(const DenseArgs& p, bool f32, int per_cu, hipStream_t s) {
  const bool tail = p.K % kI8Step != 0;
  if (tail && f32) launch_dense<C, true, true>(p, per_cu, s);
  else if (tail) launch_dense<C, true, false>(p, per_cu, s);
  else if (f32) launch_dense<C, false, true>(p, per_cu, s);
  else launch_dense<C, false, false>(p, per_cu, s);
}

template <int MT, int NT, bool kFused>
void launch_few(const DenseArgs& p, const bf16_t* x, int64_t ldx, bool f32, hipStream_t s) {
  const dim3 grid(cdiv(p.M, 16 * MT) * cdiv(p.N, 16 * NT)), block(64 * kFewWaves);
  const int lds = kFused ? p.M * (p.K + 16) : 0;
  if (f32) hipLaunchKernelGGL((k_i8_few<MT, NT, kFused, true>), grid, block, lds, s, p, x, ldx);
  else hipLaunchKernelGGL((k_i8_few<MT, NT, kFused, false>), grid, block, lds, s, p, x, ldx);
}

template <class C, template <class, bool> class Job, bool kGather>
void launch_grouped(const GroupedArgs& p, int rows_cap, int K, int col_tiles, int per_cu, hipStream_t s) {
  const int64_t tiles = (cdiv64(rows_cap, C::BM) + p.E) * col_tiles;
  const dim3 grid(grid_of(2 * tiles, per_cu));
  hipLaunchKernelGGL((k_i8_grouped<C, Job, kGather>), grid, dim3(C::kThreads), 0, s, p, K, col_tiles);
}

template <class C>
void launch_gateup(const GroupedArgs& p, int rows_cap, int per_cu, hipStream_t s) {
  const int col_tiles = p.F / (C::BN / 2);
  if (p.rows != nullptr) launch_grouped<C, GateUpJob, true>(p, rows_cap, p.H, col_tiles, per_cu, s);
  else launch_grouped<C, GateUpJob, false>(p, rows_cap, p.H, col_tiles, per_cu, s);
}

template <class C>
void launch_down(const GroupedArgs& p, int rows_cap, int per_cu, hipStream_t s) {
  launch_grouped<C, DownJob, false>(p, rows_cap, p.F, cdiv(p.H, C::BN), per_cu, s);
}

// The lowest tile that runs in one round of two workgroups per CU, counting half
// a part-filled row tile per expert; Low and Small also while most of a higher
// tile would be empty.  us of the gate/up product as Low, Small, Tall (H 2048,
// F 768; E x rows per expert): 8 x 200 18 19 22; 8 x 512 31 21 24; 8 x 1024 54
// 37 35; 128 x 16 73 76 83; 128 x 64 99 86 92; 128 x 128 150 113 105; down: 8 x
// 128 9 11 13; 16 x 200 17 13 17; 128 x 96 56 44 49; 128 x 512 306 202 173.
enum class Rows { kLow, kSmall, kTall };

Rows rows_of(int rows_cap, int E, int width) {
  const auto one_round = [&](int bm, int bn) {
    return (static_cast<double>(rows_cap) / bm + 0.5 * E) * cdiv(width, bn) < 2 * kCus;
  };
  if (rows_cap <= 16ll * E || one_round(Low::BM, Low::BN)) return Rows::kLow;
  if (rows_cap <= 96ll * E || one_round(Small::BM, Small::BN)) return Rows::kSmall;
  return Rows::kTall;
}

}  // namespace

hipError_t launch_i8_matmul(const int8_t* a, const float* sa, const int8_t* b, const float* sb, int M, int N, int K,
                            void* out, int64_t ldo, bool f32, hipStream_t s) {
  TraceScope trace_scope(K_I8_MATMUL, s);
  const DenseArgs p{a, sa, b, sb, M, N, K, out, ldo};
  // Few tiles: 8 waves split k within a tile, up to one tile per CU (a weight
  // for up to 64 rows: two).  us at K 8192, as 16 MT x 16, 32 x 64, 64 x 64 and
  // streamed: 16 x 5120 16 21 28 40; 64 x 1024 20 25 33 39; 64 x 5120 39 25 33
  // 40; 512 x 1024 - 26 34 40; 1024 x 1024 - 47 35 41; 128 x 16384 - 92 68 45.
  // The longer K, the more: 512 x 1024 takes 9 13 13 at K 2048, 7 10 6 at 512.
  // Tall tiles gain once there is one for every CU: 320 of them at K 2048 53
  // against 54, 512 70 against 79, but 160 32 against 29.
  const auto tiles = [&](int bm, int bn) { return static_cast<int64_t>(cdiv(M, bm)) * cdiv(N, bn); };
  if (M <= 64 && cdiv(M, 16) * tiles(64, 16) <= 2 * kCus) {
    if (M <= 16) launch_few<1, 1, false>(p, nullptr, 0, f32, s);
    else if (M <= 32) launch_few<2, 1, false>(p, nullptr, 0, f32, s);
    else launch_few<4, 1, false>(p, nullptr, 0, f32, s);
  } else if (M <= 32 || (K >= 1024 && tiles(32, 64) <= kCus)) {
    launch_few<2, 4, false>(p, nullptr, 0, f32, s);
  } else if (K >= 4096 && tiles(64, 64) <= kCus) {
    launch_few<4, 4, false>(p, nullptr, 0, f32, s);
  } else if (tiles(256, 256) >= kCus) {
    launch_dense<Tall>(p, f32, 1, s);
  } else {
    launch_dense<Small>(p, f32, 2, s);
  }
  return hipGetLastError();
}

bool launch_i8_linear_fused(const bf16_t* x, int64_t ldx, const int8_t* b, const float* sb, int M, int N, int K,
                            void* out, int64_t ldo, bool f32, hipStream_t s) {
  if (M > kFusedRows || static_cast<int64_t>(M) * (K + 16) > kFusedBytes) return false;
  TraceScope trace_scope(K_I8_MATMUL, s);
  launch_few<1, 1, true>(DenseArgs{nullptr, nullptr, b, sb, M, N, K, out, ldo}, x, ldx, f32, s);
  return true;
}

hipError_t launch_i8_gateup(const I8Rows& r, const int8_t* x, const float* sx, const int32_t* rows,
                            const moe_i8_experts& w, int H, int F, float* a, float* a_top, hipStream_t s) {
  TraceScope trace_scope(K_I8_GATEUP, s);
  const GroupedArgs p{r.offsets, r.E, x, sx, rows, w, H, F, a, a_top, nullptr};
  switch (rows_of(r.rows_cap, r.E, F * 2)) {
    case Rows::kLow: launch_gateup<Low>(p, r.rows_cap, 2, s); break;
    case Rows::kSmall: launch_gateup<Small>(p, r.rows_cap, 2, s); break;
    case Rows::kTall: launch_gateup<Tall>(p, r.rows_cap, 1, s); break;
  }
  return hipGetLastError();
}

hipError_t launch_i8_down(const I8Rows& r, const int8_t* a, const float* sa, const moe_i8_experts& w, int H, int F,
                          bf16_t* o, hipStream_t s) {
  TraceScope trace_scope(K_I8_DOWN, s);
  const GroupedArgs p{r.offsets, r.E, a, sa, nullptr, w, H, F, nullptr, nullptr, o};
  switch (rows_of(r.rows_cap, r.E, H)) {
    case Rows::kLow: launch_down<Low>(p, r.rows_cap, 2, s); break;
    case Rows::kSmall: launch_down<Small>(p, r.rows_cap, 2, s); break;
    case Rows::kTall: launch_down<Tall>(p, r.rows_cap, 1, s); break;
  }
  return hipGetLastError();
}

}  // namespace moe
