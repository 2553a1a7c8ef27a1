// The next token of each row of logits, from a given uniform number:
// temperature, then the top_k largest, then the shortest prefix of those that
// holds top_p of their weight, then those of at least min_p of the largest
// weight; of what is left the first in index order at which the running sum of
// the weights passes u times their sum.  Larger logits come first, equal ones
// by lower index.
//
// Sums of weights decide which token it is, so they do not depend on an order:
// with x = logit log2(e) / temperature in fp64 and N = floor of the row's
// largest x, a weight is the integer rint(2^(x - N) 2^42), at most 2^43, and
// sums of up to 2^20 of them are exact in 64 bits (weights under 2^-44 of the
// largest are 0).  2^f is a Taylor polynomial about f = 1/2: its remainder of
// 6e-15 is below the rounding to an integer.
//
// Two launches.  The first reads the logits once, chunk by chunk, and leaves
// what a row's choice needs of each chunk; the second, a workgroup per row,
// settles the filters from that and reads again only those pieces of the row
// that hold candidates.  A piece is a wave's 1024 elements, a group the 16 of
// them that a lane holds; a group's largest key tells whether it matters.
#include <algorithm>

#include "step.hpp"
#include "trace.hpp"

namespace moe {

namespace {

typedef unsigned long long u64;

constexpr int kGroup = 16, kPiece = kGroup * kWave;  // elements of a lane and of a wave
constexpr int kChunkWaves = 8, kChunk = kChunkWaves * kPiece;
constexpr int kOctaves = 44, kPerOctave = 8, kBins = kOctaves * kPerOctave;
constexpr int kUnit = 42;      // weights are in units of 2^-42 of 2^N
constexpr int kRowThreads = 1024, kRowWaves = kRowThreads / kWave;
constexpr int kList = 4096;    // candidates held in LDS
constexpr int kFastK = 2048;   // the top_k that the list is for
constexpr int kHeldMax = 8;    // largest keys per thread in the search for the k-th

// What the first launch leaves of a row, `chunks` of each.
struct RowStats {
  u64* best;       // [chunks] key << 32 | ~index of the largest
  double* ref;     // [chunks] N of the chunk
  u64* piece_sum;  // [chunks * 8] weights of a piece, in the chunk's unit
  uint32_t* top;   // [chunks * 512] largest key of a group
  u64* bins;       // [chunks * kBins] weights by eighths of an octave below 2^(N + 1)
};

__host__ __device__ inline int chunks_of(int V) { return (V + 7 + kChunk - 1) / kChunk; }  // a row may begin 7 elements into a vector

struct Ws {
  char* base;
  int B, chunks;
  __host__ __device__ RowStats row(int b) const {
    const size_t n = static_cast<size_t>(B) * chunks, at = static_cast<size_t>(b) * chunks;
    RowStats r;
    char* p = base;
    r.best = reinterpret_cast<u64*>(p) + at;
    p += n * 8;
    r.ref = reinterpret_cast<double*>(p) + at;
    p += n * 8;
    r.piece_sum = reinterpret_cast<u64*>(p) + at * kChunkWaves;
    p += n * kChunkWaves * 8;
    r.bins = reinterpret_cast<u64*>(p) + at * kBins;
    p += n * kBins * 8;
    r.top = reinterpret_cast<uint32_t*>(p) + at * (kChunkWaves * kWave);
    return r;
  }
  static size_t bytes(int B, int chunks) {
    return static_cast<size_t>(B) * chunks * (8 + 8 + kChunkWaves * 8 + kBins * 8 + kChunkWaves * kWave * 4);
  }
};

// Order-preserving key; 0 for what is never taken (-infinity, NaN, absent).
__device__ __forceinline__ uint32_t key_of(float v) {
  if (!(v > -INFINITY)) return 0u;
  const uint32_t u = v == 0.0f ? 0u : __float_as_uint(v);
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float((key >> 31) ? (key & 0x7fffffffu) : ~key);
}

// A row's settings.
struct Settings {
  bool greedy, filter_k, filter_p, filter_m;
  int k;
  double c, p, m;  // log2(e) / temperature, top_p, min_p
};
__device__ __forceinline__ Settings settings_of(const SampleArgs& a, int b) {
  Settings s;
  const float t = a.temperature != nullptr ? a.temperature[b] : 1.0f;
  s.greedy = !(t > 0.0f);
  s.c = 1.4426950408889634 / static_cast<double>(t);
  s.k = a.top_k != nullptr ? a.top_k[b] : 0;
  s.filter_k = s.k > 0 && s.k < a.V;
  s.p = a.top_p != nullptr ? a.top_p[b] : 1.0;
  s.filter_p = s.p < 1.0;
  s.m = a.min_p != nullptr ? a.min_p[b] : 0.0;
  s.filter_m = s.m > 0.0;
  if (s.m > 1.0) s.m = 1.0;
  return s;
}

// x of a value; infinity is past every finite one, so that it alone has weight.
__device__ __forceinline__ double x_of(float v, double c) { return v == INFINITY ? 1e300 : static_cast<double>(v) * c; }

// The integer weight of x <= N + 1.
__device__ __forceinline__ u64 weight(double x, double N) {
  const double n = floor(x), d = N - n;
  if (!(d <= kUnit + 1.0)) return 0;
  const double y = (x - n - 0.5) * 0.6931471805599453;
  double p = 1.0 / 39916800;
  p = fma(p, y, 1.0 / 3628800);
  p = fma(p, y, 1.0 / 362880);
  p = fma(p, y, 1.0 / 40320);
  p = fma(p, y, 1.0 / 5040);
  p = fma(p, y, 1.0 / 720);
  p = fma(p, y, 1.0 / 120);
  p = fma(p, y, 1.0 / 24);
  p = fma(p, y, 1.0 / 6);
  p = fma(p, y, 0.5);
  p = fma(p, y, 1.0);
  p = fma(p, y, 1.0);
  const int e = kUnit - static_cast<int>(d);
  const double scale = __longlong_as_double(static_cast<long long>(1023 + e) << 52) * 1.4142135623730951;
  // the sum's unit is 1: its low bits are the rounded integer
  return static_cast<u64>(__double_as_longlong(fma(p, scale, 0x1p52))) & ((1ull << 52) - 1);
}

// Eighth of an octave below 2^(N + 1) that x lies in.
__device__ __forceinline__ double bin_of(double x, double N) { return 8.0 * (N + 1.0) - 1.0 - floor(8.0 * x); }

// A sum in units of 2^(ref - 42) in those of 2^(N - 42), N >= ref, rounded.
__device__ __forceinline__ u64 rescale(u64 sum, double ref, double N) {
  const double d = N - ref;
  if (!(d < 64.0)) return 0;
  const int i = static_cast<int>(d);
  return i == 0 ? sum : (sum >> i) + ((sum >> (i - 1)) & 1);
}

__device__ __forceinline__ u64 wave_add(u64 v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v += shfl_xor(v, m);
  return v;
}
__device__ __forceinline__ u64 wave_most(u64 v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = max(v, shfl_xor(v, m));
  return v;
}
// Sum over the lanes below.
__device__ __forceinline__ u64 wave_before(u64 v) {
  const int lane = threadIdx.x & 63;
  u64 t = v;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const u64 o = __shfl_up(t, d, kWave);
    if (lane >= d) t += o;
  }
  return t - v;
}

// A row in memory.  Element i lies at place i + skew, place 0 on 16 bytes, so
// that whole vectors are read whatever the row's alignment.
template <bool F32>
struct Row {
  static constexpr int W = F32 ? 4 : 8;  // elements of a vector
  const char* at;                        // place 0
  int skew, end;                         // the row is places skew .. end
  __device__ __forceinline__ Row(const SampleArgs& a, int b) {
    constexpr int size = F32 ? 4 : 2;
    const char* p = static_cast<const char*>(a.logits) + static_cast<int64_t>(b) * a.ld * size;
    skew = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / size);
    at = p - skew * size;
    end = skew + a.V;
  }
  // Place of element e of this lane's group in the piece.
  static __device__ __forceinline__ int place(int piece, int e) {
    return piece * kPiece + (e / W) * (kWave * W) + (threadIdx.x & 63) * W + e % W;
  }
  __device__ __forceinline__ float one(int p) const {
    if (p < skew || p >= end) return -INFINITY;
    if constexpr (F32) return reinterpret_cast<const float*>(at)[p];
    else return bf2f(reinterpret_cast<const bf16_t*>(at)[p]);
  }
  // This lane's group of a piece.
  __device__ __forceinline__ void load(int piece, float (&v)[kGroup]) const {
#pragma unroll
    for (int i = 0; i < kGroup / W; ++i) {
      const int p = place(piece, i * W);
      if (p >= skew && p + W <= end) {
        const uint4 w = *reinterpret_cast<const uint4*>(at + static_cast<int64_t>(p) * (16 / W));
        if constexpr (F32) {
          v[i * W] = __uint_as_float(w.x), v[i * W + 1] = __uint_as_float(w.y);
          v[i * W + 2] = __uint_as_float(w.z), v[i * W + 3] = __uint_as_float(w.w);
        } else {
          v[i * W] = lo_bf(w.x), v[i * W + 1] = hi_bf(w.x), v[i * W + 2] = lo_bf(w.y), v[i * W + 3] = hi_bf(w.y);
          v[i * W + W - 4] = lo_bf(w.z), v[i * W + W - 3] = hi_bf(w.z);
          v[i * W + W - 2] = lo_bf(w.w), v[i * W + W - 1] = hi_bf(w.w);
        }
      } else {
#pragma unroll
        for (int j = 0; j < W; ++j) v[i * W + j] = one(p + j);
      }
    }
  }
};

// First launch: a chunk of a row per workgroup.
template <bool F32>
__global__ __launch_bounds__(kChunkWaves* kWave) void k_sample_chunks(SampleArgs a, Ws ws) {
  __shared__ u64 bests[kChunkWaves];
  __shared__ u64 bins[kBins];
  const int chunk = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const RowStats st = ws.row(b);
  const Settings s = settings_of(a, b);
  const Row<F32> row(a, b);
  const int piece = chunk * kChunkWaves + wave;
  float v[kGroup];
  row.load(piece, v);
  u64 best = 0;
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < kGroup; ++e) {
    const uint32_t key = key_of(v[e]);
    top = max(top, key);
    best = max(best, static_cast<u64>(key) << 32 | static_cast<uint32_t>(~(row.place(piece, e) - row.skew)));
  }
  best = wave_most(best);
  if (lane == 0) bests[wave] = best;
  const bool binned = s.filter_p && !s.greedy && !s.filter_k;
  if (binned)
    for (int i = tid; i < kBins; i += kChunkWaves * kWave) bins[i] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kChunkWaves; ++w) best = max(best, bests[w]);
  if (tid == 0) st.best[chunk] = best;
  if (s.greedy) return;
  st.top[chunk * (kChunkWaves * kWave) + tid] = top;
  const bool summed = !s.filter_k && !s.filter_p && !s.filter_m;
  if (!summed && !binned) return;
  const uint32_t most = static_cast<uint32_t>(best >> 32);
  const double N = most == 0 ? -1e305 : floor(x_of(value_of(most), s.c));
  if (tid == 0) st.ref[chunk] = N;
  u64 sum = 0;
#pragma unroll
  for (int e = 0; e < kGroup; ++e) {
    if (key_of(v[e]) == 0) continue;
    const double x = x_of(v[e], s.c);
    const u64 w = weight(x, N);
    sum += w;
    if (binned && w != 0) atomicAdd(&bins[static_cast<int>(fmin(bin_of(x, N), kBins - 1.0))], w);
  }
  if (summed) {
    sum = wave_add(sum);
    if (lane == 0) st.piece_sum[piece] = sum;
    return;
  }
  __syncthreads();
  for (int i = tid; i < kBins; i += kChunkWaves * kWave) st.bins[static_cast<int64_t>(chunk) * kBins + i] = bins[i];
}

// ---- second launch
constexpr int kMaxPieces = (MOE_SAMPLE_MAX_V + 7 + kChunk - 1) / kChunk * kChunkWaves;
static_assert(kMaxPieces <= 2 * kRowThreads, "two pieces per thread in the choice of the draw's piece");
struct Shared {
  u64 list[kList];
  u64 sums[kMaxPieces];  // of the pieces
  u64 bins[kBins];
  u64 waves[kRowWaves];
  u64 found, found2;
  int count;
};

// Of a workgroup's values, in thread order: the sum before each, and of all.
__device__ __forceinline__ u64 block_before(u64 v, u64* waves, u64& all) {
  const int wave = threadIdx.x >> 6;
  u64 t = wave_before(v);
  __syncthreads();  // `waves` has been read
  if ((threadIdx.x & 63) == 63) waves[wave] = t + v;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    if (w < wave) t += waves[w];
    all += waves[w];
  }
  return t;
}
__device__ __forceinline__ u64 block_add(u64 v, u64* waves) {
  v = wave_add(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 t = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) t += waves[w];
  return t;
}

// Sorts list[0 .. n) descending (bitonic, padded with zeros).  Ends with a barrier.
__device__ void sort_list(u64* list, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += kRowThreads) list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int i = threadIdx.x; i < size / 2; i += kRowThreads) {
        const int lo = (i & (j - 1)) | ((i & ~(j - 1)) << 1), hi = lo | j;
        const u64 p = list[lo], q = list[hi];
        if ((p < q) == ((lo & k) == 0)) list[lo] = q, list[hi] = p;
      }
      __syncthreads();
    }
}

__device__ __forceinline__ u64 part_of(double share, u64 all) {  // floor(share all)
  return static_cast<u64>(share * static_cast<double>(all));
}

template <bool F32>
struct Choice {
  const SampleArgs& a;
  const int b, pieces, lane, wave;
  const Settings s;
  const Row<F32> row;
  const RowStats st;
  Shared& sh;
  int32_t first;              // the largest element,
  double x_most, N, x_least;  // its x, the floor of that, the least x that min_p keeps

  __device__ Choice(const SampleArgs& a_, const Ws& ws, Shared& sh_)
      : a(a_), b(blockIdx.x), pieces(ws.chunks * kChunkWaves), lane(threadIdx.x & 63), wave(threadIdx.x >> 6),
        s(settings_of(a_, b)), row(a_, b), st(ws.row(b)), sh(sh_) {}

  // One element: its key and index, larger is earlier in the order.
  __device__ __forceinline__ u64 rank_of(float v, int place) const {
    return static_cast<u64>(key_of(v)) << 32 | static_cast<uint32_t>(~(place - row.skew));
  }
  __device__ __forceinline__ double x_at(u64 rank) const { return x_of(value_of(static_cast<uint32_t>(rank >> 32)), s.c); }

  __device__ void write(int32_t token, double logprob) const {
    a.token[b] = token;
    if (a.logprob != nullptr) a.logprob[b] = static_cast<float>(logprob);
  }
  __device__ void write(int32_t token, double x, u64 all) const {
    write(token, (x - N) * 0.6931471805599453 - log(static_cast<double>(all) * 0x1p-42));
  }
  // The draw: the running sum that the token's has to pass.
  __device__ __forceinline__ u64 draw(u64 all) const {
    const double u = a.u[b];
    return u > 0.0 ? min(part_of(u, all), all - 1) : 0;
  }

  // Elements of a piece that stay: rank >= least and x >= x_least.
  __device__ __forceinline__ u64 kept(float v, int place, u64 least) const {
    if (key_of(v) == 0 || rank_of(v, place) < least) return 0;
    const double x = x_of(v, s.c);
    return s.filter_m && x < x_least ? 0 : weight(x, N);
  }

  // The token of the running sum `r` within a piece, by the calling wave.
  __device__ void pick(int piece, u64 r, u64 least, u64 all) const {
    float v[kGroup];
    row.load(piece, v);
    constexpr int W = Row<F32>::W;
    bool done = false;
    u64 last = 0;  // the last element with weight, should rounding have left r past them all
#pragma unroll
    for (int i = 0; i < kGroup / W; ++i) {
      u64 w[W], t = 0;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        w[j] = kept(v[i * W + j], row.place(piece, i * W + j), least);
        t += w[j];
        if (w[j] != 0)
          last = max(last, static_cast<u64>(row.place(piece, i * W + j) + 1) << 32 | key_of(v[i * W + j]));
      }
      u64 before = wave_before(t);
      const u64 total = __shfl(before + t, kWave - 1, kWave);
      if (!done && r < total) {
        done = true;
        if (before <= r && r < before + t)
#pragma unroll
          for (int j = 0; j < W; ++j) {
            if (before <= r && r < before + w[j])
              write(row.place(piece, i * W + j) - row.skew, x_of(v[i * W + j], s.c), all);
            before += w[j];
          }
      }
      if (!done) r -= total;
    }
    if (!done) {
      last = wave_most(last);
      if (lane == 0) {
        if (last != 0) write(static_cast<int>(last >> 32) - 1 - row.skew, x_of(value_of(static_cast<uint32_t>(last)), s.c), all);
        else write(first, x_most, all);
      }
    }
  }

  // sums[0 .. pieces) hold the pieces' weights: finds the draw's piece and picks there.
  __device__ void pick_by_sums(u64 least) {
    __syncthreads();
    u64 mine[2], all;
    const int i0 = threadIdx.x * 2;
    for (int j = 0; j < 2; ++j) mine[j] = i0 + j < pieces ? sh.sums[i0 + j] : 0;
    u64 before = block_before(mine[0] + mine[1], sh.waves, all);
    const u64 r = draw(all);
    for (int j = 0; j < 2; ++j) {
      if (before <= r && r < before + mine[j]) {
        sh.found = i0 + j;
        sh.found2 = r - before;
      }
      before += mine[j];
    }
    __syncthreads();
    if (wave == 0) pick(static_cast<int>(sh.found), sh.found2, least, all);
  }

  // Weights of what stays, piece by piece; pieces without a group at least as
  // large as `least` are not read.
  __device__ void sum_pieces(u64 least) {
    uint32_t key = static_cast<uint32_t>(least >> 32);
    for (int piece = wave; piece < pieces; piece += kRowWaves) {
      const uint32_t top = st.top[piece * kWave + lane];
      const bool may = top != 0 && top >= key && !(s.filter_m && x_of(value_of(top), s.c) < x_least);
      u64 t = 0;
      if (__any(may)) {
        float v[kGroup];
        row.load(piece, v);
        if (may)
#pragma unroll
          for (int e = 0; e < kGroup; ++e) t += kept(v[e], row.place(piece, e), least);
        t = wave_add(t);
      }
      if (lane == 0) sh.sums[piece] = t;
    }
  }

  // Collects what `want` says of groups that `may` says: the count, of which
  // the first kList are in the list.
  template <class May, class Want>
  __device__ int collect(May may, Want want) {
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    for (int piece = wave; piece < pieces; piece += kRowWaves) {
      const uint32_t top = st.top[piece * kWave + lane];
      const bool on = top != 0 && may(top);
      if (!__any(on)) continue;
      float v[kGroup];
      row.load(piece, v);
      if (!on) continue;
#pragma unroll
      for (int e = 0; e < kGroup; ++e)
        if (const uint32_t key = key_of(v[e]); key != 0 && want(key)) {
          const int at = atomicAdd(&sh.count, 1);
          if (at < kList) sh.list[at] = rank_of(v[e], row.place(piece, e));
        }
    }
    __syncthreads();
    return sh.count;
  }

  // A key that k groups (or runs of groups) reach: at least k elements do.
  __device__ uint32_t floor_of_kth(int k) {
    const int groups = pieces * kWave, run = cdiv(groups, kRowThreads * kHeldMax);
    uint32_t top[kHeldMax];
#pragma unroll
    for (int i = 0; i < kHeldMax; ++i) {
      top[i] = 0;
      for (int j = 0; j < run; ++j) {
        const int g = (i * run + j) * kRowThreads + static_cast<int>(threadIdx.x);
        if (g < groups) top[i] = max(top[i], st.top[g]);
      }
    }
    uint32_t kth = 0;
    for (int bit = 31; bit >= 8; --bit) {
      const uint32_t at = kth | 1u << bit;
      int n = 0;
#pragma unroll
      for (int i = 0; i < kHeldMax; ++i) n += top[i] >= at ? 1 : 0;
      if (block_add(n, sh.waves) >= static_cast<u64>(k)) kth = at;
    }
    return kth;
  }

  // The candidates are the list's n largest: filters them in order, draws.
  __device__ void choose_from_list(int n, int k) {
    sort_list(sh.list, n);
    const int m = min(n, k), i0 = threadIdx.x * 4;
    u64 w[4], t = 0, all;
    double x[4];
    for (int j = 0; j < 4; ++j) {
      const u64 rank = i0 + j < m ? sh.list[i0 + j] : 0;
      x[j] = rank != 0 ? x_at(rank) : -1e305;
      w[j] = rank != 0 ? weight(x[j], N) : 0;
      t += w[j];
    }
    u64 before = block_before(t, sh.waves, all);
    const u64 need = s.filter_p ? max(part_of_up(s.p, all), 1ull) : all;
    int stay = 0;
    for (int j = 0; j < 4; ++j) {
      if (i0 + j < m && w[j] != 0 && before < need && !(s.filter_m && x[j] < x_least)) ++stay;
      before += w[j];
    }
    const int left = static_cast<int>(block_add(stay, sh.waves));  // a prefix: the filters go by the order
    // the same in index order
    u64 again[4];
    for (int j = 0; j < 4; ++j) {
      const u64 rank = i0 + j < left ? sh.list[i0 + j] : 0;
      again[j] = rank << 32 | rank >> 32;  // ~index above the key
    }
    __syncthreads();
    for (int j = 0; j < 4; ++j)
      if (i0 + j < left) sh.list[i0 + j] = again[j];
    __syncthreads();
    sort_list(sh.list, left);
    t = 0;
    for (int j = 0; j < 4; ++j) {
      again[j] = i0 + j < left ? sh.list[i0 + j] : 0;
      x[j] = again[j] != 0 ? x_of(value_of(static_cast<uint32_t>(again[j])), s.c) : -1e305;
      w[j] = again[j] != 0 ? weight(x[j], N) : 0;
      t += w[j];
    }
    before = block_before(t, sh.waves, all);
    const u64 r = draw(all);
    for (int j = 0; j < 4; ++j) {
      if (before <= r && r < before + w[j]) write(static_cast<int32_t>(~static_cast<uint32_t>(again[j] >> 32)), x[j], all);
      before += w[j];
    }
  }

  // ceil(share all), for a share below 1
  static __device__ __forceinline__ u64 part_of_up(double share, u64 all) {
    return share > 0.0 ? static_cast<u64>(ceil(share * static_cast<double>(all))) : 0;
  }

  // Rank of the last element of the shortest prefix that holds `need` of the
  // weight, by eighths of an octave; 0 where too many elements share one.
  __device__ u64 border_by_bins(u64& least) {
    for (int i = threadIdx.x; i < kBins; i += kRowThreads) sh.bins[i] = 0;
    __syncthreads();
    const int chunks = pieces / kChunkWaves;
    for (int i = threadIdx.x; i < chunks * kBins; i += kRowThreads) {
      const double ref = st.ref[i / kBins];
      const double at = i % kBins + kPerOctave * (N - ref);
      if (at < kBins) {
        const u64 w = rescale(st.bins[i], ref, N);
        if (w != 0) atomicAdd(&sh.bins[static_cast<int>(at)], w);
      }
    }
    __syncthreads();
    u64 all;
    const u64 mine = threadIdx.x < kBins ? sh.bins[threadIdx.x] : 0;
    const u64 before = block_before(mine, sh.waves, all);
    const u64 need = max(part_of_up(s.p, all), 1ull);
    if (before < need && need <= before + mine) {
      sh.found = threadIdx.x;
      sh.found2 = need - before;
    }
    __syncthreads();
    const double bin = static_cast<double>(sh.found);
    const u64 rest = sh.found2;
    const int n = collect([&](uint32_t top) { return bin_of(x_of(value_of(top), s.c), N) <= bin; },
                          [&](uint32_t key) { return bin_of(x_of(value_of(key), s.c), N) == bin; });
    if (n > kList || n == 0) return 0;
    sort_list(sh.list, n);
    u64 w[4], t = 0;
    const int i0 = threadIdx.x * 4;
    for (int j = 0; j < 4; ++j) {
      w[j] = i0 + j < n ? weight(x_at(sh.list[i0 + j]), N) : 0;
      t += w[j];
    }
    u64 sum, at = block_before(t, sh.waves, sum);
    if (threadIdx.x == 0) sh.found = sh.list[n - 1];  // should rounding have left `rest` past them all
    __syncthreads();
    for (int j = 0; j < 4; ++j) {
      if (at < rest && rest <= at + w[j]) sh.found = sh.list[i0 + j];
      at += w[j];
    }
    __syncthreads();
    least = sh.found;
    return least;
  }

  // Count or weight of the elements of rank >= at (and >= least).
  template <bool COUNT>
  __device__ u64 measure(u64 at) {
    const uint32_t key = static_cast<uint32_t>(at >> 32);
    u64 t = 0;
    for (int piece = wave; piece < pieces; piece += kRowWaves) {
      const uint32_t top = st.top[piece * kWave + lane];
      const bool may = top != 0 && top >= key;
      if (!__any(may)) continue;
      float v[kGroup];
      row.load(piece, v);
      if (!may) continue;
#pragma unroll
      for (int e = 0; e < kGroup; ++e)
        if (key_of(v[e]) != 0 && rank_of(v[e], row.place(piece, e)) >= at) t += COUNT ? 1 : weight(x_of(v[e], s.c), N);
    }
    return block_add(t, sh.waves);
  }
  // The largest rank whose elements measure `need`, bit by bit: for what the
  // lists do not hold (thousands of equal logits, a top_k of thousands).  A
  // row of up to 16 pieces stays in registers meanwhile.
  template <bool COUNT>
  __device__ u64 search(u64 need) {
    u64 at = 0;
    if (pieces <= kRowWaves) {
      float v[kGroup];
      u64 rank[kGroup], w[kGroup];
      if (wave < pieces) row.load(wave, v);
#pragma unroll
      for (int e = 0; e < kGroup; ++e) {
        const bool on = wave < pieces && key_of(v[e]) != 0;
        rank[e] = on ? rank_of(v[e], row.place(wave, e)) : 0;
        w[e] = !on ? 0 : COUNT ? 1 : weight(x_of(v[e], s.c), N);
      }
      for (int bit = 63; bit >= 0; --bit) {
        const u64 next = at | 1ull << bit;
        u64 t = 0;
#pragma unroll
        for (int e = 0; e < kGroup; ++e) t += rank[e] >= next ? w[e] : 0;
        if (block_add(t, sh.waves) >= need) at = next;
      }
      return at;
    }
    for (int bit = 63; bit >= 0; --bit) {
      const u64 next = at | 1ull << bit;
      if (measure<COUNT>(next) >= need) at = next;
    }
    return at;
  }

  __device__ void run() {
    // the row's largest
    u64 best = 0;
    for (int i = lane; i < pieces / kChunkWaves; i += kWave) best = max(best, st.best[i]);
    best = wave_most(best);
    const uint32_t most = static_cast<uint32_t>(best >> 32);
    first = static_cast<int32_t>(~static_cast<uint32_t>(best));
    if (most == 0) {  // nothing to take
      if (threadIdx.x == 0) write(-1, -INFINITY);
      return;
    }
    if (s.greedy) {
      if (threadIdx.x == 0) write(first, 0.0);
      return;
    }
    x_most = x_of(value_of(most), s.c);
    N = floor(x_most);
    x_least = s.filter_m ? x_most + log2(s.m) : 0.0;
    if (!s.filter_k && !s.filter_p && !s.filter_m) {
      for (int i = threadIdx.x; i < pieces; i += kRowThreads)
        sh.sums[i] = rescale(st.piece_sum[i], st.ref[i / kChunkWaves], N);
      pick_by_sums(0);
      return;
    }
    u64 least = 0;
    if (s.filter_k) {
      if (s.k <= kFastK) {
        const uint32_t at = floor_of_kth(s.k);
        const int n = collect([&](uint32_t top) { return top >= at; }, [&](uint32_t key) { return key >= at; });
        if (n <= kList) {
          choose_from_list(n, s.k);
          return;
        }
      }
      least = search<true>(s.k);
      if (s.filter_p) least = max(least, search<false>(max(part_of_up(s.p, measure<false>(least)), 1ull)));
    } else if (s.filter_p && border_by_bins(least) == 0) {
      least = search<false>(max(part_of_up(s.p, measure<false>(0)), 1ull));
    }
    sum_pieces(least);
    pick_by_sums(least);
  }
};

template <bool F32>
__global__ __launch_bounds__(kRowThreads) void k_sample_rows(SampleArgs a, Ws ws) {
  __shared__ Shared sh;
  Choice<F32>(a, ws, sh).run();
}

}  // namespace

size_t sample_ws(int B, int V) { return Ws::bytes(B, chunks_of(V)); }

hipError_t launch_sample(const SampleArgs& a, void* base, hipStream_t s) {
  const Ws ws{static_cast<char*>(base), a.B, chunks_of(a.V)};
  TraceScope trace_scope(K_SAMPLE, s);
  if (a.fp32) {
    hipLaunchKernelGGL(k_sample_chunks<true>, dim3(ws.chunks, a.B), dim3(kChunkWaves * kWave), 0, s, a, ws);
    hipLaunchKernelGGL(k_sample_rows<true>, dim3(a.B), dim3(kRowThreads), 0, s, a, ws);
  } else {
    hipLaunchKernelGGL(k_sample_chunks<false>, dim3(ws.chunks, a.B), dim3(kChunkWaves * kWave), 0, s, a, ws);
    hipLaunchKernelGGL(k_sample_rows<false>, dim3(a.B), dim3(kRowThreads), 0, s, a, ws);
  }
  return hipGetLastError();
}

}  // namespace moe
