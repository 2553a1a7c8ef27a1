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
// largest are 0).  What the first launch sums is in the unit of a chunk's own N and
// rounded once, as a sum, to the row's; the draw goes on in the chunk's unit within
// a piece that such a sum has led to, so that what the sum counts is there.
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
constexpr int kUnit = 42;  // weights are in units of 2^-42 of 2^N
// 1024 threads a row: two waves more a SIMD won 1 to 2 us of 256 rows and lost 1 to 2
// of one row and of a small top-k.
constexpr int kRowThreads = 512, kRowWaves = kRowThreads / kWave;
constexpr int kList = 4096;   // candidates held in LDS
constexpr int kMine = kList / kRowThreads;
// Groups with candidates, one or two in each of a long row, of which the list is likely
// to hold all; a row of up to 32 pieces has no more, and where it is flat is counted twice.
constexpr int kFewGroups = 2048;
constexpr int kFastK = 2048;  // the top_k that the list is for
constexpr int kFine = 1024;   // parts of the list's range
constexpr int kHeldPieces = 256, kHeldGroups = kHeldPieces * kWave;  // of a row whose groups' keys are held in LDS
constexpr int kMaxParts = 8;

// Workgroups per row of the second launch: as many as leave the chip's 256
// compute units one each.
__host__ __device__ inline int parts_of(int B) { return B > 128 ? 1 : B > 32 ? 256 / B : kMaxParts; }

// What the first launch leaves of a row, `chunks` of each; and what a row's
// workgroups leave each other.
struct RowStats {
  u64* best;       // [chunks] key << 32 | ~index of the largest
  double* ref;     // [chunks] N of the chunk
  u64* piece_sum;  // [chunks * 8] weights of a piece, in the chunk's unit
  uint32_t* top;   // [chunks * 512] largest key of a group
  u64* bins;       // [chunks * kBins] weights by eighths of an octave below 2^(N + 1)
  int32_t* done;   // [1 + kMaxParts] workgroups that are through, their candidates
  u64* lists;      // [parts, kList]
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
    r.lists = reinterpret_cast<u64*>(p) + static_cast<size_t>(b) * parts_of(B) * kList;
    p += static_cast<size_t>(lists(B)) * kList * 8;
    r.top = reinterpret_cast<uint32_t*>(p) + at * (kChunkWaves * kWave);
    p += n * kChunkWaves * kWave * 4;
    r.done = reinterpret_cast<int32_t*>(p) + static_cast<size_t>(b) * (1 + kMaxParts);
    return r;
  }
  // Lists of up to B rows, B parts_of(B) at its largest: more rows never need less room.
  __host__ __device__ static int lists(int B) { return B > 256 ? B : B > 32 ? 256 : kMaxParts * B; }
  static size_t bytes(int B, int chunks) {
    return static_cast<size_t>(B) * chunks * (8 + 8 + kChunkWaves * 8 + kBins * 8 + kChunkWaves * kWave * 4) +
           static_cast<size_t>(lists(B)) * kList * 8 + static_cast<size_t>(B) * (1 + kMaxParts) * 4;
  }
};

// Order-preserving key; 0 for what is never taken (-infinity, NaN, absent).
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = v == 0.0f ? 0u : __float_as_uint(v);
  const uint32_t key = u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
  return v > -INFINITY ? key : 0u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float((key >> 31) ? (key & 0x7fffffffu) : ~key);
}

constexpr uint32_t kInfKey = 0xff800000u;  // of infinity, the largest

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

// N of a chunk with nothing to take: below every logit's (5e83 at most), above the x
// of what has no weight, so that the difference is one that weighs nothing.
constexpr double kNoLogits = -1e290;

// x of a value; infinity is past every finite one, so that it alone has weight.
// Where `in` is false, one of no weight: chosen here, because a choice after
// the weight makes the compiler put each weight behind a branch of its own, one
// chain of dependent steps at a time (at temperature 1 and top-p 0.9 one row of
// 131072: 37.1 us with it, 36.4 without; 64 rows: 60.0, 59.3; 256 of 50001 in bf16
// the same).
__device__ __forceinline__ double x_if(bool in, float v, double c) {
  const double x = static_cast<double>(v) * c;
  constexpr int kFar = 0x7e37e43c;  // upper half of 1e300
  const int hi = v == INFINITY ? kFar : __double2hiint(x);
  return __hiloint2double(in ? hi : kFar | 1 << 31, __double2loint(x));
}
__device__ __forceinline__ double x_of(float v, double c) { return x_if(true, v, c); }

// The integer weight of x < N + 1: 2^f, |f| <= 1/2, by the polynomial that
// meets it in the ten Chebyshev points (2^-45.6 of it off at most), times a
// power of two; the sum with 2^52 has the rounded integer in its low bits.
// The coefficients are made opaque so that they stay in scalar registers:
// left to itself the compiler moves each into a vector register before its
// step, two moves a step.
struct Weigh {
  double c[10];
  __device__ __forceinline__ Weigh()
      : c{1.0000000000000135,    0.6931471805599462,     0.2402265069564034,     0.05550410866465167,   0.009618129193934313,
          0.0013333558200794592, 0.0001540343375125101, 1.5252672924850737e-05, 1.325964524488711e-06, 1.0205905413765595e-07} {
#pragma unroll
    for (int i = 0; i < 10; ++i) asm("" : "+s"(c[i]));
  }
  __device__ __forceinline__ u64 operator()(double x, double N) const {
    const double n = __builtin_rint(x), f = x - n;
    double p = c[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) p = fma(p, f, c[i]);
    const double w = __builtin_ldexp(p, static_cast<int>(fmax(n - N, -100.0)) + kUnit);
    return static_cast<u64>(__double_as_longlong(w + 0x1p52)) & ((1ull << 52) - 1);
  }
};

// Eighth of an octave below 2^(N + 1) that x lies in.
__device__ __forceinline__ double bin_of(double x, double N) { return 8.0 * (N + 1.0) - 1.0 - floor(8.0 * x); }

// A sum in units of 2^(ref - 42) in those of 2^(N - 42), N >= ref, rounded.
__device__ __forceinline__ u64 rescale(u64 sum, double ref, double N) {
  const double d = N - ref;
  if (!(d < 64.0)) return 0;
  const int i = static_cast<int>(d);
  return i == 0 ? sum : (sum >> i) + ((sum >> (i - 1)) & 1);
}

// v plus that of another lane, within the vector ALU (through LDS, as a
// shuffle goes, a 64-bit sum over the wave takes five times as long).
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 add_from(u64 v) {
  const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(v >> 32), CTRL, ROWS, 0xf, false);
  return v + (static_cast<u64>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo));
}
// Sum over this lane and those below: within rows of 16 lanes by shifts of 1,
// 2, 4, 8, then the last lane's sum of a row on to the next, of a half to the other.
__device__ __forceinline__ u64 wave_upto(u64 v) {
  v = add_from<0x111, 0xf>(v);
  v = add_from<0x112, 0xf>(v);
  v = add_from<0x114, 0xf>(v);
  v = add_from<0x118, 0xf>(v);
  v = add_from<0x142, 0xa>(v);
  return add_from<0x143, 0xc>(v);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_from(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_upto(int v) {
  v = add_from<0x111, 0xf>(v);
  v = add_from<0x112, 0xf>(v);
  v = add_from<0x114, 0xf>(v);
  v = add_from<0x118, 0xf>(v);
  v = add_from<0x142, 0xa>(v);
  return add_from<0x143, 0xc>(v);
}
__device__ __forceinline__ u64 lane_value(u64 v, int lane) {  // `lane` is the same in every lane
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane);
  return static_cast<u64>(hi) << 32 | lo;
}
__device__ __forceinline__ u64 wave_add(u64 v) { return lane_value(wave_upto(v), kWave - 1); }
__device__ __forceinline__ u64 wave_before(u64 v) { return wave_upto(v) - v; }
__device__ __forceinline__ u64 wave_most(u64 v) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) v = max(v, shfl_xor(v, m));
  return v;
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
  // W elements from place p, a multiple of W.
  __device__ __forceinline__ void vec(int p, float* v) const {
    if (p >= skew && p + W <= end) {
      const uint4 w = *reinterpret_cast<const uint4*>(at + static_cast<int64_t>(p) * (16 / W));
      if constexpr (F32) {
        v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y), v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
      } else {
        v[0] = lo_bf(w.x), v[1] = hi_bf(w.x), v[2] = lo_bf(w.y), v[3] = hi_bf(w.y);
        v[W - 4] = lo_bf(w.z), v[W - 3] = hi_bf(w.z), v[W - 2] = lo_bf(w.w), v[W - 1] = hi_bf(w.w);
      }
    } else {  // an end of the row: small code rather than fast
#pragma unroll 1
      for (int j = 0; j < W; ++j) {
        const float t = one(p + j);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i == j ? t : v[i];
      }
    }
  }
  // This lane's group of a piece.
  __device__ __forceinline__ void load(int piece, float (&v)[kGroup]) const {
#pragma unroll
    for (int i = 0; i < kGroup / W; ++i) vec(place(piece, i * W), v + i * W);
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
  const Weigh weight;
  const int piece = chunk * kChunkWaves + wave;
  float v[kGroup];
  row.load(piece, v);
  float most = -INFINITY;  // of what is not NaN
#pragma unroll
  for (int e = 0; e < kGroup; ++e) most = fmaxf(most, v[e]);
  const uint32_t top = key_of(most);
  uint32_t first = 0;  // ~index of the group's first element of that value
#pragma unroll
  for (int e = 0; e < kGroup; ++e)
    if (v[e] == most) first = max(first, static_cast<uint32_t>(~(row.place(piece, e) - row.skew)));
  u64 best = wave_most(static_cast<u64>(top) << 32 | first);
  if (lane == 0) bests[wave] = best;
  const bool binned = s.filter_p && !s.greedy && !s.filter_k;
  if (binned)
    for (int i = tid; i < kBins; i += kChunkWaves * kWave) bins[i] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kChunkWaves; ++w) best = max(best, bests[w]);
  if (tid == 0) st.best[chunk] = best;
  if (tid == 0 && chunk == 0) st.done[0] = 0;
  if (s.greedy) return;
  st.top[chunk * (kChunkWaves * kWave) + tid] = top;
  const bool summed = !s.filter_k && !s.filter_p && !s.filter_m;
  if (!summed && !binned) return;
  const uint32_t largest = static_cast<uint32_t>(best >> 32);
  const double N = largest == 0 ? kNoLogits : floor(x_of(value_of(largest), s.c));
  if (tid == 0) st.ref[chunk] = N;
  if (summed) {
    u64 sum = 0;
#pragma unroll
    for (int e = 0; e < kGroup; ++e) sum += weight(x_if(v[e] > -INFINITY, v[e], s.c), N);
    sum = wave_add(sum);
    if (lane == 0) st.piece_sum[piece] = sum;
    return;
  }
#pragma unroll
  for (int e = 0; e < kGroup; ++e) {
    const double x = x_if(v[e] > -INFINITY, v[e], s.c);
    const u64 w = weight(x, N);
    if (w != 0) atomicAdd(&bins[static_cast<int>(fmin(bin_of(x, N), kBins - 1.0))], w);
  }
  __syncthreads();
  for (int i = tid; i < kBins; i += kChunkWaves * kWave) st.bins[static_cast<int64_t>(chunk) * kBins + i] = bins[i];
}

// ---- second launch
constexpr int kMaxPieces = (MOE_SAMPLE_MAX_V + 7 + kChunk - 1) / kChunk * kChunkWaves;
constexpr int kSumsPerThread = (kMaxPieces + kRowThreads - 1) / kRowThreads;
struct alignas(16) Shared {
  uint32_t top[kHeldGroups];    // largest keys of the groups, where the row has no more
  uint16_t group[kHeldGroups];  // groups with candidates
  u64 list[kList];
  u64 sums[kMaxPieces];  // of the pieces
  u64 bins[kFine];
  u64 waves[2][kRowWaves];
  u64 found, found2;
  int count, groups;
};

// Of a workgroup's values, in thread order: the sum before each, and of all.
// Two sets of sums in turn: a set is written again only after the barrier of
// the call between, hence one barrier a call.
__device__ __forceinline__ u64 block_before(u64 v, u64 (&waves)[2][kRowWaves], int& turn, u64& all) {
  const int wave = threadIdx.x >> 6;
  const u64 upto = wave_upto(v);
  turn ^= 1;
  if ((threadIdx.x & 63) == 63) waves[turn][wave] = upto;
  __syncthreads();
  u64 t = upto - v;
  all = 0;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    if (w < wave) t += waves[turn][w];
    all += waves[turn][w];
  }
  return t;
}
__device__ __forceinline__ u64 block_add(u64 v, u64 (&waves)[2][kRowWaves], int& turn) {
  u64 all;
  block_before(v, waves, turn, all);
  return all;
}

// Sorts list[0 .. n) descending (bitonic, padded with zeros).  Ends with a
// barrier.  Exchanges over up to 64 entries stay within the 128 entries that a
// wave has in hand, and a wave's LDS accesses are in order: no barrier there.
__device__ __forceinline__ void sort_list(u64* list, int n) {
  int size = 2;
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += kRowThreads) list[i] = 0;
  __syncthreads();
#pragma unroll 1
  for (int k = 2; k <= size; k <<= 1)
#pragma unroll 1
    for (int j = k >> 1; j > 0; j >>= 1) {
      if (j > kWave || (j == kWave && k > 2 * kWave)) __syncthreads();
#pragma unroll 1
      for (int i = threadIdx.x; i < size / 2; i += kRowThreads) {
        const int lo = (i & (j - 1)) | ((i & ~(j - 1)) << 1), hi = lo | j;
        const u64 p = list[lo], q = list[hi];
        if ((p < q) == ((lo & k) == 0)) list[lo] = q, list[hi] = p;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  __syncthreads();
}

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ __forceinline__ u64 part_of(double share, u64 all) {  // floor(share all)
  return static_cast<u64>(share * static_cast<double>(all));
}

template <bool F32>
struct Choice {
  const SampleArgs& a;
  const int b, part, parts, pieces, lane, wave;
  const Settings s;
  const Row<F32> row;
  const RowStats st;
  Shared& sh;
  const Weigh weight;
  int turn = 0;      // of the block's sums
  int32_t first;     // the largest element,
  double x_most, N;  // its x, the floor of that
  u64 min_rank;      // what min_p keeps is of this rank at least

  __device__ __forceinline__ Choice(const SampleArgs& a_, const Ws& ws, Shared& sh_)
      : a(a_), b(blockIdx.y), part(blockIdx.x), parts(gridDim.x), pieces(ws.chunks * kChunkWaves), lane(threadIdx.x & 63),
        wave(threadIdx.x >> 6), s(settings_of(a_, b)), row(a_, b), st(ws.row(b)), sh(sh_) {}

  __device__ __forceinline__ u64 before(u64 v, u64& all) { return block_before(v, sh.waves, turn, all); }
  __device__ __forceinline__ u64 total(u64 v) { return block_add(v, sh.waves, turn); }

  // One element: its key and index, larger is earlier in the order.
  __device__ __forceinline__ u64 rank_of(float v, int place) const {
    return static_cast<u64>(key_of(v)) << 32 | static_cast<uint32_t>(~(place - row.skew));
  }
  __device__ __forceinline__ double x_at(u64 rank) const { return x_of(value_of(static_cast<uint32_t>(rank >> 32)), s.c); }
  __device__ __forceinline__ int piece_of(u64 rank) const {
    return static_cast<int>((~static_cast<uint32_t>(rank) + row.skew) / kPiece);
  }

  __device__ __forceinline__ void write(int32_t token, double logprob) const {
    a.token[b] = token;
    if (a.logprob != nullptr) a.logprob[b] = static_cast<float>(logprob);
  }
  // By one lane, the token of place p and value v.
  __device__ __forceinline__ void write(int p, float v, u64 all) const {
    write(p - row.skew, (x_of(v, s.c) - N) * 0.6931471805599453 - log(static_cast<double>(all) * 0x1p-42));
  }
  // The draw: the running sum that the token's has to pass.
  __device__ __forceinline__ u64 draw(u64 all) const {
    const double u = a.u[b];
    return u >= 1.0 ? all - 1 : u > 0.0 ? min(part_of(u, all), all - 1) : 0;  // no integer of what passes 64 bits
  }
  // The sum that the shortest prefix reaches.
  __device__ __forceinline__ u64 needed(u64 all) const {
    return s.p > 0.0 ? max(static_cast<u64>(ceil(s.p * static_cast<double>(all))), 1ull) : 1;
  }

  // Weight of an element that stays: rank >= least.
  __device__ __forceinline__ u64 kept(float v, int place, u64 least, double unit) const {
    return weight(x_if(key_of(v) != 0 && rank_of(v, place) >= least, v, s.c), unit);
  }

  // The least key whose x `in` takes, which takes all larger ones: a wave
  // compares 64 at a time.
  template <class In>
  __device__ __forceinline__ uint32_t least_key(In in) const {
    uint32_t base = 0;
#pragma unroll 1
    for (int shift = 26; shift >= 0; shift -= shift == 2 ? 2 : 6) {
      const uint32_t at = base + (static_cast<uint32_t>(lane) << shift) + ((1u << shift) - 1u);  // a block's last
      const u64 hit = __ballot(at > kInfKey || in(x_of(value_of(at), s.c)));
      base += static_cast<uint32_t>(__builtin_ctzll(hit | 1ull << 63)) << shift;
    }
    return base;
  }

  // ---- the draw in index order
  // The token of the running sum `r` within a piece, by the calling wave; the last
  // of any weight where r is past them all (u of 1 and more, a sum rounded up).
  __device__ __forceinline__ void pick(int piece, u64 r, u64 least, u64 all, double unit) const {
    float v[kGroup];
    row.load(piece, v);
    constexpr int W = Row<F32>::W;
    int token = -1, last = -1;
    float value = 0.0f, last_value = 0.0f;
    bool done = false;
#pragma unroll
    for (int i = 0; i < kGroup / W; ++i) {
      u64 w[W], t = 0;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        w[j] = kept(v[i * W + j], row.place(piece, i * W + j), least, unit);
        t += w[j];
        if (w[j] != 0) {
          last = row.place(piece, i * W + j);
          last_value = v[i * W + j];
        }
      }
      u64 at = wave_before(t);
      const u64 sum = lane_value(at + t, kWave - 1);
      if (!done && r < sum) {
        done = true;
#pragma unroll
        for (int j = 0; j < W; ++j) {
          if (at <= r && r < at + w[j]) {
            token = row.place(piece, i * W + j);
            value = v[i * W + j];
          }
          at += w[j];
        }
      }
      if (!done) r -= sum;
    }
    if (!done) {
      int most = last;
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1) most = max(most, shfl_xor(most, m));
      if (last == most) token = last, value = last_value;
    }
    if (token >= 0) write(token, value, all);
  }

  // sums[0 .. pieces) hold the pieces' weights (or, of_chunks, each chunk's first
  // the chunk's): finds the draw's piece and picks there.  `rescaled`: they are
  // rounded from sums in their chunk's unit, in which the draw then goes on.
  __device__ __forceinline__ void pick_by_sums(u64 least, bool of_chunks, bool rescaled) {
    __syncthreads();
    u64 mine[kSumsPerThread], t = 0, all;
    const int i0 = threadIdx.x * kSumsPerThread;
#pragma unroll
    for (int j = 0; j < kSumsPerThread; ++j) {
      mine[j] = i0 + j < pieces ? sh.sums[i0 + j] : 0;
      t += mine[j];
    }
    u64 at = before(t, all);
    const u64 r = draw(all);
#pragma unroll
    for (int j = 0; j < kSumsPerThread; ++j) {
      if (at <= r && r < at + mine[j]) {
        sh.found = i0 + j;
        sh.found2 = r - at;
      }
      at += mine[j];
    }
    __syncthreads();
    int piece = static_cast<int>(sh.found);
    const double unit = rescaled ? st.ref[piece / kChunkWaves] : N;
    // a sum that is not 0 is of a unit within 2^-64, and its part no more than it was there
    u64 rest = a.u[b] >= 1.0f ? ~0ull : sh.found2 << static_cast<int>(N - unit);
    if (of_chunks) {  // its pieces, a wave each
      static_assert(kChunkWaves == kRowWaves, "a wave per piece");
      float v[kGroup];
      row.load(piece + wave_index(), v);
      u64 sum = 0;
#pragma unroll
      for (int e = 0; e < kGroup; ++e) sum += kept(v[e], row.place(piece + wave_index(), e), least, unit);
      sum = wave_add(sum);
      turn ^= 1;
      if (lane == 0) sh.waves[turn][wave] = sum;
      __syncthreads();
      bool found = false;
      int w = 0;  // the piece, or the last of any weight
#pragma unroll
      for (int i = 0; i < kRowWaves; ++i) {
        const u64 here = sh.waves[turn][i];
        if (!found && here != 0) {
          w = i;
          found = rest < here;
          if (!found) rest -= here;
        }
      }
      piece += w;
      if (!found) rest = ~0ull;
    }
    if (wave == 0) pick(piece, rest, least, all, unit);
  }

  // ---- groups.  A row of up to kHeldPieces pieces has its groups' keys in
  // LDS; of a longer one they are read where they are.
  __device__ __forceinline__ bool held() const { return pieces <= kHeldPieces; }
  __device__ __forceinline__ uint32_t top_of(int g) const { return held() ? sh.top[g] : st.top[g]; }

  __device__ __forceinline__ void hold() {
    if (!held()) return;
    const int vecs = pieces * (kWave / 4);  // a multiple of 128
#pragma unroll 4
    for (int i = threadIdx.x; i < vecs; i += kRowThreads)
      reinterpret_cast<uint4*>(sh.top)[i] = reinterpret_cast<const uint4*>(st.top)[i];
    __syncthreads();
  }

  // Lists the groups whose largest key is at least lo, and counts them; -1 where
  // the row's keys are not held.
  __device__ __forceinline__ int list_groups(uint32_t lo) {
    if (!held()) return -1;
    __syncthreads();
    if (threadIdx.x == 0) sh.groups = 0;
    __syncthreads();
    const int groups = pieces * kWave;
    constexpr int kAtOnce = 8;  // per addition to the count
#pragma unroll 1
    for (int i0 = 0; i0 < groups; i0 += kAtOnce * kRowThreads) {
      bool on[kAtOnce];
      u64 m[kAtOnce];
      int n = 0;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int g = i0 + i * kRowThreads + static_cast<int>(threadIdx.x);
        const uint32_t top = g < groups ? sh.top[g] : 0;
        on[i] = top != 0 && top >= lo;
        m[i] = __ballot(on[i]);
        n += __popcll(m[i]);
      }
      if (n == 0) continue;
      int at = 0;
      if (lane == 0) at = atomicAdd(&sh.groups, n);
      at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (on[i]) sh.group[at + __popcll(m[i] & ((1ull << lane) - 1))] = static_cast<uint16_t>(i0 + i * kRowThreads + threadIdx.x);
        at += __popcll(m[i]);
      }
    }
    __syncthreads();
    return sh.groups;
  }

  // f(v, p) for the vectors v from place p on of the listed groups, spread over
  // all threads; whole waves call it, lanes without a vector with -infinities.
  template <class F>
  __device__ __forceinline__ void each_listed(F f) {
    constexpr int W = Row<F32>::W, kVecs = kGroup / W;
    const int n = sh.groups * kVecs;
#pragma unroll 1
    for (int first = wave * kWave; first < n; first += 2 * kRowThreads) {
      float v[2][W];
      int p[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int i = first + j * kRowThreads + lane;
        const int g = sh.group[min(i, n - 1) / kVecs];
        p[j] = g / kWave * kPiece + i % kVecs * (kWave * W) + g % kWave * W;
        row.vec(p[j], v[j]);
        if (i >= n)
#pragma unroll
          for (int e = 0; e < W; ++e) v[j][e] = -INFINITY;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) f(v[j], p[j]);
    }
  }
  // The same for the whole pieces from, from + step, ... that have a group of lo
  // or more, a wave each, and add(the sum of what f returned, piece).
  template <class F, class Add>
  __device__ __forceinline__ void each_piece(uint32_t lo, int from, int step, F f, Add add) {
    constexpr int W = Row<F32>::W;
#pragma unroll 1
    for (int piece = from + wave; piece < pieces; piece += step) {
      const uint32_t top = top_of(piece * kWave + lane);
      u64 t = 0;
      if (__any(top != 0 && top >= lo)) {
        float v[kGroup];
        row.load(piece, v);
#pragma unroll
        for (int e = 0; e < kGroup; e += W) t += f(v + e, row.place(piece, e));
      }
      add(t, piece);
    }
  }

  __device__ __forceinline__ void clear_sums() {
    for (int i = threadIdx.x; i < pieces; i += kRowThreads) sh.sums[i] = 0;
  }

  // Weights of what stays, by pieces.
  __device__ __forceinline__ void sum_pieces(u64 least) {
    each_piece(static_cast<uint32_t>(least >> 32), 0, kRowWaves,
               [&](const float* v, int p) {
                 u64 t = 0;
#pragma unroll
                 for (int e = 0; e < Row<F32>::W; ++e) t += kept(v[e], p + e, least, N);
                 return t;
               },
               [&](u64 t, int piece) {
                 t = wave_add(t);
                 if (lane == 0) sh.sums[piece] = t;
               });
  }

  // Elements of a vector whose keys are lo .. hi - 1 (hi 0: all from lo on) to the
  // list; a wave's places in it come from one addition to the count.
  __device__ __forceinline__ void put_in_list(const float* v, int p, uint32_t lo, uint32_t hi) {
    constexpr int W = Row<F32>::W;
    uint32_t hits = 0;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const uint32_t key = key_of(v[e]);
      hits |= key != 0 && key >= lo && (hi == 0 || key < hi) ? 1u << e : 0u;
    }
    if (!__any(hits != 0)) return;
    const int n = __popc(hits), upto = wave_upto(n);
    int base = 0;
    if (lane == kWave - 1) base = atomicAdd(&sh.count, upto);
    int at = __builtin_amdgcn_readlane(base, kWave - 1) + upto - n;
#pragma unroll
    for (int e = 0; e < W; ++e)
      if (hits >> e & 1) {
        if (at < kList) sh.list[at] = rank_of(v[e], p + e);
        ++at;
      }
  }

  // A count begins again at zero behind a barrier of its own: every wave has read
  // the count before it by then, and whether that fits the list decides its way.
  __device__ __forceinline__ void start_count() {
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
  }

  // Collects the elements of keys from lo on (`whole`: of all pieces, else of
  // the listed groups): the count, of which the first kList are in the list.
  __device__ __forceinline__ int collect(uint32_t lo, bool whole) {
    start_count();
    auto f = [&](const float* v, int p) -> u64 {
      put_in_list(v, p, lo, 0);
      return 0;
    };
    if (whole) each_piece(lo, 0, kRowWaves, f, [](u64, int) {});
    else each_listed(f);
    __syncthreads();
    return sh.count;
  }

  // Collects the elements of keys lo .. hi - 1, and (`sums`) sums, by pieces, the
  // weights of those from hi on that min_p keeps, from whole pieces.  The row's
  // workgroups may share them: each leaves its pieces' sums and its list in
  // memory, and the last to be through goes on with all of it.  -1 where this
  // workgroup has nothing more to do.
  __device__ __forceinline__ int collect_and_sum(uint32_t lo, uint32_t hi, bool shared, bool sums) {
    const uint32_t least = max(hi, static_cast<uint32_t>(min_rank >> 32));
    start_count();
    auto f = [&](const float* v, int p) {
      u64 t = 0;
      if (sums) {
#pragma unroll
        for (int e = 0; e < Row<F32>::W; ++e) t += weight(x_if(key_of(v[e]) >= least, v[e], s.c), N);
      }
      if (lo < hi) put_in_list(v, p, lo, hi);
      return t;
    };
    each_piece(lo, shared ? part * kRowWaves : 0, shared ? parts * kRowWaves : kRowWaves, f, [&](u64 t, int piece) {
      if (!sums) return;
      t = wave_add(t);
      if (lane != 0) return;
      if (shared) st.piece_sum[piece] = t;
      else sh.sums[piece] = t;
    });
    __syncthreads();
    if (!shared) return sh.count;
    const int mine = sh.count;
    for (int i = threadIdx.x; i < min(mine, kList); i += kRowThreads) st.lists[static_cast<int64_t>(part) * kList + i] = sh.list[i];
    if (threadIdx.x == 0) st.done[1 + part] = mine;
    // One thread releases what all wrote before the barrier, and acquires what
    // the others did for all: a fence by every wave writes the caches back
    // eight times over (64 us where 64 rows share the chip).  Each wave's own
    // stores have reached the cache that is written back by then.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
      sh.count = __hip_atomic_fetch_add(st.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (sh.count != parts - 1) return -1;
    if (sums)
      for (int i = threadIdx.x; i < pieces; i += kRowThreads) sh.sums[i] = st.piece_sum[i];
    // a wave per part
    static_assert(kMaxParts <= kRowWaves, "a part each");
    const int here = lane < parts ? st.done[1 + lane] : 0, upto = wave_upto(here);
    if (const int p = wave_index(); p < parts) {
      const int at = __builtin_amdgcn_readlane(upto - here, p);
      const int m = min(__builtin_amdgcn_readlane(here, p), kList - at);  // lists that are cut short make n pass kList
#pragma unroll 4
      for (int i = lane; i < m; i += kWave) sh.list[at + i] = st.lists[static_cast<int64_t>(p) * kList + i];
    }
    __syncthreads();
    return __builtin_amdgcn_readlane(upto, kWave - 1);
  }

  // A key that k groups (or sets of groups) reach: at least k elements do.
  __device__ __forceinline__ uint32_t floor_of_kth(int k) {
    const int groups = pieces * kWave;
    if (k <= 128) {
      // 256 sets of groups do for a small k; the first wave halves the range of keys step by step
      uint32_t most = 0;
#pragma unroll 4
      for (int g = threadIdx.x; g < groups; g += kRowThreads) most = max(most, top_of(g));
      sh.list[threadIdx.x] = most;
      __syncthreads();
      if (wave == 0) {
        uint32_t top[kRowThreads / (2 * kWave)];
#pragma unroll
        for (int i = 0; i < kRowThreads / (2 * kWave); ++i)
          top[i] = static_cast<uint32_t>(max(sh.list[2 * i * kWave + lane], sh.list[(2 * i + 1) * kWave + lane]));
        uint32_t kth = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 10; --bit) {
          const uint32_t at = kth | 1u << bit;
          int n = 0;
#pragma unroll
          for (int i = 0; i < kRowThreads / (2 * kWave); ++i) n += __popcll(__ballot(top[i] >= at));
          if (n >= k) kth = at;
        }
        if (lane == 0) sh.found = kth;
      }
      __syncthreads();
      return static_cast<uint32_t>(sh.found);
    }
    // more: a histogram of the groups, by 32nds of an octave below the largest
    auto bin = [&](double x) { return static_cast<int>(fmin((x_most - x) * 32.0, kFine - 1.0)); };
    clear_bins();
    __syncthreads();
    for (int g = threadIdx.x; g < groups; g += kRowThreads)
      if (const uint32_t top = top_of(g); top != 0) atomicAdd(&sh.bins[bin(x_of(value_of(top), s.c))], 1ull);
    const int at = find_bin(k);
    return at < 0 || at == kFine - 1 ? 0 : least_key([&](double x) { return x_most - x < 1e18 && bin(x) <= at; });
  }

  __device__ __forceinline__ void clear_bins() {
    for (int i = threadIdx.x; i < kFine; i += kRowThreads) sh.bins[i] = 0;
  }
  // The bin at which the bins' running sum reaches `need`, and in found2 what
  // of it is left before that bin; -1 where it does not.  Begins and ends with a barrier.
  __device__ __forceinline__ int find_bin(u64 need) {
    __syncthreads();
    if (threadIdx.x == 0) sh.found = kFine;
    constexpr int per = kFine / kRowThreads;
    u64 mine[per], t = 0, all;
#pragma unroll
    for (int j = 0; j < per; ++j) {
      mine[j] = sh.bins[threadIdx.x * per + j];
      t += mine[j];
    }
    u64 at = before(t, all);
#pragma unroll
    for (int j = 0; j < per; ++j) {
      if (at < need && need <= at + mine[j]) {
        sh.found = threadIdx.x * per + j;
        sh.found2 = need - at;
      }
      at += mine[j];
    }
    __syncthreads();
    return sh.found == kFine ? -1 : static_cast<int>(sh.found);
  }

  // Of the list's n elements of rank >= least, all of x_top - x < kFine / scale,
  // the rank of the last of the shortest prefix that counts (COUNT) or weighs
  // `need`: by fine bins, then by the order within one.  `none` where they do not reach it.
  template <bool COUNT>
  __device__ __forceinline__ u64 border(int n, u64 least, u64 need, double x_top, double scale, u64 none) {
    u64* const few = reinterpret_cast<u64*>(sh.top);  // the groups' keys have served
    static_assert(sizeof(sh.top) >= sizeof(sh.list), "a bin may hold all of the list");
    auto bin = [&](u64 rank) { return static_cast<int>(fmin(fmax((x_top - x_at(rank)) * scale, 0.0), kFine - 1.0)); };
    auto measure = [&](u64 rank) -> u64 {
      if constexpr (COUNT) return 1;
      else return weight(x_at(rank), N);
    };
    __syncthreads();
    clear_bins();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += kRowThreads)
      if (const u64 rank = sh.list[i]; rank >= least) atomicAdd(&sh.bins[bin(rank)], measure(rank));
    const int at = find_bin(need);
    if (at < 0) return none;
    const u64 rest = sh.found2;
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += kRowThreads)
      if (const u64 rank = sh.list[i]; rank >= least && bin(rank) == at) few[atomicAdd(&sh.count, 1)] = rank;
    __syncthreads();
    const int m = sh.count;
    if (threadIdx.x == 0) sh.found = none;
    if (m <= kWave) {
      if (wave == 0) {
        const u64 rank = lane < m ? few[lane] : 0, w = rank != 0 ? measure(rank) : 0;
        u64 less = 0;
#pragma unroll 1
        for (int j = 0; j < m; ++j) {
          const u64 other = lane_value(rank, j), ow = lane_value(w, j);
          less += other > rank ? ow : 0;
        }
        if (less < rest && rest <= less + w) sh.found = rank;
      }
    } else {
      sort_list(few, m);
      const int i0 = threadIdx.x * kMine;
      u64 t = 0, all;
#pragma unroll 1
      for (int j = i0; j < min(i0 + kMine, m); ++j) t += measure(few[j]);
      u64 less = before(t, all);
#pragma unroll 1
      for (int j = i0; j < min(i0 + kMine, m); ++j) {
        const u64 w = measure(few[j]);
        if (less < rest && rest <= less + w) sh.found = few[j];
        less += w;
      }
    }
    __syncthreads();
    return sh.found;
  }
  // The weights of the list's elements of rank >= least, to the sums of their pieces or chunks.
  __device__ __forceinline__ void add_to_sums(int n, u64 least, bool of_chunks) {
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += kRowThreads)
      if (const u64 rank = sh.list[i]; rank >= least) atomicAdd(&sh.sums[piece_of(rank) & (of_chunks ? -kChunkWaves : -1)], weight(x_at(rank), N));
  }

  // Fine bins per unit of x from the largest down to key lo's.
  __device__ __forceinline__ double scale_from(uint32_t lo) const {
    const double x_lo = lo != 0 ? x_of(value_of(lo), s.c) : x_most - kOctaves, span = x_most - x_lo;
    return span > 0.0 && span < 1e18 ? kFine / span : 0.0;
  }
  // Filters and draws from a list of up to a wave of candidates, a lane each: places and sums in
  // the order, then sums in index order, from a comparison with each of the
  // others, an eighth of them by each of the waves.
  __device__ __forceinline__ void choose_from_few(int n, int k) {
    static_assert(kRowWaves * 8 == kWave && 2 * kRowThreads <= kFine, "eight others a wave, two sets of sums in bins");
    const u64 rank = lane < n ? sh.list[lane] : 0;
    u64 w = rank != 0 ? weight(x_at(rank), N) : 0, t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = wave_index() * 8 + i;
      const u64 other = lane_value(rank, j), ow = lane_value(w, j);
      t += other > rank ? ow | 1ull << 56 : 0;  // weights sum to less than 2^50, places above them
    }
    t = add_up(t, 0);
    if (static_cast<int>(t >> 56) >= k) w = 0;
    if (s.filter_p && (t & ((1ull << 56) - 1)) >= needed(wave_add(w))) w = 0;
    if (rank < min_rank) w = 0;
    const u64 all = wave_add(w), r = draw(all);
    const uint32_t index = ~static_cast<uint32_t>(rank);
    t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = wave_index() * 8 + i;
      const u64 ow = lane_value(w, j);
      t += static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(index), j)) < index ? ow : 0;
    }
    t = add_up(t, 1);
    if (wave == 0 && t <= r && r < t + w)
      write(static_cast<int>(index) + row.skew, value_of(static_cast<uint32_t>(rank >> 32)), all);
  }
  // The sum of the waves' values of a lane, in set 0 or 1 of the bins.
  __device__ __forceinline__ u64 add_up(u64 v, int set) {
    u64* const at = sh.bins + set * kRowThreads;
    at[threadIdx.x] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < kRowWaves; ++i) v += at[i * kWave + lane];
    return v;
  }

  // The eighth of an octave in which the shortest prefix ends that holds top_p
  // of the weight: its keys lo .. hi - 1, and the weight that is needed of it.
  __device__ __forceinline__ u64 border_bin(uint32_t& lo, uint32_t& hi, int& bin, u64& need) {
    const int chunks = pieces / kChunkWaves;
    __syncthreads();
    clear_bins();
    __syncthreads();
    // a thread per bin, eight chunks' on their way at a time
    if (threadIdx.x < kBins) {
      u64 t = 0;
#pragma unroll 1
      for (int c = 0; c < chunks; c += 8) {
        u64 w[8];
        double ref[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) ref[j] = c + j < chunks ? st.ref[c + j] : kNoLogits;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const double from = static_cast<int>(threadIdx.x) - kPerOctave * (N - ref[j]);
          w[j] = from >= 0.0 ? st.bins[static_cast<int64_t>(c + j) * kBins + static_cast<int>(from)] : 0;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) t += rescale(w[j], ref[j], N);
      }
      sh.bins[threadIdx.x] = t;
    }
    __syncthreads();
    u64 t = 0;
    for (int i = threadIdx.x; i < kBins; i += kRowThreads) t += sh.bins[i];
    need = needed(total(t));
    bin = find_bin(need);
    const double at = bin;
    lo = least_key([&](double x) { return bin_of(x, N) <= at; });
    hi = least_key([&](double x) { return bin_of(x, N) < at; });
    return sh.found2;
  }

  // The chunks' weights in bins before `bin`, each as its first piece's sum.
  __device__ __forceinline__ void sum_chunks(int bin) {
    __syncthreads();
    clear_sums();
    __syncthreads();
#pragma unroll 1
    for (int c = wave_index(); c < pieces / kChunkWaves; c += kRowWaves) {
      const double ref = st.ref[c], shift = kPerOctave * (N - ref);
      u64 t = 0;
#pragma unroll
      for (int i0 = 0; i0 < kBins; i0 += kWave)
        if (const int i = i0 + lane; i < kBins && i + shift < bin) t += st.bins[static_cast<int64_t>(c) * kBins + i];
      t = wave_add(t);
      if (lane == 0) sh.sums[c * kChunkWaves] = rescale(t, ref, N);
    }
  }

  // ---- what the lists do not hold (more than kList elements in the border's bin of a
  // flat row, thousands of equal logits, a top_k of thousands): 64 passes over the row,
  // 3 to 4 ms at 160000 to 200000 normal logits of temperature 1 and top-p 0.95, where
  // 120000 take 40 us.  Count or weight of the elements of rank >= at.
  template <bool COUNT>
  __device__ __forceinline__ u64 measure(u64 at) {
    u64 t = 0;
    each_piece(static_cast<uint32_t>(at >> 32), 0, kRowWaves,
               [&](const float* v, int p) {
                 u64 n = 0;
#pragma unroll
                 for (int e = 0; e < Row<F32>::W; ++e)
                   if (const bool in = key_of(v[e]) != 0 && rank_of(v[e], p + e) >= at; COUNT) n += in;
                   else n += weight(x_if(in, v[e], s.c), N);
                 return n;
               },
               [&](u64 n, int) { t += n; });
    return total(t);
  }
  // The largest rank whose elements measure `need`, bit by bit.  A row of up
  // to 8 pieces stays in registers meanwhile.
  template <bool COUNT>
  __device__ __forceinline__ u64 search(u64 need) {
    u64 at = 0;
    if (pieces <= kRowWaves) {
      float v[kGroup];
      u64 rank[kGroup], w[kGroup];
      row.load(wave, v);
#pragma unroll
      for (int e = 0; e < kGroup; ++e) {
        const bool on = wave < pieces && key_of(v[e]) != 0;
        rank[e] = on ? rank_of(v[e], row.place(wave, e)) : 0;
        w[e] = COUNT ? on : weight(x_if(on, v[e], s.c), N);
      }
#pragma unroll 1
      for (int bit = 63; bit >= 0; --bit) {
        const u64 next = at | 1ull << bit;
        u64 t = 0;
#pragma unroll
        for (int e = 0; e < kGroup; ++e) t += rank[e] >= next ? w[e] : 0;
        if (total(t) >= need) at = next;
      }
      return at;
    }
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
      const u64 next = at | 1ull << bit;
      if (measure<COUNT>(next) >= need) at = next;
    }
    return at;
  }

  __device__ __forceinline__ void run() {
    if (!s.greedy && (s.filter_k || s.filter_p || s.filter_m) && !(part != 0 && s.filter_k)) hold();
    // the row's largest
    u64 best = 0;
    for (int i = lane; i < pieces / kChunkWaves; i += kWave) best = max(best, st.best[i]);
    best = wave_most(best);
    const uint32_t most = static_cast<uint32_t>(best >> 32);
    first = static_cast<int32_t>(~static_cast<uint32_t>(best));
    const bool alone = s.greedy || most == 0 || s.filter_k || !(s.filter_p || s.filter_m);
    if (alone && part != 0) return;
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
    min_rank = 0;
    if (s.filter_m) {
      const double x_least = x_most + log2(s.m);
      min_rank = static_cast<u64>(least_key([&](double x) { return x >= x_least; })) << 32;
    }
    // Each way ends in the same steps, which stand once at the end: what a
    // workgroup runs it runs once, so that the size of its code counts.
    u64 least = 0;
    int n = 0;            // candidates in the list, where it holds them all,
    bool listed = false;  // of which top_p's border comes at `need` past x_top;
    bool apart = false;   // the list is all there is, the pieces' sums are not begun
    bool summed = false;  // the pieces' sums are complete
    bool chunked = false;  // the sums are the chunks', from their bins: no weight is computed again but in the draw's
    bool rescaled = false;  // the sums are rounded from their chunks' units
    u64 need = 0, none = 0;
    double x_top = x_most, scale = 0.0;
    if (s.filter_k) {
      if (s.k <= kFastK) {
        const uint32_t lo = floor_of_kth(s.k);
        const int groups = list_groups(lo);
        n = collect(lo, groups < 0 || groups > pieces * kWave / 4);
        if (n <= kWave) {
          choose_from_few(n, s.k);
          return;
        }
        listed = apart = n <= kList;
        if (listed) {
          scale = scale_from(lo);
          if (n > s.k) least = border<true>(n, 0, s.k, x_top, scale, 0);
          if (s.filter_p) {
            u64 t = 0;
#pragma unroll 1
            for (int i = threadIdx.x; i < n; i += kRowThreads)
              if (const u64 rank = sh.list[i]; rank >= least) t += weight(x_at(rank), N);
            need = needed(total(t));
          }
        }
      }
      if (!listed) least = search<true>(s.k);
    } else if (s.filter_p || s.filter_m) {
      uint32_t lo = static_cast<uint32_t>(min_rank >> 32), hi = lo;
      int bin = 0;
      u64 rest = 0;
      if (s.filter_p) rest = border_bin(lo, hi, bin, need);
      none = static_cast<u64>(lo) << 32;
      // few groups: all that is left is likely to fit the list
      const int groups = list_groups(lo);
      const bool few = groups >= 0 && groups <= kFewGroups;
      if (few) {
        if (part != 0) return;
        n = collect(lo, false);
        listed = apart = n <= kList;
        scale = scale_from(lo);
      }
      if (!listed) {
        // Where min_p takes nothing off before the border's bin, the bins' weights are
        // what stays.  Using them pays from about four pieces a wave where a row has few
        // workgroups (at temperature 1 and top-p 0.9 256 rows of 50001 in bf16: 73 us, 69
        // with them; 64 of 131072: 61, 59), and costs steps of its own where it has many
        // (one row of 131072: 35.6, 36.5).  The row's length
        // alone decides, so that its bits do not depend on how many rows there are.
        chunked = s.filter_p && static_cast<uint32_t>(min_rank >> 32) <= hi && pieces > 4 * kRowWaves;
        n = collect_and_sum(lo, hi, !few && parts > 1, !chunked);
        if (n < 0) return;
        summed = !s.filter_p;
        listed = !summed && n > 0 && n <= kList;
        chunked = chunked && listed;
        if (chunked) sum_chunks(bin);
        rescaled = chunked;
        need = rest, x_top = N + 1.0 - bin * (1.0 / kPerOctave), scale = kFine * kPerOctave;
      }
    } else {
      for (int i = threadIdx.x; i < pieces; i += kRowThreads)
        sh.sums[i] = rescale(st.piece_sum[i], st.ref[i / kChunkWaves], N);
      summed = rescaled = true;
    }
    if (listed) {
      if (s.filter_p) least = max(least, border<false>(n, least, need, x_top, scale, none));
      least = max(least, min_rank);
      __syncthreads();
      if (apart) clear_sums();
      __syncthreads();
      add_to_sums(n, least, chunked);
    } else if (!summed) {
      if (s.filter_p) least = max(least, search<false>(needed(measure<false>(least))));
      least = max(least, min_rank);
      sum_pieces(least);
    } else {
      least = min_rank;
    }
    pick_by_sums(least, chunked, rescaled);
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
    hipLaunchKernelGGL(k_sample_rows<true>, dim3(parts_of(a.B), a.B), dim3(kRowThreads), 0, s, a, ws);
  } else {
    hipLaunchKernelGGL(k_sample_chunks<false>, dim3(ws.chunks, a.B), dim3(kChunkWaves * kWave), 0, s, a, ws);
    hipLaunchKernelGGL(k_sample_rows<false>, dim3(parts_of(a.B), a.B), dim3(kRowThreads), 0, s, a, ws);
  }
  return hipGetLastError();
}

}  // namespace moe
