// Attention over the paged 8-bit cache, single tokens and prompt chunks.
//
// A request's new tokens and the heads that share a kv head form one matrix of
// rows r = (token, head), so that few tokens still fill a matrix-core tile.
// The int8 keys and values become fp16, which is exact; a block's scale
// multiplies its scores (keys) and its probabilities (values), so the products
// themselves see integers.  Queries become fp16 divided by a power of two per
// row (their 8 significant bits fit in 11).
//
// Scores are formed transposed, S^T = K Q^T, and the output as O^T = V^T P^T:
// what one lane holds of S^T after the first product (4 tokens of one row per
// fragment) is what it must supply of P^T to the second, so probabilities
// never leave their lane.  For that, fragment j of a 64-token tile takes its 16
// tokens in the order 16 (m / 4) + 4 j + m % 4: lane group g (l / 16) then owns
// tokens 16 g .. 16 g + 15 of the tile, 16 consecutive values of each value row.
//
// Softmax statistics are fp32.  Probabilities are rounded to fp16 for the
// second product (11 bits, an eighth of the output's own rounding), times the
// value scale: with s a key's score and c its value scale, the running maximum
// is that of s + log2 c, so the weights w = 2^7 c exp2(s - max) are bounded by
// the format whatever c is, and keep all their bits down to 2^-21 of the
// largest.  The sum of the probabilities (times 2^7) is that of w / c, one
// factor per 16 tokens.
#include "serve.hpp"
#include "trace.hpp"

namespace moe {

namespace {

constexpr int kTile = 64;  // tokens per step
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kBoostLog2 = 7.0f;     // weights of the maximum are 2^7 ...
constexpr float kSlack = 8.0f;         // ... and at most 2^15: fp16 ends at 2^16
// Least scale of values (a block of zeros has 0): 2^30 weights of 2^15 over it,
// the most that a sum can hold, stay in fp32.
constexpr float kMinScale = 0x1p-80f;

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct AttnArgs {
  moe_kv_cache c;
  moe_kv_batch b;
  const bf16_t* q;
  int64_t ldq;
  bf16_t* out;
  int64_t ldo;
  int heads, group;   // query heads, and per kv head
  int max_q, max_kv;
  int few;            // rows that count as few
  int chunk, chunks;  // keys per workgroup, workgroups per row tile
  float scale2;       // |scale| log2(e)
  bool negative;      // scale < 0: the queries change sign
  bool causal;
  float* part_o;      // [items][rows][D]
  float* part_ml;     // [items][rows][2]
};

__device__ __forceinline__ f32x4 mfma_f16(const uint4& p, const uint4& q, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p), __builtin_bit_cast(f16x8, q), acc, 0, 0,
                                                0);
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}

// 8 int8 -> 8 fp16 (exact): byte + 128 becomes the low bits of 1024 + (byte + 128).
__device__ __forceinline__ uint4 f16_of(uint32_t lo, uint32_t hi) {
  const f16x2 bias = {static_cast<_Float16>(-1152.0f), static_cast<_Float16>(-1152.0f)};
  auto two = [&](uint32_t w, uint32_t sel) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, sel)) + bias);
  };
  lo ^= 0x80808080u;
  hi ^= 0x80808080u;
  return make_uint4(two(lo, 0x04010400u), two(lo, 0x04030402u), two(hi, 0x04010400u), two(hi, 0x04030402u));
}

// 8 bf16 times f -> 8 fp16.
__device__ __forceinline__ uint4 f16_of_bf16(const uint4& v, float f) {
  return make_uint4(pack_f16(lo_bf(v.x) * f, hi_bf(v.x) * f), pack_f16(lo_bf(v.y) * f, hi_bf(v.y) * f),
                    pack_f16(lo_bf(v.z) * f, hi_bf(v.z) * f), pack_f16(lo_bf(v.w) * f, hi_bf(v.w) * f));
}

// Rows of one request and the keys they see.
struct Request {
  int first, n, rows;  // packed row, new tokens, rows of this kv head
  int kv, pos0;        // tokens in the cache, position of the first new token
};

__device__ __forceinline__ int row_start(const AttnArgs& p, int i) { return min(max(p.b.row_start[i], 0), p.b.T); }

__device__ __forceinline__ Request request(const AttnArgs& p, int b) {
  Request r;
  r.first = row_start(p, b);
  const int end = p.b.row_start[b + 1];
  const int all = max(min(end, p.b.T) - r.first, 0);
  const int len = max(p.b.kv_len[b], 0) - max(end - p.b.T, 0);  // without the tokens past the last row
  r.n = min(all, p.max_q);
  r.rows = r.n * p.group;
  r.kv = max(0, min(min(len, p.max_kv), p.b.W * p.c.block_tokens));
  r.pos0 = len - all;
  return r;
}

// Keys that token i of the request sees: [0, limit).
__device__ __forceinline__ int key_limit(const AttnArgs& p, const Request& r, int i) {
  return p.causal ? min(r.kv, r.pos0 + i + 1) : r.kv;
}

// Few rows (single tokens, or a few of one kv head; at most 16, or 32 where
// some request has more than 16): one workgroup per request, kv head and chunk
// of keys; its four waves take the chunk's 64-token steps in turn, each key read
// once into registers, and merge at the end.
// More: kMany rows per workgroup, 32 per wave; keys and values pass through LDS
// as fp16.
constexpr int kMany = 128;
constexpr int kBlocks = 2;

// Unit u of the row tiles of many rows: its request and tile (-1: none).  Work
// per tile goes with the request's keys, so the requests with the most keys
// come first (a last round of long ones took 28% of 16 ragged requests).  Up to
// 64 requests are ranked here, a lane each; beyond that there are workgroups
// enough, and a request whose rows start at packed row s simply owns units
// s g / kMany + b and following.
constexpr int kRanked = 64;

struct Unit {
  int b, tile;
};
__device__ __forceinline__ Unit row_unit(const AttnArgs& p, int u) {
  if (p.b.B <= kRanked) {
    const int lane = threadIdx.x & 63;
    int units = 0, keys = 0;
    if (lane < p.b.B) {
      const Request r = request(p, lane);
      units = r.rows > p.few ? cdiv(r.rows, kMany) : 0;
      keys = r.kv;
    }
    int before = 0;
    for (int i = 0; i < p.b.B; ++i) {
      const int k = __builtin_amdgcn_readlane(keys, i), n = __builtin_amdgcn_readlane(units, i);
      before += k > keys || (k == keys && i < lane) ? n : 0;
    }
    const unsigned long long mine = __ballot(u >= before && u < before + units);
    if (mine == 0) return {0, -1};
    const int b = __builtin_ctzll(mine);
    return {b, u - __builtin_amdgcn_readlane(before, b)};
  }
  auto at = [&](int m) { return static_cast<int>(static_cast<int64_t>(row_start(p, m)) * p.group / kMany) + m; };
  int lo = 0, hi = p.b.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at(mid) <= u) lo = mid;
    else hi = mid;
  }
  return {lo, u - at(lo)};
}

// Query fragments of one row, slices of 8 dims from dim(i), and the factor
// that turns a product with them into the score's base-2 exponent.
template <int N, class Dim>
__device__ __forceinline__ float load_query(const AttnArgs& p, const bf16_t* row, Dim dim, uint4 (&f)[N]) {
  uint4 v[N];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = *reinterpret_cast<const uint4*>(row + dim(i));
    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = max(m, max(w[j] & 0x7f800000u, (w[j] << 16) & 0x7f800000u));
  }
  m = max(m, static_cast<uint32_t>(shfl_xor(static_cast<int>(m), 16)));
  m = max(m, static_cast<uint32_t>(shfl_xor(static_cast<int>(m), 32)));
  // 2^e of the largest magnitude, kept where 2^e and 2^-e are normal (a row
  // with an infinity stays infinite)
  const uint32_t e = min(max(m >> 23, 1u), 253u);
  const float down = __uint_as_float((254u - e) << 23);
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = f16_of_bf16(v[i], p.negative ? -down : down);
  return __uint_as_float(e << 23) * p.scale2;
}

// The scales of the 16 tokens that a lane holds of a tile.
struct Scales {
  float key, value_log2, value_inv;
  __device__ __forceinline__ void set(float ks, float vs) {
    vs = vs != vs ? vs : fmaxf(vs, kMinScale);
    key = ks;
    value_log2 = __builtin_amdgcn_logf(vs);
    value_inv = __builtin_amdgcn_rcpf(vs);
  }
};

// One row's softmax state.  `weigh` turns the 16 scores s[j][i] (times the key
// scale and c) that a lane holds of the row into weights; `first` is the token
// of s[0][0].  The sums are relative to `m`, which follows the running maximum
// only when that has grown by kSlack: a lane finds that by itself, and only
// then do the lanes of a row meet.  `shrink` is then the factor for earlier
// sums, 1 otherwise.
struct Softmax {
  float m = -INFINITY, l = 0.0f, shrink = 1.0f;
  template <bool kMask>
  __device__ __forceinline__ void weigh(f32x4 (&s)[4], float c, Scales sc, int first, int limit) {
    c *= sc.key;
    if (kMask) {
      // a block that the row does not see may hold anything; masked scores
      // stay -infinity, so c must not be 0
      if (first >= limit) {
        c = 1.0f;
        sc.set(1.0f, 1.0f);
      }
      c = c == 0.0f ? kMinScale : c;
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (kMask && first + 4 * j + i >= limit) s[j][i] = -INFINITY;
        top = fmaxf(top, s[j][i]);
      }
    top = fmaf(top, c, sc.value_log2);
    shrink = 1.0f;
    if (__any(top > m + kSlack)) {
      top = fmaxf(top, shfl_xor(top, 16));
      top = fmaxf(top, shfl_xor(top, 32));
      if (top > m + kSlack) {
        shrink = __builtin_amdgcn_exp2f(m - top);
        l *= shrink;
        m = top;
      }
    }
    // no key seen yet: every weight is 0
    const float shift = kMask && m == -INFINITY ? 0.0f : sc.value_log2 + kBoostLog2 - m;
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[j][i] = __builtin_amdgcn_exp2f(fmaf(s[j][i], c, shift));
        sum[i & 1] += s[j][i];
      }
    l = fmaf(sum[0] + sum[1], sc.value_inv, l);
  }
};

// Weights of 16 tokens as the second product's operand.
__device__ __forceinline__ void pack_weights(const f32x4 (&s)[4], uint4 (&pf)[2]) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    pf[i] = make_uint4(pack_f16(s[2 * i][0], s[2 * i][1]), pack_f16(s[2 * i][2], s[2 * i][3]),
                       pack_f16(s[2 * i + 1][0], s[2 * i + 1][1]), pack_f16(s[2 * i + 1][2], s[2 * i + 1][3]));
}

// Row r of the request and kv head in the output.
__device__ __forceinline__ bf16_t* out_row(const AttnArgs& p, const Request& rq, int h, int r, int D) {
  return p.out + static_cast<int64_t>(rq.first + r / p.group) * p.ldo + (h * p.group + r % p.group) * D;
}

// Factor that turns a row's sums into its output (0 for a row without a key).
__device__ __forceinline__ float normaliser(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

// NB blocks of 16 rows.  64 single tokens over up to 32768 keys (32 / 4 heads of
// 128): 250 us, 5.2 TB/s of HBM reads, a copy's rate.  The registers of 32 rows
// leave one wave a SIMD instead of two: 64 x 4 tokens over 4096 keys 104 us, 64
// x 1 49.
template <int D, int NB>
__global__ __launch_bounds__(256) void k_kv_attention(AttnArgs p) {
  constexpr int kP = D / 64, kDt = D / 16;
  __shared__ float lds_o[4][16][D];
  __shared__ float lds_m[NB][4][16], lds_l[NB][4][16];
  const int chunk = blockIdx.x % p.chunks, b = blockIdx.x / p.chunks, h = blockIdx.y;
  const Request rq = request(p, b);
  if (rq.rows == 0 || rq.rows > p.few) return;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, g = lane >> 4;
  const int t0 = chunk * p.chunk;
  const int t1 = min(t0 + p.chunk, key_limit(p, rq, rq.n - 1));
  if (t0 >= t1 && chunk > 0) return;
  const int bt = p.c.block_tokens, shift = __builtin_ctz(bt);

  // this lane's rows; dims 64 i + 16 g + 8 s of slice (i, s): the order in which
  // one 16-byte load of a key supplies two slices
  int limit[NB];
  float c[NB];
  uint4 qf[NB][2 * kP];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int row = min(n * 16 + (lane & 15), rq.rows - 1), tok = row / p.group;
    limit[n] = key_limit(p, rq, tok);
    c[n] = load_query(p, p.q + static_cast<int64_t>(rq.first + tok) * p.ldq + (h * p.group + row % p.group) * D,
                      [&](int i) { return 64 * (i >> 1) + 16 * g + 8 * (i & 1); }, qf[n]);
  }

  Softmax sm[NB];
  f32x4 o[NB][kDt];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int d = 0; d < kDt; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int32_t* table = p.b.block_table + static_cast<int64_t>(b) * p.b.W;
  const int last = p.b.W - 1;
  const int gk = (lane & 15) >> 2;  // the 16-token group this lane loads keys of
  for (int t = t0 + wv * kTile; t < t1; t += 4 * kTile) {
    // blocks of the key group and of the value group; tokens past the table are past every limit
    const int bk = table[min((t + 16 * gk) >> shift, last)], bv = table[min((t + 16 * g) >> shift, last)];
    const bool seen = bv >= 0 && bv < p.c.n_blocks;
    const int64_t pk = static_cast<int64_t>(bk >= 0 && bk < p.c.n_blocks ? bk : 0) * p.c.kv_heads + h;
    const int64_t pv = static_cast<int64_t>(seen ? bv : 0) * p.c.kv_heads + h;
    const int8_t* kp = p.c.k + pk * bt * D + ((t + 16 * gk + (lane & 3)) & (bt - 1)) * D + 16 * g;
    const int8_t* vp = p.c.v + pv * bt * D + (lane & 15) * bt + ((t + 16 * g) & (bt - 1));
    uint4 kf[4][kP], vf[kDt];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < kP; ++i) kf[j][i] = *reinterpret_cast<const uint4*>(kp + 4 * j * D + 64 * i);
#pragma unroll
    for (int d = 0; d < kDt; ++d) vf[d] = *reinterpret_cast<const uint4*>(vp + d * 16 * bt);
    const float ks = p.c.k_scale[pv], vs = p.c.v_scale[pv];

    f32x4 s[NB][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int n = 0; n < NB; ++n) s[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kP; ++i) {
        const uint4 lo = f16_of(kf[j][i].x, kf[j][i].y), hi = f16_of(kf[j][i].z, kf[j][i].w);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          s[n][j] = mfma_f16(lo, qf[n][2 * i], s[n][j]);
          s[n][j] = mfma_f16(hi, qf[n][2 * i + 1], s[n][j]);
        }
      }
    }
    Scales sc;
    sc.set(ks, vs);
    uint4 pf[NB][2];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      sm[n].template weigh<true>(s[n], c[n], sc, t + 16 * g, seen ? limit[n] : 0);
      if (__any(sm[n].shrink != 1.0f)) {
#pragma unroll
        for (int d = 0; d < kDt; ++d) o[n][d] *= sm[n].shrink;
      }
      pack_weights(s[n], pf[n]);
    }
#pragma unroll
    for (int d = 0; d < kDt; ++d) {
      const uint4 lo = f16_of(vf[d].x, vf[d].y), hi = f16_of(vf[d].z, vf[d].w);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        o[n][d] = mfma_f16(lo, pf[n][0], o[n][d]);
        o[n][d] = mfma_f16(hi, pf[n][1], o[n][d]);
      }
    }
  }

  // merge the waves: o[n][d][i] is dimension 16 d + 4 g + i of row 16 n + lane % 16
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    float l = sm[n].l;
    l += shfl_xor(l, 16);
    l += shfl_xor(l, 32);
    if (lane < 16) {
      lds_m[n][wv][lane] = sm[n].m;
      lds_l[n][wv][lane] = l;
    }
  }
  constexpr int kPer = D / 16;  // dimensions per thread
  const int r = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * kPer;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    if (n > 0) {
      if (n * 16 >= rq.rows) return;
      __syncthreads();  // the block before is merged
    }
#pragma unroll
    for (int d = 0; d < kDt; ++d) *reinterpret_cast<f32x4*>(&lds_o[wv][lane & 15][16 * d + 4 * g]) = o[n][d];
    __syncthreads();
    const int row = n * 16 + r;
    if (row >= rq.rows) continue;
    float mm = -INFINITY, ll = 0.0f, acc[kPer] = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, lds_m[n][w][r]);
    const float base = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(lds_m[n][w][r] - base);
      ll += f * lds_l[n][w][r];
#pragma unroll
      for (int i = 0; i < kPer; ++i) acc[i] += f * lds_o[w][r][d0 + i];
    }
    if (p.chunks == 1) {
      const float inv = normaliser(ll);
      bf16_t* dst = out_row(p, rq, h, row, D) + d0;
#pragma unroll
      for (int i = 0; i < kPer; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = pack_bf16x2(acc[i] * inv, acc[i + 1] * inv);
      continue;
    }
    const int64_t at = ((static_cast<int64_t>(b) * p.c.kv_heads + h) * p.chunks + chunk) * (16 * NB) + row;
    if ((threadIdx.x & 15) == 0) {
      p.part_ml[at * 2] = mm;
      p.part_ml[at * 2 + 1] = ll;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) p.part_o[at * D + d0 + i] = acc[i];
  }
}

// NB 16-row blocks per wave.  16 x 512 tokens over up to 4096 keys (32 / 4 heads
// of 128): 254 us.  VALU instructions (conversion, softmax) issue for 49% of the
// SIMDs' cycles and matrix instructions for 30%, with under 2 waves a SIMD to
// overlap them; LDS is read 31% of the time, HBM is idle (0.6 TB/s).
template <int D, int NB>
__global__ __launch_bounds__(64 * kMany / 16 / NB, NB == 1 ? 4 : 2) void k_kv_attention_rows(AttnArgs p) {
  constexpr int kThreads = 64 * kMany / 16 / NB;
  constexpr int kS = D / 32, kDt = D / 16;
  // keys [64][D], chunks of 8 dims XOR-swizzled; values [D][64], likewise
  __shared__ __attribute__((aligned(16))) uint4 lds_k[2][kTile * D / 8];
  __shared__ __attribute__((aligned(16))) uint4 lds_v[2][kTile * D / 8];
  const int heads = p.c.kv_heads, h = blockIdx.x % heads, chunk = blockIdx.x / heads % p.chunks;
  const int u = blockIdx.x / heads / p.chunks;
  const Unit unit = row_unit(p, u);
  const Request rq = request(p, unit.b);
  const int tiles = cdiv(rq.rows, kMany);
  if (rq.rows <= p.few || unit.tile < 0 || unit.tile >= tiles) return;
  const int r0 = (tiles - 1 - unit.tile) * kMany;  // the longest rows first
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, g = lane >> 4, m = lane & 15;
  const int t0 = chunk * p.chunk;
  const int t1 = min(t0 + p.chunk, key_limit(p, rq, min(r0 + kMany - 1, rq.rows - 1) / p.group));
  if (t0 >= t1 && chunk > 0) return;
  const int bt = p.c.block_tokens, shift = __builtin_ctz(bt);

  // this lane's rows, one per 16-row block of the wave
  const int wr0 = r0 + wv * 16 * NB;
  int limit[NB];
  float c[NB];
  uint4 qf[NB][kS];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int row = min(wr0 + n * 16 + m, rq.rows - 1), tok = row / p.group;
    limit[n] = key_limit(p, rq, tok);
    c[n] = load_query(p, p.q + static_cast<int64_t>(rq.first + tok) * p.ldq + (h * p.group + row % p.group) * D,
                      [&](int i) { return 32 * i + 8 * g; }, qf[n]);
  }
  const bool idle = wr0 >= rq.rows;  // this wave only stages
  // keys below this are seen by every row of the wave
  const int all_see = key_limit(p, rq, min(wr0, rq.rows - 1) / p.group);

  // Staging: a wave copies pieces of 64 x 16 bytes, of keys (kTok tokens of one
  // 16-token group: one block, found through the scalar cache) or of values (16
  // dims; lane group g copies tokens 16 g .., the ones it needs the scales of).
  const int32_t* table = p.b.block_table + static_cast<int64_t>(unit.b) * p.b.W;
  const int last = p.b.W - 1;
  constexpr int kTok = 1024 / D, kWaves = kThreads / 64;
  constexpr int kPieces = D / 16 / kWaves;  // of keys, and of values, per wave
  static_assert(kPieces >= 1 && kPieces * kWaves * 16 == D, "pieces must split evenly over the waves");
  const int wave = __builtin_amdgcn_readfirstlane(wv);
  auto k_tok = [&](int i) { return (wave + i * kWaves) * kTok; };  // first token of a piece
  const int64_t stride = static_cast<int64_t>(p.c.kv_heads) * bt * D;  // of blocks
  const int8_t* const k_head = p.c.k + static_cast<int64_t>(h) * bt * D;
  const int8_t* const v_head = p.c.v + static_cast<int64_t>(h) * bt * D;
  int v_off[kPieces], k_off[kPieces];  // within a block, but for the tile's place in it
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    k_off[i] = ((k_tok(i) + lane / (D / 16)) & (bt - 1)) * D + lane % (D / 16) * 16;
    v_off[i] = (16 * (wv + i * kWaves) + m) * bt + (16 * g & (bt - 1));
  }
  // Block numbers of a tile; tokens past the table are past every limit.
  struct Ids {
    int key[kPieces], own;
  };
  auto load_ids = [&](int t) {
    Ids x;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) x.key[i] = uniform_load(table + min((t + k_tok(i)) >> shift, last));
    x.own = table[min((t + 16 * g) >> shift, last)];
    return x;
  };
  auto valid = [&](int id) { return static_cast<uint32_t>(id) < static_cast<uint32_t>(p.c.n_blocks); };
  uint4 kreg[kPieces] = {}, vreg[kPieces] = {};
  float ks = 0.0f, vs = 0.0f;
  bool seen = false;
  auto load_tile = [&](int t, const Ids& x) {
    const int at = t & (bt - 1);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      kreg[i] = *reinterpret_cast<const uint4*>(k_head + (valid(x.key[i]) ? x.key[i] : 0) * stride + at * D + k_off[i]);
    seen = valid(x.own);
    const int own = seen ? x.own : 0;
    const int8_t* vp = v_head + own * stride + at;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) vreg[i] = *reinterpret_cast<const uint4*>(vp + v_off[i]);
    ks = p.c.k_scale[static_cast<int64_t>(own) * p.c.kv_heads + h];
    vs = p.c.v_scale[static_cast<int64_t>(own) * p.c.kv_heads + h];
  };
  // LDS positions (of 16 bytes).  Reads take 16 lanes at a time, 4 consecutive
  // ones from each of 4 places of two lane groups; the swizzles keep them, and
  // the writes, in distinct banks.
  auto k_at = [&](int tok, int c8) { return tok * (D / 8) + (c8 ^ ((((tok >> 4) << 2) | (tok & 3)) & (D / 8 - 1))); };
  auto v_at = [&](int dim, int c8) { return dim * 8 + (((c8 >> 1) | (c8 & 1) << 2) ^ ((dim >> 1) & 7)); };
  auto store_tile = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int tok = k_tok(i) + lane / (D / 16), c8 = lane % (D / 16) * 2, dim = 16 * (wv + i * kWaves) + m;
      lds_k[buf][k_at(tok, c8)] = f16_of(kreg[i].x, kreg[i].y);
      lds_k[buf][k_at(tok, c8 + 1)] = f16_of(kreg[i].z, kreg[i].w);
      lds_v[buf][v_at(dim, 2 * g)] = f16_of(vreg[i].x, vreg[i].y);
      lds_v[buf][v_at(dim, 2 * g + 1)] = f16_of(vreg[i].z, vreg[i].w);
    }
  };
  int k_read[kS], v_read[2];  // this lane's positions in fragment 0
#pragma unroll
  for (int i = 0; i < kS; ++i) k_read[i] = (16 * (m >> 2) + (m & 3)) * (D / 8) + ((4 * i + g) ^ (m & (D / 8 - 1)));
#pragma unroll
  for (int i = 0; i < 2; ++i) v_read[i] = v_at(m, 2 * g + i);

  Softmax sm[NB];
  f32x4 o[NB][kDt];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int d = 0; d < kDt; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};

  Ids ids = load_ids(t0);
  if (t0 < t1) load_tile(t0, ids);
  ids = load_ids(t0 + kTile);
  store_tile(0);
  Scales sc;
  sc.set(ks, vs);
  bool seen_now = seen;
  auto step = [&](int t, int buf) {
    __syncthreads();
    const bool more = t + kTile < t1;
    if (more) {
      load_tile(t + kTile, ids);
      ids = load_ids(t + 2 * kTile);
    }
    if (!idle) {
      f32x4 s[NB][4];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 kf = lds_k[buf][k_read[i] + 4 * j * (D / 8)];
#pragma unroll
          for (int n = 0; n < NB; ++n) s[n][j] = mfma_f16(kf, qf[n][i], s[n][j]);
        }
      uint4 pf[NB][2];
      bool changed = false;
      const bool mask = t + kTile > all_see || __any(!seen_now);
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        if (mask) sm[n].template weigh<true>(s[n], c[n], sc, t + 16 * g, seen_now ? limit[n] : 0);
        else sm[n].template weigh<false>(s[n], c[n], sc, 0, 0);
        pack_weights(s[n], pf[n]);
        changed |= sm[n].shrink != 1.0f;
      }
      if (__any(changed)) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int d = 0; d < kDt; ++d) o[n][d] *= sm[n].shrink;
      }
#pragma unroll
      for (int d = 0; d < kDt; ++d)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 vf = lds_v[buf][v_read[i] + 16 * 8 * d];
#pragma unroll
          for (int n = 0; n < NB; ++n) o[n][d] = mfma_f16(vf, pf[n][i], o[n][d]);
        }
    }
    if (more) {
      store_tile(buf ^ 1);
      sc.set(ks, vs);
      seen_now = seen;
    }
  };
  for (int t = t0; t < t1; t += 2 * kTile) {  // two steps: LDS positions are constants
    step(t, 0);
    if (t + kTile < t1) step(t + kTile, 1);
  }

#pragma unroll
  for (int n = 0; n < NB; ++n) {
    float l = sm[n].l;
    l += shfl_xor(l, 16);
    l += shfl_xor(l, 32);
    const int r = wr0 + n * 16 + m;
    if (r >= rq.rows) continue;
    if (p.chunks == 1) {
      const float inv = normaliser(l);
      bf16_t* dst = out_row(p, rq, h, r, D) + 4 * g;
#pragma unroll
      for (int d = 0; d < kDt; ++d)
        *reinterpret_cast<uint2*>(dst + 16 * d) = make_uint2(pack_bf16x2(o[n][d][0] * inv, o[n][d][1] * inv),
                                                             pack_bf16x2(o[n][d][2] * inv, o[n][d][3] * inv));
      continue;
    }
    const int64_t at =
        ((static_cast<int64_t>(u) * heads + h) * p.chunks + chunk) * kMany + (r - r0);
    if (g == 0) {
      p.part_ml[at * 2] = sm[n].m;
      p.part_ml[at * 2 + 1] = l;
    }
#pragma unroll
    for (int d = 0; d < kDt; ++d) *reinterpret_cast<f32x4*>(p.part_o + at * D + 16 * d + 4 * g) = o[n][d];
  }
}

// The chunks of a row of few joined.  Their number may be large and the rows
// few: one workgroup per row, of whose 16 groups of 16 threads each takes every
// 16th chunk, in order; the groups' sums meet in LDS.  kRows rows per chunk.
template <int D, int kRows>
__global__ __launch_bounds__(256) void k_kv_combine(AttnArgs p) {
  constexpr int kPer = D / 16;
  __shared__ float lds_o[16][D], lds_l[16];
  const int b = blockIdx.x, h = blockIdx.y, r = blockIdx.z;
  const Request rq = request(p, b);
  if (rq.rows > p.few || r >= rq.rows) return;
  const int n = max(1, min(p.chunks, cdiv(key_limit(p, rq, rq.n - 1), p.chunk)));
  const int64_t at = (static_cast<int64_t>(b) * p.c.kv_heads + h) * p.chunks * kRows + r;
  const float* ml = p.part_ml + at * 2;
  const int grp = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * kPer;
  const float* po = p.part_o + at * D + d0;
  float mm = -INFINITY;
  for (int c = threadIdx.x & 15; c < n; c += 16) mm = fmaxf(mm, ml[c * kRows * 2]);
#pragma unroll
  for (int x = 8; x >= 1; x >>= 1) mm = fmaxf(mm, shfl_xor(mm, x));
  const float base = mm == -INFINITY ? 0.0f : mm;
  float ll = 0.0f, acc[kPer] = {};
#pragma unroll 2
  for (int c = grp; c < n; c += 16) {
    const float f = __builtin_amdgcn_exp2f(ml[c * kRows * 2] - base);
    ll += f * ml[c * kRows * 2 + 1];
#pragma unroll
    for (int x = 0; x < kPer; ++x) acc[x] += f * po[static_cast<int64_t>(c) * kRows * D + x];
  }
#pragma unroll
  for (int x = 0; x < kPer; ++x) lds_o[grp][d0 + x] = acc[x];
  if (d0 == 0) lds_l[grp] = ll;
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  float l = 0.0f, a0 = 0.0f, a1 = 0.0f;
  for (int x = 0; x < min(n, 16); ++x) {
    l += lds_l[x];
    a0 += lds_o[x][2 * threadIdx.x];
    a1 += lds_o[x][2 * threadIdx.x + 1];
  }
  const float inv = normaliser(l);
  *reinterpret_cast<uint32_t*>(out_row(p, rq, h, r, D) + 2 * threadIdx.x) = pack_bf16x2(a0 * inv, a1 * inv);
}

// The chunks of a row of many joined, in order: 16 threads per row, 16 rows per workgroup.
template <int D>
__global__ __launch_bounds__(256) void k_kv_combine_rows(AttnArgs p) {
  constexpr int kPer = D / 16;
  const int h = blockIdx.y;
  const Unit unit = row_unit(p, blockIdx.x);
  const Request rq = request(p, unit.b);
  const int tiles = cdiv(rq.rows, kMany);
  if (rq.rows <= p.few || unit.tile < 0 || unit.tile >= tiles) return;
  const int r0 = (tiles - 1 - unit.tile) * kMany;
  const int i = blockIdx.z * 16 + (threadIdx.x >> 4), d0 = (threadIdx.x & 15) * kPer;
  const int r = r0 + i;
  if (r >= rq.rows) return;
  const int limit = key_limit(p, rq, min(r0 + kMany - 1, rq.rows - 1) / p.group);
  const int n = max(1, min(p.chunks, cdiv(limit, p.chunk)));
  const int64_t at = (static_cast<int64_t>(blockIdx.x) * p.c.kv_heads + h) * p.chunks * kMany + i;
  const float* ml = p.part_ml + at * 2;
  float mm = -INFINITY;
  for (int c = 0; c < n; ++c) mm = fmaxf(mm, ml[c * kMany * 2]);
  const float base = mm == -INFINITY ? 0.0f : mm;
  float ll = 0.0f, acc[kPer] = {};
  const float* po = p.part_o + at * D + d0;
#pragma unroll 4
  for (int c = 0; c < n; ++c) {
    const float f = __builtin_amdgcn_exp2f(ml[c * kMany * 2] - base);
    ll += f * ml[c * kMany * 2 + 1];
#pragma unroll
    for (int x = 0; x < kPer; ++x) acc[x] += f * po[static_cast<int64_t>(c) * kMany * D + x];
  }
  const float inv = normaliser(ll);
  bf16_t* dst = out_row(p, rq, h, r, D) + d0;
#pragma unroll
  for (int x = 0; x < kPer; x += 2) *reinterpret_cast<uint32_t*>(dst + x) = pack_bf16x2(acc[x] * inv, acc[x + 1] * inv);
}

// How the keys are split over workgroups: about `want` workgroups in all,
// at least `least` keys each.  More than one chunk only while the row tiles
// are fewer than `want`, so there are at most 2 `want` partial results.
struct Split {
  int64_t tiles;  // row tiles, times kv heads
  int chunk, chunks;
  int64_t items() const { return chunks > 1 ? tiles * chunks : 0; }
};

Split split(int64_t tiles, int64_t max_kv, int want, int least) {
  Split s;
  s.tiles = tiles;
  const int64_t per = max_kv * tiles / want;
  s.chunk = static_cast<int>(cdiv64(per < least ? least : per, least) * least);
  s.chunks = static_cast<int>(cdiv64(max_kv, s.chunk));
  return s;
}

constexpr int kFewItems = 3072, kFewLeast = 512;
constexpr int kManyItems = 512, kManyLeast = 512;

struct Plan {
  int64_t most;  // rows of a kv head that one request may have
  bool many;     // more than `few_rows`
  int units;     // row tiles of those
  int few_rows;
  Split few, rows;
};

Plan plan(const moe_kv_cache& c, const moe_kv_batch& b, const moe_kv_attn& a) {
  const int64_t places = static_cast<int64_t>(b.W) * c.block_tokens;
  const int64_t max_kv = a.max_kv < places ? a.max_kv : places;
  const int64_t group = a.heads / c.kv_heads;
  Plan p;
  p.most = (a.max_q < b.T ? a.max_q : b.T) * group;
  p.few_rows = p.most <= 16 ? 16 : 32;
  p.many = p.most > p.few_rows;
  p.units = static_cast<int>(b.T * group / kMany) + b.B;
  p.few = split(static_cast<int64_t>(b.B) * c.kv_heads, max_kv, kFewItems, kFewLeast);
  p.rows = split(static_cast<int64_t>(p.units) * c.kv_heads, max_kv, kManyItems, kManyLeast);
  return p;
}

template <int D, int NB>
void launch_few(AttnArgs p, const Plan& pl, float* ws, hipStream_t s) {
  constexpr int kRows = 16 * NB;
  const Split& sp = pl.few;
  p.chunk = sp.chunk;
  p.chunks = sp.chunks;
  p.part_o = ws;
  p.part_ml = ws + sp.items() * kRows * D;
  {
    TraceScope trace_scope(K_KV_ATTENTION, s);
    hipLaunchKernelGGL((k_kv_attention<D, NB>), dim3(p.b.B * p.chunks, p.c.kv_heads), dim3(256), 0, s, p);
  }
  if (p.chunks > 1) {
    TraceScope trace_scope(K_KV_COMBINE, s);
    const int rows = pl.most < kRows ? static_cast<int>(pl.most) : kRows;
    hipLaunchKernelGGL((k_kv_combine<D, kRows>), dim3(p.b.B, p.c.kv_heads, rows), dim3(256), 0, s, p);
  }
}

template <int D>
void launch(AttnArgs p, const Plan& pl, float* ws, hipStream_t s) {
  const int heads = p.c.kv_heads;
  p.few = pl.few_rows;
  if (pl.many) {
    AttnArgs q = p;
    q.chunk = pl.rows.chunk;
    q.chunks = pl.rows.chunks;
    q.part_o = ws;
    q.part_ml = ws + pl.rows.items() * kMany * D;
    ws = q.part_ml + pl.rows.items() * kMany * 2;
    {
      TraceScope trace_scope(K_KV_ATTENTION, s);
      hipLaunchKernelGGL((k_kv_attention_rows<D, kBlocks>), dim3(pl.units * q.chunks * heads),
                         dim3(64 * kMany / 16 / kBlocks), 0, s, q);
    }
    if (q.chunks > 1) {
      TraceScope trace_scope(K_KV_COMBINE, s);
      hipLaunchKernelGGL(k_kv_combine_rows<D>, dim3(pl.units, heads, kMany / 16), dim3(256), 0, s, q);
    }
  }
  if (pl.few_rows == 16) launch_few<D, 1>(p, pl, ws, s);
  else launch_few<D, 2>(p, pl, ws, s);
}

}  // namespace

// An upper bound that does not shrink with T, W or max_kv, so that one
// workspace serves every smaller batch.
size_t kv_attention_ws(const moe_kv_cache& c, const moe_kv_batch& b, const moe_kv_attn& a) {
  const Plan p = plan(c, b, a);
  auto items = [&](const Split& s, int64_t want, int64_t least) {
    const int64_t all = s.tiles * cdiv64(a.max_kv, least);
    return all < 2 * want ? all : 2 * want;
  };
  int64_t rows = items(p.few, kFewItems, kFewLeast) * 32;
  if (p.many) rows += items(p.rows, kManyItems, kManyLeast) * kMany;
  return static_cast<size_t>(rows) * (c.head_dim + 2) * sizeof(float);
}

hipError_t launch_kv_attention(const moe_kv_cache& c, const moe_kv_batch& b, const moe_kv_attn& a, const bf16_t* q,
                               int64_t ldq, bf16_t* out, int64_t ldo, void* ws, hipStream_t s) {
  const AttnArgs p{c,       b,       q,       ldq, out, ldo, a.heads, a.heads / c.kv_heads,
                   a.max_q, a.max_kv, 0, 0, 0, (a.scale < 0 ? -a.scale : a.scale) * kLog2e,
                   a.scale < 0, (a.flags & MOE_F_CAUSAL) != 0, nullptr, nullptr};
  if (c.head_dim == 64) launch<64>(p, plan(c, b, a), static_cast<float*>(ws), s);
  else launch<128>(p, plan(c, b, a), static_cast<float*>(ws), s);
  return hipGetLastError();
}

}  // namespace moe
