// Attention over the paged 8-bit cache, single tokens and prompt chunks.
//
// A request's new tokens and the heads that share a kv head form one matrix of
// rows r = (token, head), so that few tokens still fill a matrix-core tile.
// The int8 keys and values become bf16 in registers, which is exact; a
// block's scale multiplies its scores (keys) and its probabilities (values),
// so the products themselves see small integers.
//
// Scores are formed transposed, S^T = K Q^T, and the output as O^T = V^T P^T:
// what one lane holds of S^T after the first product (4 tokens of one row per
// fragment) is what it must supply of P^T to the second, so probabilities
// never leave their lane.  For that, fragment j of a 64-token tile takes its 16
// tokens in the order 16 (m / 4) + 4 j + m % 4: lane group g (l / 16) then owns
// tokens 16 g .. 16 g + 15 of the tile, one 16-byte load of each value row.
//
// Softmax statistics are fp32; probabilities are rounded to bf16 for the
// second product (at most 2^-8 each, independent of each other), their sum is not.
#include "serve.hpp"
#include "trace.hpp"

namespace moe {

namespace {

constexpr int kTile = 64;  // tokens per step
constexpr float kLog2e = 1.4426950408889634f;

struct AttnArgs {
  moe_kv_cache c;
  moe_kv_batch b;
  const bf16_t* q;
  int64_t ldq;
  bf16_t* out;
  int64_t ldo;
  int heads, group;   // query heads, and per kv head
  int max_q, max_kv;
  int row_tiles;      // 16-row tiles per request and kv head
  int chunk, chunks;  // tokens per workgroup, chunks per row tile
  float scale2;       // scale log2(e)
  bool causal;
  float* part_o;      // [items][16][D]
  float* part_ml;     // [items][16][2]
};

// 8 int8 -> 8 bf16 (exact).
__device__ __forceinline__ uint4 bf16_of(uint32_t lo, uint32_t hi) {
  auto f = [](uint32_t w, int i) { return static_cast<float>(static_cast<int8_t>(w >> (8 * i))); };
  return make_uint4(pack_bf16x2(f(lo, 0), f(lo, 1)), pack_bf16x2(f(lo, 2), f(lo, 3)), pack_bf16x2(f(hi, 0), f(hi, 1)),
                    pack_bf16x2(f(hi, 2), f(hi, 3)));
}

// Rows of one request and the keys they see.
struct Request {
  int first, n, rows;  // packed row, new tokens, rows of this kv head
  int kv, pos0;        // tokens in the cache, position of the first new token
};

__device__ __forceinline__ Request request(const AttnArgs& p, int b) {
  auto start = [&](int i) { return min(max(p.b.row_start[i], 0), p.b.T); };
  Request r;
  r.first = start(b);
  const int all = max(start(b + 1) - r.first, 0), len = p.b.kv_len[b];
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

// One workgroup: 16 rows against one chunk of keys; its four waves take the
// chunk's 64-token steps in turn and merge at the end.
template <int D>
__global__ __launch_bounds__(256) void k_kv_attention(AttnArgs p) {
  constexpr int kP = D / 64, kDt = D / 16;
  __shared__ float lds_o[4][16][D];
  __shared__ float lds_m[4][16], lds_l[4][16];
  const int chunk = blockIdx.x % p.chunks, rt = blockIdx.x / p.chunks % p.row_tiles;
  const int b = blockIdx.x / p.chunks / p.row_tiles, h = blockIdx.y;
  const Request rq = request(p, b);
  const int r0 = rt * 16;
  if (r0 >= rq.rows) return;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, g = lane >> 4;
  const int t0 = chunk * p.chunk;
  const int t1 = min(t0 + p.chunk, key_limit(p, rq, min(r0 + 15, rq.rows - 1) / p.group));
  if (t0 >= t1 && chunk > 0) return;
  const int bt = p.c.block_tokens, shift = __builtin_ctz(bt);

  // this lane's row
  const int row = min(r0 + (lane & 15), rq.rows - 1);
  const int tok = row / p.group, head = h * p.group + row % p.group;
  const int limit = key_limit(p, rq, tok);
  uint4 qf[kP][2];
  const bf16_t* qrow = p.q + (rq.first + tok) * p.ldq + head * D;
#pragma unroll
  for (int i = 0; i < kP; ++i)
#pragma unroll
    for (int s = 0; s < 2; ++s) qf[i][s] = *reinterpret_cast<const uint4*>(qrow + 64 * i + 16 * g + 8 * s);

  float m = -INFINITY, l = 0.0f;
  f32x4 o[kDt];
#pragma unroll
  for (int d = 0; d < kDt; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int32_t* table = p.b.block_table + static_cast<int64_t>(b) * p.b.W;
  const int last = p.b.W - 1;
  const int gk = (lane & 15) >> 2;  // the 16-token group this lane loads keys of
  for (int t = t0 + wv * kTile; t < t1; t += 4 * kTile) {
    // blocks of the key group and of the value group; past the table: none
    const int ik = (t + 16 * gk) >> shift, iv = (t + 16 * g) >> shift;
    const int bk = table[min(ik, last)], bv = table[min(iv, last)];
    const bool seen = iv <= last && bv >= 0 && bv < p.c.n_blocks;
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
    const float ks = p.c.k_scale[pv] * p.scale2, vs = p.c.v_scale[pv];

    float sc[4][4];
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kP; ++i) {
        acc = mfma16x16x32(bf16_of(kf[j][i].x, kf[j][i].y), qf[i][0], acc);
        acc = mfma16x16x32(bf16_of(kf[j][i].z, kf[j][i].w), qf[i][1], acc);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[j][i] = seen && t + 16 * g + 4 * j + i < limit ? acc[i] * ks : -INFINITY;
        top = fmaxf(top, sc[j][i]);
      }
    }
    top = fmaxf(top, shfl_xor(top, 16));
    top = fmaxf(top, shfl_xor(top, 32));
    const float m1 = fmaxf(m, top);
    const float base = m1 == -INFINITY ? 0.0f : m1;  // no key seen yet: every term is 0
    const float shrink = exp2f(m - base);
    m = m1;
    l *= shrink;
#pragma unroll
    for (int d = 0; d < kDt; ++d) o[d] *= shrink;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = exp2f(sc[j][i] - base);
        l += e;
        sc[j][i] = e == 0.0f ? 0.0f : e * vs;  // a masked place stays 0 whatever its scale
      }
    uint4 pf[2];
#pragma unroll
    for (int s = 0; s < 2; ++s)
      pf[s] = make_uint4(pack_bf16x2(sc[2 * s][0], sc[2 * s][1]), pack_bf16x2(sc[2 * s][2], sc[2 * s][3]),
                         pack_bf16x2(sc[2 * s + 1][0], sc[2 * s + 1][1]), pack_bf16x2(sc[2 * s + 1][2], sc[2 * s + 1][3]));
#pragma unroll
    for (int d = 0; d < kDt; ++d) {
      o[d] = mfma16x16x32(bf16_of(vf[d].x, vf[d].y), pf[0], o[d]);
      o[d] = mfma16x16x32(bf16_of(vf[d].z, vf[d].w), pf[1], o[d]);
    }
  }
  l += shfl_xor(l, 16);
  l += shfl_xor(l, 32);

  // merge the waves: o[d][i] is dimension 16 d + 4 g + i of row lane % 16
  if (lane < 16) {
    lds_m[wv][lane] = m;
    lds_l[wv][lane] = l;
  }
#pragma unroll
  for (int d = 0; d < kDt; ++d) *reinterpret_cast<f32x4*>(&lds_o[wv][lane & 15][16 * d + 4 * g]) = o[d];
  __syncthreads();
  constexpr int kPer = D / 16;  // dimensions per thread
  const int r = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * kPer;
  if (r0 + r >= rq.rows) return;
  float mm = -INFINITY, ll = 0.0f, acc[kPer] = {};
#pragma unroll
  for (int w = 0; w < 4; ++w) mm = fmaxf(mm, lds_m[w][r]);
  const float base = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = exp2f(lds_m[w][r] - base);
    ll += f * lds_l[w][r];
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] += f * lds_o[w][r][d0 + i];
  }
  if (p.chunks == 1) {
    const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
    bf16_t* dst = p.out + (rq.first + (r0 + r) / p.group) * p.ldo + (h * p.group + (r0 + r) % p.group) * D + d0;
#pragma unroll
    for (int i = 0; i < kPer; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = pack_bf16x2(acc[i] * inv, acc[i + 1] * inv);
    return;
  }
  const int64_t item = (static_cast<int64_t>(b) * p.c.kv_heads + h) * p.row_tiles * p.chunks + rt * p.chunks + chunk;
  if ((threadIdx.x & 15) == 0) {
    p.part_ml[(item * 16 + r) * 2] = mm;
    p.part_ml[(item * 16 + r) * 2 + 1] = ll;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) p.part_o[(item * 16 + r) * D + d0 + i] = acc[i];
}

// One workgroup per 16 rows: the chunks joined in order.
template <int D>
__global__ __launch_bounds__(256) void k_kv_combine(AttnArgs p) {
  constexpr int kPer = D / 16;
  const int rt = blockIdx.x % p.row_tiles, b = blockIdx.x / p.row_tiles, h = blockIdx.y;
  const Request rq = request(p, b);
  const int r0 = rt * 16, r = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * kPer;
  if (r0 + r >= rq.rows) return;
  const int limit = key_limit(p, rq, min(r0 + 15, rq.rows - 1) / p.group);
  const int n = max(1, min(p.chunks, cdiv(limit, p.chunk)));
  const int64_t item = ((static_cast<int64_t>(b) * p.c.kv_heads + h) * p.row_tiles + rt) * p.chunks;
  float mm = -INFINITY;
  for (int c = 0; c < n; ++c) mm = fmaxf(mm, p.part_ml[((item + c) * 16 + r) * 2]);
  const float base = mm == -INFINITY ? 0.0f : mm;
  float ll = 0.0f, acc[kPer] = {};
  for (int c = 0; c < n; ++c) {
    const int64_t at = (item + c) * 16 + r;
    const float f = exp2f(p.part_ml[at * 2] - base);
    ll += f * p.part_ml[at * 2 + 1];
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] += f * p.part_o[at * D + d0 + i];
  }
  const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
  bf16_t* dst = p.out + (rq.first + (r0 + r) / p.group) * p.ldo + (h * p.group + (r0 + r) % p.group) * D + d0;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) *reinterpret_cast<uint32_t*>(dst + i) = pack_bf16x2(acc[i] * inv, acc[i + 1] * inv);
}

struct Split {
  int row_tiles, chunk, chunks;
};

// Keys per workgroup: about kItems workgroups in all (12 per CU: enough for
// lengths to even out), at least 256 keys each.  Where a row tile has more
// than one chunk there are fewer than kItems row tiles, so at most 2 kItems
// partial results.
constexpr int kItems = 3072;

Split split(const moe_kv_cache& c, const moe_kv_batch& b, const moe_kv_attn& a) {
  Split s;
  const int64_t places = static_cast<int64_t>(b.W) * c.block_tokens;
  const int64_t max_kv = a.max_kv < places ? a.max_kv : places;
  s.row_tiles = cdiv((a.max_q < b.T ? a.max_q : b.T) * (a.heads / c.kv_heads), 16);
  const int64_t tiles = static_cast<int64_t>(s.row_tiles) * b.B * c.kv_heads;
  const int64_t per = max_kv * tiles / kItems;
  s.chunk = static_cast<int>(cdiv64(per < 256 ? 256 : per, 256) * 256);
  s.chunks = static_cast<int>(cdiv64(max_kv < 1 ? 1 : max_kv, s.chunk));
  return s;
}

}  // namespace

size_t kv_attention_ws(const moe_kv_cache& c) {
  return static_cast<size_t>(2 * kItems) * 16 * (c.head_dim + 2) * sizeof(float);
}

hipError_t launch_kv_attention(const moe_kv_cache& c, const moe_kv_batch& b, const moe_kv_attn& a, const bf16_t* q,
                               int64_t ldq, bf16_t* out, int64_t ldo, void* ws, hipStream_t s) {
  const Split sp = split(c, b, a);
  const int64_t items = static_cast<int64_t>(sp.row_tiles) * sp.chunks * b.B * c.kv_heads;
  AttnArgs p{c, b, q, ldq, out, ldo, a.heads, a.heads / c.kv_heads, a.max_q, a.max_kv, sp.row_tiles, sp.chunk, sp.chunks,
             a.scale * kLog2e, (a.flags & MOE_F_CAUSAL) != 0, static_cast<float*>(ws), nullptr};
  p.part_ml = p.part_o + items * 16 * c.head_dim;
  {
    TraceScope trace_scope(K_KV_ATTENTION, s);
    const dim3 grid(sp.row_tiles * sp.chunks * b.B, c.kv_heads);
    if (c.head_dim == 64) hipLaunchKernelGGL(k_kv_attention<64>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(k_kv_attention<128>, grid, dim3(256), 0, s, p);
  }
  if (sp.chunks > 1) {
    TraceScope trace_scope(K_KV_COMBINE, s);
    const dim3 grid(sp.row_tiles * b.B, c.kv_heads);
    if (c.head_dim == 64) hipLaunchKernelGGL(k_kv_combine<64>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(k_kv_combine<128>, grid, dim3(256), 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace moe
