// The paged 8-bit cache: tables of a step from request lengths, the write of
// new keys and values, and the read back.
//
// Work is found from the packed row starts alone: a request with n rows
// starting at row s gets the units floor(s / u) + c b, ... of a grid, which
// never overlap the next request's because n rows need at most
// floor(n / u) + c of them; a unit finds its request by a search.  The calls of
// single tokens are chains of dependent loads, so a search probes 64 places at
// once (6 binary steps take 4 us, one of these 1), and block sizes, powers of
// two, are shifts.
#include "i8_round.hpp"
#include "serve.hpp"
#include "trace.hpp"

namespace moe {

namespace {

// ---------------------------------------------------------------- plan
constexpr int kPlanPer = 16;                // requests per thread and round (1 for up to 256 requests)
constexpr int kPlanMost = (1 << 30) - 1;    // longest request: sums of two fit in 32 bits

// Largest b in [0, n) with at(b) <= x (at is non-decreasing, at(0) <= x).
template <class At>
__device__ __forceinline__ int last_not_above(int n, int64_t x, At at) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at(mid) <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The same by a whole wave, 64 places at a time.
template <class At>
__device__ __forceinline__ int wave_last_not_above(int n, int x, At at) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int stride = (hi - lo + 63) >> 6, m = lo + lane * stride;
    const int below = __popcll(__ballot(m < hi && at(m) <= x));
    lo += max(below - 1, 0) * stride;
    hi = min(hi, lo + stride);
  }
  return lo;
}

__device__ __forceinline__ int log2_of(int block_tokens) { return __ffs(block_tokens) - 1; }

struct PlanArgs {
  moe_kv_plan_dims d;
  const int32_t *old_len, *new_len;
  int32_t* block_table;
  const int32_t *free_ids, *n_free;
  int32_t *row_start, *kv_len, *positions, *slots, *seq, *state;
  bool in_place;  // kv_len or state is an input too: k_kv_plan_lengths writes them
};

// Blocks the table of a request with `len` tokens holds, of W places.
__device__ __forceinline__ int blocks_of(int len, int sh, int W) {
  return min((len >> sh) + ((len & ((1 << sh) - 1)) != 0), W);
}

// Sum of two non-negative numbers, at most 2^31 - 1.
__device__ __forceinline__ int add(int a, int b) {
  return static_cast<int>(min(static_cast<uint32_t>(a) + static_cast<uint32_t>(b), 0x7fffffffu));
}

__device__ __forceinline__ int length(int x) { return min(max(x, 0), kPlanMost); }

// Blocks that a request takes from the stack, and those past its table's width.
struct Need {
  int taken, lost;
  __device__ __forceinline__ Need(int old, int fresh, int sh, int W) {
    const int held = blocks_of(old + fresh, sh, W);
    taken = held - blocks_of(old, sh, W);
    lost = blocks_of(old + fresh, sh, 0x7fffffff) - held;
  }
};

__device__ __forceinline__ void write_state(const PlanArgs& p, int n_free, int blocks, int lost) {
  p.state[0] = max(n_free - blocks, 0);
  p.state[1] = add(max(blocks - n_free, 0), lost);
}

// Every workgroup scans all requests' lengths (8 bytes each, from L2) and
// keeps them and the running sums of new tokens and of blocks taken in LDS,
// then fills its share of the outputs, four tokens a thread: one launch, no
// order between workgroups.  A chain of loads bounds it: 5 us for 16 requests,
// 12 us for 4096 requests of 64 new tokens (4 MB).
template <int kPer>
__global__ __launch_bounds__(256) void k_kv_plan(PlanArgs p) {
  constexpr int kRound = 256 * kPer;
  __shared__ int starts[kRound + 1], needs[kRound + 1], olds[kRound];
  __shared__ int tmp[2][4];
  const int B = p.d.B, T = p.d.T, W = p.d.W, sh = log2_of(p.d.block_tokens), bt = 1 << sh;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int n_free = min(max(*p.n_free, 0), p.d.free_cap);
  const int step = gridDim.x * 256, first = blockIdx.x * 256 + tid;
  auto taken = [&](int j) {  // the j-th block taken from the stack, or -1
    if (j >= n_free) return -1;
    const int id = p.free_ids[n_free - 1 - j];
    return id >= 0 && id < p.d.n_blocks ? id : -1;
  };
  int rows = 0, blocks = 0;  // of the rounds before
  int lost = 0;              // blocks past the table's width (thread's own share)
  for (int b0 = 0; b0 < B; b0 += kRound) {
    const int cnt = min(B - b0, kRound);
    int n[kPer], nb[kPer], o[kPer];
    int sum_n = 0, sum_b = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int b = min(tid * kPer + i, cnt - 1) + b0;
      o[i] = length(p.old_len[b]);
      n[i] = length(p.new_len[b]);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (tid * kPer + i >= cnt) o[i] = n[i] = 0;
      const Need need(o[i], n[i], sh, W);
      nb[i] = need.taken;
      lost = add(lost, need.lost);
      sum_n = add(sum_n, n[i]);
      sum_b = add(sum_b, nb[i]);
    }
    int in = sum_n, ib = sum_b;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int un = __shfl_up(in, off, 64), ub = __shfl_up(ib, off, 64);
      in = add(in, lane >= off ? un : 0);
      ib = add(ib, lane >= off ? ub : 0);
    }
    // of the lanes before
    int xn = __shfl_up(in, 1, 64), xb = __shfl_up(ib, 1, 64);
    if (lane == 0) xn = xb = 0;
    __syncthreads();  // the round before is done with the shared arrays
    if (lane == 63) {
      tmp[0][wv] = in;
      tmp[1][wv] = ib;
    }
    __syncthreads();
    int all_n = rows, all_b = blocks;
    xn = add(xn, rows);
    xb = add(xb, blocks);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      xn = add(xn, w < wv ? tmp[0][w] : 0);
      xb = add(xb, w < wv ? tmp[1][w] : 0);
      all_n = add(all_n, tmp[0][w]);
      all_b = add(all_b, tmp[1][w]);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      starts[tid * kPer + i] = xn;
      needs[tid * kPer + i] = xb;
      olds[tid * kPer + i] = o[i];
      xn = add(xn, n[i]);
      xb = add(xb, nb[i]);
    }
    __syncthreads();
    for (int i = first; i < cnt; i += step) {
      p.row_start[b0 + i] = starts[i];
      if (!p.in_place)
        p.kv_len[b0 + i] = olds[i] + (kPer == 1 ? n[0] : length(p.new_len[b0 + i]));  // kPer 1: i = tid
    }
    const int end = min(all_n, T);
    for (int64_t t0 = rows + static_cast<int64_t>(first) * 4; t0 < end; t0 += static_cast<int64_t>(step) * 4) {
      int i = last_not_above(cnt, t0, [&](int m) { return starts[m]; });
      int seen = -1, id = -1;  // the place whose block is at hand
      for (int t = static_cast<int>(t0); t < min(t0 + 4, static_cast<int64_t>(end)); ++t) {
        while (i + 1 < cnt && starts[i + 1] <= t) ++i, seen = -1;
        const int pos = olds[i] + t - starts[i], at = pos >> sh;
        if (at != seen) {
          const int have = blocks_of(olds[i], sh, W);
          id = -1;
          if (at < have) id = p.block_table[static_cast<int64_t>(b0 + i) * W + at];
          else if (at < W) id = taken(needs[i] + at - have);
          seen = at;
        }
        p.positions[t] = pos;
        p.slots[t] = id >= 0 && id < p.d.n_blocks ? id * bt + (pos & (bt - 1)) : -1;
        p.seq[t] = b0 + i;
      }
    }
    for (int64_t j = blocks + first; j < all_b; j += step) {
      const int i = last_not_above(cnt, j, [&](int m) { return needs[m]; });
      const int have = blocks_of(olds[i], sh, W);
      p.block_table[static_cast<int64_t>(b0 + i) * W + have + (j - needs[i])] = taken(static_cast<int>(j));
    }
    rows = all_n;
    blocks = all_b;
  }
  for (int64_t t = static_cast<int64_t>(rows) + first; t < T; t += step) p.positions[t] = p.slots[t] = p.seq[t] = -1;
  if (blockIdx.x != 0) return;
  for (int m = 32; m >= 1; m >>= 1) lost = add(lost, shfl_xor(lost, m));
  __syncthreads();
  if (lane == 0) tmp[0][wv] = lost;
  __syncthreads();
  if (tid == 0) {
    p.row_start[B] = rows;
    if (!p.in_place) write_state(p, n_free, blocks, add(add(tmp[0][0], tmp[0][1]), add(tmp[0][2], tmp[0][3])));
  }
}

// kv_len and state, where one of them lies where old_len, new_len or n_free
// does: k_kv_plan's workgroups read those in no order, so they are written
// after it, by one workgroup whose threads read a request before they write it.
constexpr int kLengthThreads = 1024;
__global__ __launch_bounds__(kLengthThreads) void k_kv_plan_lengths(PlanArgs p) {
  __shared__ int sums[2][kLengthThreads / 64];
  const int sh = log2_of(p.d.block_tokens), tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  int blocks = 0, lost = 0;
  for (int b = tid; b < p.d.B; b += kLengthThreads) {
    const int old = length(p.old_len[b]), fresh = length(p.new_len[b]);
    const Need need(old, fresh, sh, p.d.W);
    blocks = add(blocks, need.taken);
    lost = add(lost, need.lost);
    p.kv_len[b] = old + fresh;
  }
  for (int m = 32; m >= 1; m >>= 1) {
    blocks = add(blocks, shfl_xor(blocks, m));
    lost = add(lost, shfl_xor(lost, m));
  }
  if (lane == 0) {
    sums[0][wv] = blocks;
    sums[1][wv] = lost;
  }
  __syncthreads();
  if (tid != 0) return;
  for (int w = 1; w < kLengthThreads / 64; ++w) {
    blocks = add(blocks, sums[0][w]);
    lost = add(lost, sums[1][w]);
  }
  write_state(p, min(max(*p.n_free, 0), p.d.free_cap), blocks, lost);
}

// ---------------------------------------------------------------- write
__device__ __forceinline__ int round8(float x) { return static_cast<int>(fminf(fmaxf(__builtin_rintf(x), -127.0f), 127.0f)); }

// One workgroup per block that the batch writes to, kv head, and keys
// (blockIdx.z = 0) or values (1).  The block's old contents are needed only
// where it keeps some (values: also for the bytes beside the new ones).  With
// the read: 12 us for 64 single tokens, where the chain row start - block -
// scale - bytes bounds it, 20 us for 16 x 512 tokens of 4 heads (33 MB, 6.5 us
// at the copy rate); the write alone 7 and 12, with kept tokens to round again 9
// and 14 by trace.  Holding a block's tokens in registers between the two
// passes was slower at both (14, 20), as was a read with all loads ahead (13, 20).
template <int D>
__global__ __launch_bounds__(256) void k_kv_append(moe_kv_cache c, moe_kv_batch bt_, const bf16_t* __restrict__ k,
                                                   const bf16_t* __restrict__ v, int64_t ld) {
  constexpr int kLanes = D / 8;           // threads per token
  constexpr int kTokens = 256 / kLanes;   // tokens per pass
  constexpr int kMaxBlock = 128;
  __shared__ __attribute__((aligned(16))) int8_t tile[D * kMaxBlock];  // values only: [D][bt]
  __shared__ uint32_t tops[4];
  const int bt = c.block_tokens, sh = log2_of(bt), tid = threadIdx.x;
  auto start = [&](int b) { return min(max(bt_.row_start[b], 0), bt_.T); };
  const int u = blockIdx.x;
  const int b = wave_last_not_above(bt_.B, u, [&](int m) { return (start(m) >> sh) + 2 * m; });
  const int s = start(b), end = bt_.row_start[b + 1], n = min(max(end, 0), bt_.T) - s;
  const int old = max(bt_.kv_len[b], 0) - max(end - bt_.T, 0) - n;  // kv_len counts the tokens past the last row too
  const int blk0 = max(old, 0) >> sh;
  const int blk = blk0 + u - ((s >> sh) + 2 * b);
  // the request's new tokens that lie in this block: [p0, p1) of its positions
  const int p0 = max(max(old, 0), blk * bt), p1 = min(old + n, (blk + 1) * bt);
  if (n <= 0 || p0 >= p1 || blk >= bt_.W) return;
  const int id = bt_.block_table[static_cast<int64_t>(b) * bt_.W + blk];
  if (id < 0 || id >= c.n_blocks) return;
  const int h = blockIdx.y;
  const bool values = blockIdx.z != 0;
  const int off = p0 - blk * bt, cnt = p1 - p0;
  const bf16_t* src = (values ? v : k) + static_cast<int64_t>(s + p0 - old) * ld + h * D;
  const int64_t at = static_cast<int64_t>(id) * c.kv_heads + h;
  int8_t* dst = (values ? c.v : c.k) + at * bt * D;
  float* scale = (values ? c.v_scale : c.k_scale) + at;
  const float s0 = off > 0 ? *scale : 0.0f;
  const int tok = tid / kLanes, d0 = tid % kLanes * 8;

  uint32_t m = 0;
  for (int t = tok; t < cnt; t += kTokens) m = max(m, top8(*reinterpret_cast<const uint4*>(src + t * ld + d0)));
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = max(m, static_cast<uint32_t>(shfl_xor(static_cast<int>(m), o)));
  if ((tid & 63) == 0) tops[tid >> 6] = m;
  if (values && cnt < bt)  // a block's first tokens leave zeros behind them
    for (int i = tid * 16; i < D * bt; i += 256 * 16)
      *reinterpret_cast<uint4*>(tile + i) = off > 0 ? *reinterpret_cast<const uint4*>(dst + i) : make_uint4(0, 0, 0, 0);
  __syncthreads();  // also: every thread has read the old scale
  m = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  const float s1 = m >= kInfBits || s0 != s0 ? __uint_as_float(0x7fc00000u) : fmaxf(s0, __uint_as_float(m) / 127.0f);
  if (tid == 0) *scale = s1;
  const bool live = s1 > 0.0f;  // neither all zeros nor NaN
  const float shrink = live ? s0 / s1 : 0.0f;
  const bool again = off > 0 && shrink != 1.0f;

  if (again && !values)
    for (int i = tid * 4; i < off * D; i += 256 * 4) {
      char4 q = *reinterpret_cast<const char4*>(dst + i);
      q = make_char4(round8(q.x * shrink), round8(q.y * shrink), round8(q.z * shrink), round8(q.w * shrink));
      *reinterpret_cast<char4*>(dst + i) = q;
    }
  if (again && values) {
    for (int i = tid; i < D * bt; i += 256)
      if ((i & (bt - 1)) < off) tile[i] = static_cast<int8_t>(round8(tile[i] * shrink));
  }
  for (int t = tok; t < cnt; t += kTokens) {  // from the caches: registers for 128 tokens cost more
    const uint4 x = *reinterpret_cast<const uint4*>(src + t * ld + d0);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    int q[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q[2 * i] = live ? round8(lo_bf(w[i]) / s1) : 0;
      q[2 * i + 1] = live ? round8(hi_bf(w[i]) / s1) : 0;
    }
    if (!values) {
      uint2 o;
      o.x = (q[0] & 255) | ((q[1] & 255) << 8) | ((q[2] & 255) << 16) | (static_cast<uint32_t>(q[3]) << 24);
      o.y = (q[4] & 255) | ((q[5] & 255) << 8) | ((q[6] & 255) << 16) | (static_cast<uint32_t>(q[7]) << 24);
      *reinterpret_cast<uint2*>(dst + (off + t) * D + d0) = o;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) tile[(d0 + i) * bt + off + t] = static_cast<int8_t>(q[i]);
    }
  }
  if (!values) return;
  __syncthreads();
  for (int i = tid * 16; i < D * bt; i += 256 * 16)
    *reinterpret_cast<uint4*>(dst + i) = *reinterpret_cast<const uint4*>(tile + i);
}

// ---------------------------------------------------------------- read
// One workgroup per 64 tokens of a request, kv head, and keys or values: 9 us
// for the 17 MB of 16 x 512 tokens and what lies before them, of which the
// chain start - block - bytes and the byte-wide transpose are most.
template <int D>
__global__ __launch_bounds__(256) void k_kv_read(moe_kv_cache c, int B, int W, const int32_t* __restrict__ block_table,
                                                 const int32_t* __restrict__ kv_start, int total,
                                                 bf16_t* __restrict__ k_out, bf16_t* __restrict__ v_out) {
  __shared__ __attribute__((aligned(16))) int8_t tile[D][64 + 16];
  const int bt = c.block_tokens, sh = log2_of(bt), tid = threadIdx.x, h = blockIdx.y;
  auto start = [&](int b) { return min(max(kv_start[b], 0), total); };
  const int u = blockIdx.x;
  const int b = wave_last_not_above(B, u, [&](int m) { return start(m) / 64 + m; });
  const int s = start(b), n = start(b + 1) - s;
  const int t0 = (u - (s / 64 + b)) * 64;
  if (t0 < 0 || t0 >= n) return;  // before the first request's rows, or none of this one
  const int32_t* table = block_table + static_cast<int64_t>(b) * W;
  auto block = [&](int t) {  // of token t, or -1
    const int i = t >> sh;
    const int id = i < W ? table[i] : -1;
    return id >= 0 && id < c.n_blocks ? id : -1;
  };
  const bool values = blockIdx.z != 0;
  const int64_t row0 = static_cast<int64_t>(s + t0) * c.kv_heads + h;
  bf16_t* out = values ? v_out : k_out;
  if (values) {  // rows of the block are head_dim, so transpose: 16 tokens of one dim per thread
    for (int i = tid; i < D * 4; i += 256) {
      const int d = i >> 2, t = (i & 3) * 16;
      const int id = block(t0 + t);
      uint4 x = make_uint4(0, 0, 0, 0);
      if (id >= 0)
        x = *reinterpret_cast<const uint4*>(c.v + (static_cast<int64_t>(id) * c.kv_heads + h) * bt * D + d * bt +
                                            ((t0 + t) & (bt - 1)));
      *reinterpret_cast<uint4*>(&tile[d][t]) = x;
    }
    __syncthreads();
  }
  for (int i = tid; i < 64 * (D / 8); i += 256) {
    const int t = i / (D / 8), d0 = i % (D / 8) * 8;
    if (t0 + t >= n) continue;
    const int id = block(t0 + t);
    uint32_t w[4] = {0, 0, 0, 0};
    if (id >= 0) {
      const int64_t at = static_cast<int64_t>(id) * c.kv_heads + h;
      const float sc = (values ? c.v_scale : c.k_scale)[at];
      int8_t q[8];
      if (values) {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = tile[d0 + j][t];
      } else {
        *reinterpret_cast<uint2*>(q) = *reinterpret_cast<const uint2*>(c.k + at * bt * D + ((t0 + t) & (bt - 1)) * D + d0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(q[2 * j] * sc, q[2 * j + 1] * sc);
    }
    *reinterpret_cast<uint4*>(out + (row0 + static_cast<int64_t>(t) * c.kv_heads) * D + d0) =
        make_uint4(w[0], w[1], w[2], w[3]);
  }
}

}  // namespace

hipError_t launch_kv_plan(const moe_kv_plan_dims& d, const int32_t* old_len, const int32_t* new_len,
                          int32_t* block_table, const int32_t* free_ids, const int32_t* n_free, int32_t* row_start,
                          int32_t* kv_len, int32_t* positions, int32_t* slots, int32_t* seq, int32_t* state,
                          hipStream_t s) {
  TraceScope trace_scope(K_KV_PLAN, s);
  const int work = d.T > d.B ? d.T : d.B;
  int grid = cdiv(work, 1024);
  grid = grid < 1 ? 1 : grid > 256 ? 256 : grid;
  const PlanArgs p{d,      old_len,   new_len, block_table, free_ids,
                   n_free, row_start, kv_len,  positions,   slots,
                   seq,    state,     kv_len == old_len || kv_len == new_len || state == n_free};
  if (d.B <= 256) hipLaunchKernelGGL(k_kv_plan<1>, dim3(grid), dim3(256), 0, s, p);
  else hipLaunchKernelGGL(k_kv_plan<kPlanPer>, dim3(grid), dim3(256), 0, s, p);
  if (p.in_place) hipLaunchKernelGGL(k_kv_plan_lengths, dim3(1), dim3(kLengthThreads), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_kv_append(const moe_kv_cache& c, const moe_kv_batch& b, const bf16_t* k, const bf16_t* v, int64_t ld,
                            hipStream_t s) {
  TraceScope trace_scope(K_KV_APPEND, s);
  const dim3 grid(b.T / c.block_tokens + 2 * b.B, c.kv_heads, 2);
  if (c.head_dim == 64) hipLaunchKernelGGL(k_kv_append<64>, grid, dim3(256), 0, s, c, b, k, v, ld);
  else hipLaunchKernelGGL(k_kv_append<128>, grid, dim3(256), 0, s, c, b, k, v, ld);
  return hipGetLastError();
}

hipError_t launch_kv_read(const moe_kv_cache& c, int B, int W, const int32_t* block_table, const int32_t* kv_start,
                          int total, bf16_t* k_out, bf16_t* v_out, hipStream_t s) {
  TraceScope trace_scope(K_KV_READ, s);
  const dim3 grid(total / 64 + B, c.kv_heads, 2);
  if (c.head_dim == 64)
    hipLaunchKernelGGL(k_kv_read<64>, grid, dim3(256), 0, s, c, B, W, block_table, kv_start, total, k_out, v_out);
  else
    hipLaunchKernelGGL(k_kv_read<128>, grid, dim3(256), 0, s, c, B, W, block_table, kv_start, total, k_out, v_out);
  return hipGetLastError();
}

}  // namespace moe
