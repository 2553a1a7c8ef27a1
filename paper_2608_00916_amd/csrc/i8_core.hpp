// Core of the int8 products on the gfx950 matrix cores: tiles of
// C[m][n] = sum_k A[m][k] B[n][k], exact in int32, streamed by persistent
// workgroups.
//
// Both operands are K-contiguous, so a step is 128 bytes of each of a tile's
// BM + BN rows.  They go straight from global memory into LDS (16 bytes per
// lane, no registers); v_mfma_i32_16x16x64_i8 takes 16 consecutive k per lane,
// one ds_read_b128.  A row's eight 16-byte chunks are XOR-swizzled so that the
// 16 rows of one fragment read lie in distinct banks; the copy into LDS is
// linear in the lanes, so the swizzle is applied to the global address.
//
// The B fragment is fed first, so a lane holds four consecutive fragment rows
// of B.  Fragment n of a wave takes rows col(n) + 8 (i / 4) + i % 4 (i < 16):
// lane l then holds C[m = l % 16][col(n) + 8 (l / 16) + i], two runs of 8
// columns over its FN = 4 fragments; of either run the four lanes of a row
// store 64 consecutive bytes of bf16.
//
// Two LDS stages: the copies of step k + 1 run under the products of step k,
// and those of the next tile's first step under this tile's last one.  Loads
// and stores share one in-order counter: the copies of the next tile's first
// step are waited for before this tile's stores, which then have that step to
// drain.  A taller tile brings fewer bytes from L2 per product, hence the 256 x
// 256 tile over 8 waves (128 x 64 each): 4096 x 16384 x 8192 at 2570 TOPS, 128
// x 128 tiles over 4 waves at 2080; at K 2048 2200 and 1840, where the stores of
// all workgroups meet at the memory every 16 steps.  At 8192 x 5120 x 2048 the
// matrix cores are busy 43% of the time, and waves wait 40% of theirs, for
// copies and at the barrier; LDS (16%) and VALU (22%) have room.  Measured and
// not taken: four stages of 64 bytes of k (13% slower, twice the barriers), a
// barrier within the step with the next fragments read under its last products
// (the same), lines brought into L2 ahead of the copies (20% slower),
// workgroups out of phase (the same), stores past the caches (the same).
//
// The copies are buffer loads whose resource ends with the operand's last row
// in the tile: rows past it read zeros, and so do chunks past K, so no load
// leaves its operand.
#pragma once

#include "common.hpp"
#include "moe.h"

namespace moe {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kI8Step = 128;  // k per step

__device__ __forceinline__ i32x4 mfma_i8(const uint4& p, const uint4& q, i32x4 acc) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, p), __builtin_bit_cast(i32x4, q), acc, 0, 0,
                                               0);
}

// The one sum that leaves int32: MOE_I8_MAX_K products of -128 and -128 are 2^31,
// which arrives as -2^31, a sum that no operands have.  2^31 - 1 is the same
// number in fp32.
__device__ __forceinline__ int unwrap(int sum) { return sum == INT32_MIN ? INT32_MAX : sum; }

// 16 bytes per lane from a buffer resource to LDS at base + 16 lane; offsets at
// or past the resource's size read zeros (the check covers the per-lane offset
// only, so all of the offset is in it).  The instructions are written out
// because the compiler, which cannot tell the stages apart, makes every LDS
// read wait for the copies that it knows of: the products then overlap with no
// copy.  Their waits are wait_vm's below.  The nop covers the distance from a
// VALU write of the resource's or base's registers, and from that of m0.
__device__ __forceinline__ void copy_to_lds(i32x4 r, uint32_t off, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds_base), "v"(off), "s"(r)
               : "memory");
}

__device__ __forceinline__ void copy_to_lds(const int8_t* p, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(lds_base), "v"(p)
               : "memory");
}

__device__ __forceinline__ uint32_t lds_address(int8_t* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) int8_t*)(p)));
}

constexpr uint32_t kI8Oob = 0x80000000u;  // an offset past every resource

// Rows of one operand's tile: contiguous (row r at base + r K, `rows` of them),
// or, for a gathered A, row r at base + index[r] K.
struct I8Source {
  const int8_t* base;
  int rows;
  const int32_t* index = nullptr;
};

// All but the last N of this wave's vector loads (copies into LDS are counted
// as such) and stores are done.
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N < 64, "the counter has 6 bits");
  asm volatile("" ::: "memory");
  // the builtin, so that the compiler too takes its own loads as done
  __builtin_amdgcn_s_waitcnt((N & 15) | N >> 4 << 14 | 7 << 4 | 15 << 8);
  asm volatile("" ::: "memory");
}

// All waves are here; LDS reads before it have returned (their products were
// issued).  Unlike __syncthreads it leaves vector memory in flight.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// BM x BN tile over WM x WN waves.
template <int BM_, int BN_, int WM_, int WN_>
struct I8Tile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int kWaves = WM * WN;
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  static constexpr int col(int n) { return (n >> 1) * 32 + (n & 1) * 4; }  // of a lane's four columns of fragment n
  static constexpr int kStage = (BM + BN) * kI8Step;
  static constexpr int kCopies = (BM + BN) / 8 / kWaves;  // of 8 rows, per wave and step
  static constexpr int kCopiesA = BM / 8 / kWaves;
  static_assert(BM % (8 * kWaves) == 0 && BN % (8 * kWaves) == 0, "rows must split evenly over the waves");
  static_assert(FN == 4, "a lane holds two runs of 8 columns");
};

// Chunk position of chunk c of row r of either operand.  LDS has 64 banks (256
// bytes, two rows): the XOR separates the row pairs of one fragment.
__device__ __forceinline__ int a_swizzle(int r, int c) { return c ^ ((r >> 1) & 7); }
__device__ __forceinline__ int b_swizzle(int r, int c) {  // fragment rows: 4 together, 8 apart
  return c ^ (((r >> 1) & 1) | (((r >> 3) & 3) << 1));
}

// Work items of a persistent grid over n tiles.  Where the last, incomplete
// round would fill at most half of the workgroups, its tiles are cut into two
// halves of BM / 2 rows, on which half of the waves work.  Odd workgroups take
// their half tile first: their epilogues, whose stores would otherwise all meet
// at the memory, then fall between those of the even ones.
struct Items {
  int tiles, full;  // tiles, and those left whole (a multiple of the grid unless all are)
  __device__ __forceinline__ Items(bool cut, int n) : tiles(n) {
    const int rem = n % static_cast<int>(gridDim.x);
    full = cut && 2 * rem <= static_cast<int>(gridDim.x) ? n - rem : n;
  }
  __device__ __forceinline__ int count() const { return 2 * tiles - full; }
  // tile of item i, and its half (-1: whole)
  __device__ __forceinline__ void at(int i, int* tile, int* half) const {
    const int w = blockIdx.x, grid = gridDim.x;
    if ((w & 1) && w < count() - full) i = i == w ? full + w : i - grid;
    *half = i < full ? -1 : (i - full) & 1;
    *tile = i < full ? i : full + (i - full) / 2;
  }
};

// Streams work items blockIdx.x, + gridDim.x, ... of `items`.  Job:
//   Tile tile(int i)              an item's tile (uniform), with .rows valid rows of A (<= 0: nothing to do)
//   I8Source a(const Tile&)       the tile's rows of A
//   I8Source b(const Tile&, int)  of B, part 0 .. kParts - 1: B row q is row
//   int b_part(q), b_row(q)       b_row(q) of part b_part(q)
//   void prefetch(const Tile&)    called before the tile's first step: loads within the loop
//                                 would make every round wait for its copies
//   bool kSkip                    waves without a valid row skip the products
//   bool kAnyInt8                 operands may hold -128 (else -127 .. 127)
//   void finish(const Tile&, acc) its results; waves without a valid row skip it
// kGather: rows of A through an index, at 64-bit offsets.
template <class C, bool kTail, bool kGather, class Job>
__device__ __forceinline__ void i8_stream(int K, int items, Job& job, int8_t* st) {
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wv / C::WN, wn = wv % C::WN;
  const int steps = cdiv(K, kI8Step);
  // copy i of this wave covers stage rows 8 (i kWaves + wv) ..: lane / 8, chunk lane % 8
  auto row0 = [&](int i) { return (i * C::kWaves + wv) * 8; };
  auto a_chunk = [&](int i) { return a_swizzle(row0(i) + (lane >> 3), lane & 7) * 16; };
  auto b_chunk = [&](int i) { return b_swizzle(row0(i) - C::BM + (lane >> 3), lane & 7) * 16; };
  I8Source sa{nullptr, 0}, sb[Job::kParts];
  const int8_t* gather[kGather ? C::kCopiesA : 1];
  auto sources = [&](const typename Job::Tile& t) {
    sa = job.a(t);
#pragma unroll
    for (int q = 0; q < Job::kParts; ++q) sb[q] = job.b(t, q);
    if constexpr (kGather) {
#pragma unroll
      for (int i = 0; i < C::kCopiesA; ++i)
        gather[i] = sa.base + static_cast<int64_t>(sa.index[min(row0(i) + (lane >> 3), sa.rows - 1)]) * K + a_chunk(i);
    }
  };
  auto rsrc = [&](const I8Source& x) {
    const uint64_t p = reinterpret_cast<uint64_t>(x.base);
    return i32x4{static_cast<int>(p), static_cast<int>(p >> 32 & 0xffff), x.rows * K, 0x00020000};
  };
  auto load = [&](int kt, int8_t* to) {
    const bool part = kTail && (kt + 1) * kI8Step > K;
    const i32x4 ra = rsrc(sa);
    i32x4 rb[Job::kParts];
#pragma unroll
    for (int q = 0; q < Job::kParts; ++q) rb[q] = rsrc(sb[q]);
#pragma unroll
    for (int i = 0; i < C::kCopies; ++i) {
      const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_address(to)) + row0(i) * kI8Step;
      if (i < C::kCopiesA) {
        if constexpr (kGather) {
          copy_to_lds(gather[i] + kt * kI8Step, dst);
        } else {
          uint32_t off = static_cast<uint32_t>((lane >> 3) * K + a_chunk(i) + (row0(i) * K + kt * kI8Step));
          if (part && kt * kI8Step + a_chunk(i) >= K) off = kI8Oob;
          copy_to_lds(ra, off, dst);
        }
      } else {
        const int q = row0(i) - C::BM;  // 8 rows of B, of one part
        const int pt = Job::b_part(q);
        uint32_t off = static_cast<uint32_t>((lane >> 3) * K + b_chunk(i) + (Job::b_row(q) * K + kt * kI8Step));
        if (part && kt * kI8Step + b_chunk(i) >= K) off = kI8Oob;
        copy_to_lds(Job::kParts > 1 && pt ? rb[Job::kParts - 1] : rb[0], off, dst);
      }
    }
  };
  const int g = lane >> 4, i16 = lane & 15;
  i32x4 acc[C::FM][C::FN];
  auto compute = [&](const int8_t* from) {
    const int8_t* at = from + (wm * C::FM * 16 + i16) * kI8Step;
    const int brow = 8 * (i16 >> 2) + (i16 & 3);
    const int8_t* bt = from + (C::BM + wn * C::FN * 16 + brow) * kI8Step;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint4 b[C::FN];
      const int ca = a_swizzle(i16, s * 4 + g) * 16;
#pragma unroll
      for (int n = 0; n < C::FN; ++n)
        b[n] = *reinterpret_cast<const uint4*>(bt + C::col(n) * kI8Step + b_swizzle(brow, s * 4 + g) * 16);
#pragma unroll
      for (int m = 0; m < C::FM; ++m) {
        const uint4 a = *reinterpret_cast<const uint4*>(at + m * 16 * kI8Step + ca);
#pragma unroll
        for (int n = 0; n < C::FN; ++n) acc[m][n] = mfma_i8(b[n], a, acc[m][n]);
      }
      // the fragments of two rows ahead are read under the products of one
      if (s == 0) __builtin_amdgcn_sched_group_barrier(0x100, C::FN + 2, 0);
#pragma unroll
      for (int m = 0; m < C::FM; ++m) {
        __builtin_amdgcn_sched_group_barrier(0x008, C::FN, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
    }
  };

  // the first item with rows from i on
  auto find = [&](int i, typename Job::Tile& x) {
    for (; i < items; i += gridDim.x) {
      x = job.tile(i);
      if (x.rows > 0) break;
    }
    return i;
  };
  typename Job::Tile cur;
  int t = find(blockIdx.x, cur);
  if (t >= items) return;
  sources(cur);
  load(0, st);
  wait_vm<0>();
  int8_t *now = st, *then = st + C::kStage;
  auto swap = [&] {
    int8_t* x = now;
    now = then;
    then = x;
  };
  while (true) {
    const bool live = !Job::kSkip || wm * C::FM * 16 < cur.rows;
#pragma unroll
    for (int m = 0; m < C::FM; ++m)
#pragma unroll
      for (int n = 0; n < C::FN; ++n) acc[m][n] = i32x4{0, 0, 0, 0};
    lds_barrier();
    for (int kt = 0; kt + 1 < steps; ++kt) {
      load(kt + 1, then);
      if (live) compute(now);
      wait_vm<0>();
      lds_barrier();
      swap();
    }
    // The last step stands apart: loads into registers within the loop would
    // make each of its rounds wait for its copies.
    job.prefetch(cur);
    typename Job::Tile next = cur;
    const int tn = find(t + gridDim.x, next);
    if (tn < items) {
      sources(next);
      load(0, then);
    }
    if (live) compute(now);
    wait_vm<0>();  // the scales and the copies, but not the stores that follow
    if constexpr (Job::kAnyInt8) {
      if (K == MOE_I8_MAX_K) {
#pragma unroll
        for (int m = 0; m < C::FM; ++m)
#pragma unroll
          for (int n = 0; n < C::FN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[m][n][i] = unwrap(acc[m][n][i]);
      }
    }
    if (live) job.finish(cur, acc);
    if (tn >= items) break;
    swap();
    t = tn;
    cur = next;
  }
}

// Tile i of n in the order of the XCDs: workgroups go to the 8 XCDs in turn,
// and each XCD takes a contiguous run of tiles.
__device__ __forceinline__ int xcd_order(int i, int n) {
  const int x = i & 7, per = n >> 3, rest = n & 7;
  return x * per + min(x, rest) + (i >> 3);
}

}  // namespace moe
