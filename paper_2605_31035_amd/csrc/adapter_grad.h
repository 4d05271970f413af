// The gradients of the adapters: dA_l = sum u_i^T (keep_i x_i) and
// dB_l = sum dy_i^T t_i over the rows i of adapter l, products whose
// contraction runs along the rows.
#pragma once

#include <type_traits>

#include "adapter.h"

namespace mixfp4 {

constexpr int kGradThreads = 256;

// Columns of x or dy of a workgroup: the more, the fewer reads of the terms;
// the sums of 256 columns by a rank of 64 take 64 registers of each lane.
constexpr int cols_of(int padded) { return padded <= 64 ? 256 : 128; }

// Positions of the pieces: whole tiles, split evenly over those in use.
__device__ __forceinline__ int64_t piece_begin(int64_t tiles, int s, int splits) {
  return tiles * s / splits;
}

// One workgroup: 256 or 128 columns, all of the rank, one piece of the positions.
// It walks the adapters that its piece holds, kDepth positions at a time.
// The columns of x or dy are transposed through registers into LDS (8 rows by
// 8 or 4 columns per thread; dropout's draws are made on the rows), the terms
// come transposed from the join, so that an operand's 8 consecutive positions
// are one LDS read.  The next step's reads are under way while a step is
// multiplied.  An adapter within one piece is written at once, one across
// pieces as partial sums (at most two per piece: the one that enters it and
// the one that leaves it) for sum_kernel.  A rank above 128 takes two
// workgroups (r0), so that the sums stay in registers.  Bound by one step's
// rows under way per workgroup and the products' LDS reads, three terms of t
// or u for each of x or dy: 2048x(4096 + 4096) by themselves 34 us with rank
// 128, 54 with 256.
template <int kRank, bool kDb>
__device__ __forceinline__ void grad_body(const GradSide& a, const GradArgs& q, int block, int piece,
                                          int r0, uint4* lds) {
  constexpr int kTiles = kRank / 16;
  constexpr int kCols = cols_of(kRank), kSide = kCols / 64; // 16-column tiles of a wave
  constexpr int kDepth = 64;
  constexpr int kSlots = kDepth / 8;
  constexpr int kWidth = kCols / 32;                       // columns of a thread's piece
  constexpr int kGroups = kCols / kWidth;
  constexpr int kTerms = 3 * kRank * kSlots;
  constexpr int kPer = (kTerms + kGradThreads - 1) / kGradThreads;
  using Row = std::conditional_t<kWidth == 8, uint4, uint2>;
  uint4* xt = lds;
  uint4* ut = lds + kCols * kSlots;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r16 = lane & 15, g = lane >> 4;
  const int col0 = block * kCols;
  const int64_t tiles = q.plan.seg[q.adapters];
  const int64_t t0 = piece_begin(tiles, piece, q.splits), t1 = piece_begin(tiles, piece + 1, q.splits);
  const int64_t matrix = (int64_t)q.rank * a.cols;
  const int cg = tid % kGroups, pg = tid / kGroups;
  const int col = col0 + cg * kWidth;

  f32x4 acc[kTiles][kSide];
  const int wave_col = wave * 16 * kSide;
  // Behind the adapter's own rank stand zeros: the terms are zero there, but
  // zero times an infinite x or dy is not.
  const auto store = [&](float* to, int own) {
    // opaque, so that the addresses are made here and not kept in registers
    // over the steps
    int r16 = lane & 15, g = lane >> 4;
    asm volatile("" : "+v"(r16), "+v"(g));
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      if constexpr (kDb) {
        const int r = r0 + 16 * i + 4 * g;
#pragma unroll
        for (int j = 0; j < kSide; ++j) {
          const int n = col0 + wave_col + 16 * j + r16;
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = r + e < own ? acc[i][j][e] : 0.0f;
          if (n < a.cols && r < q.rank) *reinterpret_cast<f32x4*>(to + (int64_t)n * q.rank + r) = v;
        }
      } else {
        const int r = r0 + 16 * i + r16;
#pragma unroll
        for (int j = 0; j < kSide; ++j) {
          const int c = col0 + wave_col + 32 * (j >> 1) + 8 * g;
          if (r < q.rank && c < a.cols)
            *reinterpret_cast<f32x4*>(to + (int64_t)r * a.cols + c + 4 * (j & 1)) =
                r < own ? acc[i][j] : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
      }
    }
  };
  const auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int j = 0; j < kSide; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  };

  if (piece == 0)                  // adapters without rows
    for (int l = 0; l < q.adapters; ++l)
      if (q.plan.seg[l] == q.plan.seg[l + 1]) {
        clear();
        store(a.out + l * matrix, 0);
      }
  if (t0 >= t1) return;

  int rows[8], at_rows[8];         // of the next step's reads, of the reads under way
  Row x[8];
  uint4 u[kPer];
  const auto load_rows = [&](int64_t p, int64_t p1) {
    const int64_t at = p + pg * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) rows[j] = -1;
    if (at < p1) {
      const int4 lo = *reinterpret_cast<const int4*>(q.plan.order + at);
      const int4 hi = *reinterpret_cast<const int4*>(q.plan.order + at + 4);
      rows[0] = lo.x, rows[1] = lo.y, rows[2] = lo.z, rows[3] = lo.w;
      rows[4] = hi.x, rows[5] = hi.y, rows[6] = hi.z, rows[7] = hi.w;
    }
  };
  const bool inside = col + kWidth <= a.cols;
  const auto load = [&](int64_t p, int64_t p1) {
#pragma unroll
    for (int j = 0; j < 8; ++j) at_rows[j] = rows[j];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t row = rows[j] < 0 ? 0u : (uint32_t)rows[j];
      x[j] = *reinterpret_cast<const Row*>(
          inside ? a.src + (uint64_t)row * (uint32_t)a.ld + col : a.terms_t);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = tid + i * kGradThreads;
      const int64_t pos = p + e % kSlots * 8;
      const int h = e / (kRank * kSlots), r = e / kSlots - h * kRank;
      const uint16_t* from =
          a.terms_t + (int64_t)(h * q.padded + r0 + r) * q.positions + (pos < p1 ? pos : p);
      if (kTerms % kGradThreads == 0 || e < kTerms) u[i] = *reinterpret_cast<const uint4*>(from);
    }
  };

  for (int l = q.plan.tile_adapter[t0]; l < q.adapters && q.plan.seg[l] < t1; ++l) {
    const int64_t first = q.plan.seg[l], last = q.plan.seg[l + 1];
    if (first == last) continue;
    const int64_t p0 = (first > t0 ? first : t0) * q.tile_rows;
    const int64_t p1 = (last < t1 ? last : t1) * q.tile_rows;
    clear();
    load_rows(p0, p1);
    load(p0, p1);
    load_rows(p0 + kDepth, p1);
    for (int64_t p = p0; p < p1; p += kDepth) {
      if (!inside) {
        // the last columns, by element: nothing behind them is read
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t row = at_rows[j] < 0 ? 0u : (uint32_t)at_rows[j];
          const uint4 v = load8(a.src + (uint64_t)row * (uint32_t)a.ld, col, a.cols);
          if constexpr (kWidth == 8) x[j] = v; else x[j] = make_uint2(v.x, v.y);
        }
        wait_loads();
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (at_rows[j] < 0) {
          x[j] = Row{};
        } else if (!kDb && q.drop.threshold) {
          const uint4 m = keep_masks(block_draws((int64_t)at_rows[j] * (a.cols / 8) + col / 8, q.drop.key),
                                     q.drop.threshold);
          if constexpr (kWidth == 8) {
            x[j] = and4(x[j], m);
          } else {
            x[j].x &= col & 4 ? m.z : m.x;
            x[j].y &= col & 4 ? m.w : m.y;
          }
        }
      }
      __syncthreads();
      if constexpr (kWidth == 8) {
        uint4 v[8];
        transpose8(x, v);
#pragma unroll
        for (int c = 0; c < 8; ++c) xt[lds_slot8<kSlots>(cg * 8 + c, pg)] = v[c];
      } else {
        uint4 v[4];
        transpose8x4(x, v);
#pragma unroll
        for (int c = 0; c < 4; ++c) xt[lds_slot8<kSlots>(cg * 4 + c, pg)] = v[c];
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = tid + i * kGradThreads;
        if (p + e % kSlots * 8 >= p1) u[i] = make_uint4(0, 0, 0, 0);
        if (kTerms % kGradThreads == 0 || e < kTerms) ut[lds_slot<kSlots>(e / kSlots, e % kSlots)] = u[i];
      }
      __syncthreads();
      if (p + kDepth < p1) {
        load(p + kDepth, p1);
        load_rows(p + 2 * kDepth, p1);
      }
#pragma unroll
      for (int s = 0; s < kDepth / 32; ++s) {
        if (p + 32 * s >= p1) break;
        uint4 xf[kSide];
#pragma unroll
        for (int j = 0; j < kSide; ++j) {
          const int c = kDb ? 16 * j + r16 : 32 * (j >> 1) + 8 * (r16 >> 2) + 4 * (j & 1) + (r16 & 3);
          xf[j] = xt[lds_slot8<kSlots>(wave_col + c, 4 * s + g)];
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int h = 2; h >= 0; --h) {             // the smallest term first
            const uint4 uf = ut[lds_slot<kSlots>(h * kRank + 16 * i + r16, 4 * s + g)];
#pragma unroll
            for (int j = 0; j < kSide; ++j)
              acc[i][j] = kDb ? mfma16(uf, xf[j], acc[i][j]) : mfma16(xf[j], uf, acc[i][j]);
          }
      }
    }
    const int own = rank_of(q.ranks, l, q.rank);
    if (first >= t0 && last <= t1)
      store(a.out + l * matrix, own);
    else
      store(a.part + (2 * piece + (first >= t0)) * matrix, own);
  }
}

// 16-byte units of LDS of a workgroup.
constexpr int grad_lds(int padded) { return (cols_of(padded) + 3 * padded) * 8; }

// Workgroup `index` of the gradients: those of a piece side by side, which
// read the same rows.
template <int kRank>
__device__ __forceinline__ void grad_block(const GradArgs& q, int index, int r0, uint4* lds) {
  constexpr int kCols = cols_of(kRank);
  const int blocks_a = (q.a.cols + kCols - 1) / kCols, blocks = blocks_a + (q.b.cols + kCols - 1) / kCols;
  const int piece = index / blocks, block = index % blocks;
  if (block < blocks_a)
    grad_body<kRank, false>(q.a, q, block, piece, r0, lds);
  else
    grad_body<kRank, true>(q.b, q, block - blocks_a, piece, r0, lds);
}

}  // namespace mixfp4
