// The narrow products of the adapters: t = (keep x) A_l^T and u = dy B_l,
// [rows, depth] times [depth, rank], and the join of their pieces.
#include "adapter.h"

namespace mixfp4 {

namespace {

constexpr int kThreads = 256;

// One workgroup: one tile of rows of one adapter, one piece of the
// contraction, in chunks of kC: the chunks of x and W go through registers
// (two of them under way) into LDS, where the operands are read.  There x's
// 16 bytes are one group of dropout's draws, and B_l [depth, rank] is
// transposed, 8 rows by 4 columns at a time.  Loads are made without branches,
// from an element that is there in place of one that is not, and cleared or
// (the last, partial 16 bytes of a row) read again on their way into LDS: a
// load in a branch would make the loads under way wait for each other.  With
// tiles of 16 rows each wave takes a quarter of every chunk, joined at the
// end; with tiles of 64 rows 16 of them, or half of them and half of a rank
// above 64.  Bound by memory with many rows: dy 8192x14336 rank 64 57 us,
// 4.1 TB/s (a bare read of these rows 41); x 8192x4096 with draws 26 us.  With
// few by the latency of a piece's chunks: x 2048x4096 rank 64 11 us.
template <int kT, int kRank, bool kTransposed>
__global__ __launch_bounds__(kThreads, kRank <= 64 ? 3 : 2) void shrink_kernel(ShrinkArgs a, int tiles) {
  constexpr int kC = kT == 16 || kRank <= 64 ? 128 : 64;
  constexpr int kSlots = kC / 8;
  constexpr int kTiles = kRank / 16;
  constexpr int kHalf = kT == 64 && kRank > 64 ? 2 : 1;       // parts of the rank
  constexpr int kMine = kTiles / kHalf;                       // a wave's tiles of it
  constexpr int kSteps = kT == 16 ? kC / 128 : kC / 32;       // its matrix steps in a chunk
  constexpr int kX = kT * kSlots / kThreads;                  // 16-byte pieces of x per thread
  constexpr int kPieces = kTransposed ? kRank * kSlots / 4 : kRank * kSlots;
  constexpr int kPer = (kPieces + kThreads - 1) / kThreads;
  constexpr int kAhead = kT == 16 && kRank > 128 ? 1 : 2;     // chunks under way
  constexpr int kJoin = kT == 16 ? 4 * kTiles * 64 : 0;
  constexpr int kLds = (kRank + kT) * kSlots > kJoin ? (kRank + kT) * kSlots : kJoin;
  __shared__ uint4 lds[kLds];
  uint4* xs = lds + kRank * kSlots;
  const int tile = blockIdx.z * gridDim.y + blockIdx.y, piece = blockIdx.x;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r16 = lane & 15, g = lane >> 4;
  if (tile >= tiles) return;
  const int l = a.plan.tile_adapter[tile];
  if (l < 0 || l >= a.adapters) return;
  const int rank = rank_of(a.ranks, l, a.rank);
  const int64_t p0 = (int64_t)tile * kT;
  const uint16_t* w = a.w + (int64_t)l * a.rank * a.depth;

  const int chunks = (a.depth + kC - 1) / kC;
  const int c0 = (int)((int64_t)chunks * piece / a.splits);
  const int c1 = (int)((int64_t)chunks * (piece + 1) / a.splits);
  const int count = c1 - c0;

  const int xslot = tid % kSlots, xrow = tid / kSlots;
  int row[kX];
  const uint16_t* src[kX];
#pragma unroll
  for (int i = 0; i < kX; ++i) {
    row[i] = a.plan.order[p0 + xrow + i * (kThreads / kSlots)];
    src[i] = a.src + (row[i] < 0 ? 0u : (uint64_t)(uint32_t)row[i] * (uint32_t)a.ld);
  }

  struct Chunk {
    uint4 x[kX];
    uint4 w[kTransposed ? 1 : kPer];
    uint2 t[kTransposed ? kPer : 1][8];
  };
  // Chunks behind the last are "loaded" too, from one address: were the loads
  // in a branch, each wait would have to assume that none are under way.
  const auto load = [&](int chunk, bool there, Chunk& c) {
    const int col = chunk * kC + xslot * 8;
    const bool whole = there && col + 8 <= a.depth;
#pragma unroll
    for (int i = 0; i < kX; ++i) c.x[i] = *reinterpret_cast<const uint4*>(whole ? src[i] + col : w);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = tid + i * kThreads;
      if constexpr (kTransposed) {
        const int rb = p % (kRank / 4) * 4, at = chunk * kC + p / (kRank / 4) % kSlots * 8;
        const uint16_t* from = w + (rb < a.rank ? rb : 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int n = !there ? 0 : at + j < a.depth ? at + j : a.depth - 1;
          c.t[i][j] = *reinterpret_cast<const uint2*>(from + (int64_t)n * a.rank);
        }
      } else {
        const int r = p / kSlots, at = chunk * kC + p % kSlots * 8;
        c.w[i] = *reinterpret_cast<const uint4*>(w + (int64_t)(there && r < rank ? r : 0) * a.depth +
                                                 (there && at < a.depth ? at : 0));
      }
    }
  };
  const auto fill = [&](int chunk, Chunk& c) {
    const int col = chunk * kC + xslot * 8;
#pragma unroll
    for (int i = 0; i < kX; ++i) {
      uint4 v = c.x[i];
      if (col + 8 > a.depth) {
        v = load8(src[i], col, a.depth);
        wait_loads();
      }
      if (!kTransposed && a.drop.threshold)
        v = and4(v, keep_masks(block_draws((int64_t)row[i] * (a.depth / 8) + col / 8, a.drop.key),
                               a.drop.threshold));
      if (row[i] < 0) v = make_uint4(0, 0, 0, 0);
      xs[lds_slot<kSlots>(xrow + i * (kThreads / kSlots), xslot)] = v;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = tid + i * kThreads;
      if (kPieces % kThreads != 0 && p >= kPieces) break;
      if constexpr (kTransposed) {
        const int rb = p % (kRank / 4) * 4, nb = p / (kRank / 4), at = chunk * kC + nb * 8;
        if (at + 8 > a.depth || rb + 4 > rank) {
          const uint32_t lo = (rank > rb ? 0xFFFFu : 0u) | (rank > rb + 1 ? 0xFFFF0000u : 0u);
          const uint32_t hi = (rank > rb + 2 ? 0xFFFFu : 0u) | (rank > rb + 3 ? 0xFFFF0000u : 0u);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t there = at + j < a.depth ? 0xFFFFFFFFu : 0u;
            c.t[i][j].x &= lo & there;
            c.t[i][j].y &= hi & there;
          }
        }
        uint4 v[4];
        transpose8x4(c.t[i], v);
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[lds_slot<kSlots>(rb + e, nb)] = v[e];
      } else {
        const int r = p / kSlots, at = chunk * kC + p % kSlots * 8;
        if (r >= rank || at >= a.depth) c.w[i] = make_uint4(0, 0, 0, 0);
        lds[lds_slot<kSlots>(r, p % kSlots)] = c.w[i];
      }
    }
  };

  f32x4 acc[kHalf][kMine];
#pragma unroll
  for (int h = 0; h < kHalf; ++h)
#pragma unroll
    for (int i = 0; i < kMine; ++i) acc[h][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // a wave's rows (kHalf tiles of 16) and its part of the rank
  const int row0 = kT == 16 ? 0 : kHalf == 1 ? wave * 16 : (wave & 1) * 32;
  const int rank0 = kHalf == 1 ? 0 : (wave >> 1) * (kRank / 2);
  // each tile begins elsewhere in the piece (see tile_grid on memory channels)
  const int start = count > 0 ? tile % count : 0;
  const auto at = [&](int i) { return c0 + (start + i < count ? start + i : start + i - count); };
  Chunk c[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    load(at(i), i < count, c[i]);
  for (int done = 0; done < count; done += kAhead) {
#pragma unroll
    for (int b = 0; b < kAhead; ++b) {
      const int i = done + b;
      if (i >= count) break;
      __syncthreads();
      fill(at(i), c[b]);
      __syncthreads();
      load(at(i + kAhead), i + kAhead < count, c[b]);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int slot = (kT == 16 ? wave * 4 : s * 4) + g;
        uint4 xf[kHalf];
#pragma unroll
        for (int h = 0; h < kHalf; ++h) xf[h] = xs[lds_slot<kSlots>(row0 + 16 * h + r16, slot)];
#pragma unroll
        for (int t = 0; t < kMine; ++t) {
          const uint4 wf = lds[lds_slot<kSlots>(rank0 + t * 16 + r16, slot)];
#pragma unroll
          for (int h = 0; h < kHalf; ++h) acc[h][t] = mfma16(wf, xf[h], acc[h][t]);
        }
      }
    }
  }

  float* part = a.part + (int64_t)piece * a.positions * a.rank;
  if constexpr (kT == 16) {
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(lds);
#pragma unroll
    for (int i = 0; i < kTiles; ++i) sums[(wave * kTiles + i) * 64 + lane] = acc[0][i];
    __syncthreads();
    for (int i = wave; i < kTiles; i += 4) {
      f32x4 v = sums[i * 64 + lane];
#pragma unroll
      for (int q = 1; q < 4; ++q) v += sums[(q * kTiles + i) * 64 + lane];
      const int r = i * 16 + 4 * g;
      if (r < a.rank) *reinterpret_cast<f32x4*>(part + (p0 + r16) * a.rank + r) = v;
    }
  } else {
#pragma unroll
    for (int h = 0; h < kHalf; ++h)
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int r = rank0 + i * 16 + 4 * g;
        if (r < a.rank)
          *reinterpret_cast<f32x4*>(part + (p0 + row0 + 16 * h + r16) * a.rank + r) = acc[h][i];
      }
  }
}

template <int kT, bool kTransposed>
void launch(const ShrinkArgs& a, int64_t tiles, hipStream_t stream) {
  const dim3 grid = tile_grid(a.splits, tiles);
  const int count = (int)tiles;
  switch (padded_rank(a.rank)) {
    case 16: shrink_kernel<kT, 16, kTransposed><<<grid, kThreads, 0, stream>>>(a, count); break;
    case 32: shrink_kernel<kT, 32, kTransposed><<<grid, kThreads, 0, stream>>>(a, count); break;
    case 64: shrink_kernel<kT, 64, kTransposed><<<grid, kThreads, 0, stream>>>(a, count); break;
    case 128: shrink_kernel<kT, 128, kTransposed><<<grid, kThreads, 0, stream>>>(a, count); break;
    default: shrink_kernel<kT, 256, kTransposed><<<grid, kThreads, 0, stream>>>(a, count); break;
  }
}

// 16 positions per workgroup (they are of one adapter).  Mode 0 sums the
// pieces, mode 1 takes t_in's rows.  A thread sums four consecutive values;
// with a small rank, several threads share the pieces and their sums are
// added in a fixed order.  Pieces are read eight at a time, so that their
// latencies overlap: 4.7 us for 48 rows, 5.3 for 8192 of rank 64, 8.9 with both
// transposes of the backward pass; 16 for 2048 of rank 256 with them.
template <int kRank>
__global__ __launch_bounds__(kThreads) void join_kernel(JoinArgs a, int tile_rows) {
  constexpr int kItems = 16 * kRank / 4;                    // float4 of the 16 positions
  constexpr int kShare = kItems < kThreads ? kThreads / kItems : 1;
  constexpr int kWide = kRank < 32 ? 32 : kRank;
  constexpr int kPitch = kRank + 4;
  __shared__ float v[16 * kPitch];
  __shared__ f32x4 shared[kShare > 1 ? kThreads : 1];
  const int64_t p0 = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * 16;
  const int mode = blockIdx.y;
  if (p0 >= a.positions) return;
  const int l = a.plan.tile_adapter[p0 / tile_rows];
  if (l < 0) return;
  const int tid = threadIdx.x;
  const bool none = l >= a.adapters;
  const int rank = none ? 0 : rank_of(a.ranks, l, a.rank);
  const float s = none || !a.scaling ? 1.0f : a.scaling[l];
  const int64_t piece = a.positions * a.rank;
  for (int i = tid; i < kItems * kShare; i += kThreads) {
    const int item = i % kItems, part = i / kItems;
    const int q = item / (kRank / 4), r = item % (kRank / 4) * 4;
    const int row = a.plan.order[p0 + q];
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (r < rank && row >= 0) {
      if (mode == 1) {
        if (part == 0) {
          const float* t = a.t_in + (int64_t)row * a.rank + r;   // any 4-byte alignment
          sum = f32x4{t[0], t[1], t[2], t[3]};
        }
      } else {
        const float* from = a.part + (p0 + q) * a.rank + r;
        int j = part;
        for (; j + 7 * kShare < a.splits; j += 8 * kShare) {
          f32x4 u[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            u[e] = *reinterpret_cast<const f32x4*>(from + (j + e * kShare) * piece);
#pragma unroll
          for (int e = 0; e < 8; ++e) sum += u[e];
        }
        for (; j < a.splits; j += kShare) sum += *reinterpret_cast<const f32x4*>(from + j * piece);
      }
    }
    if constexpr (kShare > 1) {
      shared[tid] = sum;
      __syncthreads();                                     // one round: kItems * kShare threads
      if (part > 0) break;
#pragma unroll
      for (int e = 1; e < kShare; ++e) sum += shared[tid + e * kItems];
    }
    if (mode == 0) sum *= a.z;
    f32x4 scaled = s * sum;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r + e >= rank || row < 0) sum[e] = scaled[e] = 0.0f;   // whatever s is
    if (mode == 0 && a.t && row >= 0 && r < a.rank) {
      float* t = a.t + (int64_t)row * a.rank + r;
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = sum[e];
    }
    *reinterpret_cast<f32x4*>(&v[q * kPitch + r]) = scaled;
  }
  if (none) return;
  __syncthreads();
  if (mode == 0) {
    for (int i = tid; i < 16 * kWide / 2; i += kThreads) {
      const int q = i / (kWide / 2), r = i % (kWide / 2) * 2;
      uint32_t hi[2] = {0u, 0u}, lo[2] = {0u, 0u};
      if (r < kRank) {
        split_bf16(v[q * kPitch + r], hi[0], lo[0]);
        split_bf16(v[q * kPitch + r + 1], hi[1], lo[1]);
      }
      uint32_t* to = reinterpret_cast<uint32_t*>(a.terms + (p0 + q) * 2 * kWide + r);
      to[0] = hi[0] | hi[1] << 16;
      to[kWide / 2] = lo[0] | lo[1] << 16;
    }
  }
  uint16_t* transposed = mode == 0 ? a.terms_t : a.t_in_t;
  if (transposed)
    for (int i = tid; i < 8 * kRank; i += kThreads) {
      const int q = i % 8 * 2, r = i / 8;
      uint32_t x[3], y[3];
      split_bf16(v[q * kPitch + r], x);
      split_bf16(v[(q + 1) * kPitch + r], y);
#pragma unroll
      for (int h = 0; h < 3; ++h)
        *reinterpret_cast<uint32_t*>(transposed + ((int64_t)h * kRank + r) * a.positions + p0 + q) =
            x[h] | y[h] << 16;
    }
}

}  // namespace

// Pieces of the contraction: enough workgroups to fill the device (one per
// compute unit with a rank above 128, whose pieces are large: the forward pass
// of 1537x4096x4096 rank 256 took 43 us with 8 of them, 46 with 16), each with
// two chunks at least.
int adapter_shrink_splits(int64_t tiles, int64_t depth, int64_t rank) {
  if (tiles < 1) return 1;
  const int64_t chunks = (depth + 127) / 128;
  int64_t s = padded_rank(rank) > 128 ? compute_units() / tiles : (768 + tiles - 1) / tiles;
  if (s > chunks / 2) s = chunks / 2;
  return s < 1 ? 1 : (int)s;
}

hipError_t launch_adapter_shrink(const ShrinkArgs& a, int tile_rows, int64_t tiles, bool transposed,
                                 hipStream_t stream) {
  if (tile_rows == 16)
    transposed ? launch<16, true>(a, tiles, stream) : launch<16, false>(a, tiles, stream);
  else
    transposed ? launch<64, true>(a, tiles, stream) : launch<64, false>(a, tiles, stream);
  return hipGetLastError();
}

hipError_t launch_adapter_join(const JoinArgs& a, int tile_rows, hipStream_t stream) {
  // a dimension of a launch holds less than 2^32 threads
  constexpr int64_t kMost = int64_t(1) << 23;
  const int64_t blocks = a.positions / 16, x = blocks < kMost ? blocks : kMost;
  const dim3 grid((unsigned)x, a.t_in ? 2 : 1, (unsigned)((blocks + x - 1) / x));
  switch (padded_rank(a.rank)) {
    case 16: join_kernel<16><<<grid, kThreads, 0, stream>>>(a, tile_rows); break;
    case 32: join_kernel<32><<<grid, kThreads, 0, stream>>>(a, tile_rows); break;
    case 64: join_kernel<64><<<grid, kThreads, 0, stream>>>(a, tile_rows); break;
    case 128: join_kernel<128><<<grid, kThreads, 0, stream>>>(a, tile_rows); break;
    default: join_kernel<256><<<grid, kThreads, 0, stream>>>(a, tile_rows); break;
  }
  return hipGetLastError();
}

}  // namespace mixfp4
