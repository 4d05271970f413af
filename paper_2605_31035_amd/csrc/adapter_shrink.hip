// The narrow products of the adapters: t = (keep x) A_l^T and u = dy B_l,
// [rows, depth] times [depth, rank], and the join of their pieces.
#include "adapter.h"

namespace mixfp4 {

namespace {

constexpr int kThreads = 256;

// One workgroup: one tile of rows of one adapter, one piece of the
// contraction.  Chunks of kC of it: W's chunk [rank, kC] goes through LDS (for
// B_l [depth, rank] transposed on the way, 8 x 8 at a time), x's straight from
// memory into the operand registers, which is each element once: a lane's
// operand of one matrix instruction is 8 consecutive elements of its row, one
// group of dropout's draws.  With tiles of 64 rows each wave takes 16 of
// them, with tiles of 16 a quarter of every chunk, joined at the end.
template <int kT, int kRank, bool kTransposed>
__global__ __launch_bounds__(kThreads) void shrink_kernel(ShrinkArgs a) {
  constexpr int kC = kT == 16 || kRank <= 64 ? 128 : 64;
  constexpr int kSlots = kC / 8;
  constexpr int kTiles = kRank / 16;
  constexpr int kSteps = kT == 16 ? kC / 128 : kC / 32;   // matrix steps of a wave in a chunk
  // pieces of W per thread and chunk: 16 bytes each, or 8 x 8 blocks
  constexpr int kPieces = kTransposed ? kRank * kSlots / 8 : kRank * kSlots;
  constexpr int kPer = (kPieces + kThreads - 1) / kThreads;
  constexpr int kLds = kRank * kSlots > (kT == 16 ? 4 * kTiles * 64 : 0) ? kRank * kSlots
                                                                        : 4 * kTiles * 64;
  __shared__ uint4 lds[kLds];
  const int tile = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r16 = lane & 15, g = lane >> 4;
  const int l = a.plan.tile_adapter[tile];
  if (l < 0 || l >= a.adapters) return;
  const int rank = rank_of(a.ranks, l, a.rank);
  const int64_t position = (int64_t)tile * kT + (kT == 16 ? 0 : wave * 16) + r16;
  const int row = a.plan.order[position];
  const uint16_t* src = a.src + (row < 0 ? 0 : (int64_t)row * a.ld);
  const uint16_t* w = a.w + (int64_t)l * a.rank * a.depth;
  const int64_t draw = (int64_t)row * (a.depth / 8);       // dropout: depth % 8 == 0

  const int chunks = (a.depth + kC - 1) / kC;
  const int c0 = (int)((int64_t)chunks * blockIdx.y / a.splits);
  const int c1 = (int)((int64_t)chunks * (blockIdx.y + 1) / a.splits);

  uint4 xr[kSteps];
  uint4 wr[kPer][kTransposed ? 8 : 1];
  const auto column = [&](int chunk, int s) {
    return chunk * kC + (kT == 16 ? wave * 32 : s * 32) + 8 * g;
  };
  const auto load = [&](int chunk) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
      xr[s] = row < 0 ? make_uint4(0, 0, 0, 0) : load8(src, column(chunk, s), a.depth);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = tid + i * kThreads;
      if constexpr (kTransposed) {
        const int rb = p % (kRank / 8), nb = p / (kRank / 8);
        const int at = chunk * kC + nb * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          wr[i][j] = p < kPieces && at + j < a.depth && rb * 8 < rank
                         ? clear_from(*reinterpret_cast<const uint4*>(
                                          w + (int64_t)(at + j) * a.rank + rb * 8), rank - rb * 8)
                         : make_uint4(0, 0, 0, 0);
      } else {
        const int r = p / kSlots, at = chunk * kC + p % kSlots * 8;
        wr[i][0] = p < kPieces && r < rank ? load8(w + (int64_t)r * a.depth, at, a.depth)
                                           : make_uint4(0, 0, 0, 0);
      }
    }
  };

  f32x4 acc[kTiles];
#pragma unroll
  for (int i = 0; i < kTiles; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (c0 < c1) load(c0);
  for (int chunk = c0; chunk < c1; ++chunk) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = tid + i * kThreads;
      if (p >= kPieces) break;
      if constexpr (kTransposed) {
        const int rb = p % (kRank / 8), nb = p / (kRank / 8);
        uint4 v[8];
        transpose8(wr[i], v);
#pragma unroll
        for (int c = 0; c < 8; ++c) lds[lds_slot<kSlots>(rb * 8 + c, nb)] = v[c];
      } else {
        lds[lds_slot<kSlots>(p / kSlots, p % kSlots)] = wr[i][0];
      }
    }
    uint4 xf[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      xf[s] = xr[s];
      if (a.drop.threshold && row >= 0)
        xf[s] = and4(xf[s], keep_masks(block_draws(draw + column(chunk, s) / 8, a.drop.key),
                                       a.drop.threshold));
    }
    __syncthreads();
    if (chunk + 1 < c1) load(chunk + 1);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int slot = (kT == 16 ? wave * 4 : s * 4) + g;
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
        acc[i] = mfma16(lds[lds_slot<kSlots>(i * 16 + r16, slot)], xf[s], acc[i]);
    }
  }

  float* part = a.part + (int64_t)blockIdx.y * a.positions * a.rank;
  if constexpr (kT == 16) {
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(lds);
#pragma unroll
    for (int i = 0; i < kTiles; ++i) sums[(wave * kTiles + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < kTiles; i += 4) {
      f32x4 v = sums[i * 64 + lane];
#pragma unroll
      for (int q = 1; q < 4; ++q) v += sums[(q * kTiles + i) * 64 + lane];
      const int r = i * 16 + 4 * g;
      if (r < a.rank) *reinterpret_cast<f32x4*>(part + position * a.rank + r) = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int r = i * 16 + 4 * g;
      if (r < a.rank) *reinterpret_cast<f32x4*>(part + position * a.rank + r) = acc[i];
    }
  }
}

template <int kT, bool kTransposed>
void launch(const ShrinkArgs& a, int64_t tiles, hipStream_t stream) {
  const dim3 grid((unsigned)tiles, (unsigned)a.splits);
  switch (padded_rank(a.rank)) {
    case 16: shrink_kernel<kT, 16, kTransposed><<<grid, kThreads, 0, stream>>>(a); break;
    case 32: shrink_kernel<kT, 32, kTransposed><<<grid, kThreads, 0, stream>>>(a); break;
    case 64: shrink_kernel<kT, 64, kTransposed><<<grid, kThreads, 0, stream>>>(a); break;
    case 128: shrink_kernel<kT, 128, kTransposed><<<grid, kThreads, 0, stream>>>(a); break;
    default: shrink_kernel<kT, 256, kTransposed><<<grid, kThreads, 0, stream>>>(a); break;
  }
}

// 16 positions per workgroup (they are of one adapter).  Mode 0 sums the
// pieces, mode 1 takes t_in's rows.
__global__ __launch_bounds__(kThreads) void join_kernel(JoinArgs a, int tile_rows, int padded) {
  __shared__ float v[16][256 + 1];
  const int64_t p0 = (int64_t)blockIdx.x * 16;
  const int mode = blockIdx.y;
  const int l = a.plan.tile_adapter[p0 / tile_rows];
  if (l < 0) return;
  const int tid = threadIdx.x;
  const bool none = l >= a.adapters;
  const int rank = none ? 0 : rank_of(a.ranks, l, a.rank);
  const float s = none || !a.scaling ? 1.0f : a.scaling[l];
  for (int i = tid; i < 16 * padded; i += kThreads) {
    const int q = i / padded, r = i % padded;
    const int row = a.plan.order[p0 + q];
    float sum = 0.0f;
    if (r < rank && row >= 0) {
      if (mode == 1) {
        sum = a.t_in[(int64_t)row * a.rank + r];
      } else {
        const float* part = a.part + (p0 + q) * a.rank + r;
        for (int j = 0; j < a.splits; ++j) sum += part[(int64_t)j * a.positions * a.rank];
        sum *= a.z;
      }
    }
    if (mode == 0 && a.t && row >= 0 && r < a.rank) a.t[(int64_t)row * a.rank + r] = sum;
    v[q][r] = s * sum;
  }
  if (none) return;
  __syncthreads();
  if (mode == 0 && a.terms) {
    const int width = padded < 32 ? 32 : padded;
    for (int i = tid; i < 16 * width; i += kThreads) {
      const int q = i / width, r = i % width;
      uint32_t hi = 0u, lo = 0u;
      if (r < padded) split_bf16(v[q][r], hi, lo);
      uint16_t* to = a.terms + (p0 + q) * 2 * width + r;
      to[0] = (uint16_t)hi;
      to[width] = (uint16_t)lo;
    }
  }
  uint16_t* transposed = mode == 0 ? a.terms_t : a.t_in_t;
  if (transposed)
    for (int i = tid; i < 16 * padded; i += kThreads) {
      const int q = i % 16, r = i / 16;
      uint32_t part[3];
      split_bf16(v[q][r], part[0], part[1], part[2]);
#pragma unroll
      for (int h = 0; h < 3; ++h)
        transposed[((int64_t)h * padded + r) * a.positions + p0 + q] = (uint16_t)part[h];
    }
}

}  // namespace

// Pieces of the contraction: enough workgroups to fill the device, each with
// two chunks at least.
int adapter_shrink_splits(int64_t tiles, int64_t depth, int64_t rank) {
  const int64_t chunks = (depth + 127) / 128;
  if (tiles < 1) return 1;
  int64_t s = (512 + tiles - 1) / tiles;
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
  join_kernel<<<dim3((unsigned)(a.positions / 16), a.t_in ? 2 : 1), kThreads, 0, stream>>>(
      a, tile_rows, padded_rank(a.rank));
  return hipGetLastError();
}

}  // namespace mixfp4
