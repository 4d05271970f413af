// The wide products of the adapters: out = c + terms B_l^T and
// dx = dx0 + keep (terms A_l), where the terms are s_l t or s_l z u in two
// bf16 parts (adapter.h).
#pragma once

#include <type_traits>

#include "adapter.h"

namespace mixfp4 {

// A wave takes 32 columns of a block of 128, and all rows of the tile, or half
// of them: of a tile of 64 rows, whose sums and base would hold half of the
// registers, so that too few waves are there to hide the memory's latency
// (whole forward passes: 1537x4096x4096 rank 256 67 -> 55 us, 2048x4096x11008
// rank 64 61 -> 59).  The input gradient with a small rank gains nothing by it
// (its draws need more registers): 8192x4096 rank 64 57 us either way.
constexpr int threads_of(int tile_rows, int rank, bool dx) {
  return tile_rows == 64 && (!dx || rank > 64) ? 512 : 256;
}
constexpr int waves_of(int tile_rows, int rank, bool dx) {
  return tile_rows == 16 && rank > 128 ? 1 : rank <= 64 && !dx ? 4 : 2;
}

// 16-byte units of LDS of a workgroup.
constexpr int expand_lds(int tile_rows, int rank, bool dx) {
  const int slots = (rank < 32 ? 32 : rank) / 8;
  return tile_rows * 2 * slots + 128 * slots + threads_of(tile_rows, rank, dx) / 64 * 128 + tile_rows / 4;
}

// One workgroup: one tile of rows, `width` columns, 128 at a time and 32 of
// them per wave.  The terms of the tile stand in LDS.  W is the left operand
// of the matrix instructions, so that a lane of the result holds one row; of
// two instructions with columns 8 q + 0..3 and 8 q + 4..7 it holds 8
// consecutive columns, one group of dropout's draws.  The wave then turns
// its 16 x 32 results in LDS of its own, so that 8 lanes read the base and
// write out of one row, a whole 128-byte line (kAligned; otherwise 32 lanes,
// 4 bytes each).  There the fp32 base and result pass the caches by: they are
// used once, and W and the terms stay (8192x14336: 193 us against 202; rows
// that do not fill lines lose by it).  What the next block needs from memory
// is requested before this block is stored: loads behind stores wait for
// them.  Loads are made without branches, from a row or column that is there
// in place of one that is not (behind the last block, from one address): with
// loads in a branch each wait would have to assume that none are under way.
// Only tiles and blocks that are not full look at each store.  Bound by
// memory: 8192x14336 rank 64 162 us, 5.8 TB/s; 2048x11008 40 us, 4.5 TB/s.
template <int kT, int kRank, bool kDx, bool kOut16, bool kAligned, bool kJoin>
__device__ __forceinline__ void expand_body(const ExpandArgs& a, int width, int tile, int chunk,
                                            uint4* lds) {
  constexpr int kWide = kRank < 32 ? 32 : kRank;     // terms per part
  constexpr int kSteps = kWide / 32;
  constexpr int kThreads = threads_of(kT, kRank, kDx);
  constexpr bool kShared = kThreads == 512;          // two waves per 32 columns
  constexpr int kRows = kT / 16 / (kShared ? 2 : 1); // 16-row tiles of a wave
  constexpr int kSlots = kWide / 8;
  // pieces of W per thread and block: 16 bytes of B_l, or 8 rows by 4 columns
  // of A_l
  constexpr int kPieces = kDx ? (32 * kSlots + kThreads - 1) / kThreads : 128 * kSlots / kThreads;
  constexpr bool kAhead = kRank <= 128 || kThreads == 512;   // registers for W of the next block
  uint4* terms = lds;                                          // [kT][2 kSlots]
  uint4* wt = terms + kT * 2 * kSlots;                         // [128][kSlots]
  f32x4* turn = reinterpret_cast<f32x4*>(wt + 128 * kSlots);   // [waves][16 * 8]
  int32_t* order = reinterpret_cast<int32_t*>(turn + kThreads / 64 * 128);   // [kT]
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r16 = lane & 15, g = lane >> 4;
  const int wave_col = (wave & 3) * 32, row0 = (wave >> 2) * 32;
  const int l = a.plan.tile_adapter[tile];
  if (l < 0) return;
  const bool none = l >= a.adapters;
  const int rank = none ? 0 : rank_of(a.ranks, l, a.rank);
  const int64_t p0 = (int64_t)tile * kT;
  const uint16_t* w = a.w + (none ? 0 : (int64_t)l * a.rank * a.cols);
  const int begin = chunk * width;
  const int end = a.cols - begin < width ? a.cols : begin + width;

  // pieces of 16 bytes of B_l: column and slot of each, the same in every
  // block; a wave loads its own 32 columns unless another shares them
  const int slots = a.rank >> 3;
  const int p_first = kShared ? tid : lane, p_step = kShared ? kThreads : 64;
  constexpr int kSpan = kShared ? 128 : 32;
  const int span0 = kShared ? 0 : wave_col;
  int piece_col[kDx ? 1 : kPieces], piece_at[kDx ? 1 : kPieces];
  if constexpr (!kDx) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int p = p_first + p_step * i, col = p / slots, slot = p - col * slots;
      piece_col[i] = col < kSpan ? col : kSpan;
      piece_at[i] = col < kSpan ? lds_slot<kSlots>(span0 + col, slot) : 0;
      if (slot * 8 >= rank) piece_col[i] |= 0x100;              // behind the adapter's rank
      else if (slot * 8 + 8 > rank) piece_col[i] |= 0x200;
    }
  }
  uint4 wf[kDx ? 1 : kPieces];
  uint2 wp[kDx ? kPieces : 1][8];
  const auto load_w = [&](int block, bool there) {
    if constexpr (kDx) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int p = tid + i * kThreads, cb = p % 32, rb = p / 32;
        int col = block + cb * 4;
        col = col < end ? col : end - 4;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = rb * 8 + j < rank ? rb * 8 + j : 0;
          wp[i][j] = *reinterpret_cast<const uint2*>(w + (there ? (int64_t)r * a.cols + col : 0));
        }
      }
    } else {
      // columns of B_l stand side by side
      const int c0 = block + span0;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int p = p_first + p_step * i;
        const bool is = there && (piece_col[i] & 0xFF) < kSpan && c0 + (piece_col[i] & 0xFF) < end;
        wf[i] = *reinterpret_cast<const uint4*>(w + (is ? (int64_t)c0 * a.rank + p * 8 : 0));
      }
    }
  };
  load_w(begin, true);

  if (tid < kT) order[tid] = a.plan.order[p0 + tid];
  if constexpr (kJoin) {
    // the terms of the few rows from the pieces of their sums, sixteen reads
    // at a time (from the first piece where there are no more)
    const float f = none || !a.scaling ? 1.0f : a.scaling[l];
    const int64_t size = a.positions * a.rank;
    for (int e = tid; e < kT * kWide / 4; e += kThreads) {
      const int q = e / (kWide / 4), r = e % (kWide / 4) * 4;
      const int row = a.plan.order[p0 + q];
      if (row < 0) break;                    // and all behind it
      f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
      if (r < rank) {
        const float* from = a.part + (p0 + q) * a.rank + r;
        for (int j = 0; j < a.splits; j += 16) {
          f32x4 v[16];
#pragma unroll
          for (int h = 0; h < 16; ++h)
            v[h] = *reinterpret_cast<const f32x4*>(from + (j + h < a.splits ? j + h : 0) * size);
#pragma unroll
          for (int h = 0; h < 16; ++h)
            if (j + h < a.splits) sum += v[h];
        }
        sum *= a.z;
#pragma unroll
        for (int h = 0; h < 4; ++h)
          if (r + h >= rank) sum[h] = 0.0f;
      }
      if (a.t && chunk == 0 && r < a.rank) {
        float* t = a.t + (int64_t)row * a.rank + r;
#pragma unroll
        for (int h = 0; h < 4; ++h) t[h] = sum[h];
      }
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) split_bf16(r + h < rank ? f * sum[h] : 0.0f, hi[h], lo[h]);
      uint2* to = reinterpret_cast<uint2*>(terms);
      to[2 * lds_slot<2 * kSlots>(q, r >> 3) + (r >> 2 & 1)] =
          make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
      to[2 * lds_slot<2 * kSlots>(q, kSlots + (r >> 3)) + (r >> 2 & 1)] =
          make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
    }
  } else if (rank > 0) {
    const uint4* from = reinterpret_cast<const uint4*>(a.terms + p0 * 2 * kWide);
#pragma unroll
    for (int i = 0; i < (kT * 2 * kSlots + kThreads - 1) / kThreads; ++i) {
      const int p = tid + i * kThreads;
      if (p < kT * 2 * kSlots) terms[lds_slot<2 * kSlots>(p / (2 * kSlots), p % (2 * kSlots))] = from[p];
    }
  }
  if constexpr (!kDx) {
    if (a.rank < kWide)                      // the rank padded to whole matrix steps
      for (int p = tid; p < 128 * kSlots; p += kThreads)
        if (p % kSlots >= slots) wt[lds_slot<kSlots>(p / kSlots, p % kSlots)] = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();

  // this lane's rows: of its loads and stores, those that are not there
  // replaced by the tile's first for loads
  constexpr int kLoads = kAligned ? 2 * kRows : 8 * kRows;
  constexpr int kLanes = kAligned ? 8 : 32;
  const int sub = lane / kLanes, lane_col = lane % kLanes * (kAligned ? 4 : 1);
  const bool whole = order[kT - 1] >= 0;      // rows are missing at the end only
  const auto row_of = [&](int i) { return order[row0 + i * (64 / kLanes) + sub]; };
  f32x4 base[kRows][2];
  const float* base_at = a.base ? a.base : reinterpret_cast<const float*>(a.w);
  const bool has_base = a.base != nullptr;
  const auto load_base = [&](int block, bool there) {
    there = there && has_base;
    int col = block + wave_col + lane_col;
    col = col < end ? col : end - (kAligned ? 4 : 1);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int row = row_of(i);
      row = row < 0 ? order[0] : row;
      const float* p = base_at + (there ? (uint64_t)(uint32_t)row * (uint32_t)a.ldb + col : 0u);
      if constexpr (kAligned)
        base[i >> 1][i & 1] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
      else
        base[i >> 3][(i >> 2) & 1][i & 3] = *p;
    }
  };
  load_base(begin, true);

  // all blocks; kCheck: rows or columns may be missing
  const auto run = [&](auto check) {
    constexpr bool kCheck = decltype(check)::value;
    for (int block = begin; block < end; block += 128) {
      const int c0 = block + wave_col;
      const bool more = block + 128 < end;
      f32x4 acc[kRows][2];
#pragma unroll
      for (int i = 0; i < kRows; ++i) acc[i][0] = acc[i][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if constexpr (kDx) {
        if (block > begin) __syncthreads();
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int p = tid + i * kThreads, cb = p % 32, rb = p / 32;
          uint4 q[4];
          if (rank < kWide) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (rb * 8 + j >= rank) wp[i][j] = make_uint2(0, 0);
          }
          transpose8x4(wp[i], q);
          if (32 * kSlots % kThreads == 0 || rb < kSlots)
#pragma unroll
            for (int c = 0; c < 4; ++c) wt[lds_slot<kSlots>(cb * 4 + c, rb)] = q[c];
        }
        __syncthreads();
      } else {
        if (kShared && block > begin) __syncthreads();
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          uint4 v = wf[i];
          if (rank < a.rank) {
            if (piece_col[i] & 0x100) v = make_uint4(0, 0, 0, 0);
            if (piece_col[i] & 0x200) v = clear_from(v, rank & 7);
          }
          if ((piece_col[i] & 0xFF) < kSpan) wt[piece_at[i]] = v;
        }
        __builtin_amdgcn_wave_barrier();
        if (kShared) __syncthreads();
      }
      if (kAhead) load_w(block + 128, more);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if (s * 32 >= rank) break;
        uint4 f[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
          f[j] = wt[lds_slot<kSlots>(wave_col + 8 * (r16 >> 2) + 4 * j + (r16 & 3), 4 * s + g)];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const uint4 hi = terms[lds_slot<2 * kSlots>(row0 + i * 16 + r16, 4 * s + g)];
          const uint4 lo = terms[lds_slot<2 * kSlots>(row0 + i * 16 + r16, kSlots + 4 * s + g)];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            acc[i][j] = mfma16(f[j], lo, acc[i][j]);
            acc[i][j] = mfma16(f[j], hi, acc[i][j]);
          }
        }
      }
      if (!kAhead) load_w(block + 128, more);
      // An infinite W times a second term of zero, or of the other sign than
      // the first, is NaN where the product is infinite: what is NaN is made
      // again of the first terms, whose products have the infinities and NaN of
      // the whole.  To look costs nothing where memory bounds, and up to 1 of
      // 41 us where few waves with a rank above 128 wait for their products.
      bool lost = false;
#pragma unroll
      for (int e = 0; e < 8 * kRows; ++e) {
        const float v = acc[e >> 3][e >> 2 & 1][e & 3];
        lost |= v != v;
      }
      if (__builtin_expect(__any(lost), 0)) {
        int r = r16, k = g;        // opaque, so that the addresses are made here
        asm volatile("" : "+v"(r), "+v"(k));
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            f32x4 first = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (int s = 0; s * 32 < rank; ++s)
              first = mfma16(wt[lds_slot<kSlots>(wave_col + 8 * (r >> 2) + 4 * j + (r & 3), 4 * s + k)],
                             terms[lds_slot<2 * kSlots>(row0 + i * 16 + r, 4 * s + k)], first);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = acc[i][j][e] == acc[i][j][e] ? acc[i][j][e] : first[e];
          }
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        if constexpr (kDx) {
          if (a.drop.threshold) {
            const int row = order[row0 + i * 16 + r16], col = c0 + 8 * g;
            const uint4 d = block_draws((int64_t)row * (a.cols / 8) + col / 8, a.drop.key);
            const uint32_t u[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if ((e & 1 ? u[e >> 1] >> 16 : u[e >> 1] & 0xFFFFu) < a.drop.threshold)
                acc[i][e >> 2][e & 3] = 0.0f;
          }
        }
        f32x4* mine = turn + wave * 128;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < 2; ++j) mine[r16 * 8 + ((2 * g + j) ^ (r16 & 7))] = acc[i][j];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < kLoads / kRows; ++h) {
          const int q = h * (64 / kLanes) + sub;
          if constexpr (kAligned)
            acc[i][h] = mine[q * 8 + ((lane & 7) ^ (q & 7))];
          else
            acc[i][h >> 2][h & 3] = reinterpret_cast<const float*>(
                mine)[(q * 8 + ((lane_col >> 2) ^ (q & 7))) * 4 + (lane_col & 3)];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (has_base) acc[i][h] += base[i][h];
      }
      load_base(block + 128, more);
      const int col = c0 + lane_col;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = row_of(i);
        if (kCheck && (row < 0 || col >= end)) continue;
        const int64_t at = (int64_t)((uint64_t)(uint32_t)row * (uint32_t)a.ldo) + col;
        if constexpr (kAligned) {
          const f32x4 v = acc[i >> 1][i & 1];
          if constexpr (kOut16)
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at) = make_uint2(
                bf16_bits(v[0]) | bf16_bits(v[1]) << 16, bf16_bits(v[2]) | bf16_bits(v[3]) << 16);
          else
            __builtin_nontemporal_store(v, reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at));
        } else {
          const float v = acc[i >> 3][(i >> 2) & 1][i & 3];
          if constexpr (kOut16)
            static_cast<uint16_t*>(a.out)[at] = (uint16_t)bf16_bits(v);
          else
            static_cast<float*>(a.out)[at] = v;
        }
      }
    }
  };
  if (whole && (end - begin) % 128 == 0)
    run(std::false_type{});
  else
    run(std::true_type{});
}

}  // namespace mixfp4
