// Kernels of the adapters' wide products (adapter_expand.h).
#include "adapter_expand.h"

namespace mixfp4 {

namespace {

template <int kT, int kRank, bool kDx, bool kOut16, bool kAligned, bool kJoin>
__global__ __launch_bounds__(threads_of(kT, kRank, kDx), waves_of(kT, kRank, kDx)) void expand_kernel(
    ExpandArgs a, int width, int tiles) {
  __shared__ uint4 lds[expand_lds(kT, kRank, kDx)];
  const int tile = blockIdx.z * gridDim.y + blockIdx.y;
  if (tile < tiles)
    expand_body<kT, kRank, kDx, kOut16, kAligned, kJoin>(a, width, tile, blockIdx.x, lds);
}

template <int kT, bool kDx, bool kOut16, bool kAligned, bool kJoin = false>
void launch(const ExpandArgs& a, int64_t tiles, int width, hipStream_t stream) {
  const dim3 grid = tile_grid((a.cols + width - 1) / width, tiles);
  const int n = (int)tiles;
  const auto go = [&](auto rank) {
    constexpr int kRank = decltype(rank)::value;
    expand_kernel<kT, kRank, kDx, kOut16, kAligned, kJoin>
        <<<grid, threads_of(kT, kRank, kDx), 0, stream>>>(a, width, n);
  };
  switch (padded_rank(a.rank)) {
    case 16: go(std::integral_constant<int, 16>{}); break;
    case 32: go(std::integral_constant<int, 32>{}); break;
    case 64: go(std::integral_constant<int, 64>{}); break;
    case 128: go(std::integral_constant<int, 128>{}); break;
    default: go(std::integral_constant<int, 256>{}); break;
  }
}

template <int kT, bool kDx, bool kOut16>
void launch(const ExpandArgs& a, int64_t tiles, int width, bool aligned, hipStream_t stream) {
  if constexpr (kT == 16 && !kDx) {
    if (a.part) {
      aligned ? launch<kT, kDx, kOut16, true, true>(a, tiles, width, stream)
              : launch<kT, kDx, kOut16, false, true>(a, tiles, width, stream);
      return;
    }
  }
  aligned ? launch<kT, kDx, kOut16, true>(a, tiles, width, stream)
          : launch<kT, kDx, kOut16, false>(a, tiles, width, stream);
}

}  // namespace

// Whether the wide product joins the pieces itself: every workgroup of a tile
// then reads them, which beats the join's launch (4.7 us) as long as that is
// little, up to 4 MB in all (17 MB cost 6.6 us).
bool adapter_expand_joins(int64_t m, int64_t n, int64_t rank, int tile_rows, int splits) {
  return tile_rows == 16 && (n + 127) / 128 * m * rank * 4 * splits <= (int64_t(4) << 20);
}

int adapter_expand_width(const ExpandArgs& a, int tile_rows, int64_t tiles, bool dx) {
  // Blocks of 128 columns per workgroup: several, so that the terms are read
  // seldom and a block's memory is requested under the one before, as long as
  // the device stays full.  A rank above 128 leaves room for one workgroup per
  // compute unit: as many as there are units (the forward pass of
  // 1537x4096x4096 rank 256: 55 us with one block each, 46 with four, 49 with
  // five).  Else two (that of 8192x4096x14336 rank 64: 200 us with one, 191 with
  // two, 204 with three), one below 6000 workgroups (2048x4096x11008: the same
  // with one to three); the input gradient pays more for a workgroup's start
  // (by itself 8192x4096: 62 us with one, 56 with two).  Tiles of 16 rows: 1024
  // workgroups (the pass of 48x4096x11008 rank 64: 22 us with one, 19 with three).
  const bool small = tile_rows == 16;
  const int64_t blocks = (a.cols + 127) / 128, units = blocks * tiles;
  int64_t w;
  if (small)
    w = units / 1024 < 4 ? units / 1024 : 4;
  else if (padded_rank(a.rank) > 128)
    w = (units + compute_units() - 1) / compute_units();
  else
    w = units >= (dx ? 3000 : 6000) ? 2 : 1;
  if (w > 8) w = 8;
  return 128 * (w < 1 ? 1 : (int)w);
}

// 16-byte accesses of the base and the result: every row begins on 16 bytes
// (8 for a bf16 result) and holds whole pieces.
bool adapter_expand_aligned(const ExpandArgs& a, bool out16) {
  return a.cols % 4 == 0 && ((uintptr_t)a.out & (out16 ? 7 : 15)) == 0 && a.ldo % 4 == 0 &&
         (!a.base || (((uintptr_t)a.base & 15) == 0 && a.ldb % 4 == 0));
}

hipError_t launch_adapter_expand(const ExpandArgs& a, int tile_rows, int64_t tiles, bool dx,
                                 bool out16, hipStream_t stream) {
  const bool small = tile_rows == 16, aligned = adapter_expand_aligned(a, out16);
  const int wd = adapter_expand_width(a, tile_rows, tiles, dx);
  if (dx) {
    small ? launch<16, true, false>(a, tiles, wd, aligned, stream)
          : launch<64, true, false>(a, tiles, wd, aligned, stream);
  } else if (out16) {
    small ? launch<16, false, true>(a, tiles, wd, aligned, stream)
          : launch<64, false, true>(a, tiles, wd, aligned, stream);
  } else {
    small ? launch<16, false, false>(a, tiles, wd, aligned, stream)
          : launch<64, false, false>(a, tiles, wd, aligned, stream);
  }
  return hipGetLastError();
}

}  // namespace mixfp4
