// The gradients of the adapters: dA_l = sum u_i^T (keep_i x_i) and
// dB_l = sum dy_i^T t_i over the rows i of adapter l, products whose
// contraction runs along the rows.
#include "adapter.h"

namespace mixfp4 {

namespace {

constexpr int kThreads = 256;
constexpr int kCols = 128;     // columns of x or dy of a workgroup
constexpr int kDepth = 128;    // positions of a step
constexpr int kSlots = kDepth / 8;

// Positions of the pieces: whole tiles, split evenly over those in use.
__device__ __forceinline__ int64_t piece_begin(int64_t tiles, int s, int splits) {
  return tiles * s / splits;
}

// One workgroup: 128 columns, all of the rank, one piece of the positions.
// It walks the adapters that its piece holds.  Each step transposes 128
// positions x 128 columns through registers into LDS (8 x 8 per thread: eight
// 16-byte loads of eight rows, on which dropout's draws are made, one group
// each), so that an operand's 8 consecutive positions are one LDS read; the
// terms come transposed from the join.  An adapter within one piece is
// written at once, one across pieces as partial sums (at most two per piece:
// the one that enters it and the one that leaves it) for sum_kernel.
template <int kRank, bool kDb>
__global__ __launch_bounds__(kThreads) void grad_kernel(GradArgs a) {
  constexpr int kTiles = kRank / 16;
  __shared__ uint4 xt[kCols * kSlots];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r16 = lane & 15, g = lane >> 4;
  const int col0 = blockIdx.x * kCols;
  const int piece = blockIdx.y;
  const int64_t tiles = a.plan.seg[a.adapters];
  const int64_t t0 = piece_begin(tiles, piece, a.splits), t1 = piece_begin(tiles, piece + 1, a.splits);
  const int64_t matrix = (int64_t)a.rank * a.cols;
  const int cg = tid % 16, pg = tid / 16;
  const int col = col0 + cg * 8;

  f32x4 acc[kTiles][2];
  const auto store = [&](float* to) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      if constexpr (kDb) {
        const int r = 16 * i + 4 * g;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int n = col0 + wave * 32 + 16 * j + r16;
          if (n < a.cols && r < a.rank) *reinterpret_cast<f32x4*>(to + (int64_t)n * a.rank + r) = acc[i][j];
        }
      } else {
        const int r = 16 * i + r16, c = col0 + wave * 32 + 8 * g;
        if (r < a.rank && c < a.cols)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            *reinterpret_cast<f32x4*>(to + (int64_t)r * a.cols + c + 4 * j) = acc[i][j];
      }
    }
  };
  const auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) acc[i][0] = acc[i][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  };

  if (piece == 0)                  // adapters without rows
    for (int l = 0; l < a.adapters; ++l)
      if (a.plan.seg[l] == a.plan.seg[l + 1]) {
        clear();
        store(a.out + l * matrix);
      }
  if (t0 >= t1) return;
  for (int l = a.plan.tile_adapter[t0]; l < a.adapters && a.plan.seg[l] < t1; ++l) {
    const int64_t first = a.plan.seg[l], last = a.plan.seg[l + 1];
    if (first == last) continue;
    const int64_t p0 = (first > t0 ? first : t0) * a.tile_rows;
    const int64_t p1 = (last < t1 ? last : t1) * a.tile_rows;
    clear();
    for (int64_t p = p0; p < p1; p += kDepth) {
      uint4 v[8], q[8];
      const int64_t at = p + pg * 8;
      int row[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) row[j] = at < p1 ? a.plan.order[at + j] : -1;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = row[j] >= 0 ? load8(a.src + (int64_t)row[j] * a.ld, col, a.cols)
                           : make_uint4(0, 0, 0, 0);
      if (!kDb && a.drop.threshold)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (row[j] >= 0 && col < a.cols)
            v[j] = and4(v[j], keep_masks(block_draws((int64_t)row[j] * (a.cols / 8) + col / 8,
                                                     a.drop.key), a.drop.threshold));
      transpose8(v, q);
      __syncthreads();
#pragma unroll
      for (int c = 0; c < 8; ++c) xt[lds_slot<kSlots>(cg * 8 + c, pg)] = q[c];
      __syncthreads();
#pragma unroll
      for (int s = 0; s < kDepth / 32; ++s) {
        const int64_t pos = p + 32 * s + 8 * g;
        if (p + 32 * s >= p1) break;
        uint4 xf[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int c = kDb ? 16 * j + r16 : 8 * (r16 >> 2) + 4 * j + (r16 & 3);
          xf[j] = xt[lds_slot<kSlots>(wave * 32 + c, 4 * s + g)];
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
          const uint16_t* t = a.terms_t + (int64_t)(16 * i + r16) * a.positions + pos;
#pragma unroll
          for (int h = 2; h >= 0; --h) {             // the smallest term first
            const uint4 u = pos < p1 ? *reinterpret_cast<const uint4*>(t + (int64_t)h * kRank * a.positions)
                                     : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 2; ++j)
              acc[i][j] = kDb ? mfma16(u, xf[j], acc[i][j]) : mfma16(xf[j], u, acc[i][j]);
          }
        }
      }
    }
    if (first >= t0 && last <= t1)
      store(a.out + l * matrix);
    else
      store(a.part + (2 * piece + (first >= t0)) * matrix);
  }
}

// The adapters across pieces: their partial sums, in the order of the pieces.
__global__ __launch_bounds__(kThreads) void sum_kernel(GradArgs a) {
  const int l = blockIdx.y;
  const int64_t tiles = a.plan.seg[a.adapters];
  const int64_t first = a.plan.seg[l], last = a.plan.seg[l + 1];
  if (first == last) return;
  int s0 = 0, s1 = 0;
  for (int s = 1; s < a.splits; ++s) {
    const int64_t b = piece_begin(tiles, s, a.splits);
    if (b <= first) s0 = s;
    if (b < last) s1 = s;
  }
  if (s0 == s1) return;
  const int64_t matrix = (int64_t)a.rank * a.cols;
  for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4; i < matrix;
       i += (int64_t)gridDim.x * kThreads * 4) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = s0; s <= s1; ++s) {
      if (piece_begin(tiles, s, a.splits) == piece_begin(tiles, s + 1, a.splits)) continue;
      const int slot = 2 * s + (first >= piece_begin(tiles, s, a.splits));
      v += *reinterpret_cast<const f32x4*>(a.part + slot * matrix + i);
    }
    *reinterpret_cast<f32x4*>(a.out + l * matrix + i) = v;
  }
}

template <bool kDb>
void launch(const GradArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.cols + kCols - 1) / kCols), (unsigned)a.splits);
  switch (padded_rank(a.rank)) {
    case 16: grad_kernel<16, kDb><<<grid, kThreads, 0, stream>>>(a); break;
    case 32: grad_kernel<32, kDb><<<grid, kThreads, 0, stream>>>(a); break;
    case 64: grad_kernel<64, kDb><<<grid, kThreads, 0, stream>>>(a); break;
    case 128: grad_kernel<128, kDb><<<grid, kThreads, 0, stream>>>(a); break;
    default: grad_kernel<256, kDb><<<grid, kThreads, 0, stream>>>(a); break;
  }
}

}  // namespace

// Pieces of the positions: enough workgroups to fill the device, as long as
// the partial sums (8 bytes an element, written and read) stay below a
// quarter of src's bytes.
int adapter_grad_splits(int64_t m, int64_t cols, int64_t rank) {
  const int64_t blocks = (cols + kCols - 1) / kCols;
  int64_t s = (512 + blocks - 1) / blocks;
  if (s > m / (16 * rank)) s = m / (16 * rank);
  return s < 1 ? 1 : (int)s;
}

hipError_t launch_adapter_grad(const GradArgs& a, bool db, hipStream_t stream) {
  db ? launch<true>(a, stream) : launch<false>(a, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t blocks = ((int64_t)a.rank * a.cols + 4 * kThreads - 1) / (4 * kThreads);
  sum_kernel<<<dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)a.adapters), kThreads, 0,
               stream>>>(a);
  return hipGetLastError();
}

}  // namespace mixfp4
