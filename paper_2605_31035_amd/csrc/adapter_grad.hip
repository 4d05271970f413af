// Kernels of the backward pass behind the join: the input gradient
// (adapter_expand.h) and the adapters' gradients (adapter_grad.h).
#include "adapter_expand.h"
#include "adapter_grad.h"

namespace mixfp4 {

namespace {

constexpr int kSumThreads = 256;

// The gradients of a rank above 64 by themselves: their sums and dx's take
// the registers of one compute unit each.
__global__ __launch_bounds__(kGradThreads, 2) void grad_kernel(GradArgs q) {
  __shared__ uint4 lds[grad_lds(128)];
  grad_block<128>(q, blockIdx.x, blockIdx.y * 128, lds);
}

// The adapters across pieces: their partial sums, in the order of the pieces.
__global__ __launch_bounds__(kSumThreads) void sum_kernel(GradArgs q) {
  const GradSide& a = blockIdx.z ? q.b : q.a;
  const int l = blockIdx.y;
  const int64_t tiles = q.plan.seg[q.adapters];
  const int64_t first = q.plan.seg[l], last = q.plan.seg[l + 1];
  if (first == last) return;
  int s0 = 0, s1 = 0;
  for (int s = 1; s < q.splits; ++s) {
    const int64_t b = piece_begin(tiles, s, q.splits);
    if (b <= first) s0 = s;
    if (b < last) s1 = s;
  }
  if (s0 == s1) return;
  const int64_t matrix = (int64_t)q.rank * a.cols;
  for (int64_t i = ((int64_t)blockIdx.x * kSumThreads + threadIdx.x) * 4; i < matrix;
       i += (int64_t)gridDim.x * kSumThreads * 4) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    // eight reads at a time; pieces without tiles hold nothing
    for (int s = s0; s <= s1; s += 8) {
      f32x4 u[8];
      bool there[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int t = s + e <= s1 ? s + e : s1;
        const int64_t begin = piece_begin(tiles, t, q.splits);
        there[e] = s + e <= s1 && begin < piece_begin(tiles, t + 1, q.splits);
        const int slot = there[e] ? 2 * t + (first >= begin) : 2 * s1;   // s1's is there: it enters
        u[e] = *reinterpret_cast<const f32x4*>(a.part + slot * matrix + i);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (there[e]) v += u[e];
    }
    *reinterpret_cast<f32x4*>(a.out + l * matrix + i) = v;
  }
}

// Workgroups of a launch: dx's (`across` per tile) and the gradients'.
struct Wide {
  int width, across, dxs, grads;
};

// dx and the gradients in one launch: dx is bound by memory, the gradients
// wait for their rows and multiply, so side by side they take less than in
// turn.  The gradients' workgroups, which run long, are spread evenly over the
// front of the launch, among the first quarter of dx's (the whole pass at
// 8192x14336x4096 rank 64: 226 us in turn, 208 so, 225 among the first half,
// 244 among seven eighths; 2048x11008x4096 rank 16: 65, 55.6, 58, 64).
template <int kT, int kRank, bool kAligned>
__global__ __launch_bounds__(kGradThreads, 2) void backward_kernel(ExpandArgs x, GradArgs q, Wide w) {
  constexpr int kDx = expand_lds(kT, kRank, true), kGrad = grad_lds(kRank);
  __shared__ uint4 lds[kDx > kGrad ? kDx : kGrad];
  const uint64_t b = blockIdx.x, front = (uint64_t)w.grads + w.dxs / 4;
  if (b < front) {
    const int before = (int)(b * w.grads / front), behind = (int)((b + 1) * w.grads / front);
    if (behind > before) {
      grad_block<kRank>(q, before, 0, lds);
      return;
    }
    const int i = (int)b - before;
    expand_body<kT, kRank, true, false, kAligned, false>(x, w.width, i / w.across, i % w.across, lds);
  } else {
    const int i = (int)b - w.grads;
    expand_body<kT, kRank, true, false, kAligned, false>(x, w.width, i / w.across, i % w.across, lds);
  }
}

template <int kT, bool kAligned>
void launch(const ExpandArgs& x, const GradArgs& q, const Wide& w, hipStream_t stream) {
  const unsigned grid = (unsigned)(w.dxs + w.grads);
  switch (padded_rank(q.rank)) {
    case 16: backward_kernel<kT, 16, kAligned><<<grid, kGradThreads, 0, stream>>>(x, q, w); break;
    case 32: backward_kernel<kT, 32, kAligned><<<grid, kGradThreads, 0, stream>>>(x, q, w); break;
    default: backward_kernel<kT, 64, kAligned><<<grid, kGradThreads, 0, stream>>>(x, q, w); break;
  }
}

int64_t blocks_of(int64_t cols, int64_t rank) {
  const int c = cols_of(padded_rank(rank));
  return (cols + c - 1) / c;
}

}  // namespace

// Pieces of the positions.  More of them fill the device, in whole rounds of
// two workgroups per compute unit at best, and write and read more partial
// sums: 8 bytes an element of the gradients against 2 an element of x and dy.
int adapter_grad_splits(int64_t m, int64_t n, int64_t k, int64_t rank) {
  const int64_t blocks = (blocks_of(n, rank) + blocks_of(k, rank)) * (rank > 128 ? 2 : 1);
  const int64_t round = 2 * compute_units();
  int best = 1;
  double score = 0.0;
  for (int64_t s = 1; s <= 64 && (s == 1 || s * 64 <= m); ++s) {
    const int64_t groups = blocks * s;
    const double full = (double)groups / (double)((groups + round - 1) / round * round);
    const double v = full / (1.0 + (s > 1 ? (double)(s * rank * 4) / (double)m : 0.0));
    if (v > 1.02 * score) {
      score = v;
      best = (int)s;
    }
  }
  return best;
}

// The backward pass behind the join: dx and both gradients.  With a rank up to
// 64 in one launch.
hipError_t launch_adapter_grad(const GradArgs& q, const ExpandArgs& dx, int tile_rows, int64_t tiles,
                               hipStream_t stream) {
  const int64_t grads = (blocks_of(q.a.cols, q.rank) + blocks_of(q.b.cols, q.rank)) * q.splits;
  hipError_t e = hipSuccess;
  if (q.rank > 64) {
    if (tiles > 0) e = launch_adapter_expand(dx, tile_rows, tiles, true, false, stream);
    if (e != hipSuccess) return e;
    grad_kernel<<<dim3((unsigned)grads, q.rank > 128 ? 2 : 1), kGradThreads, 0, stream>>>(q);
  } else {
    const int width = tiles > 0 ? adapter_expand_width(dx, tile_rows, tiles, true) : 128;
    int64_t across = (dx.cols + width - 1) / width;
    const bool together = across * tiles < (1 << 23);     // workgroups of one launch
    if (!together) {
      e = launch_adapter_expand(dx, tile_rows, tiles, true, false, stream);
      if (e != hipSuccess) return e;
      across = 0;
    }
    const Wide w{width, (int)across, (int)(across * tiles), (int)grads};
    const bool aligned = adapter_expand_aligned(dx, false);
    if (tile_rows == 16)
      aligned ? launch<16, true>(dx, q, w, stream) : launch<16, false>(dx, q, w, stream);
    else
      aligned ? launch<64, true>(dx, q, w, stream) : launch<64, false>(dx, q, w, stream);
  }
  e = hipGetLastError();
  if (e != hipSuccess || q.splits == 1) return e;
  const int64_t cols = q.a.cols > q.b.cols ? q.a.cols : q.b.cols;
  const int64_t blocks = ((int64_t)q.rank * cols + 4 * kSumThreads - 1) / (4 * kSumThreads);
  sum_kernel<<<dim3((unsigned)(blocks < 1024 ? blocks : 1024), (unsigned)q.adapters, 2), kSumThreads, 0,
               stream>>>(q);
  return hipGetLastError();
}

}  // namespace mixfp4
