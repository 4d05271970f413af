// The launches of one forward or backward pass of the adapters, and their
// workspace.
#include "internal.h"

namespace mixfp4 {

namespace {

// Hands out pieces of the workspace, 256-byte aligned.
struct Carver {
  uint8_t* at;
  int64_t used = 0;
  template <typename T>
  T* take(int64_t bytes) {
    T* p = reinterpret_cast<T*>(at + used);
    used += (bytes + 255) / 256 * 256;
    return p;
  }
};

struct Pass {
  int tile_rows;
  int64_t tiles, positions;
  int padded, width;                       // terms: padded rank, at least 32 of them
  int splits, grad_splits;
  float *part, *part_a, *part_b;
  uint16_t *terms, *terms_t, *t_t;
  int64_t bytes;

  Pass(int64_t m, int64_t n, int64_t k, int64_t rank, int64_t adapters, bool backward, void* ws) {
    tile_rows = adapter_tile_rows(m, adapters);
    tiles = adapter_tiles_max(m, adapters);
    positions = tiles * tile_rows;
    padded = padded_rank(rank);
    width = padded < 32 ? 32 : padded;
    splits = adapter_shrink_splits(tiles, backward ? n : k, rank);
    grad_splits = backward ? adapter_grad_splits(m, n, k, rank) : 1;
    Carver c{static_cast<uint8_t*>(ws)};
    part = c.take<float>(4 * splits * positions * rank);
    terms = c.take<uint16_t>(4 * positions * width);
    terms_t = t_t = nullptr;
    part_a = part_b = nullptr;
    if (backward) {
      terms_t = c.take<uint16_t>(6 * positions * padded);
      t_t = c.take<uint16_t>(6 * positions * padded);
      if (grad_splits > 1) {
        part_a = c.take<float>(8 * grad_splits * rank * k);
        part_b = c.take<float>(8 * grad_splits * rank * n);
      }
    }
    bytes = c.used;
  }
};

}  // namespace

int64_t adapter_workspace(int64_t m, int64_t n, int64_t k, int64_t rank, int64_t adapters,
                          bool backward) {
  return Pass(m, n, k, rank, adapters, backward, nullptr).bytes;
}

hipError_t launch_adapter(const AdapterArgs& a, hipStream_t stream) {
  const Pass p(a.m, a.n, a.k, a.rank, a.adapters, false, a.workspace);
  const int rank = (int)a.rank, adapters = (int)a.adapters;
  hipError_t e = launch_adapter_shrink(
      {a.x, a.ldx, a.a, a.ranks, a.plan, a.drop, (int)a.k, rank, adapters, p.splits, p.positions, p.part},
      p.tile_rows, p.tiles, false, stream);
  if (e != hipSuccess) return e;
  ExpandArgs x{};
  x.w = a.b, x.ranks = a.ranks, x.plan = a.plan, x.base = a.c, x.ldb = a.ldc, x.out = a.out;
  x.ldo = a.ldo, x.cols = (int)a.n, x.rank = rank, x.adapters = adapters;
  if (adapter_expand_joins(a.m, a.n, rank, p.tile_rows, p.splits)) {
    x.part = p.part, x.scaling = a.scaling, x.t = a.t;
    x.positions = p.positions, x.splits = p.splits, x.z = a.drop.z;
  } else {
    JoinArgs j{};
    j.part = p.part, j.scaling = a.scaling, j.ranks = a.ranks, j.plan = a.plan;
    j.positions = p.positions, j.rank = rank, j.adapters = adapters, j.splits = p.splits;
    j.z = a.drop.z, j.terms = p.terms, j.t = a.t;
    e = launch_adapter_join(j, p.tile_rows, stream);
    if (e != hipSuccess) return e;
    x.terms = p.terms;
  }
  return launch_adapter_expand(x, p.tile_rows, p.tiles, false, a.out16, stream);
}

hipError_t launch_adapter_backward(const AdapterArgs& a, hipStream_t stream) {
  const Pass p(a.m, a.n, a.k, a.rank, a.adapters, true, a.workspace);
  const int rank = (int)a.rank, adapters = (int)a.adapters;
  const GradArgs grad{{a.x, a.ldx, p.terms_t, p.part_a, a.da, (int)a.k},
                      {a.dy, a.lddy, p.t_t, p.part_b, a.db, (int)a.n},
                      a.ranks, a.plan, a.drop, p.positions, rank, p.padded, adapters, p.grad_splits, p.tile_rows};
  ExpandArgs x{};
  x.terms = p.terms, x.w = a.a, x.ranks = a.ranks, x.plan = a.plan, x.drop = a.drop;
  x.base = a.dx0, x.ldb = a.lddx0, x.out = a.dx, x.ldo = a.lddx;
  x.cols = (int)a.k, x.rank = rank, x.adapters = adapters;
  if (a.m > 0) {                            // else gradients of zero
    hipError_t e = launch_adapter_shrink(
        {a.dy, a.lddy, a.b, a.ranks, a.plan, {}, (int)a.n, rank, adapters, p.splits, p.positions, p.part},
        p.tile_rows, p.tiles, true, stream);
    if (e != hipSuccess) return e;
    JoinArgs j{};
    j.part = p.part, j.scaling = a.scaling, j.ranks = a.ranks, j.plan = a.plan;
    j.positions = p.positions, j.rank = rank, j.adapters = adapters, j.splits = p.splits;
    j.z = a.drop.z, j.terms = p.terms, j.terms_t = p.terms_t, j.t_in = a.t, j.t_in_t = p.t_t;
    e = launch_adapter_join(j, p.tile_rows, stream);
    if (e != hipSuccess) return e;
  }
  return launch_adapter_grad(grad, x, p.tile_rows, p.tiles, stream);
}

}  // namespace mixfp4
