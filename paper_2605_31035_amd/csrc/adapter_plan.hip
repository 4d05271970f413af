// Rows grouped by their adapter: the plan that the adapter products share.
#include "adapter.h"

namespace mixfp4 {

namespace {

constexpr int kThreads = 1024;

// One workgroup per group (L adapters and the rows without one).  Each counts
// the rows of every group (runs of one group cost one LDS add), so that it
// knows where its tiles begin, and writes its rows in ascending order: the
// sums over a group's rows are then in a fixed order.  Bound by the latency of
// a thread's reads, twice m / 1024 of them one after the other: 4.3 us for 509
// rows, 5 for 2048, 14 to 19 for 16384 of up to 64 adapters, 46 of 1024, 92 to
// 140 for 131072 of 8.
__global__ __launch_bounds__(kThreads) void adapter_plan_kernel(const int32_t* index, int rows,
                                                                int adapters, int tile_rows,
                                                                int tiles_max, AdapterPlan plan) {
  extern __shared__ int hist[];              // adapters + 1
  __shared__ int wave_sum[kThreads / 64];
  const int tid = threadIdx.x, mine = blockIdx.x;
  for (int j = tid; j <= adapters; j += kThreads) hist[j] = 0;
  __syncthreads();
  const int per = (rows + kThreads - 1) / kThreads;
  const int64_t first64 = (int64_t)tid * per;
  const int first = first64 < rows ? (int)first64 : rows;
  const int last = rows - first < per ? rows : first + per;
  const auto group_of = [&](int i) {
    const int g = index[i];
    return g < 0 || g >= adapters ? adapters : g;
  };
  int run = -1, length = 0, own = 0;
  for (int i = first; i < last; ++i) {
    const int g = group_of(i);
    own += g == mine;
    if (g != run) {
      if (length) atomicAdd(&hist[run], length);
      run = g;
      length = 0;
    }
    ++length;
  }
  if (length) atomicAdd(&hist[run], length);
  __syncthreads();
  // tiles of the groups before this one
  int before = 0;
  for (int j = tid; j < mine; j += kThreads) before += (hist[j] + tile_rows - 1) / tile_rows;
  const int lane = tid & 63, wave = tid >> 6;
  for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
  if (lane == 0) wave_sum[wave] = before;
  __syncthreads();
  int base = 0;
  for (int w = 0; w < kThreads / 64; ++w) base += wave_sum[w];
  __syncthreads();
  // this thread's place among the rows of the group
  int upto = own;
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  int64_t at = (int64_t)base * tile_rows + upto - own;
  for (int w = 0; w < wave; ++w) at += wave_sum[w];
  if (own)
    for (int i = first; i < last; ++i)
      if (group_of(i) == mine) plan.order[at++] = i;
  const int count = hist[mine], tiles = (count + tile_rows - 1) / tile_rows;
  for (int i = count + tid; i < tiles * tile_rows; i += kThreads)
    plan.order[(int64_t)base * tile_rows + i] = -1;
  for (int i = tid; i < tiles; i += kThreads) plan.tile_adapter[base + i] = mine;
  if (tid == 0) plan.seg[mine] = base;
  if (mine == adapters) {
    if (tid == 0) plan.seg[adapters + 1] = base + tiles;
    for (int i = base + tiles + tid; i < tiles_max; i += kThreads) plan.tile_adapter[i] = -1;
  }
}

}  // namespace

// Rows of a tile: 16 where few rows meet an adapter, whose tiles of 64 would
// be mostly empty and too few to fill the device, and 64 where W is read less
// often so.  Forward and backward pass of a 4096 x 4096 layer, us, with 16 and
// with 64 rows: 255 rows of one adapter 17.8 and 19.8, 31.5 and 32.0; 512 rows
// 20.2 and 21.2, 35.9 and 36.6; 1024 rows of 32 adapters (rank 64) 28.8 and
// 32.4, 98 and 104; 4096 of 128 (rank 16) 49 and 53, 152 and 145.
int adapter_tile_rows(int64_t rows, int64_t adapters) {
  return rows <= 512 || rows <= 32 * adapters ? 16 : 64;
}

// ceil(c / T) summed over the groups is at most rows / T + groups, and at
// most one tile per row.
int64_t adapter_tiles_max(int64_t rows, int64_t adapters) {
  const int64_t t = rows / adapter_tile_rows(rows, adapters) + adapters + 1;
  return t < rows ? t : rows;
}

int64_t adapter_plan_bytes(int64_t rows, int64_t adapters) {
  const int64_t tiles = adapter_tiles_max(rows, adapters);
  const int64_t head = (adapters + 2 + tiles + 3) / 4 * 4;
  return 4 * (head + tiles * adapter_tile_rows(rows, adapters));
}

AdapterPlan adapter_plan_at(void* p, int64_t rows, int64_t adapters) {
  int32_t* w = static_cast<int32_t*>(p);
  const int64_t tiles = adapter_tiles_max(rows, adapters);
  return {w, w + adapters + 2, w + (adapters + 2 + tiles + 3) / 4 * 4};
}

hipError_t launch_adapter_plan(const int32_t* index, int64_t rows, int64_t adapters, void* plan,
                               hipStream_t stream) {
  adapter_plan_kernel<<<(unsigned)(adapters + 1), kThreads, 4 * (adapters + 1), stream>>>(
      index, (int)rows, (int)adapters, adapter_tile_rows(rows, adapters),
      (int)adapter_tiles_max(rows, adapters), adapter_plan_at(plan, rows, adapters));
  return hipGetLastError();
}

}  // namespace mixfp4
