// The wide products of the adapters: out = c + terms B_l^T and
// dx = dx0 + keep (terms A_l), where the terms are s_l t or s_l z u in two
// bf16 parts (adapter.h).
#include "adapter.h"

namespace mixfp4 {

namespace {

constexpr int kThreads = 256;
constexpr int kBlock32 = 32;   // columns of a wave's step

// One workgroup: one tile of rows, `width` columns.  The terms of the tile
// stand in LDS; a wave takes 32 columns at a time for all rows of the tile.
// W is the left operand of the matrix instructions, so that a lane of the
// result holds one row; of two instructions with columns 8 q + 0..3 and
// 8 q + 4..7 it holds 8 consecutive columns: 32 bytes of fp32, and one group
// of dropout's draws.
template <int kT, int kRank, bool kDx, bool kOut16>
__global__ __launch_bounds__(kThreads) void expand_kernel(ExpandArgs a, int width, bool aligned) {
  constexpr int kWide = kRank < 32 ? 32 : kRank;     // terms per part
  constexpr int kSteps = kWide / 32;
  constexpr int kRows = kT / 16;
  constexpr int kPitch = 2 * kWide / 8 + 1;          // 16-byte units; odd against bank conflicts
  constexpr int kSlots = kWide / 8;
  __shared__ uint4 terms[kT * kPitch];
  __shared__ uint4 wt[kDx ? 128 * kSlots : 1];
  const int tile = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r16 = lane & 15, g = lane >> 4;
  const int l = a.plan.tile_adapter[tile];
  if (l < 0) return;
  const bool none = l >= a.adapters;
  const int rank = none ? 0 : rank_of(a.ranks, l, a.rank);
  const int64_t p0 = (int64_t)tile * kT;
  if (rank > 0) {
    const uint4* from = reinterpret_cast<const uint4*>(a.terms + p0 * 2 * kWide);
    for (int i = tid; i < kT * (kPitch - 1); i += kThreads)
      terms[i / (kPitch - 1) * kPitch + i % (kPitch - 1)] = from[i];
    __syncthreads();
  }
  int rows[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) rows[i] = a.plan.order[p0 + i * 16 + r16];
  const uint16_t* w = a.w + (none ? 0 : (int64_t)l * a.rank * a.cols);
  const int begin = blockIdx.y * width;
  const int end = a.cols - begin < width ? a.cols : begin + width;

  for (int block = begin; block < end; block += 128) {
    if constexpr (kDx) {
      // A_l's columns block .. block + 128, transposed: [128][rank]
      if (rank > 0) {
        __syncthreads();
        for (int p = tid; p < 16 * kSlots; p += kThreads) {
          const int cb = p % 16, rb = p / 16;
          const int col = block + cb * 8;
          uint4 v[8], q[8];
#pragma unroll
          for (int j = 0; j < 8; ++j)
            v[j] = rb * 8 + j < rank && col < end
                       ? *reinterpret_cast<const uint4*>(w + (int64_t)(rb * 8 + j) * a.cols + col)
                       : make_uint4(0, 0, 0, 0);
          transpose8(v, q);
#pragma unroll
          for (int c = 0; c < 8; ++c) wt[lds_slot<kSlots>(cb * 8 + c, rb)] = q[c];
        }
        __syncthreads();
      }
    }
    const int c0 = block + wave * kBlock32;
    if (c0 >= end) continue;
    f32x4 acc[kRows][2];
#pragma unroll
    for (int i = 0; i < kRows; ++i) acc[i][0] = acc[i][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      if (s * 32 >= rank) break;
      uint4 wf[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int col = 8 * (r16 >> 2) + 4 * j + (r16 & 3);
        if constexpr (kDx) {
          wf[j] = wt[lds_slot<kSlots>(wave * kBlock32 + col, 4 * s + g)];
        } else {
          const int r = 32 * s + 8 * g;
          wf[j] = c0 + col < end && r < rank
                      ? clear_from(*reinterpret_cast<const uint4*>(
                                       w + (int64_t)(c0 + col) * a.rank + r), rank - r)
                      : make_uint4(0, 0, 0, 0);
        }
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const uint4 hi = terms[(i * 16 + r16) * kPitch + 4 * s + g];
        const uint4 lo = terms[(i * 16 + r16) * kPitch + kSlots + 4 * s + g];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          acc[i][j] = mfma16(wf[j], lo, acc[i][j]);
          acc[i][j] = mfma16(wf[j], hi, acc[i][j]);
        }
      }
    }
    const int col = c0 + 8 * g;
    const int valid = end - col < 8 ? end - col : 8;
    const bool wide = aligned && valid == 8;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      if (rows[i] < 0 || valid <= 0) continue;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = acc[i][e >> 2][e & 3];
      if constexpr (kDx) {
        if (a.drop.threshold) {
          const uint4 d = block_draws((int64_t)rows[i] * (a.cols / 8) + col / 8, a.drop.key);
          const uint32_t u[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if ((e & 1 ? u[e >> 1] >> 16 : u[e >> 1] & 0xFFFFu) < a.drop.threshold) v[e] = 0.0f;
        }
      }
      if (a.base) {
        const float* base = a.base + (int64_t)rows[i] * a.ldb + col;
        if (wide) {
          const f32x4 b0 = reinterpret_cast<const f32x4*>(base)[0];
          const f32x4 b1 = reinterpret_cast<const f32x4*>(base)[1];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += e < 4 ? b0[e & 3] : b1[e & 3];
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < valid) v[e] += base[e];
        }
      }
      const int64_t at = (int64_t)rows[i] * a.ldo + col;
      if constexpr (kOut16) {
        uint16_t* out = static_cast<uint16_t*>(a.out) + at;
        uint32_t b[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = bf16_bits(v[e]);
        if (wide) {
          *reinterpret_cast<uint4*>(out) = make_uint4(b[0] | b[1] << 16, b[2] | b[3] << 16,
                                                      b[4] | b[5] << 16, b[6] | b[7] << 16);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < valid) out[e] = (uint16_t)b[e];
        }
      } else {
        float* out = static_cast<float*>(a.out) + at;
        if (wide) {
          reinterpret_cast<f32x4*>(out)[0] = f32x4{v[0], v[1], v[2], v[3]};
          reinterpret_cast<f32x4*>(out)[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < valid) out[e] = v[e];
        }
      }
    }
  }
}

template <int kT, bool kDx, bool kOut16>
void launch(const ExpandArgs& a, int64_t tiles, int width, bool aligned, hipStream_t stream) {
  const dim3 grid((unsigned)tiles, (unsigned)((a.cols + width - 1) / width));
  switch (padded_rank(a.rank)) {
    case 16: expand_kernel<kT, 16, kDx, kOut16><<<grid, kThreads, 0, stream>>>(a, width, aligned); break;
    case 32: expand_kernel<kT, 32, kDx, kOut16><<<grid, kThreads, 0, stream>>>(a, width, aligned); break;
    case 64: expand_kernel<kT, 64, kDx, kOut16><<<grid, kThreads, 0, stream>>>(a, width, aligned); break;
    case 128: expand_kernel<kT, 128, kDx, kOut16><<<grid, kThreads, 0, stream>>>(a, width, aligned); break;
    default: expand_kernel<kT, 256, kDx, kOut16><<<grid, kThreads, 0, stream>>>(a, width, aligned); break;
  }
}

}  // namespace

hipError_t launch_adapter_expand(const ExpandArgs& a, int tile_rows, int64_t tiles, bool dx,
                                 bool out16, hipStream_t stream) {
  // columns per workgroup: wide enough that the terms are read seldom, as
  // long as the device stays full
  int64_t width = (a.cols * tiles / 1024 + 127) / 128 * 128;
  if (width < 128) width = 128;
  if (width > 1024) width = 1024;
  const bool aligned = ((uintptr_t)a.out & 15) == 0 && a.ldo % (out16 ? 8 : 4) == 0 &&
                       (!a.base || (((uintptr_t)a.base & 15) == 0 && a.ldb % 4 == 0));
  const bool small = tile_rows == 16;
  const int wd = (int)width;
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
