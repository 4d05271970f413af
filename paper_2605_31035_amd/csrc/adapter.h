// Low-rank adapters beside a shared projection: shared pieces of the kernels.
//
// Row i of x has adapter l = index[i] (none outside [0, L)).  With rank
// r_l <= R, A_l [R, K], B_l [n, R], scaling s_l, dropout's keep mask on x and
// z = 1 / (1 - p):
//   t_i  = z (keep_i x_i) A_l^T             out_i = c_i + s_l t_i B_l^T
//   u_i  = s_l dy_i B_l                     dx_i  = dx0_i + z keep_i (u_i A_l)
//   dA_l = z sum_i u_i^T (keep_i x_i)       dB_l  = s_l sum_i dy_i^T t_i
// Every product runs on v_mfma_f32_16x16x32_bf16.  x, dy, A and B are bf16
// and exact there.  t and u are fp32 sums; as operands they are carried as
// bf16 terms.  Two terms in the products that a matrix is added to (out, dx):
// |t - hi - lo| <= 2^-17 |t| (2^e <= |t|: a step of hi is 2^(e-7), the rest at
// most 2^(e-8) and its own step below that 2^(e-16); 2^-16.9 where t is above
// the largest bf16), about 2^-19 in the mean.
// Three in dA and dB, which stand alone: they hold t's 24 bits.  With two the
// gradients were 2.5e-6 from the exact ones, where fp32 operands give 3e-7
// (333 rows) to 2e-6 (8192 rows).
//
// Rows are grouped by adapter into tiles of T rows (AdapterPlan): a position
// is tile * T + row in the tile, and order[position] is the row of x or -1.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"
#include "philox.h"

namespace mixfp4 {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t bf16_bits(float v) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v);
}

// v = hi + lo in bf16; an infinity or NaN stays whole in hi.  A finite v above
// the largest bf16, which rounds to infinity, takes that one.
__device__ __forceinline__ void split_bf16(float v, uint32_t& hi, uint32_t& lo) {
  const bool finite = fabsf(v) < __builtin_huge_valf();
  hi = bf16_bits(v);
  if (finite && (hi & 0x7F80u) == 0x7F80u) --hi;
  const float h = __uint_as_float(hi << 16);
  lo = finite ? bf16_bits(v - h) : 0u;
}

// v = a[0] + a[1] + a[2], exactly, none of them zero unless v is and all of
// v's sign: an infinite operand's products with them are infinite where its
// product with v is.  v's 24 bits give up to three terms of eight; where there
// are fewer, the first is taken in parts.  An infinity or NaN stands in all
// three.  (Below 2^-109 the last step of bf16, 2^-133, bounds it.)
__device__ __forceinline__ void split_bf16(float v, uint32_t (&a)[3]) {
  const float first = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u), rest = v - first;
  const float second = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u), third = rest - second;
  float t[3] = {first, second, third};
  if (third == 0.0f) {
    t[0] = 0.5f * first;
    t[1] = second == 0.0f ? 0.25f * first : 0.5f * first;
    t[2] = second == 0.0f ? 0.25f * first : second;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e) a[e] = bf16_bits(fabsf(v) < __builtin_huge_valf() ? t[e] : v);
}

// The keep bits of 8 consecutive elements from their group's draws: element e
// takes the low (e even) or high half of word e / 2 and is kept from the
// threshold on.  Returned as masks of the four words of packed bf16 pairs.
__device__ __forceinline__ uint4 keep_masks(uint4 d, uint32_t threshold) {
  const auto m = [&](uint32_t w) {
    return ((w & 0xFFFFu) >= threshold ? 0xFFFFu : 0u) | ((w >> 16) >= threshold ? 0xFFFF0000u : 0u);
  };
  return make_uint4(m(d.x), m(d.y), m(d.z), m(d.w));
}
__device__ __forceinline__ uint4 and4(uint4 a, uint4 b) {
  return make_uint4(a.x & b.x, a.y & b.y, a.z & b.z, a.w & b.w);
}

// 8 bf16 of a row from column `col` on; columns from `cols` on are zero and
// not read.
__device__ __forceinline__ uint4 load8(const uint16_t* row, int col, int cols) {
  if (col + 8 <= cols) return *reinterpret_cast<const uint4*>(row + col);
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (col + e < cols) w[e >> 1] |= (uint32_t)row[col + e] << (16 * (e & 1));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Waits for all of the wave's loads: at the end of a branch that loads, so
// that the code behind it need not wait on its account (s_waitcnt vmcnt(0),
// the other counters at their maximum).
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// 8 bf16 with those from element `valid` on cleared.
__device__ __forceinline__ uint4 clear_from(uint4 v, int valid) {
  if (valid >= 8) return v;
  const auto m = [&](uint32_t w, int e) {
    return w & ((valid > e ? 0xFFFFu : 0u) | (valid > e + 1 ? 0xFFFF0000u : 0u));
  };
  return make_uint4(m(v.x, 0), m(v.y, 2), m(v.z, 4), m(v.w, 6));
}

// Transpose of 8 x 8 bf16: v[j] row j in, column c out in w[c].
__device__ __forceinline__ void transpose8(const uint4 (&v)[8], uint4 (&w)[8]) {
  const auto word = [](const uint4& q, int i) { return i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w; };
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const uint32_t sel = (c & 1) ? 0x07060302u : 0x05040100u;   // high or low halves of two rows
    w[c] = make_uint4(__builtin_amdgcn_perm(word(v[1], c >> 1), word(v[0], c >> 1), sel),
                      __builtin_amdgcn_perm(word(v[3], c >> 1), word(v[2], c >> 1), sel),
                      __builtin_amdgcn_perm(word(v[5], c >> 1), word(v[4], c >> 1), sel),
                      __builtin_amdgcn_perm(word(v[7], c >> 1), word(v[6], c >> 1), sel));
  }
}

// Transpose of 8 rows of 4 bf16: column c out in w[c].
__device__ __forceinline__ void transpose8x4(const uint2 (&v)[8], uint4 (&w)[4]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t sel = (c & 1) ? 0x07060302u : 0x05040100u;
    const auto word = [&](int j) { return c < 2 ? v[j].x : v[j].y; };
    w[c] = make_uint4(__builtin_amdgcn_perm(word(1), word(0), sel),
                      __builtin_amdgcn_perm(word(3), word(2), sel),
                      __builtin_amdgcn_perm(word(5), word(4), sel),
                      __builtin_amdgcn_perm(word(7), word(6), sel));
  }
}

// LDS tiles of rows of kSlots 16-byte slots: slot s of row r stands at s ^
// key(r), so that 8 consecutive rows at one slot (operand reads) fall into
// different banks.  The key depends on r mod 16 alone, so that the tiles of
// 16 rows differ by a constant that the read instruction adds; rows r, r + 4,
// ... at one slot (writes of transposed 8 x 4 blocks) still meet four banks.
template <int kSlots>
__device__ __forceinline__ int lds_slot(int row, int slot) {
  return row * kSlots + (slot ^ ((row ^ (row >> 2 & 2)) & (kSlots - 1)));
}
// The same for tiles written in transposed 8 x 8 blocks: rows r, r + 8, ...
// at one slot fall into different banks too.
template <int kSlots>
__device__ __forceinline__ int lds_slot8(int row, int slot) {
  return row * kSlots + (slot ^ ((row ^ (row >> 3)) & (kSlots - 1)));
}

__device__ __forceinline__ int rank_of(const int32_t* ranks, int l, int rank) {
  if (!ranks) return rank;
  const int r = ranks[l];
  return r < 0 ? 0 : r > rank ? rank : r;
}

// A grid of `across` workgroups per tile, those of one tile side by side: the
// rows of a matrix often lie a multiple of some KB apart, and workgroups that
// read all rows at the same columns at the same time meet in few memory
// channels.
inline dim3 tile_grid(int64_t across, int64_t tiles) {
  const int64_t y = tiles < 32768 ? tiles : 32768;
  return dim3((unsigned)across, (unsigned)y, (unsigned)((tiles + y - 1) / y));
}

}  // namespace mixfp4
