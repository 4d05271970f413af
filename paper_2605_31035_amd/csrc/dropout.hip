// Dropout from a counter-based generator: y = residual + z keep x.
//
// Element (i, j) of a [rows, k] matrix is kept when its 16-bit draw is at
// least threshold = round(65536 p); z = 65536 / (65536 - threshold).  Its
// draw is half j % 2 of word (j % 8) / 2 of Philox4x32-10 under the key
// `seed` and the counter (i ceil(k / 8) + j / 8, offset), so no mask is
// stored, and the backward pass is the same call on the gradient.  16 bits
// an element let one call of the generator serve 8 elements and put p within
// 2^-17 of the wanted one.
#include "adapter.h"
#include "formats.h"

namespace mixfp4 {

namespace {

constexpr int kThreads = 256;

template <bool kBf16>
__device__ __forceinline__ void load_values(const void* p, int64_t at, int valid, bool wide,
                                            float (&v)[8]) {
  if constexpr (kBf16) {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (wide) {
      const uint4 w = *reinterpret_cast<const uint4*>(q);
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = bf16_lo(u[e]);
        v[2 * e + 1] = bf16_hi(u[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < valid ? __uint_as_float((uint32_t)q[e] << 16) : 0.0f;
    }
  } else {
    const float* q = static_cast<const float*>(p) + at;
    if (wide) {
      const float4 a = reinterpret_cast<const float4*>(q)[0];
      const float4 b = reinterpret_cast<const float4*>(q)[1];
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
      v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < valid ? q[e] : 0.0f;
    }
  }
}

template <bool kBf16>
__device__ __forceinline__ void store_values(void* p, int64_t at, int valid, bool wide,
                                             const float (&v)[8]) {
  if constexpr (kBf16) {
    uint16_t* q = static_cast<uint16_t*>(p) + at;
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = bf16_bits(v[e]);
    if (wide) {
      *reinterpret_cast<uint4*>(q) = make_uint4(b[0] | b[1] << 16, b[2] | b[3] << 16,
                                                b[4] | b[5] << 16, b[6] | b[7] << 16);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < valid) q[e] = (uint16_t)b[e];
    }
  } else {
    float* q = static_cast<float*>(p) + at;
    if (wide) {
      reinterpret_cast<float4*>(q)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(q)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < valid) q[e] = v[e];
    }
  }
}

// One thread per group of 8 elements.  kResidual: 0 none, 1 fp32, 2 bf16.
template <bool kX16, int kResidual, bool kOut16>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a, uint32_t groups,
                                                           int64_t total, bool aligned) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * kThreads) {
    const int64_t row = i / groups;
    const int64_t col = (i - row * groups) * 8;
    const int valid = a.k - col < 8 ? (int)(a.k - col) : 8;
    const bool wide = aligned && valid == 8;
    float v[8], r[8];
    load_values<kX16>(a.x, row * a.ldx + col, valid, wide, v);
    if constexpr (kResidual != 0)
      load_values<kResidual == 2>(a.residual, row * a.ldr + col, valid, wide, r);
    uint32_t d[4] = {0u, 0u, 0u, 0u};
    if (a.drop.threshold) {
      const uint4 w = block_draws(i, a.drop.key);
      d[0] = w.x, d[1] = w.y, d[2] = w.z, d[3] = w.w;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t u = e & 1 ? d[e >> 1] >> 16 : d[e >> 1] & 0xFFFFu;
      const float y = u >= a.drop.threshold ? v[e] * a.drop.z : 0.0f;
      v[e] = kResidual ? r[e] + y : y;
    }
    store_values<kOut16>(a.out, row * a.ldo + col, valid, wide, v);
  }
}

template <bool kX16, int kResidual, bool kOut16>
hipError_t launch(const DropoutArgs& a, hipStream_t stream) {
  const uint32_t groups = (uint32_t)((a.k + 7) / 8);
  const int64_t total = a.rows * (int64_t)groups;
  // 16-byte accesses: every row of every operand begins on one
  const auto fits = [](const void* p, int64_t ld, bool half) {
    return ((uintptr_t)p & 15) == 0 && ld % (half ? 8 : 4) == 0;
  };
  const bool aligned = fits(a.x, a.ldx, kX16) && fits(a.out, a.ldo, kOut16) &&
                       (!kResidual || fits(a.residual, a.ldr, kResidual == 2));
  static ResidentCache cache;
  const int64_t wanted = (total + kThreads - 1) / kThreads;
  const int64_t most = 8 * resident_groups(dropout_kernel<kX16, kResidual, kOut16>, cache);
  dropout_kernel<kX16, kResidual, kOut16>
      <<<(unsigned)(wanted < most ? wanted : most), kThreads, 0, stream>>>(a, groups, total, aligned);
  return hipGetLastError();
}

template <bool kX16, int kResidual>
hipError_t launch(const DropoutArgs& a, hipStream_t stream) {
  return a.out16 ? launch<kX16, kResidual, true>(a, stream) : launch<kX16, kResidual, false>(a, stream);
}

template <bool kX16>
hipError_t launch(const DropoutArgs& a, hipStream_t stream) {
  if (!a.residual) return launch<kX16, 0>(a, stream);
  return a.residual16 ? launch<kX16, 2>(a, stream) : launch<kX16, 1>(a, stream);
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
  return a.x16 ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace mixfp4
