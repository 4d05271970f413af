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

// Wide accesses of any address that an element may have: rows of odd lengths
// begin anywhere, and the memory path takes such accesses whole.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// kPass: past the caches.
template <bool kPass, typename T>
__device__ __forceinline__ T fetch(const void* p) {
  if constexpr (kPass) return __builtin_nontemporal_load(static_cast<const T*>(p));
  return *static_cast<const T*>(p);
}
template <bool kPass, typename T>
__device__ __forceinline__ void put(void* p, T v) {
  if constexpr (kPass)
    __builtin_nontemporal_store(v, static_cast<T*>(p));
  else
    *static_cast<T*>(p) = v;
}

// kV consecutive values of a row, 16 bytes (8 of four bf16) an access.
template <bool kBf16, int kV, bool kPass = false>
__device__ __forceinline__ void load_values(const void* p, int64_t at, float (&v)[kV]) {
  if constexpr (kBf16) {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    uint32_t w[kV == 1 ? 1 : kV / 2];
    if constexpr (kV == 1) {
      v[0] = __uint_as_float((uint32_t)q[0] << 16);
      return;
    } else if constexpr (kV == 8) {
      const u32x4_any u = fetch<kPass, u32x4_any>(q);
      w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
    } else {
      const u32x2_any u = fetch<kPass, u32x2_any>(q);
      w[0] = u.x, w[1] = u.y;
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) v[e] = e & 1 ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]);
  } else {
    const float* q = static_cast<const float*>(p) + at;
    if constexpr (kV == 1) {
      v[0] = q[0];
    } else {
#pragma unroll
      for (int e = 0; e < kV; e += 4) {
        const f32x4_any a = fetch<kPass, f32x4_any>(q + e);
        v[e] = a.x, v[e + 1] = a.y, v[e + 2] = a.z, v[e + 3] = a.w;
      }
    }
  }
}

template <bool kBf16, int kV, bool kPass = false>
__device__ __forceinline__ void store_values(void* p, int64_t at, const float (&v)[kV]) {
  if constexpr (kBf16) {
    uint16_t* q = static_cast<uint16_t*>(p) + at;
    if constexpr (kV == 1) {
      q[0] = (uint16_t)bf16_bits(v[0]);
    } else {
      uint32_t w[kV / 2];
#pragma unroll
      for (int e = 0; e < kV / 2; ++e) w[e] = bf16_bits(v[2 * e]) | bf16_bits(v[2 * e + 1]) << 16;
      if constexpr (kV == 8)
        put<kPass>(q, u32x4_any{w[0], w[1], w[2], w[3]});
      else
        put<kPass>(q, u32x2_any{w[0], w[1]});
    }
  } else {
    float* q = static_cast<float*>(p) + at;
    if constexpr (kV == 1)
      q[0] = v[0];
    else
#pragma unroll
      for (int e = 0; e < kV; e += 4)
        put<kPass>(q + e, f32x4_any{v[e], v[e + 1], v[e + 2], v[e + 3]});
  }
}

// Waves' walk over the pieces of 512 elements: `chunks` per row; a step of all
// waves is step_rows rows and step_chunks pieces.
struct Walk {
  int64_t total, step_rows;
  uint32_t chunks, step_chunks;
};

// One wave per piece of 512 elements of a row: each lane makes the draws of
// one group of 8, then the lanes read and write side by side, kV elements
// each, 8 / kV times, and get the keep bits of what they hold from the lane
// that drew them.  kV is 8, or 4 if all is fp32, whose 16-byte accesses then
// lie side by side (2^26 elements fp32 to fp32: 85 us, 6.3 TB/s, against 105;
// with a bf16 operand 8 are better: 2^23 elements fp32 into a bf16 residual
// 11.5 us against 13.4).  kResidual: 0 none, 1 fp32, 2 bf16.  Bound by memory:
// 2^27 elements bf16 to bf16 87 us, 6.2 TB/s (92 through the caches, where
// what fits into the infinity cache is better off: 11.5 against 12.3 us for
// 2^23 elements); rows of 8191 bf16 124 us, of 8191 fp32 87 us (by single
// elements 299 and 253).
template <bool kX16, int kResidual, bool kOut16, int kV, bool kPass>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a, Walk walk) {
  const int lane = threadIdx.x & 63;
  // the wave's walk in scalar registers
  const int64_t first =
      (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t step = (int64_t)gridDim.x * (kThreads / 64);
  int64_t row = first / walk.chunks;
  uint32_t chunk = (uint32_t)(first - row * walk.chunks);
  const int64_t groups = (a.k + 7) / 8;
  for (int64_t i = first; i < walk.total; i += step) {
    const int64_t col0 = (int64_t)chunk * 512;
    float v[8 / kV][kV], r[8 / kV][kV];
    const auto column = [&](int h) { return col0 + (h * 64 + lane) * kV; };
    const bool whole = col0 + 512 <= a.k;          // else a lane looks at each of its parts
    const int64_t xrow = row * a.ldx, rrow = row * a.ldr, orow = row * a.ldo;
    // parts that are not there are read from the row's first element; a part
    // that the row's end cuts is read by element
    const auto there = [&](int h) { return whole || column(h) + kV <= a.k; };
#pragma unroll
    for (int h = 0; h < 8 / kV; ++h) {
      const int64_t c = there(h) ? column(h) : 0;
      if (whole || a.k >= kV) {
        load_values<kX16, kV, kPass>(a.x, xrow + c, v[h]);
        if constexpr (kResidual != 0) load_values<kResidual == 2, kV, kPass>(a.residual, rrow + c, r[h]);
      }
    }
    uint32_t bits = 0xFFu;
    if (a.drop.threshold) {
      const uint4 w = block_draws(row * groups + (int64_t)chunk * 64 + lane, a.drop.key);
      const uint32_t d[4] = {w.x, w.y, w.z, w.w};
      bits = 0u;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        bits |= ((e & 1 ? d[e >> 1] >> 16 : d[e >> 1] & 0xFFFFu) >= a.drop.threshold ? 1u : 0u) << e;
    }
    const auto result = [&](float x, float res, bool keep) {
      const float y = keep ? x * a.drop.z : 0.0f;
      return kResidual ? res + y : y;
    };
#pragma unroll
    for (int h = 0; h < 8 / kV; ++h) {
      uint32_t mine = bits;
      if constexpr (kV < 8) mine = __shfl(bits, (h * 64 + lane) * kV / 8) >> (lane * kV & 7);
      if (there(h)) {
        float y[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e)
          y[e] = result(v[h][e], kResidual ? r[h][e] : 0.0f, mine >> e & 1u);
        store_values<kOut16, kV, kPass>(a.out, orow + column(h), y);
      } else if (kV > 1 && column(h) < a.k) {
        for (int e = 0; column(h) + e < a.k; ++e) {
          float x[1], res[1] = {0.0f}, y[1];
          load_values<kX16, 1>(a.x, xrow + column(h) + e, x);
          if constexpr (kResidual != 0) load_values<kResidual == 2, 1>(a.residual, rrow + column(h) + e, res);
          y[0] = result(x[0], res[0], mine >> e & 1u);
          store_values<kOut16, 1>(a.out, orow + column(h) + e, y);
        }
      }
    }
    row += walk.step_rows;
    chunk += walk.step_chunks;
    if (chunk >= walk.chunks) {
      chunk -= walk.chunks;
      ++row;
    }
  }
}

template <bool kX16, int kResidual, bool kOut16, int kV, bool kPass>
hipError_t launch_width(const DropoutArgs& a, hipStream_t stream) {
  Walk w{};
  w.chunks = (uint32_t)((a.k + 511) / 512);
  w.total = a.rows * (int64_t)w.chunks;
  static ResidentCache cache;
  const int64_t wanted = (w.total + kThreads / 64 - 1) / (kThreads / 64);
  const int64_t most = 16 * resident_groups(dropout_kernel<kX16, kResidual, kOut16, kV, kPass>, cache);
  const int64_t grid = wanted < most ? wanted : most, step = grid * (kThreads / 64);
  w.step_rows = step / w.chunks;
  w.step_chunks = (uint32_t)(step % w.chunks);
  dropout_kernel<kX16, kResidual, kOut16, kV, kPass><<<(unsigned)grid, kThreads, 0, stream>>>(a, w);
  return hipGetLastError();
}

template <bool kX16, int kResidual, bool kOut16>
hipError_t launch(const DropoutArgs& a, hipStream_t stream) {
  constexpr int kV = !kX16 && !kOut16 && kResidual != 2 ? 4 : 8;
  constexpr int kBytes[3] = {0, 4, 2};
  const int64_t bytes = a.rows * a.k * ((kX16 ? 2 : 4) + kBytes[kResidual] + (kOut16 ? 2 : 4));
  // past the caches where the operands do not fit into the infinity cache
  // (256 MB) and rows fill whole accesses
  const auto fits = [](const void* p, int64_t ld, bool half) {
    const int64_t size = half ? 2 : 4;
    return ((uintptr_t)p & 15) == 0 && ld * size % 16 == 0;
  };
  if (bytes > (int64_t(256) << 20) && fits(a.x, a.ldx, kX16) && fits(a.out, a.ldo, kOut16) &&
      (!kResidual || fits(a.residual, a.ldr, kResidual == 2)))
    return launch_width<kX16, kResidual, kOut16, kV, true>(a, stream);
  return launch_width<kX16, kResidual, kOut16, kV, false>(a, stream);
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
