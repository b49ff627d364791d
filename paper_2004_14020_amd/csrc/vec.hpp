// Device helpers of the kernels that fill gradient tensors: widths, roundings, loads of rows that start
// on any element.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace caramel {

#define CARAMEL_GLOBAL __attribute__((address_space(1)))

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// A value that is the same in all lanes, into a scalar register.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return uint32_t(__builtin_amdgcn_readfirstlane(int(v))); }

// A stretch of memory whose accesses the hardware checks, 32 bits by 32 bits: loads behind its end give zeros, stores
// there are dropped.
constexpr int kRawBuffer = 0x00027000;      // word 3 of a buffer resource: untyped data
constexpr uint32_t kNowhere = 0x60000000u;  // an offset behind every end, also with a tile's rows added to it
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(uint64_t base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, int(bytes), kRawBuffer);
}

// fp32 -> bf16, round to nearest, ties to even, NaN stays NaN
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
// (a vector's element has to be passed by value: __builtin_bit_cast of one takes the vector's first)
__device__ __forceinline__ float as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ uint32_t as_bits(float v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ float bf16_low(uint32_t v) { return as_float(v << 16); }
__device__ __forceinline__ float bf16_high(uint32_t v) { return as_float(v & 0xFFFF0000u); }

// What a wavefront's lanes have written to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// N (1, 4 or 8) consecutive elements, widened to fp32.  Rows may start on any element (odd widths), so the
// vectors promise the alignment of one element only; the hardware takes such accesses as they are.
template <bool BF16, int N>
__device__ __forceinline__ void load_elems(uint64_t at, float* v) {
  if constexpr (BF16) {
    if constexpr (N == 1) {
      v[0] = bf16_low(*reinterpret_cast<const CARAMEL_GLOBAL uint16_t*>(at));
    } else {
      typedef uint32_t vec __attribute__((ext_vector_type(N / 2), aligned(2)));
      const vec x = *reinterpret_cast<const CARAMEL_GLOBAL vec*>(at);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        v[2 * i] = bf16_low(x[i]);
        v[2 * i + 1] = bf16_high(x[i]);
      }
    }
  } else {
    if constexpr (N == 1) {
      v[0] = *reinterpret_cast<const CARAMEL_GLOBAL float*>(at);
    } else {
      typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
      for (int q = 0; q < N; q += 4) {
        const vec x = *reinterpret_cast<const CARAMEL_GLOBAL vec*>(at + 4 * q);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[q + i] = x[i];
      }
    }
  }
}

// ... and back, rounded once; STREAM: streaming stores
template <bool BF16, int N, bool STREAM = false>
__device__ __forceinline__ void store_elems(uint64_t at, const float* v) {
// (written out: as the argument of a function, a pointer loses the alignment its type promises)
#define CARAMEL_PUT(type, to, x)                                                                          \
  if constexpr (STREAM) __builtin_nontemporal_store(x, reinterpret_cast<CARAMEL_GLOBAL type*>(to)); \
  else *reinterpret_cast<CARAMEL_GLOBAL type*>(to) = x
  if constexpr (BF16) {
    if constexpr (N == 1) {
      CARAMEL_PUT(uint16_t, at, uint16_t(bf16_pair(v[0], v[0])));
    } else {
      typedef uint32_t vec __attribute__((ext_vector_type(N / 2), aligned(2)));
      vec x;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) x[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
      CARAMEL_PUT(vec, at, x);
    }
  } else {
    if constexpr (N == 1) {
      CARAMEL_PUT(float, at, v[0]);
    } else {
      typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
      for (int q = 0; q < N; q += 4) {
        vec x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[q + i];
        CARAMEL_PUT(vec, at + 4 * q, x);
      }
    }
  }
}
#undef CARAMEL_PUT

}  // namespace caramel
