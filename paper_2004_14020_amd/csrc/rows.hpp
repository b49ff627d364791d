// Rows that stay in the registers of a team of wavefronts: loads and stores of pieces of them, and sums over them.
#pragma once

#include "vec.hpp"

namespace caramel {

// Columns that a lane takes at once: 16 bytes.
template <bool BF16>
constexpr int kPiece = BF16 ? 8 : 4;

constexpr int kStreaming = 2;  // of a buffer access: non-temporal

// A row of `columns` values, or a stretch of one.  The hardware checks every 32 bits of an access against the row's end (loads behind it give
// zeros, stores there are dropped), so no lane needs a branch, and all loads are in flight before the first is waited for.  Of an odd
// number of bf16 columns the last one shares its 32 bits with what is behind the row, and is left to accesses of its own.
template <bool BF16>
struct Row {
  static constexpr int ES = BF16 ? 2 : 4, N = kPiece<BF16>;
  __amdgpu_buffer_rsrc_t at;
  uint32_t columns;

  __device__ __forceinline__ Row(uint64_t base, uint32_t n) : at(buffer(base, n * ES)), columns(n) {}
  __device__ __forceinline__ bool odd() const { return BF16 && columns % 2; }

  // 16 bytes from column `col` on
  template <bool STREAM = false>
  __device__ __forceinline__ u32x4 get(uint32_t col) const {
    return __builtin_amdgcn_raw_buffer_load_b128(at, int(col * ES), 0, STREAM ? kStreaming : 0);
  }
  // V of them, `step` columns apart
  template <int V>
  __device__ __forceinline__ void get_all(uint32_t col, uint32_t step, bool stream, u32x4 (&v)[V]) const {
    if (stream) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = get<true>(col + i * step);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = get<false>(col + i * step);
    }
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void put(uint32_t col, u32x4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(v, at, int(col * ES), 0, STREAM ? kStreaming : 0);
  }
  // the last one of an odd number
  __device__ __forceinline__ uint32_t get_last() const {
    return uint32_t(__builtin_amdgcn_raw_buffer_load_b16(at, int((columns - 1) * ES), 0, 0));
  }
  // ... into the piece from `col` on, if it is there (what is behind it is 0 already)
  __device__ __forceinline__ void merge_last(uint32_t col, uint32_t last, u32x4& v) const {
#pragma unroll
    for (int d = 0; d < 4; ++d) v[d] = col + 2 * d == columns - 1 ? last : v[d];
  }
  __device__ __forceinline__ void put_last(uint32_t col, u32x4 v) const {
#pragma unroll
    for (int d = 0; d < 4; ++d)
      if (col + 2 * d == columns - 1) __builtin_amdgcn_raw_buffer_store_b16(uint16_t(v[d]), at, int((columns - 1) * ES), 0, 0);
  }
};

template <bool BF16>
__device__ __forceinline__ void widen(u32x4 raw, float* v) {
#pragma unroll
  for (int j = 0; j < kPiece<BF16>; ++j) {
    if constexpr (BF16) v[j] = j % 2 ? bf16_high(raw[j / 2]) : bf16_low(raw[j / 2]);
    else v[j] = as_float(raw[j]);
  }
}
template <bool BF16>
__device__ __forceinline__ u32x4 narrow(const float* v) {
  u32x4 raw;
#pragma unroll
  for (int d = 0; d < 4; ++d) raw[d] = BF16 ? bf16_pair(v[2 * d % kPiece<BF16>], v[(2 * d + 1) % kPiece<BF16>]) : as_bits(v[d]);
  return raw;
}

// The value of the lane that a step of a reduction within 16 lanes pairs this one with: a neighbour, the pair beside, the other
// half, ... (moves between lanes of a row of 16 go through no memory).
template <int STEP, typename T>
__device__ __forceinline__ T beside(T v) {
  constexpr int kControl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;  // pairs, quads, mirrored half row, mirrored row
  if constexpr (sizeof(T) == 8) {
    const u32x2 x = __builtin_bit_cast(u32x2, v);
    const u32x2 y = {uint32_t(__builtin_amdgcn_update_dpp(0, int(x[0]), kControl, 15, 15, false)),
                     uint32_t(__builtin_amdgcn_update_dpp(0, int(x[1]), kControl, 15, 15, false))};
    return __builtin_bit_cast(T, y);
  } else {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kControl, 15, 15, false));
  }
}
template <typename T>
__device__ __forceinline__ T of_lane(T v, int lane) {
  if constexpr (sizeof(T) == 8) {
    const u32x2 x = __builtin_bit_cast(u32x2, v);
    const u32x2 y = {uint32_t(__builtin_amdgcn_readlane(int(x[0]), lane)), uint32_t(__builtin_amdgcn_readlane(int(x[1]), lane))};
    return __builtin_bit_cast(T, y);
  } else {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  }
}

// Over every row of 16 lanes, in each of them; over the wavefront, in all lanes.  The same order everywhere.
template <typename T>
__device__ __forceinline__ T row_sum(T v) {
  v += beside<0>(v);
  v += beside<1>(v);
  v += beside<2>(v);
  return v + beside<3>(v);
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, beside<0>(v));
  v = fmaxf(v, beside<1>(v));
  v = fmaxf(v, beside<2>(v));
  return fmaxf(v, beside<3>(v));
}
template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
  v = row_sum(v);
  return (of_lane(v, 0) + of_lane(v, 16)) + (of_lane(v, 32) + of_lane(v, 48));
}
__device__ __forceinline__ float wave_max(float v) {
  v = row_max(v);
  return fmaxf(fmaxf(of_lane(v, 0), of_lane(v, 16)), fmaxf(of_lane(v, 32), of_lane(v, 48)));
}

// Over one number of each of COUNT (16 at most) wavefronts, `step` apart in LDS: every row of 16 lanes for itself.
template <int COUNT, typename T>
__device__ __forceinline__ T across_sum(const T* lds, int step) {
  const int k = threadIdx.x % 16;
  return row_sum(k < COUNT ? lds[k * step] : T(0));
}
template <int COUNT>
__device__ __forceinline__ float across_max(const float* lds, int step) {
  return row_max(lds[min(int(threadIdx.x % 16), COUNT - 1) * step]);
}

// The sum over a team of TEAM wavefronts, which are the whole workgroup where they are more than one.  Calls that follow each other take
// `lds` (TEAM values each) in turn, so that one barrier is enough.
template <int TEAM, typename T>
__device__ __forceinline__ T team_sum(T v, T* lds) {
  v = wave_sum(v);
  if constexpr (TEAM > 1) {
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = across_sum<TEAM>(lds, 1);
  }
  return v;
}

}  // namespace caramel
