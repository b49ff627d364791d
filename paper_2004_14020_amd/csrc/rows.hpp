// Rows that stay in the registers of a team of wavefronts: how their columns are dealt out, and sums over them.
#pragma once

#include "vec.hpp"

namespace caramel {

// Columns that a lane takes at once: 16 bytes.  Lane l of a team has the pieces l, l + lanes, l + 2 lanes, ... of a row.
template <bool BF16>
constexpr int kPiece = BF16 ? 8 : 4;

// A piece of a row that has `width` columns; zeros behind them.
template <bool BF16>
__device__ __forceinline__ void load_piece(uint64_t row, uint32_t col, uint32_t width, float* v) {
  constexpr int N = kPiece<BF16>, ES = BF16 ? 2 : 4;
  if (col + N <= width) {
    load_elems<BF16, N>(row + uint64_t(col) * ES, v);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      v[j] = 0.0f;
      if (col + j < width) load_elems<BF16, 1>(row + uint64_t(col + j) * ES, v + j);
    }
  }
}

template <bool BF16>
__device__ __forceinline__ void store_piece(uint64_t row, uint32_t col, uint32_t width, const float* v) {
  constexpr int N = kPiece<BF16>, ES = BF16 ? 2 : 4;
  if (col + N <= width) {
    store_elems<BF16, N>(row + uint64_t(col) * ES, v);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (col + j < width) store_elems<BF16, 1>(row + uint64_t(col + j) * ES, v + j);
  }
}

// The sum over a wavefront, in every lane, in the same order everywhere.
template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  return v;
}

// ... over TEAM wavefronts, which are the whole workgroup where they are more than one.  Calls that follow each other take
// `lds` (TEAM values each) in turn, so that one barrier is enough.
template <int TEAM, typename T>
__device__ __forceinline__ T team_sum(T v, T* lds) {
  v = wave_sum(v);
  if constexpr (TEAM > 1) {
    const uint32_t wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 0) lds[wave] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int k = 1; k < TEAM; ++k) v += lds[k];
  }
  return v;
}

}  // namespace caramel
