// Activation checkpoints in 8 bits.
//
// A block is 32 consecutive tokens of one feature.  With a = its largest magnitude and e the smallest
// exponent >= -126 for which a <= 127 * 2^e, a value x is kept as q = round(x / 2^e), ties to even, |q| <= 127,
// and read back as q * 2^e.  (e stops at 121, so that 127 * 2^e is still a number: what lies above is kept as 127.)  The scale is a power of two, so that every value that is read back is a bf16
// number: the weight gradient feeds the matrix cores with it without another rounding.  A block that holds
// an infinity or a NaN is marked and reads back as NaN throughout.  One scale per feature (not per token)
// keeps the few features that are much larger than the rest from taking the others' bits.
//
// Layout: codes [block][feature][32], then the scales [block][feature] as e + 127 (255: the mark).  32 tokens
// of a feature are 32 contiguous bytes, which is the order in which a matrix product over the tokens wants them.
//
// Bound: HBM, each value read and written once.  A lane keeps four features of all 32 tokens in registers: the
// largest magnitude needs no other lane.
#include "layers.hpp"
#include "vec.hpp"

namespace caramel {
namespace {

constexpr int kFeatures = 4;  // of a lane

constexpr uint32_t kTop = 0x7F7E0000u;  // 127 * 2^121

// scale byte of a block from the bits of its largest magnitude
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest) {
  const int e = int(largest >> 23) - 6 + ((largest & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);  // 127/64 = 1 + 0x7E0000 / 2^23
  return largest >= 0x7F800000u ? 255u : uint32_t(min(max(e, 1), 121 + 127));
}

template <bool BF16>
__global__ void __launch_bounds__(256) k_checkpoint_store(CheckpointArgs a) {
  constexpr int ES = BF16 ? 2 : 4;
  const uint32_t w = blockIdx.y, n = a.w.tokens[w], wide = (a.features + 256 * kFeatures - 1) / (256 * kFeatures);
  const uint32_t block = blockIdx.x / wide, blocks = (n + kCheckpointBlock - 1) / kCheckpointBlock;
  const uint32_t f = (blockIdx.x % wide * 256 + threadIdx.x) * kFeatures;
  if (block >= blocks || f >= a.features) return;
  const uint32_t rows = min(n - block * kCheckpointBlock, kCheckpointBlock);
  const uint32_t cols = min(a.features - f, uint32_t(kFeatures));
  const uint64_t src = a.w.a[w] + (uint64_t(block) * kCheckpointBlock * a.pitch + f) * ES;
  float x[kCheckpointBlock][kFeatures];
#pragma unroll
  for (uint32_t r = 0; r < kCheckpointBlock; ++r) {
    for (int j = 0; j < kFeatures; ++j) x[r][j] = 0.0f;
    if (r < rows) {
      const uint64_t at = src + r * a.pitch * ES;
      if (cols == kFeatures) {
        load_elems<BF16, kFeatures>(at, x[r]);
      } else {
#pragma unroll
        for (int j = 0; j < kFeatures; ++j)
          if (uint32_t(j) < cols) load_elems<BF16, 1>(at + j * ES, &x[r][j]);
      }
    }
  }
  const uint64_t codes = a.w.b[w], scales = codes + uint64_t(blocks) * a.features * kCheckpointBlock;
#pragma unroll
  for (int j = 0; j < kFeatures; ++j) {
    if (uint32_t(j) >= cols) break;
    uint32_t largest = 0;
#pragma unroll
    for (uint32_t r = 0; r < kCheckpointBlock; ++r)
      largest = max(largest, as_bits(x[r][j]) & 0x7FFFFFFFu);
    const uint32_t s = scale_byte(largest);
    if (largest > kTop) {
      const float top = as_float(kTop);
#pragma unroll
      for (uint32_t r = 0; r < kCheckpointBlock; ++r) x[r][j] = fminf(fmaxf(x[r][j], -top), top);
    }
    const uint32_t keep = s == 255u ? 0u : 0xFFFFFFFFu;
    // 2^-e; adding 1.5 * 2^23 leaves round(x / 2^e), ties to even, in the low bits (the product is exact)
    const float inv = as_float((254u - min(s, 253u)) << 23);
    uint32_t q[8];
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      uint32_t t[4];
      for (int k = 0; k < 4; ++k) t[k] = as_bits(__builtin_fmaf(x[4 * d + k][j], inv, 12582912.0f));
      const uint32_t lo = __builtin_amdgcn_perm(t[1], t[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(t[3], t[2], 0x04000C0Cu);
      q[d] = (lo | hi) & keep;
    }
    const uint64_t feature = uint64_t(block) * a.features + f + j;
    typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(4)));
    CARAMEL_GLOBAL vec* const to = reinterpret_cast<CARAMEL_GLOBAL vec*>(codes + feature * kCheckpointBlock);
    to[0] = vec{q[0], q[1], q[2], q[3]};
    to[1] = vec{q[4], q[5], q[6], q[7]};
    *reinterpret_cast<CARAMEL_GLOBAL uint8_t*>(scales + feature) = uint8_t(s);
  }
}

template <bool BF16>
__global__ void __launch_bounds__(256) k_checkpoint_load(CheckpointArgs a) {
  constexpr int ES = BF16 ? 2 : 4;
  const uint32_t w = blockIdx.y, n = a.w.tokens[w], wide = (a.features + 256 * kFeatures - 1) / (256 * kFeatures);
  const uint32_t block = blockIdx.x / wide, blocks = (n + kCheckpointBlock - 1) / kCheckpointBlock;
  const uint32_t f = (blockIdx.x % wide * 256 + threadIdx.x) * kFeatures;
  if (block >= blocks || f >= a.features) return;
  const uint32_t rows = min(n - block * kCheckpointBlock, kCheckpointBlock);
  const uint32_t cols = min(a.features - f, uint32_t(kFeatures));
  const uint64_t codes = a.w.b[w], scales = codes + uint64_t(blocks) * a.features * kCheckpointBlock;
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(4)));
  vec q[kFeatures][2];
  float size[kFeatures];
#pragma unroll
  for (int j = 0; j < kFeatures; ++j) {
    q[j][0] = q[j][1] = vec{0, 0, 0, 0};
    size[j] = 0.0f;
    if (uint32_t(j) < cols) {
      const uint64_t feature = uint64_t(block) * a.features + f + j;
      const CARAMEL_GLOBAL vec* const from = reinterpret_cast<const CARAMEL_GLOBAL vec*>(codes + feature * kCheckpointBlock);
      q[j][0] = from[0];
      q[j][1] = from[1];
      const uint32_t s = *reinterpret_cast<const CARAMEL_GLOBAL uint8_t*>(scales + feature);
      size[j] = as_float(s == 255u ? 0x7FC00000u : s << 23);
    }
  }
  const uint64_t dst = a.w.a[w] + (uint64_t(block) * kCheckpointBlock * a.pitch + f) * ES;
#pragma unroll
  for (uint32_t r = 0; r < kCheckpointBlock; ++r) {
    if (r < rows) {
      float y[kFeatures];
#pragma unroll
      for (int j = 0; j < kFeatures; ++j) y[j] = float(int8_t(q[j][r / 16][r % 16 / 4] >> (8 * (r % 4)))) * size[j];
      const uint64_t at = dst + r * a.pitch * ES;
      if (cols == kFeatures) {
        store_elems<BF16, kFeatures>(at, y);
      } else {
#pragma unroll
        for (int j = 0; j < kFeatures; ++j)
          if (uint32_t(j) < cols) store_elems<BF16, 1>(at + j * ES, &y[j]);
      }
    }
  }
}

dim3 grid_of(const CheckpointArgs& a) {
  return dim3((a.features + 256 * kFeatures - 1) / (256 * kFeatures) * uint32_t(checkpoint_blocks(a.max_tokens)), a.world);
}

}  // namespace

hipError_t launch_checkpoint_store(const CheckpointArgs& a, hipStream_t s) {
  if (a.max_tokens == 0) return hipSuccess;
  if (a.bf16) hipLaunchKernelGGL((k_checkpoint_store<true>), grid_of(a), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_checkpoint_store<false>), grid_of(a), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_checkpoint_load(const CheckpointArgs& a, hipStream_t s) {
  if (a.max_tokens == 0) return hipSuccess;
  if (a.bf16) hipLaunchKernelGGL((k_checkpoint_load<true>), grid_of(a), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_checkpoint_load<false>), grid_of(a), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace caramel
