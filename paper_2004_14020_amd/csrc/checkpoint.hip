// Activation checkpoints in 8 bits.
//
// A block is 32 consecutive tokens of one feature.  With a = its largest magnitude and e the smallest
// exponent >= -126 for which a <= 127 * 2^e, a value x is kept as q = round(x / 2^e), ties to even, |q| <= 127,
// and read back as q * 2^e.  (e stops at 121, so that 127 * 2^e is still a number: what lies above is
// kept as 127.)  The scale is a power of two, so that every value that is read back is a bf16 number: the weight gradient feeds the matrix cores with it without another rounding.  A block that holds
// an infinity or a NaN is marked and reads back as NaN throughout.  One scale per feature (not per token)
// keeps the few features that are much larger than the rest from taking the others' bits.
//
// Layout: codes [block][feature][32], then the scales [block][feature] as e + 127 (255: the mark).  32 tokens
// of a feature are 32 contiguous bytes, which is the order in which a matrix product over the tokens wants them.
//
// Bound: HBM, each value read and written once.  A wavefront takes one block of 256 features (128 where fp32 is
// stored, for the registers).  A lane keeps its features of all 32 tokens in registers, so the largest magnitude needs no other lane, and all 32 loads (buffer loads,
// whose range check takes care of rows behind the last token) are in flight at once.  The codes are exchanged through LDS, so that
// a wavefront's memory access on their side is 1 KiB in one piece; a lane's own codes are 32 bytes a feature.
#include "layers.hpp"
#include "vec.hpp"

namespace caramel {
namespace {

// Of a workgroup.  4 x 4096 x 4096 bf16, store and load one after the other: four wavefronts 45.8 and 44.2 us, two 41.8 and
// 31.9; with streaming stores of the codes 39.2 and 38.3 (they are then not in the last-level cache), of what load gives 48.
constexpr int kWaves = 2;
constexpr uint32_t kTop = 0x7F7E0000u;  // 127 * 2^121

// scale byte of a block from the bits of its largest magnitude
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest) {
  const int e = int(largest >> 23) - 6 + ((largest & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);  // 127/64 = 1 + 0x7E0000 / 2^23
  return largest >= 0x7F800000u ? 255u : uint32_t(min(max(e, 1), 121 + 127));
}

// Where a wavefront works: one block of tokens, FEATURES of every lane.
struct Place {
  uint32_t w, block, blocks, rows, f0, left;  // left: features from f0 on
  bool any;
};
template <int FEATURES>
__device__ __forceinline__ Place place(const CheckpointArgs& a) {
  Place p;
  const uint32_t wide = (a.features + 64 * FEATURES - 1) / (64 * FEATURES);
  const uint32_t at = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  p.w = blockIdx.y;
  p.block = at / wide;
  p.f0 = (at - p.block * wide) * 64 * FEATURES;
  const uint32_t n = a.w.tokens[p.w];
  p.blocks = (n + kCheckpointBlock - 1) / kCheckpointBlock;
  p.any = p.block < p.blocks;
  p.rows = p.any ? min(n - p.block * kCheckpointBlock, kCheckpointBlock) : 0;
  p.left = a.features - p.f0;
  return p;
}

// 64 x PIECES pieces of 16 bytes in LDS: lane l's piece c.  The exchange of c's bits spreads the lanes' pieces over the
// banks, which lie PIECES pieces apart.
template <int PIECES>
__device__ __forceinline__ uint32_t slot(uint32_t l, uint32_t c) {
  return l * PIECES + (c ^ (l & (PIECES - 1)));
}

// bf16 rows may start on any element, and loads take four elements wherever they begin.  The range check goes by pairs, so of an odd
// number of features the last row's end is loaded once more, one by one.  4 x 1955 x 8995 bf16: 47 us as with 8992; with all its
// elements loaded one by one 69.
template <bool BF16>
__global__ void __launch_bounds__(64 * kWaves) k_checkpoint_store(CheckpointArgs a) {
  constexpr int ES = BF16 ? 2 : 4, kFeatures = BF16 ? 4 : 2, kPieces = 2 * kFeatures;
  constexpr int WORDS = 2;  // 32-bit words of a lane's values of one token
  typedef uint32_t raw __attribute__((ext_vector_type(WORDS)));
  __shared__ u32x4 lds[kWaves][64 * kPieces];
  const Place p = place<kFeatures>(a);
  if (!p.any) return;
  const uint32_t lane = threadIdx.x % 64, row_bytes = uint32_t(a.pitch) * ES;
  u32x4* const mine = lds[threadIdx.x / 64];
  const __amdgpu_buffer_rsrc_t rx = buffer(a.w.a[p.w] + (uint64_t(p.block) * kCheckpointBlock * a.pitch + p.f0) * ES,
                                           (p.rows - 1) * row_bytes + p.left * ES);
  raw x[kCheckpointBlock];
#pragma unroll
  for (uint32_t r = 0; r < kCheckpointBlock; ++r) {
    x[r] = __builtin_amdgcn_raw_buffer_load_b64(rx, int(r * row_bytes + lane * kFeatures * ES), 0, 0);
  }
  if constexpr (BF16) {
    if (p.left % 2 && p.left < 64 * kFeatures) {
      const int off = int((p.rows - 1) * row_bytes + lane * kFeatures * ES);
      raw last;
#pragma unroll
      for (int d = 0; d < WORDS; ++d)
        last[d] = uint32_t(__builtin_amdgcn_raw_buffer_load_b16(rx, off + 4 * d, 0, 0)) |
                  uint32_t(__builtin_amdgcn_raw_buffer_load_b16(rx, off + 4 * d + 2, 0, 0)) << 16;
#pragma unroll
      for (uint32_t r = 0; r < kCheckpointBlock; ++r) x[r] = r + 1 == p.rows ? last : x[r];
    }
  }
  // largest magnitudes: as integers, magnitudes are in order, and NaN above infinity above the numbers
  uint32_t largest[kFeatures];
  if constexpr (BF16) {
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    u16x4 m = 0;
#pragma unroll
    for (uint32_t r = 0; r < kCheckpointBlock; ++r)
      m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x4, x[r] & 0x7FFF7FFFu));
#pragma unroll
    for (int j = 0; j < kFeatures; ++j) largest[j] = uint32_t(m[j]) << 16;
  } else {
    raw m = 0;
#pragma unroll
    for (uint32_t r = 0; r < kCheckpointBlock; ++r) m = __builtin_elementwise_max(m, x[r] & 0x7FFFFFFFu);
#pragma unroll
    for (int j = 0; j < kFeatures; ++j) largest[j] = m[j];
  }
  // numbers above 127 * 2^121 become that
  bool beyond = false;
#pragma unroll
  for (int j = 0; j < kFeatures; ++j) beyond = beyond || largest[j] > kTop;
  if (__ballot(beyond)) {
#pragma unroll
    for (uint32_t r = 0; r < kCheckpointBlock; ++r) {
      if constexpr (BF16) {
        typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
        const u16x4 top = uint16_t(kTop >> 16);
        const u16x4 m = __builtin_elementwise_min(top, __builtin_bit_cast(u16x4, x[r] & 0x7FFF7FFFu));
        x[r] = (x[r] & 0x80008000u) | __builtin_bit_cast(raw, m);
      } else {
        const raw top = kTop;
        x[r] = (x[r] & 0x80000000u) | __builtin_elementwise_min(top, x[r] & 0x7FFFFFFFu);
      }
    }
  }
  uint32_t scale[kFeatures];
#pragma unroll
  for (int j = 0; j < kFeatures; ++j) {
    const uint32_t s = scale_byte(largest[j]);
    const uint32_t keep = s == 255u ? 0u : 0xFFFFFFFFu;
    // 2^-e; adding 1.5 * 2^23 leaves round(x / 2^e), ties to even, in the low bits (the product is exact)
    const float inv = as_float((254u - min(s, 253u)) << 23);
    u32x4 q[2];
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      uint32_t t[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float v;
        if constexpr (BF16) v = j % 2 ? bf16_high(x[4 * d + k][j / 2]) : bf16_low(x[4 * d + k][j / 2]);
        else v = as_float(x[4 * d + k][j]);
        t[k] = as_bits(__builtin_fmaf(v, inv, 12582912.0f));
      }
      const uint32_t lo = __builtin_amdgcn_perm(t[1], t[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(t[3], t[2], 0x04000C0Cu);
      q[d / 4][d % 4] = (lo | hi) & keep;
    }
    mine[slot<kPieces>(lane, 2 * j)] = q[0];
    mine[slot<kPieces>(lane, 2 * j + 1)] = q[1];
    scale[j] = s;
  }
  wave_sync();
  const uint64_t codes = a.w.b[p.w], feature = uint64_t(p.block) * a.features + p.f0;
  const __amdgpu_buffer_rsrc_t rq = buffer(codes + feature * kCheckpointBlock, p.left * kCheckpointBlock);
  const __amdgpu_buffer_rsrc_t rs = buffer(codes + uint64_t(p.blocks) * a.features * kCheckpointBlock + feature, p.left);
#pragma unroll
  for (uint32_t i = 0; i < kPieces; ++i) {
    const uint32_t at = i * 64 + lane;
    __builtin_amdgcn_raw_buffer_store_b128(mine[slot<kPieces>(at / kPieces, at % kPieces)], rq, int(at * 16), 0, 0);
  }
  if (a.features % kFeatures == 0) {  // both the rows of scales and this lane's part of one start on a whole store
    if constexpr (BF16)
      __builtin_amdgcn_raw_buffer_store_b32(scale[0] | scale[1] << 8 | scale[2] << 16 | scale[3] << 24, rs, int(lane * 4), 0, 0);
    else
      __builtin_amdgcn_raw_buffer_store_b16(uint16_t(scale[0] | scale[1] << 8), rs, int(lane * 2), 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < kFeatures; ++j) __builtin_amdgcn_raw_buffer_store_b8(uint8_t(scale[j]), rs, int(lane * kFeatures + j), 0, 0);
  }
}

template <bool BF16>
__global__ void __launch_bounds__(64 * kWaves) k_checkpoint_load(CheckpointArgs a) {
  constexpr int ES = BF16 ? 2 : 4, kFeatures = 4, kPieces = 2 * kFeatures;
  __shared__ u32x4 lds[kWaves][64 * kPieces];
  const Place p = place<kFeatures>(a);
  if (!p.any) return;
  const uint32_t lane = threadIdx.x % 64, row_bytes = uint32_t(a.pitch) * ES;
  u32x4* const mine = lds[threadIdx.x / 64];
  const uint64_t codes = a.w.b[p.w], feature = uint64_t(p.block) * a.features + p.f0;
  const __amdgpu_buffer_rsrc_t rq = buffer(codes + feature * kCheckpointBlock, p.left * kCheckpointBlock);
  const __amdgpu_buffer_rsrc_t rs = buffer(codes + uint64_t(p.blocks) * a.features * kCheckpointBlock + feature, p.left);
  u32x4 in[8];
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) in[i] = __builtin_amdgcn_raw_buffer_load_b128(rq, int(i * 1024 + lane * 16), 0, 0);
  float size[kFeatures];
#pragma unroll
  for (int j = 0; j < kFeatures; ++j) {
    const uint32_t s = __builtin_amdgcn_raw_buffer_load_b8(rs, int(lane * 4 + j), 0, 0);
    size[j] = as_float(s == 255u ? 0x7FC00000u : s << 23);
  }
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) mine[slot<kPieces>(i * 8 + lane / 8, lane % 8)] = in[i];
  wave_sync();
  u32x4 q[kFeatures][2];
#pragma unroll
  for (int j = 0; j < kFeatures; ++j) {
    q[j][0] = mine[slot<kPieces>(lane, 2 * j)];
    q[j][1] = mine[slot<kPieces>(lane, 2 * j + 1)];
  }
  const uint64_t dst = a.w.a[p.w] + (uint64_t(p.block) * kCheckpointBlock * a.pitch + p.f0) * ES;
  const __amdgpu_buffer_rsrc_t rx = buffer(dst, (p.rows - 1) * row_bytes + p.left * ES);
  const uint32_t f = lane * kFeatures;
  if (f >= p.left) return;
  const bool whole = f + kFeatures <= p.left;  // else element by element (everything so: 4 x 1955 x 8995 bf16 56 us, 37)
#pragma unroll
  for (uint32_t r = 0; r < kCheckpointBlock; ++r) {
    float y[kFeatures];
#pragma unroll
    for (int j = 0; j < kFeatures; ++j) y[j] = float(int8_t(q[j][r / 16][r % 16 / 4] >> (8 * (r % 4)))) * size[j];
    const int off = int(r * row_bytes + f * ES);
    if (whole) {
      if constexpr (BF16)
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3])}, rx, off, 0, 0);
      else
        __builtin_amdgcn_raw_buffer_store_b128(u32x4{as_bits(y[0]), as_bits(y[1]), as_bits(y[2]), as_bits(y[3])}, rx, off, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < kFeatures; ++j) {
        const int at = f + j < p.left ? off + j * ES : int(kNowhere);
        if constexpr (BF16) __builtin_amdgcn_raw_buffer_store_b16(uint16_t(bf16_pair(y[j], y[j])), rx, at, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b32(as_bits(y[j]), rx, at, 0, 0);
      }
    }
  }
}

dim3 grid_of(const CheckpointArgs& a, uint32_t features) {  // of a lane
  const uint64_t waves = (a.features + 64 * features - 1) / (64 * features) * checkpoint_blocks(a.max_tokens);
  return dim3(uint32_t((waves + kWaves - 1) / kWaves), a.world);
}

}  // namespace

hipError_t launch_checkpoint_store(const CheckpointArgs& args, const AllWorkers& v, hipStream_t s) {
  if (args.max_tokens == 0) return hipSuccess;
  return in_groups(args, v, [&](const CheckpointArgs& a, uint32_t) {
    const dim3 block(64 * kWaves);
    if (a.bf16) hipLaunchKernelGGL((k_checkpoint_store<true>), grid_of(a, 4), block, 0, s, a);
    else hipLaunchKernelGGL((k_checkpoint_store<false>), grid_of(a, 2), block, 0, s, a);
    return hipGetLastError();
  });
}

hipError_t launch_checkpoint_load(const CheckpointArgs& args, const AllWorkers& v, hipStream_t s) {
  if (args.max_tokens == 0) return hipSuccess;
  return in_groups(args, v, [&](const CheckpointArgs& a, uint32_t) {
    const dim3 block(64 * kWaves);
    if (a.bf16) hipLaunchKernelGGL((k_checkpoint_load<true>), grid_of(a, 4), block, 0, s, a);
    else hipLaunchKernelGGL((k_checkpoint_load<false>), grid_of(a, 4), block, 0, s, a);
    return hipGetLastError();
  });
}

}  // namespace caramel
