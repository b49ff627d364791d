// Weight and bias gradients of a dense layer, from its input's 8-bit checkpoint.
//
//   dW[k, n] = round([dW[k, n] +] sum over the tokens m of x[m, k] * dy[m, n])
//   db[n]    = round([db[n] +]    sum over the tokens m of dy[m, n])
//
// for all workers of a plan in one launch.  The product runs on the matrix cores in bf16 with fp32 sums.  Nothing is rounded on the
// way in: a value read back from a checkpoint is a bf16 number (checkpoint.hip), and an fp32 gradient is the sum of three bf16
// numbers (24 significant bits, eight each), which go through the matrix cores one after the other.  That is three products
// instead of one, at 16 times the rate of the fp32 matrix instructions.  Below 2^-110 the third number would be smaller than bf16
// goes: bits under 2^-133 are cut off.  (The matrix cores take subnormal numbers as they are.)  A common power of two cannot help, as
// both x and dy may lie anywhere in fp32's range, and finding one for each tile would be another pass over dy.
//
// Bound: no unit by itself.  8 x (4096 tokens, 1024 x 4096) bf16 takes 261 us a call = 1053 TFLOP/s (the kernel's least 252; back to
// back 277 to 316, as the clock falls), against 1262 of a library product of 8192^3 and 675 of one of this shape.  Of the cycles, at
// the 1.9 GHz that power leaves of 2.4, the matrix cores are busy in 53 %, other vector instructions take 32 % of the SIMDs', and
// LDS, which gives every product its 128-bit operand at 256 bytes a clock, is busy in 33 %.  What the loop's instructions cost, of 251 us:
// without widening x 230, without fetching dy 225, without either and without LDS writes 200.  16384 tokens, 1024 x 1024 fp32 95 us + 12
// for joining its 16 parts (three products: 1085 TFLOP/s; an fp32 library product 153).  Few tokens: HBM, see below.
//
// Tiling.  A workgroup owns TK features x TN outputs and walks the tokens 32 at a time (one block of the
// checkpoint).  dy is brought to LDS once per workgroup, transposed on the way through registers so that
// a matrix operand (eight tokens of one output) is one 128-bit read; x goes from the checkpoint straight
// to registers, 16 bytes = 16 tokens of one feature per lane, and is widened there: its layout is already that
// of the operand.  The tokens are dealt to the operand's places in the same permuted order on both sides.
// Outputs are dealt to lanes in pairs, so that a lane ends with two neighbours to store.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "layers.hpp"
#include "vec.hpp"

namespace caramel {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kXcds = 8;

struct Tiling {
  uint32_t nk, nn;        // tiles along features and outputs
  uint32_t splits;        // parts of the tokens
  uint32_t total;         // workgroups
  uint64_t split_stride;  // bytes from one part's sums to the next (0: one part, sums go to the gradient itself)
  uint64_t bias_stride;
};

// A byte of a word as a number.  One instruction; written down, because the compiler otherwise makes vectors of shifts
// out of a row of them, which takes twice the instructions and more registers than there are.
__device__ __forceinline__ float signed_byte(uint32_t word, int n) {
  float f;
  switch (n) {
    case 0: asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(word)); break;
    case 1: asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(word)); break;
    case 2: asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(word)); break;
    default: asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(word));
  }
  return f;
}

// How bf16 rows of dy are loaded, two outputs at a time.  kPairs: an even number of outputs.  kShift: an odd number; the lane
// whose pair would reach behind the row takes the pair before and shifts.  kSingle: one output, loaded as such.  (Rows may
// start on any element.)
enum Load { kPairs, kShift, kSingle };

// The rows of dy of one workgroup: TN outputs, brought in by its 2 TN lanes 32 tokens at a time; a lane has eight tokens of two
// outputs.
template <bool BF16, Load LOAD, int TN>
struct Dy {
  static constexpr int ES = BF16 ? 2 : 4, P = BF16 ? 1 : 3;
  static constexpr int kPacks = 2 * (BF16 ? 1 : 4);
  typedef uint32_t raw __attribute__((ext_vector_type(BF16 ? 8 : 16)));
  uint64_t base;
  uint32_t row_bytes, behind, end_token, off, octet, pair;
  bool last_pair;
  float bias[2] = {0.0f, 0.0f};  // sums of this lane's two outputs
  u32x4 parts[P];                // of the output that is being packed

  __device__ __forceinline__ Dy(const WeightGradientArgs& a, uint32_t w, uint32_t n0, uint32_t end, uint32_t tid) {
    const uint32_t lead = n0 ? 2 : 0;  // outputs before the tile that kShift may reach back to
    octet = tid / (TN / 2);
    pair = tid % (TN / 2);
    end_token = uniform(end);
    row_bytes = uint32_t(a.dy_pitch) * ES;
    behind = row_bytes - (a.outputs - n0 + lead) * ES;
    base = a.w.b[w] + uint64_t(n0 - lead) * ES;
    last_pair = LOAD == kShift && n0 + pair * 2 + 1 == a.outputs;
    off = octet * 8 * row_bytes + (pair * 2 + lead - (last_pair ? 1 : 0)) * ES;
  }
  // A block's memory.  Behind the last block, loads are made as well, of an empty stretch: they give zeros and fetch nothing.
  // (A branch around them would make the compiler wait for all loads where the ways meet.)
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t block(uint32_t b) const {
    const uint32_t rows = min(end_token - min(b * kCheckpointBlock, end_token), kCheckpointBlock);
    return buffer(base + uint64_t(b) * kCheckpointBlock * row_bytes, max(int(rows * row_bytes - behind), 0));
  }
  __device__ __forceinline__ void load_row(__amdgpu_buffer_rsrc_t r, raw& v, int j) const {  // j: 0 to 7
    const int at = int(off + j * row_bytes);
    if constexpr (!BF16) {
      const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0);
      v[2 * j] = x[0];
      v[2 * j + 1] = x[1];
    } else if constexpr (LOAD == kSingle) {
      v[j] = __builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0);
    } else {
      v[j] = __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
    }
  }
  __device__ __forceinline__ raw load(uint32_t b) const {
    raw v;
    const __amdgpu_buffer_rsrc_t r = block(b);
#pragma unroll
    for (int j = 0; j < 8; ++j) load_row(r, v, j);
    return v;
  }
  // To LDS as operands, eight tokens of an output to a piece, and into the sums where the bias is due; in kPacks steps.
  template <typename BIAS>
  __device__ __forceinline__ void pack(raw& in, u32x4 (*lds)[4][TN], int n, BIAS) {
    const int odd = BF16 ? n : n / 4;
    u32x4* const to = &lds[0][octet][odd * (TN / 2) + pair];
    if constexpr (BF16) {
      if constexpr (LOAD == kShift)
        if (!odd) in >>= last_pair ? 16u : 0u;
#pragma unroll
      for (int d = 0; d < 4; ++d) parts[0][d] = __builtin_amdgcn_perm(in[2 * d + 1], in[2 * d], odd ? 0x07060302u : 0x05040100u);
      *to = parts[0];
      if constexpr (BIAS::value)
#pragma unroll
        for (int j = 0; j < 8; ++j) bias[odd] += odd ? bf16_high(in[j]) : bf16_low(in[j]);
    } else {
      // v = hi + mid + lo: the upper half of a float is a bf16 number, and the rest is exact; lo's lower half is 0 from 2^-110 on
      const int d = n % 4;
      uint32_t part[3][2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t bits = in[2 * (2 * d + e) + odd];
        const float x = as_float(bits), hi = bf16_high(bits);
        const float rest = x == hi ? 0.0f : x - hi;  // an infinity is all in its upper half
        const float mid = bf16_high(as_bits(rest));
        part[0][e] = bits;
        part[1][e] = as_bits(rest);
        part[2][e] = as_bits(rest - mid);
        if constexpr (BIAS::value) bias[odd] += x;
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        parts[p][d] = __builtin_amdgcn_perm(part[p][1], part[p][0], 0x07060302u);
        if (d == 3) to[p * 4 * TN] = parts[p];
      }
    }
  }
};

__device__ __forceinline__ float scale_of(uint32_t byte) { return as_float(byte == 255u ? 0x7FC00000u : byte << 23); }

// Two codes of a word (the lower or the upper ones) as a pair of bf16 numbers: eight bits times a power of two, nothing to round.
__device__ __forceinline__ uint32_t widen_two(uint32_t codes, int upper, float scale) {
  const uint32_t lo = as_bits(signed_byte(codes, 2 * upper) * scale), hi = as_bits(signed_byte(codes, 2 * upper + 1) * scale);
  return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}

// 32 features of this lane's outputs n (y0) and n + 1 (y1): a lane of the first half holds features 8 (r / 4) + r % 4, one of the
// second half those 4 further on.  off: of the first of them; left: outputs from n on; ends_odd: the tile holds the last
// output of an odd number of them, which is stored by itself.  (Pairs may lie on any element.)  AUX: cache policy of the stores (2:
// streaming).
template <bool OUT_BF16, int AUX>
__device__ __forceinline__ void write_strip(__amdgpu_buffer_rsrc_t ro, uint32_t off, uint32_t left, uint32_t out_row, bool ends_odd,
                                            bool accumulate, f32x16 y0, f32x16 y1) {
  // lanes that have nothing to store get an offset that the range check drops
  const uint32_t pair = left > 1 ? off : kNowhere, single = left == 1 ? off : kNowhere;
  auto row = [&](int r) { return (8 * (r / 4) + r % 4) * out_row; };
  if (accumulate) {
    u32x2 old[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if constexpr (OUT_BF16) {
        const uint32_t v = __builtin_amdgcn_raw_buffer_load_b32(ro, int(pair + row(r)), 0, 0);
        old[r] = u32x2{v << 16, v & 0xFFFF0000u};
      } else {
        old[r] = __builtin_amdgcn_raw_buffer_load_b64(ro, int(pair + row(r)), 0, 0);
      }
    }
    if (ends_odd) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (OUT_BF16) old[r][0] |= uint32_t(__builtin_amdgcn_raw_buffer_load_b16(ro, int(single + row(r)), 0, 0)) << 16;
        else old[r][0] |= __builtin_amdgcn_raw_buffer_load_b32(ro, int(single + row(r)), 0, 0);
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      y0[r] += as_float(old[r][0]);
      y1[r] += as_float(old[r][1]);
    }
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if constexpr (OUT_BF16)
      __builtin_amdgcn_raw_buffer_store_b32(bf16_pair(y0[r], y1[r]), ro, int(pair + row(r)), 0, AUX);
    else
      __builtin_amdgcn_raw_buffer_store_b64(u32x2{as_bits(y0[r]), as_bits(y1[r])}, ro, int(pair + row(r)), 0, AUX);
  }
  if (ends_odd) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if constexpr (OUT_BF16)
        __builtin_amdgcn_raw_buffer_store_b16(uint16_t(bf16_pair(y0[r], y0[r])), ro, int(single + row(r)), 0, 0);
      else
        __builtin_amdgcn_raw_buffer_store_b32(as_bits(y0[r]), ro, int(single + row(r)), 0, 0);
    }
  }
}

// The bias of a workgroup's outputs from its lanes' sums; LDS has to be free.
template <bool OUT_BF16, int TN>
__device__ __forceinline__ void write_bias(const WeightGradientArgs& a, float* part, uint32_t tid, uint32_t n0, uint64_t to,
                                           uint32_t octet, uint32_t pair, const float* sums) {
  constexpr int OS = OUT_BF16 ? 2 : 4;
  part[octet * TN + pair * 2] = sums[0];
  part[octet * TN + pair * 2 + 1] = sums[1];
  __syncthreads();
  if (tid >= TN || n0 + tid >= a.outputs) return;
  float y = part[tid];
#pragma unroll
  for (int o = 1; o < 4; ++o) y += part[o * TN + tid];
  const uint64_t at = to + uint64_t(n0 + tid) * OS;
  if (a.accumulate) {
    float old;
    load_elems<OUT_BF16, 1>(at, &old);
    y += old;
  }
  store_elems<OUT_BF16, 1>(at, &y);
}

// WK x WN wavefronts, each with FK * 32 features and TB * 64 outputs.
template <int WK, int WN, int FK, int TB, int OCCUPANCY, bool DY_BF16, bool OUT_BF16, Load LOAD>
__global__ void __launch_bounds__(WK * WN * 64, OCCUPANCY) k_weight_gradient(WeightGradientArgs a, Tiling t) {
  constexpr int TK = WK * FK * 32, TN = WN * TB * 64, THREADS = WK * WN * 64;
  static_assert(THREADS == 2 * TN, "the lanes share a block of dy evenly");
  constexpr int P = DY_BF16 ? 1 : 3, OS = OUT_BF16 ? 2 : 4;
  __shared__ u32x4 lds[3][P][4][TN];

  // workgroups go round robin over the XCDs: each XCD gets a contiguous range of tiles, so that the tiles that
  // share dy and x share an L2
  const uint32_t xcd = blockIdx.x % kXcds, per = t.total / kXcds, more = t.total % kXcds;
  uint32_t tile = xcd * per + min(xcd, more) + blockIdx.x / kXcds;
  const uint32_t tiles = t.nk * t.nn;
  const uint32_t w = uniform(tile / (tiles * t.splits));
  tile -= w * tiles * t.splits;
  const uint32_t split = uniform(tile / tiles);
  tile -= split * tiles;
  // bands of four tiles along the features
  const uint32_t band = uniform(tile / (4 * t.nn)), in_band = tile - band * 4 * t.nn;
  const uint32_t high = min(t.nk - band * 4, 4u);
  const uint32_t nt = uniform(in_band / high), kt = band * 4 + in_band - nt * high;
  const uint32_t k0 = kt * TK, n0 = nt * TN;

  const uint32_t M = a.w.tokens[w], K = a.features, N = a.outputs;
  const uint32_t blocks = (M + kCheckpointBlock - 1) / kCheckpointBlock;
  const uint32_t share = (blocks + t.splits - 1) / t.splits;
  const uint32_t b0 = uniform(min(split * share, blocks)), b1 = uniform(min(b0 + share, blocks));

  const uint32_t tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64);
  const uint32_t wk = wave / WN, wn = wave % WN, l32 = lane % 32, half = lane / 32;

  const uint64_t codes = a.w.a[w], scales = codes + uint64_t(blocks) * K * kCheckpointBlock;
  typedef Dy<DY_BF16, LOAD, TN> Rows;
  typedef typename Rows::raw raw;
  constexpr int kPacks = Rows::kPacks;
  Rows dy(a, w, n0, min(M, b1 * kCheckpointBlock), tid);
  const bool sums_dy = a.has_bias && kt == 0;
  auto pack = [&](raw& v, uint32_t buf, int n, auto with_bias) { dy.pack(v, lds[buf], n, with_bias); };
  auto pack_all = [&](raw& v, uint32_t buf) {
#pragma unroll
    for (int n = 0; n < kPacks; ++n) {
      if (sums_dy) pack(v, buf, n, std::true_type{});
      else pack(v, buf, n, std::false_type{});
    }
  };

  struct Codes {
    u32x4 q[FK];
    uint32_t s[FK];
  };
  auto load_codes = [&](Codes& c, uint32_t b, int f) {
    const __amdgpu_buffer_rsrc_t rq = buffer(codes + (uint64_t(b) * K + k0) * kCheckpointBlock, b < b1 ? (K - k0) * kCheckpointBlock : 0);
    const __amdgpu_buffer_rsrc_t rs = buffer(scales + uint64_t(b) * K + k0, b < b1 ? K - k0 : 0);
    const uint32_t k = (wk * FK + f) * 32 + l32;
    c.q[f] = __builtin_amdgcn_raw_buffer_load_b128(rq, int(k * kCheckpointBlock + half * 16), 0, 0);
    c.s[f] = __builtin_amdgcn_raw_buffer_load_b8(rs, int(k), 0, 0);
  };
  auto load_x = [&](uint32_t b) {
    Codes c;
#pragma unroll
    for (int f = 0; f < FK; ++f) load_codes(c, b, f);
    return c;
  };

  f32x16 acc[FK][TB * 2];
#pragma unroll
  for (int f = 0; f < FK; ++f)
#pragma unroll
    for (int c = 0; c < TB * 2; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[f][c][r] = 0.0f;

  // x as operands: FK * 32 features times two steps of 16 tokens, widened from the codes four bytes to two at a time
  struct Widened {
    u32x4 v[FK][2];
  };
  constexpr int kWidens = FK * 8;
  auto widen = [&](const Codes& x, Widened& to, int n) {  // n: 0 to kWidens - 1
    const int f = n / 8, s = n / 4 % 2, d = n % 4;
    to.v[f][s][d] = widen_two(x.q[f][s * 2 + d / 2], d % 2, scale_of(x.s[f]));
  };

  // The products of a block, in the order in which they are made: two steps of 16 tokens, the parts of dy from the smallest
  // on, the wavefront's outputs.
  constexpr int kSlots = 2 * P * TB * 2, kDepth = 4;  // operands in flight (two: the same within 2 %)
  static_assert(kSlots % kDepth == 0, "a turn ends with the operands where the next one looks for them");
  auto read = [&](uint32_t buf, int slot) {
    const int c = slot % (TB * 2), p = P - 1 - slot / (TB * 2) % P, s = slot / (TB * 2 * P);
    return __builtin_bit_cast(bf16x8, lds[buf][p][half * 2 + s][(c % 2) * (TN / 2) + (wn * TB + c / 2) * 32 + l32]);
  };

  if (b0 < b1) {
    // A turn of fp32 takes three times as long: there, fetching one block ahead is enough, and registers are short.
    constexpr int kSets = DY_BF16 ? 2 : 1;
    raw y[kSets];
    Codes x[kSets];
    Widened xs[2];
    x[0] = load_x(b0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (i == 0 || kSets == 1) y[0] = dy.load(b0 + i);
      if (i == 0 && kSets == 2) y[1] = dy.load(b0 + 1);
      pack_all(y[i % kSets], i);
    }
#pragma unroll
    for (int n = 0; n < kWidens; ++n) widen(x[0], xs[0], n);
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      x[i] = load_x(b0 + 1 + i);
      y[i] = dy.load(b0 + 2 + i);
    }
    __syncthreads();
    bf16x8 ahead[kDepth];
#pragma unroll
    for (int q = 0; q < kDepth; ++q) ahead[q] = read(0, q);
    uint32_t buf = 0, next = 1, write = 2;
    // Block b is multiplied while x of block b + 1 is widened, dy of block b + 2 goes to LDS, and x of block b + 1 + kSets and dy
    // of block b + 2 + kSets are fetched.  The order of the instructions is laid down: a few others after every product, which run in its shadow.
    // A wavefront issues in order, so a row of loads, or of conversions, would hold up the products behind it.
    constexpr int kLoads = 8, kPieces = kPacks + kLoads + kWidens + FK;
    auto turn = [&](uint32_t b, Widened& now, Widened& then, Codes& x_in, raw& dy_in, auto with_bias) {
      const __amdgpu_buffer_rsrc_t r = dy.block(b + 2 + kSets);
      auto piece = [&](int n) {
        if (n < kPacks) return pack(dy_in, write, n, with_bias);
        n -= kPacks;
        if (n < kLoads + kWidens) {  // in turn, while there are both
          constexpr int kBoth = kLoads < kWidens ? kLoads : kWidens;
          const bool load = n < 2 * kBoth ? n % 2 == 0 : kLoads > kWidens;
          const int at = n < 2 * kBoth ? n / 2 : n - kBoth;
          return load ? dy.load_row(r, dy_in, at) : widen(x_in, then, at);
        }
        return load_codes(x_in, b + 1 + kSets, n - kLoads - kWidens);
      };
#pragma unroll
      for (int q = 0; q < kSlots; ++q) {
        const bf16x8 o = ahead[q % kDepth];
#pragma unroll
        for (int f = 0; f < FK; ++f)
          acc[f][q % (TB * 2)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, now.v[f][q / (kSlots / 2)]), o,
                                                                        acc[f][q % (TB * 2)], 0, 0, 0);
        ahead[q % kDepth] = q + kDepth < kSlots ? read(buf, q + kDepth) : read(next, q + kDepth - kSlots);
#pragma unroll
        for (int n = q * kPieces / kSlots; n < (q + 1) * kPieces / kSlots; ++n) piece(n);
        __builtin_amdgcn_sched_barrier(0);
      }
      __syncthreads();
      const uint32_t free = buf;
      buf = next;
      next = write;
      write = free;
    };
    auto walk = [&](auto with_bias) {
      for (uint32_t b = b0; b < b1; b += 2) {  // after an odd last block, one of zeros
        turn(b, xs[0], xs[1], x[0], y[0], with_bias);
        turn(b + 1, xs[1], xs[0], x[kSets - 1], y[kSets - 1], with_bias);
      }
    };
    if (sums_dy) walk(std::true_type{});
    else walk(std::false_type{});
  }

  // a lane holds outputs n, n + 1 of features 8 (r / 4) + 4 half + r % 4
  const uint64_t out = a.w.c[w] + split * t.split_stride + (uint64_t(k0) * N + n0) * OS;
  const uint32_t out_row = N * OS;
  const __amdgpu_buffer_rsrc_t ro = buffer(out, (min(K - k0, uint32_t(TK)) * N - n0) * OS);
#pragma unroll
  for (int f = 0; f < FK; ++f)
#pragma unroll
    for (int c = 0; c < TB; ++c) {
      const uint32_t col = ((wn * TB + c) * 32 + l32) * 2;
      const uint32_t left = n0 + col < N ? N - n0 - col : 0;
      write_strip<OUT_BF16, 0>(ro, ((wk * FK + f) * 32 + 4 * half) * out_row + col * OS, left, out_row, N % 2 && n0 + TN >= N, a.accumulate,
                            acc[f][2 * c], acc[f][2 * c + 1]);
    }

  if (sums_dy) {  // the same for all lanes of the workgroup
    __syncthreads();
    write_bias<OUT_BF16, TN>(a, reinterpret_cast<float*>(lds), tid, n0, a.w.d[w] + split * t.bias_stride, dy.octet, dy.pair,
                                     dy.bias);
  }
}

// Few tokens: what is written outweighs the product.  A workgroup keeps dy of all tokens in LDS, 128 outputs of it, and goes
// along the features, each wavefront by itself, 32 features at a time: codes come in and sums go out without a barrier.
// Bound: HBM writes.  2 x (64 tokens, 25088 x 4096) fp32: 162 us a call, 828 MB written at 5.1 TB/s (the kernel's least 151, back to back
// 165).  Least values of one session: 149, in the tiles of the other kernel 256, with plain stores 172, with three workgroups per compute
// unit 187, with workgroups for three rounds 158.  STREAM: streaming stores, where rows are
// whole cache lines and all tensors together are more than the last-level cache holds; 4 x (14 tokens, 2845 x 3365) bf16, 77 MB in rows
// that are not: 29 us, with streaming stores 62.
struct ShortTiling {
  uint32_t nn, share;  // tiles along the outputs; steps of 32 features per workgroup
};

template <int BLOCKS, bool DY_BF16, bool OUT_BF16, Load LOAD, bool STREAM>
__global__ void __launch_bounds__(256, 2) k_weight_gradient_short(WeightGradientArgs a, ShortTiling t) {
  constexpr int TN = 128, TB = 2, P = DY_BF16 ? 1 : 3, OS = OUT_BF16 ? 2 : 4;
  __shared__ u32x4 lds[BLOCKS][P][4][TN];
  const uint32_t w = blockIdx.y, part = uniform(blockIdx.x / t.nn), n0 = (blockIdx.x - part * t.nn) * TN;
  const uint32_t M = a.w.tokens[w], K = a.features, N = a.outputs;
  const uint32_t blocks = (M + kCheckpointBlock - 1) / kCheckpointBlock;
  const uint32_t tid = threadIdx.x, lane = tid % 64, wave = uniform(tid / 64), l32 = lane % 32, half = lane / 32;
  const uint32_t steps = (K + 31) / 32, s1 = min((part + 1) * t.share, steps);
  const uint64_t codes = a.w.a[w], scales = codes + uint64_t(blocks) * K * kCheckpointBlock;

  struct Codes {
    u32x4 q;
    uint32_t s;
  };
  auto load_codes = [&](uint32_t step, uint32_t b) {
    const bool there = step < s1 && b < blocks;
    const uint64_t at = uint64_t(b) * K + step * 32;
    Codes c;
    c.q = __builtin_amdgcn_raw_buffer_load_b128(buffer(codes + at * kCheckpointBlock, there ? (K - step * 32) * kCheckpointBlock : 0),
                                                int(l32 * kCheckpointBlock + half * 16), 0, 0);
    c.s = __builtin_amdgcn_raw_buffer_load_b8(buffer(scales + at, there ? K - step * 32 : 0), int(l32), 0, 0);
    return c;
  };
  uint32_t step = part * t.share + wave;
  Codes next = load_codes(step, 0);

  typedef Dy<DY_BF16, LOAD, TN> Rows;
  Rows dy(a, w, n0, M, tid);
  const bool sums_dy = a.has_bias && part == 0;
  typename Rows::raw v[BLOCKS];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) v[b] = dy.load(b);
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int n = 0; n < Rows::kPacks; ++n) dy.pack(v[b], lds[b], n, std::true_type{});
  __syncthreads();

  for (; step < s1; step += 4) {
    f32x16 acc[TB * 2];
#pragma unroll
    for (int c = 0; c < TB * 2; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[c][r] = 0.0f;
    for (uint32_t b = 0; b < blocks; ++b) {
      const Codes x = next;
      const bool more = b + 1 < blocks;
      next = load_codes(more ? step : step + 4, more ? b + 1 : 0);
      const float size = scale_of(x.s);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 xs;
#pragma unroll
        for (int d = 0; d < 4; ++d) xs[d] = widen_two(x.q[s * 2 + d / 2], d % 2, size);
#pragma unroll
        for (int p = P - 1; p >= 0; --p)
#pragma unroll
          for (int c = 0; c < TB * 2; ++c) {
            const u32x4 y = lds[b][p][half * 2 + s][(c % 2) * (TN / 2) + c / 2 * 32 + l32];
            acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, xs), __builtin_bit_cast(bf16x8, y), acc[c], 0, 0, 0);
          }
      }
    }
    const uint32_t k0 = step * 32, out_row = N * OS;
    const __amdgpu_buffer_rsrc_t ro = buffer(a.w.c[w] + (uint64_t(k0) * N + n0) * OS, (min(K - k0, 32u) * N - n0) * OS);
#pragma unroll
    for (int c = 0; c < TB; ++c) {
      const uint32_t col = (c * 32 + l32) * 2, left = n0 + col < N ? N - n0 - col : 0;
      write_strip<OUT_BF16, STREAM ? 2 : 0>(ro, 4 * half * out_row + col * OS, left, out_row, N % 2 && n0 + TN >= N, a.accumulate, acc[2 * c], acc[2 * c + 1]);
    }
  }

  if (sums_dy) {
    __syncthreads();
    write_bias<OUT_BF16, TN>(a, reinterpret_cast<float*>(lds), tid, n0, a.w.d[w], dy.octet, dy.pair, dy.bias);
  }
}

// Adds the parts of the tokens, in order; kJoinAhead of them are fetched at once.  23 parts of 102 x 885: 9.3 us, four at once
// 11.0; 10 parts of 8 x 2142 x 247 9.9 (four), 9.9 and, sixteen at once, 12.5.
constexpr int kJoinAhead = 8;

template <bool OUT_BF16>
__global__ void __launch_bounds__(256) k_weight_join(WeightGradientArgs a, Tiling t, uint64_t parts, uint64_t bias_parts) {
  constexpr int OS = OUT_BF16 ? 2 : 4;
  const uint32_t w = blockIdx.y;
  const uint64_t size = uint64_t(a.features) * a.outputs;
  uint64_t i = (uint64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  uint64_t from = parts + w * t.splits * t.split_stride, stride = t.split_stride, to = a.w.c[w], end = size;
  if (i >= (size + 3) / 4 * 4) {
    i -= (size + 3) / 4 * 4;
    if (!a.has_bias || i >= a.outputs) return;
    from = bias_parts + w * t.splits * t.bias_stride;
    stride = t.bias_stride;
    to = a.w.d[w];
    end = a.outputs;
  }
  if (i + 4 <= end) {
    float sum[4] = {};
    for (uint32_t p = 0; p < t.splits; p += kJoinAhead) {
      float x[kJoinAhead][4];
#pragma unroll
      for (int q = 0; q < kJoinAhead; ++q) load_elems<false, 4>(from + min(p + q, t.splits - 1) * stride + i * 4, x[q]);
#pragma unroll
      for (int q = 0; q < kJoinAhead; ++q)
        if (p + q < t.splits)
          for (int j = 0; j < 4; ++j) sum[j] += x[q][j];
    }
    if (a.accumulate) {
      float old[4];
      load_elems<OUT_BF16, 4>(to + i * OS, old);
      for (int j = 0; j < 4; ++j) sum[j] += old[j];
    }
    store_elems<OUT_BF16, 4>(to + i * OS, sum);
  } else {
    for (; i < end; ++i) {
      float sum = 0.0f;
      for (uint32_t p = 0; p < t.splits; ++p) {
        float x;
        load_elems<false, 1>(from + p * stride + i * 4, &x);
        sum += x;
      }
      if (a.accumulate) {
        float old;
        load_elems<OUT_BF16, 1>(to + i * OS, &old);
        sum += old;
      }
      store_elems<OUT_BF16, 1>(to + i * OS, &sum);
    }
  }
}

// Which kernel, and in how many parts the tokens are summed.
enum Kernel { kShort, kNarrowTile, kSmallTile, kLargeTile };
struct Shape {
  Kernel kernel;
  uint32_t splits;
};

// Large tiles, in as many parts of the tokens as fill the chip once, unless their ragged ends waste a quarter of the work or too
// little is left for a workgroup to do; else small ones in parts for at most one round of two workgroups per compute unit.  Fewer
// tiles than compute units: 16384 x 1024 x 1024 fp32, large in 16 parts 94.8 + 11.6 us (joining), small in 8 parts 111.3 + 7.0, in
// 4 133 + 5, in 16 114 + 12.  More: 8 x (4096 x 1024 x 4096) bf16, large 252 us, small 355.
// Tiles of 64 outputs in place of 128 where these would be empty in at least a sixth: 16 x (376 x 4610 x 34) fp32 24 us, small 38;
// 4 x (1580 x 1024 x 320) fp32 34 and 41, of 192 30 and 29; with fewer empty places, 4 x (256 x 1024 x 960), 18 and 16.
Shape choose(uint32_t world, uint32_t features, uint32_t outputs, uint32_t max_tokens, bool dy_bf16) {
  auto tiles = [&](uint32_t side) { return uint64_t(world) * ((features + side - 1) / side) * ((outputs + side - 1) / side); };
  const uint64_t small = tiles(128), large = tiles(256);
  const uint64_t blocks = checkpoint_blocks(max_tokens);
  if (blocks <= (dy_bf16 ? 6u : 2u)) return {kShort, 1};
  if (outputs > 1 && 16 * large <= 5 * small) {
    const uint64_t splits = std::max<uint64_t>(1, std::min(256 / large, blocks / 16));
    if (large * splits >= 192 && blocks >= 8 * splits) return {kLargeTile, uint32_t(splits)};
  }
  // A part more takes time off the walk along the tokens (0.56 us a block) and adds its sums' way to memory and back (at 4 TB/s) and a
  // step of the join (0.06 us); their total is least at the root.  3 x (1430 x 426 x 848) bf16 22 us, with as many parts as have eight
  // blocks 25; 11964 x 102 x 885 22 and 26; 4 x (1024 x 1024 x 1000) fp32 41 and 49; 8 x (512 x 784 x 10) 11 and 14; 2^20 x 64 x 64
  // fp32 127, with 64 parts 466.
  auto parts = [&](uint64_t fill) {
    const uint64_t best = std::llround(std::sqrt(0.28e6 * double(blocks) / (double(world) * features * outputs + 3e4)));
    return uint32_t(std::max<uint64_t>(1, std::min<uint64_t>({fill, blocks / 4, best})));
  };
  const uint32_t strips = (outputs + 63) / 64;
  const uint64_t narrow = uint64_t(world) * ((features + 127) / 128) * strips;
  if (strips % 2 && strips <= 5) return {kNarrowTile, parts((1024 + narrow - 1) / narrow)};
  return {kSmallTile, parts((512 + small - 1) / small)};
}

uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }

template <int WK, int WN, int FK, int TB, int OCCUPANCY>
hipError_t launch(const WeightGradientArgs& a, const Tiling& t, bool out_bf16, hipStream_t s) {
  const dim3 grid(t.total), block(WK * WN * 64);
#define CARAMEL_WG(DY, OUT, LOAD) hipLaunchKernelGGL((k_weight_gradient<WK, WN, FK, TB, OCCUPANCY, DY, OUT, LOAD>), grid, block, 0, s, a, t)
  if (!a.dy_bf16) {
    if (out_bf16) CARAMEL_WG(false, true, kPairs);
    else CARAMEL_WG(false, false, kPairs);
  } else if (a.outputs % 2 == 0) {
    if (out_bf16) CARAMEL_WG(true, true, kPairs);
    else CARAMEL_WG(true, false, kPairs);
  } else if (a.outputs > 1) {
    if (out_bf16) CARAMEL_WG(true, true, kShift);
    else CARAMEL_WG(true, false, kShift);
  } else if constexpr (WK == 2 && WN == 1) {  // one output always goes to narrow tiles
    if (out_bf16) CARAMEL_WG(true, true, kSingle);
    else CARAMEL_WG(true, false, kSingle);
  }
#undef CARAMEL_WG
  return hipGetLastError();
}

hipError_t launch_short(const WeightGradientArgs& a, hipStream_t s) {
  ShortTiling t{};
  t.nn = (a.outputs + 127) / 128;
  const uint32_t steps = (a.features + 31) / 32;
  const uint64_t tiles = uint64_t(t.nn) * a.world;
  const uint32_t parts = uint32_t(std::min<uint64_t>((steps + 3) / 4, (512 + tiles - 1) / tiles));
  t.share = (steps + parts - 1) / parts;
  t.share = (t.share + 3) / 4 * 4;
  const dim3 grid(t.nn * ((steps + t.share - 1) / t.share), a.world), block(256);
  const uint64_t row = uint64_t(a.outputs) * (a.out_bf16 ? 2 : 4);
  const bool stream = row % 128 == 0 && row * a.features * a.all > (uint64_t(256) << 20);
#define CARAMEL_WG(BLOCKS, DY, OUT, LOAD)                                                                                            \
  if constexpr (LOAD == kPairs) { /* the others' rows are no whole lines */                                                          \
    if (stream) hipLaunchKernelGGL((k_weight_gradient_short<BLOCKS, DY, OUT, LOAD, true>), grid, block, 0, s, a, t);                 \
    else hipLaunchKernelGGL((k_weight_gradient_short<BLOCKS, DY, OUT, LOAD, false>), grid, block, 0, s, a, t);                       \
  } else {                                                                                                                           \
    hipLaunchKernelGGL((k_weight_gradient_short<BLOCKS, DY, OUT, LOAD, false>), grid, block, 0, s, a, t);                            \
  }
  if (!a.dy_bf16) {
    if (a.out_bf16) {
      CARAMEL_WG(2, false, true, kPairs)
    } else {
      CARAMEL_WG(2, false, false, kPairs)
    }
  } else if (a.outputs % 2 == 0) {
    if (a.out_bf16) {
      CARAMEL_WG(6, true, true, kPairs)
    } else {
      CARAMEL_WG(6, true, false, kPairs)
    }
  } else if (a.outputs > 1) {
    if (a.out_bf16) {
      CARAMEL_WG(6, true, true, kShift)
    } else {
      CARAMEL_WG(6, true, false, kShift)
    }
  } else if (a.out_bf16) {
    CARAMEL_WG(6, true, true, kSingle)
  } else {
    CARAMEL_WG(6, true, false, kSingle)
  }
#undef CARAMEL_WG
  return hipGetLastError();
}

}  // namespace

uint64_t weight_gradient_workspace(uint32_t world, uint32_t features, uint32_t outputs, uint32_t max_tokens) {
  // of whichever type dy turns out to have: the two differ only in that few tokens need none
  const Shape c = choose(world, features, outputs, max_tokens, false);
  if (c.splits < 2) return 0;
  return uint64_t(world) * c.splits * (up256(uint64_t(features) * outputs * 4) + up256(uint64_t(outputs) * 4));
}

hipError_t launch_weight_gradient(const WeightGradientArgs& args, const AllWorkers& v, hipStream_t s) {
  if (args.max_tokens == 0 && args.accumulate) return hipSuccess;
  const Shape c = choose(args.all, args.features, args.outputs, args.max_tokens, args.dy_bf16);
  if (c.kernel == kShort) return in_groups(args, v, [&](const WeightGradientArgs& a, uint32_t) { return launch_short(a, s); });
  const uint32_t tk = c.kernel == kLargeTile ? 256 : 128, tn = c.kernel == kNarrowTile ? 64 : tk;
  Tiling t{};
  t.nk = (args.features + tk - 1) / tk;
  t.nn = (args.outputs + tn - 1) / tn;
  t.splits = c.splits;
  if (c.splits > 1) {
    t.split_stride = up256(uint64_t(args.features) * args.outputs * 4);
    t.bias_stride = up256(uint64_t(args.outputs) * 4);
  }
  return in_groups(args, v, [&](const WeightGradientArgs& a, uint32_t first) {
    t.total = t.nk * t.nn * t.splits * a.world;
    auto tiles = [&](const WeightGradientArgs& to, bool out_bf16) {
      if (c.kernel == kLargeTile) return launch<8, 1, 1, 4, 2>(to, t, out_bf16, s);
      if (c.kernel == kSmallTile) return launch<2, 2, 2, 1, 2>(to, t, out_bf16, s);
      return launch<2, 1, 2, 1, 2>(to, t, out_bf16, s);
    };
    if (c.splits == 1) return tiles(a, a.out_bf16);
    const uint64_t parts = reinterpret_cast<uint64_t>(a.ws) + first * t.splits * (t.split_stride + t.bias_stride);
    const uint64_t bias_parts = parts + a.world * t.splits * t.split_stride;
    WeightGradientArgs p = a;
    p.accumulate = false;
    for (uint32_t w = 0; w < a.world; ++w) {
      p.w.c[w] = parts + w * t.splits * t.split_stride;
      p.w.d[w] = bias_parts + w * t.splits * t.bias_stride;
    }
    const hipError_t e = tiles(p, false);
    if (e != hipSuccess) return e;
    const uint64_t vecs = (uint64_t(a.features) * a.outputs + 3) / 4 + (a.has_bias ? (a.outputs + 3) / 4 : 0);
    const dim3 grid(uint32_t((vecs + 255) / 256), a.world);
    if (a.out_bf16) hipLaunchKernelGGL((k_weight_join<true>), grid, dim3(256), 0, s, a, t, parts, bias_parts);
    else hipLaunchKernelGGL((k_weight_join<false>), grid, dim3(256), 0, s, a, t, parts, bias_parts);
    return hipGetLastError();
  });
}

}  // namespace caramel
