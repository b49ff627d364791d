// Weight and bias gradients of a dense layer, from its input's 8-bit checkpoint.
//
//   dW[k, n] = round([dW[k, n] +] sum over the tokens m of x[m, k] * dy[m, n])
//   db[n]    = round([db[n] +]    sum over the tokens m of dy[m, n])
//
// for all workers of a plan in one launch.  The product runs on the matrix cores in bf16 with fp32 sums, and
// loses nothing on the way in: a value read back from a checkpoint is a bf16 number (checkpoint.hip), and an
// fp32 gradient is the sum of three bf16 numbers (24 significant bits, eight each), which go through the
// matrix cores one after the other.  That is three products instead of one, at 16 times the rate of
// the fp32 matrix instructions.
//
// Tiling.  A workgroup owns TK features x TN outputs and walks the tokens 32 at a time (one block of the
// checkpoint).  dy is brought to LDS once per workgroup, transposed on the way through registers so that
// a matrix operand (eight tokens of one output) is one 128-bit read; x goes from the checkpoint straight
// to registers, 16 bytes = 16 tokens of one feature per lane, and is widened there: its layout is already that
// of the operand.  The tokens are dealt to the operand's places in the same permuted order on both sides.
// Outputs are dealt to lanes in pairs, so that a lane ends with two neighbours to store.
#include <algorithm>

#include "layers.hpp"
#include "vec.hpp"

namespace caramel {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kXcds = 8;
constexpr uint32_t kNowhere = 0x7FFFFFF0u;  // an offset that every range check drops

struct Tiling {
  uint32_t nk, nn;        // tiles along features and outputs
  uint32_t splits;        // parts of the tokens
  uint32_t total;         // workgroups
  uint64_t split_stride;  // bytes from one part's sums to the next (0: one part, sums go to the gradient itself)
  uint64_t bias_stride;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(uint64_t base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, int(bytes), kRawBuffer);
}

// WK x WN wavefronts, each with FK * 32 features and TB * 64 outputs.  ODD: bf16 rows of dy start on odd
// elements or end in the middle of a pair, so elements are loaded one by one.
template <int WK, int WN, int FK, bool DY_BF16, bool OUT_BF16, bool ODD>
__global__ void __launch_bounds__(WK * WN * 64, 2) k_weight_gradient(WeightGradientArgs a, Tiling t) {
  constexpr int TB = WK / 2, TK = WK * FK * 32, TN = WN * TB * 64, THREADS = WK * WN * 64;
  static_assert(TN * 2 == THREADS, "each lane brings eight tokens of two outputs per step");
  constexpr int P = DY_BF16 ? 1 : 3, ES = DY_BF16 ? 2 : 4, OS = OUT_BF16 ? 2 : 4;
  __shared__ u32x4 lds[2][P][4][TN];

  // workgroups go round robin over the XCDs: each XCD gets a contiguous range of tiles, so that the tiles that
  // share dy and x share an L2
  const uint32_t xcd = blockIdx.x % kXcds, per = t.total / kXcds, more = t.total % kXcds;
  uint32_t tile = xcd * per + min(xcd, more) + blockIdx.x / kXcds;
  const uint32_t tiles = t.nk * t.nn;
  const uint32_t w = tile / (tiles * t.splits);
  tile -= w * tiles * t.splits;
  const uint32_t split = tile / tiles;
  tile -= split * tiles;
  // bands of four tiles along the features
  const uint32_t band = tile / (4 * t.nn), in_band = tile - band * 4 * t.nn;
  const uint32_t high = min(t.nk - band * 4, 4u);
  const uint32_t kt = band * 4 + in_band % high, nt = in_band / high;
  const uint32_t k0 = kt * TK, n0 = nt * TN;

  const uint32_t M = a.w.tokens[w], K = a.features, N = a.outputs;
  const uint32_t blocks = (M + kCheckpointBlock - 1) / kCheckpointBlock;
  const uint32_t share = (blocks + t.splits - 1) / t.splits;
  const uint32_t b0 = min(split * share, blocks), b1 = min(b0 + share, blocks);

  const uint32_t tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const uint32_t wk = wave / WN, wn = wave % WN, l32 = lane % 32, half = lane / 32;
  const uint32_t octet = tid / (TN / 2), pair = tid % (TN / 2);

  const uint64_t codes = a.w.a[w], scales = codes + uint64_t(blocks) * K * kCheckpointBlock;
  const uint64_t dy = a.w.b[w] + uint64_t(n0) * ES;
  const uint32_t row_bytes = uint32_t(a.dy_pitch) * ES;
  const uint32_t dy_off = octet * 8 * row_bytes + pair * 2 * ES;

  typedef uint32_t raw __attribute__((ext_vector_type(DY_BF16 ? 8 : 16)));
  auto load_dy = [&](uint32_t b) {
    const uint32_t rows = min(M - b * kCheckpointBlock, kCheckpointBlock);
    const __amdgpu_buffer_rsrc_t r = buffer(dy + uint64_t(b) * kCheckpointBlock * row_bytes, (rows - 1) * row_bytes + (N - n0) * ES);
    raw v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int off = int(dy_off + j * row_bytes);
      if constexpr (!DY_BF16) {
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
        v[2 * j] = x[0];
        v[2 * j + 1] = x[1];
      } else if constexpr (ODD) {
        v[j] = uint32_t(__builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0)) |
               uint32_t(__builtin_amdgcn_raw_buffer_load_b16(r, off + 2, 0, 0)) << 16;
      } else {
        v[j] = __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0);
      }
    }
    return v;
  };

  const bool sums_dy = a.has_bias && kt == 0;
  float bias[2] = {0.0f, 0.0f};
  auto keep_dy = [&](const raw& v, int buf) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (DY_BF16) {
        u32x4 y;
#pragma unroll
        for (int d = 0; d < 4; ++d) y[d] = __builtin_amdgcn_perm(v[2 * d + 1], v[2 * d], i ? 0x07060302u : 0x05040100u);
        lds[buf][0][octet][i * (TN / 2) + pair] = y;
      } else {
        // v = hi + mid + lo: the upper half of a float is a bf16 number, and the rest is exact
        u32x4 y[3];
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          uint32_t part[3][2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t bits = v[2 * (2 * d + e) + i];
            const float x = as_float(bits), hi = bf16_high(bits);
            const float rest = x == hi ? 0.0f : x - hi;  // an infinity is all in its upper half
            const float mid = bf16_high(as_bits(rest));
            part[0][e] = bits;
            part[1][e] = as_bits(rest);
            part[2][e] = as_bits(rest - mid);
          }
#pragma unroll
          for (int p = 0; p < 3; ++p) y[p][d] = __builtin_amdgcn_perm(part[p][1], part[p][0], 0x07060302u);
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) lds[buf][p][octet][i * (TN / 2) + pair] = y[p];
      }
    }
    if (sums_dy) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (DY_BF16) {
          bias[0] += bf16_low(v[j]);
          bias[1] += bf16_high(v[j]);
        } else {
          bias[0] += as_float(v[2 * j]);
          bias[1] += as_float(v[2 * j + 1]);
        }
      }
    }
  };

  struct Codes {
    u32x4 q[FK];
    uint32_t s[FK];
  };
  auto load_x = [&](uint32_t b) {
    Codes c;
    const __amdgpu_buffer_rsrc_t rq = buffer(codes + (uint64_t(b) * K + k0) * kCheckpointBlock, (K - k0) * kCheckpointBlock);
    const __amdgpu_buffer_rsrc_t rs = buffer(scales + uint64_t(b) * K + k0, K - k0);
#pragma unroll
    for (int f = 0; f < FK; ++f) {
      const uint32_t k = (wk * FK + f) * 32 + l32;
      c.q[f] = __builtin_amdgcn_raw_buffer_load_b128(rq, int(k * kCheckpointBlock + half * 16), 0, 0);
      c.s[f] = __builtin_amdgcn_raw_buffer_load_b8(rs, int(k), 0, 0);
    }
    return c;
  };

  f32x16 acc[FK][TB * 2];
#pragma unroll
  for (int f = 0; f < FK; ++f)
#pragma unroll
    for (int c = 0; c < TB * 2; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[f][c][r] = 0.0f;

  if (b0 < b1) {
    raw next = load_dy(b0);
    Codes x = load_x(b0);
    keep_dy(next, 0);
    if (b0 + 1 < b1) next = load_dy(b0 + 1);
    int buf = 0;
    for (uint32_t b = b0; b < b1; ++b) {
      __syncthreads();
      bf16x8 xs[FK][2];
#pragma unroll
      for (int f = 0; f < FK; ++f) {
        const float size = as_float(x.s[f] == 255u ? 0x7FC00000u : x.s[f] << 23);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          u32x4 y;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            uint32_t v[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int byte = s * 8 + d * 2 + e;
              v[e] = as_bits(float(int8_t(x.q[f][byte / 4] >> (8 * (byte % 4)))) * size);
            }
            y[d] = __builtin_amdgcn_perm(v[1], v[0], 0x07060302u);
          }
          xs[f][s] = __builtin_bit_cast(bf16x8, y);
        }
      }
      if (b + 1 < b1) x = load_x(b + 1);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int p = P - 1; p >= 0; --p)
#pragma unroll
          for (int c = 0; c < TB * 2; ++c) {
            const uint32_t slot = (c % 2) * (TN / 2) + (wn * TB + c / 2) * 32 + l32;
            const bf16x8 y = __builtin_bit_cast(bf16x8, lds[buf][p][half * 2 + s][slot]);
#pragma unroll
            for (int f = 0; f < FK; ++f) acc[f][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xs[f][s], y, acc[f][c], 0, 0, 0);
          }
      if (b + 1 < b1) {
        keep_dy(next, buf ^ 1);
        if (b + 2 < b1) next = load_dy(b + 2);
      }
      buf ^= 1;
    }
  }

  // a lane holds outputs n, n + 1 of features 8 (r / 4) + 4 half + r % 4
  const uint64_t out = a.w.c[w] + split * t.split_stride + (uint64_t(k0) * N + n0) * OS;
  const uint32_t out_row = N * OS;
  const __amdgpu_buffer_rsrc_t ro = buffer(out, (min(K - k0, uint32_t(TK)) * N - n0) * OS);
  const bool pairs = N % 2 == 0;
#pragma unroll
  for (int f = 0; f < FK; ++f)
#pragma unroll
    for (int c = 0; c < TB; ++c) {
      const uint32_t col = ((wn * TB + c) * 32 + l32) * 2;
      const uint32_t left = n0 + col < N ? N - n0 - col : 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const uint32_t row = (wk * FK + f) * 32 + 8 * (r / 4) + 4 * half + r % 4;
        const uint32_t off = row * out_row + col * OS;
        float y0 = acc[f][2 * c][r], y1 = acc[f][2 * c + 1][r];
        // lanes behind the last output get an offset that the range check drops
        const int at0 = int(left > 0 ? off : kNowhere), at1 = int(left > 1 ? off + OS : kNowhere);
        if (pairs) {
          if constexpr (OUT_BF16) {
            if (a.accumulate) {
              const uint32_t old = __builtin_amdgcn_raw_buffer_load_b32(ro, at0, 0, 0);
              y0 += bf16_low(old);
              y1 += bf16_high(old);
            }
            __builtin_amdgcn_raw_buffer_store_b32(bf16_pair(y0, y1), ro, at0, 0, 0);
          } else {
            if (a.accumulate) {
              const u32x2 old = __builtin_amdgcn_raw_buffer_load_b64(ro, at0, 0, 0);
              y0 += as_float(old[0]);
              y1 += as_float(old[1]);
            }
            __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{y0, y1}), ro, at0, 0, 0);
          }
        } else if constexpr (OUT_BF16) {
          if (a.accumulate) {
            y0 += bf16_low(uint32_t(__builtin_amdgcn_raw_buffer_load_b16(ro, at0, 0, 0)));
            y1 += bf16_low(uint32_t(__builtin_amdgcn_raw_buffer_load_b16(ro, at1, 0, 0)));
          }
          const uint32_t v = bf16_pair(y0, y1);
          __builtin_amdgcn_raw_buffer_store_b16(uint16_t(v), ro, at0, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b16(uint16_t(v >> 16), ro, at1, 0, 0);
        } else {
          if (a.accumulate) {
            y0 += as_float(__builtin_amdgcn_raw_buffer_load_b32(ro, at0, 0, 0));
            y1 += as_float(__builtin_amdgcn_raw_buffer_load_b32(ro, at1, 0, 0));
          }
          __builtin_amdgcn_raw_buffer_store_b32(as_bits(y0), ro, at0, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b32(as_bits(y1), ro, at1, 0, 0);
        }
      }
    }

  if (sums_dy) {  // the same for all lanes of the workgroup
    __syncthreads();
    float* const part = reinterpret_cast<float*>(lds);
    part[octet * TN + pair * 2] = bias[0];
    part[octet * TN + pair * 2 + 1] = bias[1];
    __syncthreads();
    if (tid < TN && n0 + tid < N) {
      float y = ((part[tid] + part[TN + tid]) + part[2 * TN + tid]) + part[3 * TN + tid];
      const uint64_t at = a.bias[w] + split * t.bias_stride + uint64_t(n0 + tid) * OS;
      if (a.accumulate) {
        float old;
        load_elems<OUT_BF16, 1>(at, &old);
        y += old;
      }
      store_elems<OUT_BF16, 1>(at, &y);
    }
  }
}

// Adds the parts of the tokens, in order.
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
    to = a.bias[w];
    end = a.outputs;
  }
  if (i + 4 <= end) {
    float sum[4] = {};
#pragma unroll 4
    for (uint32_t p = 0; p < t.splits; ++p) {
      float x[4];
      load_elems<false, 4>(from + p * stride + i * 4, x);
      for (int j = 0; j < 4; ++j) sum[j] += x[j];
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

// Which tile, and in how many parts the tokens are summed.
struct Shape {
  bool large;  // 256 x 256 by eight wavefronts, or 128 x 128 by four
  uint32_t splits;
};

Shape choose(uint32_t world, uint32_t features, uint32_t outputs, uint32_t max_tokens) {
  auto tiles = [&](uint32_t side) { return uint64_t(world) * ((features + side - 1) / side) * ((outputs + side - 1) / side); };
  const uint32_t blocks = uint32_t(checkpoint_blocks(max_tokens));
  if (tiles(256) >= 192 && blocks >= 8) return {true, 1};
  const uint64_t want = (512 + tiles(128) - 1) / tiles(128);
  return {false, uint32_t(std::max<uint64_t>(1, std::min<uint64_t>(want, blocks / 8)))};
}

uint64_t up256(uint64_t x) { return (x + 255) / 256 * 256; }

template <int WK, int WN, int FK>
hipError_t launch(const WeightGradientArgs& a, const Tiling& t, bool out_bf16, hipStream_t s) {
  const dim3 grid(t.total), block(WK * WN * 64);
  // pairs of bf16 outputs are loaded together where every row starts and ends on a pair
  bool odd = a.dy_pitch % 2 || a.outputs % 2;
  for (uint32_t w = 0; w < a.world; ++w) odd = odd || a.w.b[w] % 4;
#define CARAMEL_WG(DY, OUT, ODD) hipLaunchKernelGGL((k_weight_gradient<WK, WN, FK, DY, OUT, ODD>), grid, block, 0, s, a, t)
  if (a.dy_bf16) {
    if (odd) {
      if (out_bf16) CARAMEL_WG(true, true, true);
      else CARAMEL_WG(true, false, true);
    } else {
      if (out_bf16) CARAMEL_WG(true, true, false);
      else CARAMEL_WG(true, false, false);
    }
  } else {
    if (out_bf16) CARAMEL_WG(false, true, false);
    else CARAMEL_WG(false, false, false);
  }
#undef CARAMEL_WG
  return hipGetLastError();
}

}  // namespace

uint64_t weight_gradient_workspace(uint32_t world, uint32_t features, uint32_t outputs, uint32_t max_tokens) {
  const Shape c = choose(world, features, outputs, max_tokens);
  if (c.splits < 2) return 0;
  return uint64_t(world) * c.splits * (up256(uint64_t(features) * outputs * 4) + up256(uint64_t(outputs) * 4));
}

hipError_t launch_weight_gradient(const WeightGradientArgs& a, hipStream_t s) {
  if (a.max_tokens == 0 && a.accumulate) return hipSuccess;
  const Shape c = choose(a.world, a.features, a.outputs, a.max_tokens);
  const uint32_t side = c.large ? 256 : 128;
  Tiling t{};
  t.nk = (a.features + side - 1) / side;
  t.nn = (a.outputs + side - 1) / side;
  t.splits = c.splits;
  t.total = t.nk * t.nn * t.splits * a.world;
  if (c.splits == 1) return c.large ? launch<4, 2, 2>(a, t, a.out_bf16, s) : launch<2, 2, 2>(a, t, a.out_bf16, s);

  t.split_stride = up256(uint64_t(a.features) * a.outputs * 4);
  t.bias_stride = up256(uint64_t(a.outputs) * 4);
  const uint64_t parts = reinterpret_cast<uint64_t>(a.ws), bias_parts = parts + a.world * t.splits * t.split_stride;
  WeightGradientArgs p = a;
  p.accumulate = false;
  for (uint32_t w = 0; w < a.world; ++w) {
    p.w.c[w] = parts + w * t.splits * t.split_stride;
    p.bias[w] = bias_parts + w * t.splits * t.bias_stride;
  }
  const hipError_t e = c.large ? launch<4, 2, 2>(p, t, false, s) : launch<2, 2, 2>(p, t, false, s);
  if (e != hipSuccess) return e;
  const uint64_t vecs = (uint64_t(a.features) * a.outputs + 3) / 4 + (a.has_bias ? (a.outputs + 3) / 4 : 0);
  const dim3 grid(uint32_t((vecs + 255) / 256), a.world);
  if (a.out_bf16) hipLaunchKernelGGL((k_weight_join<true>), grid, dim3(256), 0, s, a, t, parts, bias_parts);
  else hipLaunchKernelGGL((k_weight_join<false>), grid, dim3(256), 0, s, a, t, parts, bias_parts);
  return hipGetLastError();
}

}  // namespace caramel
