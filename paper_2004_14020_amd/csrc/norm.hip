// Residual root-mean-square norm, and its gradient.
//
//   h = x + residual, rounded to its type;   r_i = 1 / sqrt(mean_j h_ij^2 + eps)
//   y_ij = round((h_ij r_i) g_j)
//   gradient, with u = dy g and n = h r:   dx = [dsum +] r (u - n mean_j(u n)),   dg_j = [dg_j +] sum_i dy_ij n_ij
//
// The mean square is a sum in 64 bits: r is then the same fp32 number in whatever order the columns are added, but for one
// row in some ten million, and so is everything that follows from it, down to the 8-bit codes of values that lie next to the
// border between two of them.  (64-bit multiply-adds run at the rate of 32-bit ones here, and there is one per column.)  The
// sums of the gradient are fp32.
//
// A row stays in the registers of a team of wavefronts, so that every matrix is read and written once.  Bound by memory: 8 workers x 4096 rows x
// 1024 bf16 with a residual 44.8 us, 6.0 TB/s; the gradient, with dsum, 47.1 us, 5.7 TB/s, and 4.7 us for joining the gain's parts (a copy of
// 1 GiB: 6.08 TB/s).
#include <algorithm>
#include <type_traits>

#include "layers.hpp"
#include "rows.hpp"

namespace caramel {
namespace {

// The pieces of a lane: V of a row of a team of LANES.
template <bool BF16, int V, int LANES>
struct Pieces {
  static constexpr int N = kPiece<BF16>;
  u32x4 raw[V];
  uint32_t last;

  static __device__ __forceinline__ uint32_t column(uint32_t lane, int v) { return (v * LANES + lane) * N; }
  __device__ __forceinline__ void load(const Row<BF16>& row, uint32_t lane, bool stream) {
    row.get_all(lane * N, LANES * N, stream, raw);
    if (row.odd()) last = row.get_last();
  }
  // before the first use of an odd row's values
  __device__ __forceinline__ void finish(const Row<BF16>& row, uint32_t lane) {
    if (row.odd()) {
#pragma unroll
      for (int v = 0; v < V; ++v) row.merge_last(column(lane, v), last, raw[v]);
    }
  }
};

template <bool BF16>
__device__ __forceinline__ void store_piece(const Row<BF16>& row, uint32_t col, const float* v, bool stream) {
  const u32x4 raw = narrow<BF16>(v);
  if (stream) row.template put<true>(col, raw);
  else row.template put<false>(col, raw);
  if (row.odd()) row.put_last(col, raw);
}

// The gains of a piece of a row; they are in the plan's type, which need not be that of the rows.
template <int N>
__device__ __forceinline__ void load_gains(uint64_t at, bool bf16, uint32_t width, uint32_t col, float* g) {
  if (bf16) {
    const Row<true> row(at, width);
    u32x4 raw = row.get(col);  // (of fp32 rows, twice as many as are needed)
    if (row.odd()) row.merge_last(col, row.get_last(), raw);
    float all[8];
    widen<true>(raw, all);
#pragma unroll
    for (int j = 0; j < N; ++j) g[j] = all[j];
  } else {
    const Row<false> row(at, width);
#pragma unroll
    for (int q = 0; q < N; q += 4) widen<false>(row.get(col + q), g + q);
  }
}

// Those of all pieces of a lane: kept for all rows where that takes few registers, else loaded (from the caches) when they are needed.
template <bool BF16, int V, int LANES>
struct Gains {
  static constexpr int N = kPiece<BF16>;
  static constexpr bool kKept = V * N <= 16;
  uint64_t at;
  bool bf16;
  uint32_t width, lane;
  float kept[kKept ? V : 1][N];

  __device__ __forceinline__ Gains(uint64_t from, bool is_bf16, uint32_t columns, uint32_t l)
      : at(from), bf16(is_bf16), width(columns), lane(l) {
    if constexpr (kKept) {
#pragma unroll
      for (int v = 0; v < V; ++v) load_gains<N>(at, bf16, width, (v * LANES + lane) * N, kept[v]);
    }
  }
  __device__ __forceinline__ void get(int v, float* g) const {
    if constexpr (kKept) {
#pragma unroll
      for (int j = 0; j < N; ++j) g[j] = kept[v][j];
    } else {
      load_gains<N>(at, bf16, width, (v * LANES + lane) * N, g);
    }
  }
};

// 1 / sqrt(sum / width + eps): the hardware's 64-bit estimate, off by 2^-24 (measured, as the others here), and two steps of Newton's method,
// right to 2^-51 and then rounded.  (After one step it is off by 2^-47: of 2 x 262144 rows next to where two fp32 numbers meet, 200
// were rounded the wrong way.)
__device__ __forceinline__ float rstd_of(double sum, double inverse_width, float eps) {
  const double m = __builtin_fma(sum, inverse_width, double(eps));
  double r = __builtin_amdgcn_rsq(m);
#pragma unroll
  for (int i = 0; i < 2; ++i) r = __builtin_fma(0.5 * r, __builtin_fma(-m * r, r, 1.0), r);
  return float(m == __builtin_inf() ? 0.0 : r);
}

// Of matrices of so many bytes a call reads and writes past the caches what nobody reads again soon, so that what somebody does stays
// there: y, and dx.  Forward, 8 workers x 4096 rows x 1024 bf16: 49.6 us where all go through the caches, 43.7 with x, the residual and
// the sum past them, 45.7 with y past them too (with an 8-bit copy of y, which reads it again, 92.4, 83.2 and 90.8); its gradient 48.1
// and 39.7.  Of smaller matrices the inputs are in the caches as often as not: gradient 19.0 us and 20.1 at 8 x 1500 x 1024, 25.6
// and 23.2 at 8 x 2048 x 1024.
constexpr uint64_t kLarge = uint64_t(28) << 20;
constexpr uint32_t kGridGroups = 1u << 20;  // workgroups along x: a grid has less than 2^32 lanes in a direction

// V pieces a lane, TEAM wavefronts to a row.
template <bool BF16, int V, int TEAM>
__global__ void __launch_bounds__(TEAM <= 4 ? 256 : 1024) k_norm(NormArgs a) {
  constexpr int N = kPiece<BF16>, ES = BF16 ? 2 : 4, kWaves = TEAM <= 4 ? 4 : 16;
  __shared__ double lds[TEAM];
  const uint32_t w = blockIdx.y, group = blockIdx.x + blockIdx.z * kGridGroups;
  const uint32_t row = group * (kWaves / TEAM) + uniform(threadIdx.x / 64) / TEAM;
  if (row >= a.w.tokens[w]) return;
  constexpr int LANES = 64 * TEAM;
  const uint32_t lane = threadIdx.x % LANES;
  const uint64_t at = uint64_t(row) * a.pitch * ES;
  using P = Pieces<BF16, V, LANES>;
  const Row<BF16> rx(a.w.at[kNormX][w] + at, a.width), rr(a.w.at[kNormResidual][w] + at, a.width);
  P x, r;
  x.load(rx, lane, a.stream);
  if (a.residual) r.load(rr, lane, a.stream);
  const Gains<BF16, V, LANES> gain(a.w.at[kNormGain][w], a.gain_bf16, a.width, lane);
  x.finish(rx, lane);
  float h[V][N];
#pragma unroll
  for (int v = 0; v < V; ++v) widen<BF16>(x.raw[v], h[v]);
  if (a.residual) {
    const Row<BF16> rs(a.w.at[kNormSum][w] + at, a.width);
    r.finish(rr, lane);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float y[N];
      widen<BF16>(r.raw[v], y);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        h[v][j] += y[j];
        if constexpr (BF16) h[v][j] = bf16_low(bf16_pair(h[v][j], 0.0f));
      }
      store_piece<BF16>(rs, P::column(lane, v), h[v], a.stream);
    }
  }
  double ss = 0.0;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < N; ++j) ss = __builtin_fma(double(h[v][j]), double(h[v][j]), ss);
  ss = team_sum<TEAM>(ss, lds);
  const float rstd = rstd_of(ss, a.inverse_width, a.eps);
  if (lane == 0) reinterpret_cast<CARAMEL_GLOBAL float*>(a.w.at[kNormRstd][w])[row] = rstd;
  const Row<BF16> ry(a.w.at[kNormY][w] + at, a.width);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float g[N];
    gain.get(v, g);
#pragma unroll
    for (int j = 0; j < N; ++j) h[v][j] = (h[v][j] * rstd) * g[j];
    store_piece<BF16>(ry, P::column(lane, v), h[v], false);
  }
}

// ---- gradient -------------------------------------------------------------------------------

// A worker's tokens are cut into parts; the teams of a workgroup share a part's rows and keep sums of dy n for their
// columns in registers.  Parts are joined by a second launch.
constexpr uint32_t kNormParts = 1024;  // of all workers, about
constexpr uint32_t kNormRows = 8;      // rows of a part, at least

uint32_t norm_parts(uint32_t world, uint32_t max_tokens) {
  const uint32_t most = std::max(1u, kNormParts / std::min(world, kGroup));
  return std::max(1u, std::min(most, (max_tokens + kNormRows - 1) / kNormRows));
}

template <bool BF16, int V, int TEAM>
__global__ void __launch_bounds__(TEAM <= 4 ? 256 : 1024) k_norm_gradient(NormGradientArgs a, uint32_t span, uint64_t stride) {
  constexpr int N = kPiece<BF16>, ES = BF16 ? 2 : 4, kWaves = TEAM <= 4 ? 4 : 16, kTeams = kWaves / TEAM;
  __shared__ float lds[2][TEAM];
  __shared__ float sums[kTeams > 1 ? (kTeams - 1) * 64 * TEAM * N : 1];
  const uint32_t w = blockIdx.y, n = a.w.tokens[w], first = blockIdx.x * span, last = min(first + span, n);
  if (first >= n) return;
  constexpr int LANES = 64 * TEAM;
  const uint32_t lane = threadIdx.x % LANES, team = uniform(threadIdx.x / 64) / TEAM;
  using P = Pieces<BF16, V, LANES>;
  const Gains<BF16, V, LANES> gain(a.w.at[kNormGradGain][w], a.gain_bf16, a.width, lane);
  constexpr bool kLate = TEAM == 16 && V * N >= 32;  // dsum is loaded when it is added, for the registers
  float sum[V][N] = {};
  uint32_t turn = 0;
  for (uint32_t row = first + team; row < last; row += kTeams) {
    const uint64_t at = uint64_t(row) * a.pitch * ES;
    const Row<BF16> rx(a.w.at[kNormGradX][w] + at, a.width), ry(a.w.at[kNormGradDy][w] + at, a.width);
    const Row<BF16> rd(a.w.at[kNormGradDsum][w] + at, a.width), ro(a.w.at[kNormGradDx][w] + at, a.width);
    P x, y, d;
    x.load(rx, lane, a.stream);
    y.load(ry, lane, a.stream);
    if (a.dsum && !kLate) d.load(rd, lane, a.stream);
    const float r = reinterpret_cast<const CARAMEL_GLOBAL float*>(a.w.at[kNormGradRstd][w])[row];
    x.finish(rx, lane);
    y.finish(ry, lane);
    float c = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float n[N], u[N], g[N];
      widen<BF16>(x.raw[v], n);
      widen<BF16>(y.raw[v], u);
      gain.get(v, g);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        n[j] *= r;
        sum[v][j] = __builtin_fmaf(u[j], n[j], sum[v][j]);
        c = __builtin_fmaf(u[j] * g[j], n[j], c);
      }
    }
    c = team_sum<TEAM>(c, lds[turn]) / float(a.width);
    turn ^= 1;
    if (a.dsum && !kLate) d.finish(rd, lane);
    // (left to itself, the compiler keeps what it has widened, in twice the registers of what it came from)
    if constexpr (BF16) {
#pragma unroll
      for (int v = 0; v < V; ++v) asm volatile("" : "+v"(x.raw[v]), "+v"(y.raw[v]));
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float n[N], u[N], g[N], o[N];
      widen<BF16>(x.raw[v], n);
      widen<BF16>(y.raw[v], u);
      gain.get(v, g);
      if (a.dsum) {
        if constexpr (kLate) {
          d.raw[v] = rd.get(P::column(lane, v));
          if (rd.odd()) rd.merge_last(P::column(lane, v), rd.get_last(), d.raw[v]);
        }
        widen<BF16>(d.raw[v], o);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < N; ++j) o[j] = __builtin_fmaf(r, __builtin_fmaf(-(n[j] * r), c, u[j] * g[j]), o[j]);
      store_piece<BF16>(ro, P::column(lane, v), o, false);
    }
  }
  // the workgroup's teams, one piece of every lane after the other
  const Row<false> out(reinterpret_cast<uint64_t>(a.ws) + (w * stride + uint64_t(blockIdx.x) * a.width) * 4, a.width);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (kTeams > 1) {
      if (team) {
#pragma unroll
        for (int j = 0; j < N; ++j) sums[((team - 1) * N + j) * LANES + lane] = sum[v][j];
      }
      __syncthreads();
      if (!team) {
#pragma unroll
        for (int k = 0; k < kTeams - 1; ++k)
#pragma unroll
          for (int j = 0; j < N; ++j) sum[v][j] += sums[(k * N + j) * LANES + lane];
      }
      __syncthreads();
    }
    if (!team) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) out.put(P::column(lane, v) + 4 * q, narrow<false>(sum[v] + 4 * q));
    }
  }
}

// 64 columns to a workgroup; its sixteen wavefronts share the parts, and their sums are added in order.
__global__ void __launch_bounds__(1024) k_norm_join(NormGradientArgs a, uint32_t span, uint64_t stride) {
  __shared__ float lds[16][64];
  const uint32_t w = blockIdx.y, parts = (a.w.tokens[w] + span - 1) / span, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t col = blockIdx.x * 64 + lane;
  const uint32_t each = (parts + 15) / 16, first = wave * each, last = min(first + each, parts);
  const CARAMEL_GLOBAL float* const in = reinterpret_cast<const CARAMEL_GLOBAL float*>(reinterpret_cast<uint64_t>(a.ws)) + w * stride;
  float sum = 0.0f;
  if (col < a.width) {
    uint32_t k = first;
    for (; k + 8 <= last; k += 8) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = in[uint64_t(k + i) * a.width + col];
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += v[i];
    }
    for (; k < last; ++k) sum += in[uint64_t(k) * a.width + col];
  }
  lds[wave][lane] = sum;
  __syncthreads();
  if (wave || col >= a.width) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) sum += lds[k][lane];
  const uint64_t out = a.w.at[kNormGradOut][w] + uint64_t(col) * (a.gain_bf16 ? 2 : 4);
  float old = 0.0f;
  if (a.gain_bf16) {
    if (a.accumulate) load_elems<true, 1>(out, &old);
    sum += old;
    store_elems<true, 1>(out, &sum);
  } else {
    if (a.accumulate) load_elems<false, 1>(out, &old);
    sum += old;
    store_elems<false, 1>(out, &sum);
  }
}

template <int V, int TEAM>
struct Shape {
  static constexpr int kV = V, kTeam = TEAM;
};

// Wavefronts and pieces that hold a row of `width` columns: launch(pieces, wavefronts) as compile-time numbers.  As few wavefronts as can do, but no
// more than four pieces a lane, for the registers (8 x 2048 x 2048 bf16 48.9 us and 52.3 with eight; the gradient 63 and 119;
// two a lane and four wavefronts 54.8 and 61.8).
template <int PIECE, typename LAUNCH>
void row_shape(uint32_t width, LAUNCH&& launch) {
  constexpr uint32_t kWave = 64 * PIECE;
  if (width <= kWave) launch(Shape<1, 1>{});
  else if (width <= 2 * kWave) launch(Shape<2, 1>{});
  else if (width <= 4 * kWave) launch(Shape<4, 1>{});
  else if (width <= 4 * 2 * kWave) launch(Shape<2, 4>{});
  else if (width <= 4 * 4 * kWave) launch(Shape<4, 4>{});
  else if (width <= 16 * 2 * kWave) launch(Shape<2, 16>{});
  else if (width <= 16 * 4 * kWave) launch(Shape<4, 16>{});
  else if constexpr (16 * 4 * kWave < kNormWidth) launch(Shape<8, 16>{});
}
// The gradient holds more: bf16 rows whose four pieces would leave two wavefronts per SIMD take three (3 x 1500 x 4104 52 us, with four 70) or
// sixteen wavefronts (8 x 1000 x 8192 119, with four 126).
template <int PIECE, typename LAUNCH>
void gradient_shape(uint32_t width, LAUNCH&& launch) {
  constexpr uint32_t kWave = 64 * PIECE;
  if constexpr (PIECE == 8) {
    if (width <= kWave) launch(Shape<1, 1>{});
    else if (width <= 2 * kWave) launch(Shape<2, 1>{});
    else if (width <= 4 * kWave) launch(Shape<4, 1>{});
    else if (width <= 4 * 2 * kWave) launch(Shape<2, 4>{});
    else if (width <= 4 * 3 * kWave) launch(Shape<3, 4>{});
    else if (width <= 16 * kWave) launch(Shape<1, 16>{});
    else if (width <= 16 * 2 * kWave) launch(Shape<2, 16>{});
    else launch(Shape<4, 16>{});
  } else {
    row_shape<PIECE>(width, launch);
  }
}

}  // namespace

hipError_t launch_norm(const NormArgs& all, const AllBuffers<kNormBuffers>& v, hipStream_t s) {
  if (all.max_tokens == 0) return hipSuccess;
  NormArgs args = all;
  args.inverse_width = 1.0 / double(all.width);
  args.stream = uint64_t(all.all) * all.max_tokens * all.width * (all.bf16 ? 2 : 4) >= kLarge;
  const hipError_t e = in_groups(args, v, [&](const NormArgs& a, uint32_t) {
    auto rows = [&](auto bf16, auto shape) {
      constexpr int V = decltype(shape)::kV, TEAM = decltype(shape)::kTeam;
      constexpr uint32_t kRows = (TEAM <= 4 ? 4 : 16) / TEAM;
      const uint32_t groups = (a.max_tokens + kRows - 1) / kRows;
      const dim3 grid(std::min(groups, kGridGroups), a.world, (groups + kGridGroups - 1) / kGridGroups), block(TEAM <= 4 ? 256 : 1024);
      hipLaunchKernelGGL((k_norm<decltype(bf16)::value, V, TEAM>), grid, block, 0, s, a);
    };
    if (a.bf16) row_shape<kPiece<true>>(a.width, [&](auto shape) { rows(std::true_type{}, shape); });
    else row_shape<kPiece<false>>(a.width, [&](auto shape) { rows(std::false_type{}, shape); });
    return hipGetLastError();
  });
  if (e != hipSuccess || !args.checkpoint) return e;
  CheckpointArgs c{};
  AllWorkers to{};
  c.all = args.all;
  c.max_tokens = args.max_tokens;
  c.features = args.width;
  c.pitch = args.pitch;
  c.bf16 = args.bf16;
  for (uint32_t w = 0; w < args.all; ++w) {
    to.a[w] = v.at[kNormY][w];
    to.b[w] = v.at[kNormCheckpoint][w];
    to.tokens[w] = v.tokens[w];
  }
  return launch_checkpoint_store(c, to, s);
}

uint64_t norm_gradient_workspace(uint32_t world, uint32_t width, uint32_t max_tokens) {
  return uint64_t(world) * norm_parts(world, max_tokens) * width * 4;
}

hipError_t launch_norm_gradient(const NormGradientArgs& all, const AllBuffers<kNormGradBuffers>& v, hipStream_t s) {
  NormGradientArgs args = all;
  args.stream = uint64_t(all.all) * all.max_tokens * all.width * (all.bf16 ? 2 : 4) >= kLarge;
  const uint32_t parts = norm_parts(args.all, args.max_tokens), span = std::max(1u, (args.max_tokens + parts - 1) / parts);
  const uint64_t stride = uint64_t(parts) * args.width;
  return in_groups(args, v, [&](NormGradientArgs a, uint32_t g) {
    a.ws += g * stride * 4;
    if (a.max_tokens) {
      auto rows = [&](auto bf16, auto shape) {
        constexpr int V = decltype(shape)::kV, TEAM = decltype(shape)::kTeam;
        const dim3 grid(parts, a.world), block(TEAM <= 4 ? 256 : 1024);
        hipLaunchKernelGGL((k_norm_gradient<decltype(bf16)::value, V, TEAM>), grid, block, 0, s, a, span, stride);
      };
      if (a.bf16) gradient_shape<kPiece<true>>(a.width, [&](auto shape) { rows(std::true_type{}, shape); });
      else gradient_shape<kPiece<false>>(a.width, [&](auto shape) { rows(std::false_type{}, shape); });
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(k_norm_join, dim3((a.width + 63) / 64, a.world), dim3(1024), 0, s, a, span, stride);
    return hipGetLastError();
  });
}

}  // namespace caramel
