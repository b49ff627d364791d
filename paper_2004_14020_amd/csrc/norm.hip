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
// A row stays in the registers of a team of wavefronts, so that every matrix is read and written once.
#include <algorithm>

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
  __device__ __forceinline__ void load(const Row<BF16>& row, uint32_t lane) {
#pragma unroll
    for (int v = 0; v < V; ++v) raw[v] = row.get(column(lane, v));
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

template <bool BF16, bool STREAM>
__device__ __forceinline__ void store_piece(const Row<BF16>& row, uint32_t col, const float* v) {
  const u32x4 raw = narrow<BF16>(v);
  row.template put<STREAM>(col, raw);
  if (row.odd()) row.put_last(col, raw);
}

// Gains are in the plan's type, which need not be that of the rows: the N of a piece of the rows.
template <bool BF16, int V, int LANES>
struct Gains {
  static constexpr int N = kPiece<BF16>;
  u32x4 raw[V][2];
  uint32_t last;

  // (bf16 gains of fp32 rows: the 16 bytes hold twice as many as are needed, and what is behind the row is not read)
  __device__ __forceinline__ void load(uint64_t at, bool bf16, uint32_t width, uint32_t lane) {
    if (bf16) {
      const Row<true> row(at, width);
#pragma unroll
      for (int v = 0; v < V; ++v) raw[v][0] = row.get((v * LANES + lane) * N);
      if (row.odd()) last = row.get_last();
    } else {
      const Row<false> row(at, width);
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int q = 0; q < N / 4; ++q) raw[v][q] = row.get((v * LANES + lane) * N + 4 * q);
    }
  }
  __device__ __forceinline__ void get(bool bf16, uint32_t width, uint32_t lane, int v, float* g) const {
    if (bf16) {
      u32x4 r = raw[v][0];
      if (width % 2) Row<true>(0, width).merge_last((v * LANES + lane) * N, last, r);
      float all[8];
      widen<true>(r, all);
#pragma unroll
      for (int j = 0; j < N; ++j) g[j] = all[j];
    } else {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) widen<false>(raw[v][q], g + 4 * q);
    }
  }
};

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
  x.load(rx, lane);
  if (a.residual) r.load(rr, lane);
  Gains<BF16, V, LANES> gain;
  gain.load(a.w.at[kNormGain][w], a.gain_bf16, a.width, lane);
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
      store_piece<BF16, false>(rs, P::column(lane, v), h[v]);
    }
  }
  double ss = 0.0;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < N; ++j) ss = __builtin_fma(double(h[v][j]), double(h[v][j]), ss);
  ss = team_sum<TEAM>(ss, lds);
  const float rstd = float(1.0 / sqrt(ss / double(a.width) + double(a.eps)));
  if (lane == 0) reinterpret_cast<CARAMEL_GLOBAL float*>(a.w.at[kNormRstd][w])[row] = rstd;
  const Row<BF16> ry(a.w.at[kNormY][w] + at, a.width);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float g[N];
    gain.get(a.gain_bf16, a.width, lane, v, g);
#pragma unroll
    for (int j = 0; j < N; ++j) h[v][j] = (h[v][j] * rstd) * g[j];
    store_piece<BF16, false>(ry, P::column(lane, v), h[v]);
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
  Gains<BF16, V, LANES> gain;
  gain.load(a.w.at[kNormGradGain][w], a.gain_bf16, a.width, lane);
  float sum[V][N] = {};
  uint32_t turn = 0;
  for (uint32_t row = first + team; row < last; row += kTeams) {
    const uint64_t at = uint64_t(row) * a.pitch * ES;
    const Row<BF16> rx(a.w.at[kNormGradX][w] + at, a.width), ry(a.w.at[kNormGradDy][w] + at, a.width);
    const Row<BF16> rd(a.w.at[kNormGradDsum][w] + at, a.width), ro(a.w.at[kNormGradDx][w] + at, a.width);
    P x, y, d;
    x.load(rx, lane);
    y.load(ry, lane);
    if (a.dsum) d.load(rd, lane);
    const float r = reinterpret_cast<const CARAMEL_GLOBAL float*>(a.w.at[kNormGradRstd][w])[row];
    x.finish(rx, lane);
    y.finish(ry, lane);
    float c = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float n[N], u[N], g[N];
      widen<BF16>(x.raw[v], n);
      widen<BF16>(y.raw[v], u);
      gain.get(a.gain_bf16, a.width, lane, v, g);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        n[j] *= r;
        sum[v][j] = __builtin_fmaf(u[j], n[j], sum[v][j]);
        c = __builtin_fmaf(u[j] * g[j], n[j], c);
      }
    }
    c = team_sum<TEAM>(c, lds[turn]) / float(a.width);
    turn ^= 1;
    if (a.dsum) d.finish(rd, lane);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float n[N], u[N], g[N], o[N];
      widen<BF16>(x.raw[v], n);
      widen<BF16>(y.raw[v], u);
      gain.get(a.gain_bf16, a.width, lane, v, g);
      if (a.dsum) {
        widen<BF16>(d.raw[v], o);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < N; ++j) o[j] = __builtin_fmaf(r, __builtin_fmaf(-(n[j] * r), c, u[j] * g[j]), o[j]);
      store_piece<BF16, false>(ro, P::column(lane, v), o);
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

// 64 columns to a workgroup; its four wavefronts share the parts, and their sums are added in order.
__global__ void __launch_bounds__(256) k_norm_join(NormGradientArgs a, uint32_t span, uint64_t stride) {
  __shared__ float lds[4][64];
  const uint32_t w = blockIdx.y, parts = (a.w.tokens[w] + span - 1) / span, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t col = blockIdx.x * 64 + lane;
  const uint32_t each = (parts + 3) / 4, first = wave * each, last = min(first + each, parts);
  const CARAMEL_GLOBAL float* const in = reinterpret_cast<const CARAMEL_GLOBAL float*>(reinterpret_cast<uint64_t>(a.ws)) + w * stride;
  float sum = 0.0f;
  if (col < a.width)
    for (uint32_t k = first; k < last; ++k) sum += in[uint64_t(k) * a.width + col];
  lds[wave][lane] = sum;
  __syncthreads();
  if (wave || col >= a.width) return;
  sum = ((lds[0][lane] + lds[1][lane]) + lds[2][lane]) + lds[3][lane];
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

// The fewest wavefronts and pieces that hold a row of `width` columns: launch(pieces, wavefronts) as compile-time numbers.
template <int V, int TEAM>
struct Shape {
  static constexpr int kV = V, kTeam = TEAM;
};
template <typename LAUNCH>
void by_shape(uint32_t width, int piece, LAUNCH&& launch) {
  const uint32_t wave = 64 * uint32_t(piece);
  if (width <= wave) launch(Shape<1, 1>{});
  else if (width <= 2 * wave) launch(Shape<2, 1>{});
  else if (width <= 4 * wave) launch(Shape<4, 1>{});
  else if (width <= 8 * wave) launch(Shape<2, 4>{});
  else if (width <= 16 * wave) launch(Shape<4, 4>{});
  else if (width <= 64 * wave) launch(Shape<4, 16>{});
  else launch(Shape<8, 16>{});
}

}  // namespace

hipError_t launch_norm(const NormArgs& args, const AllBuffers<kNormBuffers>& v, hipStream_t s) {
  if (args.max_tokens == 0) return hipSuccess;
  const hipError_t e = in_groups(args, v, [&](const NormArgs& a, uint32_t) {
    by_shape(a.width, a.bf16 ? 8 : 4, [&](auto shape) {
      constexpr int V = decltype(shape)::kV, TEAM = decltype(shape)::kTeam;
      constexpr uint32_t kRows = (TEAM <= 4 ? 4 : 16) / TEAM;
      const uint32_t groups = (a.max_tokens + kRows - 1) / kRows;
      const dim3 grid(std::min(groups, kGridGroups), a.world, (groups + kGridGroups - 1) / kGridGroups), block(TEAM <= 4 ? 256 : 1024);
      if (a.bf16) hipLaunchKernelGGL((k_norm<true, V, TEAM>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((k_norm<false, V, TEAM>), grid, block, 0, s, a);
    });
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

hipError_t launch_norm_gradient(const NormGradientArgs& args, const AllBuffers<kNormGradBuffers>& v, hipStream_t s) {
  const uint32_t parts = norm_parts(args.all, args.max_tokens), span = std::max(1u, (args.max_tokens + parts - 1) / parts);
  const uint64_t stride = uint64_t(parts) * args.width;
  return in_groups(args, v, [&](NormGradientArgs a, uint32_t g) {
    a.ws += g * stride * 4;
    if (a.max_tokens) {
      by_shape(a.width, a.bf16 ? 8 : 4, [&](auto shape) {
        constexpr int V = decltype(shape)::kV, TEAM = decltype(shape)::kTeam;
        const dim3 grid(parts, a.world), block(TEAM <= 4 ? 256 : 1024);
        if (a.bf16) hipLaunchKernelGGL((k_norm_gradient<true, V, TEAM>), grid, block, 0, s, a, span, stride);
        else hipLaunchKernelGGL((k_norm_gradient<false, V, TEAM>), grid, block, 0, s, a, span, stride);
      });
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(k_norm_join, dim3((a.width + 63) / 64, a.world), dim3(256), 0, s, a, span, stride);
    return hipGetLastError();
  });
}

}  // namespace caramel
