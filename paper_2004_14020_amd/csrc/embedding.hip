// Embedding lookup, and its gradient by sorted tokens.
//
//   lookup     out[i, :] = round(scale * table[id[i], :])
//   gradient   g[v, :]   = round([g[v, :] +] scale * sum of dy[i, :] over the tokens i with id[i] = v)
//
// Tokens whose id lies outside the table are padding: their output is zero, and they add to no row.  The
// sums are fp32 in the order of the tokens, cut at fixed places of the sorted list, so results are
// reproducible bit for bit.
#include <algorithm>

#include "layers.hpp"
#include "vec.hpp"

namespace caramel {
namespace {

// ---- lookup ---------------------------------------------------------------------------------

// Bound: HBM (rows named once, read and written).  `lanes` lanes (a power of two) take one row, four rows
// each, so that four independent loads are in flight per lane.
constexpr int kLookupRows = 4;

template <bool BF16, bool IDS64>
__global__ void __launch_bounds__(256) k_embedding_lookup(LookupArgs a, uint32_t lanes) {
  constexpr int N = BF16 ? 8 : 4, ES = BF16 ? 2 : 4;
  const uint32_t w = blockIdx.y, n = a.w.tokens[w];
  const uint32_t groups = 256 / lanes, lane = threadIdx.x & (lanes - 1);
  const uint32_t first = blockIdx.x * groups * kLookupRows + threadIdx.x / lanes;
  const uint64_t ids = a.w.b[w];
  uint64_t src[kLookupRows];
  bool there[kLookupRows];
#pragma unroll
  for (int r = 0; r < kLookupRows; ++r) {
    const uint32_t i = first + r * groups;
    there[r] = false;
    src[r] = 0;
    if (i < n) {
      const uint64_t id = IDS64 ? reinterpret_cast<const CARAMEL_GLOBAL uint64_t*>(ids)[i]
                                : reinterpret_cast<const CARAMEL_GLOBAL uint32_t*>(ids)[i];
      there[r] = id < a.vocab;  // a negative id is a huge one
      src[r] = a.w.a[w] + id * a.width * ES;
    }
  }
  const uint64_t dst = a.w.c[w];
  for (uint32_t col = lane * N; col < a.width; col += lanes * N) {
    if (col + N <= a.width) {
      float x[kLookupRows][N];
#pragma unroll
      for (int r = 0; r < kLookupRows; ++r) {
        for (int j = 0; j < N; ++j) x[r][j] = 0.0f;
        if (there[r]) load_elems<BF16, N>(src[r] + uint64_t(col) * ES, x[r]);
      }
#pragma unroll
      for (int r = 0; r < kLookupRows; ++r) {
        const uint32_t i = first + r * groups;
        if (i >= n) continue;
        if (there[r])
          for (int j = 0; j < N; ++j) x[r][j] *= a.scale;
        store_elems<BF16, N>(dst + (i * a.out_pitch + col) * ES, x[r]);
      }
    } else {
      for (int r = 0; r < kLookupRows; ++r) {
        const uint32_t i = first + r * groups;
        if (i >= n) continue;
        for (uint32_t k = col; k < a.width; ++k) {
          float x = 0.0f;
          if (there[r]) {
            load_elems<BF16, 1>(src[r] + uint64_t(k) * ES, &x);
            x *= a.scale;
          }
          store_elems<BF16, 1>(dst + (i * a.out_pitch + k) * ES, &x);
        }
      }
    }
  }
}

// ---- gradient -------------------------------------------------------------------------------

// Three launches.
//   k_embedding_sort   a stable counting sort of the tokens by id.  A workgroup owns a range of ids and reads
//                      all of its worker's ids twice (they are a few ten KiB and stay in the caches), so no
//                      workgroup needs another's counts.
//   k_embedding_sum    the sorted list is cut into chunks of equal length, so that work is even however
//                      often a token occurs; a chunk's lanes walk it and write each row that ends inside.
//                      Rows cut by a chunk's border leave partial sums.  Other workgroups clear the rows that
//                      no token names.
//   k_embedding_join   adds the partial sums of the rows that were cut, in the chunks' order.

constexpr int kSortWaves = 16;
constexpr uint32_t kSortRange = 960;  // most ids of a workgroup: one lane each in the scan, 60 KiB of counters

struct Layout {
  uint64_t start, order, sorted, partial, stride;  // bytes; stride from worker to worker
  uint32_t chunk, chunks;                          // tokens per chunk; chunks of the longest worker
};

// Bytes are laid out for the longest worker, so that offsets are the same for all.
Layout layout(uint32_t world, uint32_t vocab, uint32_t width, uint32_t max_tokens) {
  auto up = [](uint64_t x) { return (x + 255) / 256 * 256; };
  Layout l{};
  l.chunk = uint64_t(world) * max_tokens >= 16384 ? 32 : 8;
  l.chunks = (max_tokens + l.chunk - 1) / l.chunk;
  l.start = 0;
  l.order = up((uint64_t(vocab) + 1) * 4);
  l.sorted = l.order + up(uint64_t(max_tokens) * 4);
  l.partial = l.sorted + up(uint64_t(max_tokens) * 4);
  l.stride = l.partial + up(uint64_t(2) * l.chunks * width * 4);
  return l;
}

template <bool IDS64>
__device__ __forceinline__ uint32_t read_id(uint64_t ids, uint32_t i, uint32_t vocab) {
  if constexpr (IDS64) {
    const uint64_t id = reinterpret_cast<const CARAMEL_GLOBAL uint64_t*>(ids)[i];
    return id < vocab ? uint32_t(id) : 0xFFFFFFFFu;
  } else {
    const uint32_t id = reinterpret_cast<const CARAMEL_GLOBAL uint32_t*>(ids)[i];
    return id < vocab ? id : 0xFFFFFFFFu;
  }
}

template <bool IDS64>
__global__ void __launch_bounds__(64 * kSortWaves) k_embedding_sort(EmbeddingGradientArgs a, Layout l, uint32_t range) {
  extern __shared__ uint32_t lds[];
  uint32_t* const count = lds;                        // [wave][id - lo]
  uint32_t* const sums = lds + kSortWaves * range;    // one per wave
  uint32_t* const lower = sums + kSortWaves;
  const uint32_t w = blockIdx.y, n = a.w.tokens[w];
  const uint32_t lo = blockIdx.x * range, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const uint64_t ids = a.w.a[w];
  unsigned char* const ws = a.ws + w * l.stride;
  for (uint32_t i = threadIdx.x; i < kSortWaves * range; i += blockDim.x) count[i] = 0;
  if (threadIdx.x == 0) *lower = 0;
  __syncthreads();
  // each wave counts a stretch of the tokens
  const uint32_t part = (n + 64 * kSortWaves - 1) / (64 * kSortWaves) * 64;
  const uint32_t begin = min(wave * part, n), end = min(begin + part, n);
  uint32_t below = 0;
  for (uint32_t i = begin + lane; i < end; i += 64) {
    const uint32_t id = read_id<IDS64>(ids, i, a.vocab);
    if (id - lo < range) {
      if (id != 0xFFFFFFFFu) atomicAdd(&count[wave * range + id - lo], 1u);
    } else if (id < lo) {
      ++below;
    }
  }
  if (below) atomicAdd(lower, below);
  __syncthreads();
  // one lane per id: where its tokens go, wave by wave
  uint32_t mine = 0;
  if (threadIdx.x < range)
    for (int v = 0; v < kSortWaves; ++v) {
      const uint32_t c = count[v * range + threadIdx.x];
      count[v * range + threadIdx.x] = mine;
      mine += c;
    }
  uint32_t incl = mine;
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t up = __shfl_up(incl, d);
    if (lane >= uint32_t(d)) incl += up;
  }
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  uint32_t base = *lower + incl - mine;
  for (uint32_t v = 0; v < wave; ++v) base += sums[v];
  uint32_t* const start = reinterpret_cast<uint32_t*>(ws + l.start);
  if (threadIdx.x < range) {
    for (int v = 0; v < kSortWaves; ++v) count[v * range + threadIdx.x] += base;
    if (lo + threadIdx.x < a.vocab) {
      start[lo + threadIdx.x] = base;
      if (lo + threadIdx.x == a.vocab - 1) start[a.vocab] = base + mine;
    }
  }
  __syncthreads();
  // each wave deals out its stretch, in order
  uint32_t* const order = reinterpret_cast<uint32_t*>(ws + l.order);
  uint32_t* const sorted = reinterpret_cast<uint32_t*>(ws + l.sorted);
  volatile uint32_t* const next = count + wave * range;  // one lane moves it on for the others of its wavefront
  for (uint32_t i0 = begin; i0 < end; i0 += 64) {
    const uint32_t i = i0 + lane;
    const uint32_t id = i < end ? read_id<IDS64>(ids, i, a.vocab) : 0xFFFFFFFFu;
    const bool in = id != 0xFFFFFFFFu && id - lo < range;
    uint64_t left = __ballot(in);
    while (left) {  // one round per different id among the 64
      const uint32_t who = __ffsll((unsigned long long)left) - 1;
      const uint32_t v = __builtin_amdgcn_readlane(id, who);
      const uint64_t same = __ballot(in && id == v);
      const uint32_t at = next[v - lo];
      if (in && id == v) {
        const uint32_t rank = __popcll(same & ((uint64_t(1) << lane) - 1));
        order[at + rank] = i;
        sorted[at + rank] = v;
      }
      if (lane == who) next[v - lo] = at + uint32_t(__popcll(same));
      left &= ~same;
    }
  }
}

template <bool OUT_BF16, int N>
__device__ __forceinline__ void write_row(const EmbeddingGradientArgs& a, uint64_t out, uint32_t row, uint32_t col,
                                          uint32_t cols, const float* sum) {
  constexpr int ES = OUT_BF16 ? 2 : 4;
  const uint64_t at = out + (uint64_t(row) * a.width + col) * ES;
  if (cols >= N) {
    float y[N];
    if (a.accumulate) {
      load_elems<OUT_BF16, N>(at, y);
      for (int j = 0; j < N; ++j) y[j] += a.scale * sum[j];
    } else {
      for (int j = 0; j < N; ++j) y[j] = a.scale * sum[j];
    }
    store_elems<OUT_BF16, N>(at, y);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (uint32_t(j) >= cols) break;
      float y = a.scale * sum[j], old = 0.0f;
      if (a.accumulate) {
        load_elems<OUT_BF16, 1>(at + j * ES, &old);
        y += old;
      }
      store_elems<OUT_BF16, 1>(at + j * ES, &y);
    }
  }
}

constexpr int kSumBlock = 256;
constexpr int kAhead = 8;  // tokens whose rows are fetched at once

template <bool DY_BF16, bool OUT_BF16>
__global__ void __launch_bounds__(kSumBlock) k_embedding_sum(EmbeddingGradientArgs a, Layout l, uint32_t lanes,
                                                             uint32_t sum_blocks) {
  constexpr int N = DY_BF16 ? 8 : 4, ES = DY_BF16 ? 2 : 4, OS = OUT_BF16 ? 2 : 4;
  const uint32_t w = blockIdx.y;
  const unsigned char* const ws = a.ws + w * l.stride;
  const uint32_t* const start = reinterpret_cast<const uint32_t*>(ws + l.start);
  const uint64_t out = a.w.c[w];
  const uint32_t lane = threadIdx.x & (lanes - 1);
  const uint32_t col = (blockIdx.z * lanes + lane) * N;
  if (blockIdx.x >= sum_blocks) {
    // rows that no token names: a wavefront looks at 64 of them
    const uint32_t row0 = ((blockIdx.x - sum_blocks) * (kSumBlock / 64) + threadIdx.x / 64) * 64;
    if (row0 >= a.vocab) return;
    const uint32_t r = row0 + threadIdx.x % 64;
    uint64_t empty = __ballot(r < a.vocab && start[min(r, a.vocab - 1)] == start[min(r, a.vocab - 1) + 1]);
    const uint32_t c0 = blockIdx.z * lanes * N, c1 = min(c0 + lanes * N, a.width);
    const float zero[N] = {};
    while (empty) {
      const uint32_t row = row0 + __ffsll((unsigned long long)empty) - 1;
      empty &= empty - 1;
      const uint64_t at = out + uint64_t(row) * a.width * OS;
      for (uint32_t c = c0 + threadIdx.x % 64 * N; c < c1; c += 64 * N) {
        if (c + N <= c1) {
          store_elems<OUT_BF16, N>(at + uint64_t(c) * OS, zero);
        } else {
          for (uint32_t k = c; k < c1; ++k) store_elems<OUT_BF16, 1>(at + uint64_t(k) * OS, zero);
        }
      }
    }
    return;
  }
  const uint32_t total = start[a.vocab];
  const uint32_t chunk = blockIdx.x * (kSumBlock / lanes) + threadIdx.x / lanes;
  const uint32_t c0 = min(chunk, l.chunks) * l.chunk;
  if (c0 >= total || col >= a.width) return;
  const uint32_t c1 = min(c0 + l.chunk, total);
  const uint32_t cols = min(a.width - col, uint32_t(N));
  const uint32_t* const order = reinterpret_cast<const uint32_t*>(ws + l.order);
  const uint32_t* const sorted = reinterpret_cast<const uint32_t*>(ws + l.sorted);
  const uint64_t partial = reinterpret_cast<uint64_t>(ws + l.partial);
  const uint64_t dy = a.w.b[w] + uint64_t(col) * ES;
  float sum[N] = {};
  uint32_t row = sorted[c0];
  auto leave = [&](bool cut_end) {
    const bool cut_begin = start[row] < c0;
    if (!cut_begin && !cut_end) {
      write_row<OUT_BF16, N>(a, out, row, col, cols, sum);
    } else {
      // the part of a row that began earlier goes into the chunk's first place, one that begins here into the second
      const uint64_t at = partial + ((uint64_t(chunk) * 2 + (cut_begin ? 0 : 1)) * a.width + col) * 4;
      if (cols >= N) store_elems<false, N>(at, sum);
      else
        for (uint32_t j = 0; j < cols; ++j) store_elems<false, 1>(at + 4 * j, sum + j);
    }
  };
  for (uint32_t e = c0; e < c1; e += kAhead) {
    float x[kAhead][N];
    uint32_t id[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      id[j] = 0xFFFFFFFFu;
      if (e + j < c1) {
        id[j] = sorted[e + j];
        const uint64_t at = dy + uint64_t(order[e + j]) * a.dy_pitch * ES;
        if (cols >= N) {
          load_elems<DY_BF16, N>(at, x[j]);
        } else {
          for (int k = 0; k < N; ++k) {
            x[j][k] = 0.0f;
            if (uint32_t(k) < cols) load_elems<DY_BF16, 1>(at + k * ES, &x[j][k]);
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (e + j >= c1) break;
      if (id[j] != row) {
        leave(false);
        for (int k = 0; k < N; ++k) sum[k] = 0.0f;
        row = id[j];
      }
      for (int k = 0; k < N; ++k) sum[k] += x[j][k];
    }
  }
  leave(start[row + 1] > c1);
}

constexpr int kJoinWaves = 8;

// One workgroup per chunk and 256 columns; it works if a row begins in the chunk and runs past its end.  The
// wavefronts take equal stretches of that row's partial sums.
template <bool OUT_BF16>
__global__ void __launch_bounds__(64 * kJoinWaves) k_embedding_join(EmbeddingGradientArgs a, Layout l) {
  __shared__ float part[kJoinWaves][256];
  const uint32_t w = blockIdx.y, chunk = blockIdx.x;
  const unsigned char* const ws = a.ws + w * l.stride;
  const uint32_t* const start = reinterpret_cast<const uint32_t*>(ws + l.start);
  const uint32_t* const sorted = reinterpret_cast<const uint32_t*>(ws + l.sorted);
  const uint32_t c1 = (chunk + 1) * l.chunk;
  if (c1 >= start[a.vocab]) return;
  const uint32_t row = sorted[c1 - 1], end = start[row + 1];
  if (end <= c1 || start[row] < chunk * l.chunk) return;
  const uint32_t pieces = (end - 1) / l.chunk - chunk + 1;
  const uint32_t wave = threadIdx.x / 64, col = blockIdx.z * 256 + threadIdx.x % 64 * 4;
  const uint32_t cols = col < a.width ? min(a.width - col, 4u) : 0u;
  const uint32_t share = (pieces + kJoinWaves - 1) / kJoinWaves;
  const uint32_t p0 = min(wave * share, pieces), p1 = min(p0 + share, pieces);
  const uint64_t partial = reinterpret_cast<uint64_t>(ws + l.partial) + uint64_t(col) * 4;
  float sum[4] = {};
#pragma unroll 4
  for (uint32_t p = p0; p < p1; ++p) {
    // the first piece lies in the second place of its chunk, the others in the first
    const uint64_t at = partial + (uint64_t(chunk + p) * 2 + (p == 0 ? 1 : 0)) * a.width * 4;
    float x[4] = {};
    if (cols == 4) load_elems<false, 4>(at, x);
    else
      for (uint32_t j = 0; j < cols; ++j) load_elems<false, 1>(at + 4 * j, x + j);
    for (int j = 0; j < 4; ++j) sum[j] += x[j];
  }
  for (int j = 0; j < 4; ++j) part[wave][threadIdx.x % 64 * 4 + j] = sum[j];
  __syncthreads();
  if (wave || !cols) return;
  for (int v = 1; v < kJoinWaves; ++v)
    for (int j = 0; j < 4; ++j) sum[j] += part[v][threadIdx.x * 4 + j];
  write_row<OUT_BF16, 4>(a, a.w.c[w], row, col, cols, sum);
}

uint32_t lanes_for(uint32_t width, uint32_t per_lane, uint32_t most) {
  uint32_t lanes = 1;
  while (lanes < most && lanes * per_lane < width) lanes *= 2;
  return lanes;
}

}  // namespace

hipError_t launch_embedding_lookup(const LookupArgs& a, hipStream_t s) {
  if (a.max_tokens == 0) return hipSuccess;
  const uint32_t lanes = lanes_for(a.width, a.bf16 ? 8 : 4, 256);
  const uint32_t rows = 256 / lanes * kLookupRows;
  const dim3 grid((a.max_tokens + rows - 1) / rows, a.world);
  if (a.bf16) {
    if (a.ids64) hipLaunchKernelGGL((k_embedding_lookup<true, true>), grid, dim3(256), 0, s, a, lanes);
    else hipLaunchKernelGGL((k_embedding_lookup<true, false>), grid, dim3(256), 0, s, a, lanes);
  } else {
    if (a.ids64) hipLaunchKernelGGL((k_embedding_lookup<false, true>), grid, dim3(256), 0, s, a, lanes);
    else hipLaunchKernelGGL((k_embedding_lookup<false, false>), grid, dim3(256), 0, s, a, lanes);
  }
  return hipGetLastError();
}

uint64_t embedding_gradient_workspace(uint32_t world, uint32_t vocab, uint32_t width, uint32_t max_tokens) {
  return layout(world, vocab, width, max_tokens).stride * world;
}

hipError_t launch_embedding_gradient(const EmbeddingGradientArgs& a, hipStream_t s) {
  if (a.max_tokens == 0 && a.accumulate) return hipSuccess;
  const Layout l = layout(a.world, a.vocab, a.width, a.max_tokens);
  // enough workgroups to fill the chip, each with as few ids as that allows
  const uint64_t even = (uint64_t(a.vocab) * a.world + 255) / 256;
  const uint32_t range = uint32_t(std::min<uint64_t>(kSortRange, std::max<uint64_t>(64, even)));
  const dim3 sort_grid((a.vocab + range - 1) / range, a.world);
  const size_t lds = (kSortWaves * range + kSortWaves + 1) * sizeof(uint32_t);
  if (a.ids64) hipLaunchKernelGGL((k_embedding_sort<true>), sort_grid, dim3(64 * kSortWaves), lds, s, a, l, range);
  else hipLaunchKernelGGL((k_embedding_sort<false>), sort_grid, dim3(64 * kSortWaves), lds, s, a, l, range);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const uint32_t per_lane = a.dy_bf16 ? 8 : 4, lanes = lanes_for(a.width, per_lane, 64);
  const uint32_t groups = kSumBlock / lanes, sum_blocks = (l.chunks + groups - 1) / groups;
  const uint32_t fill_blocks = a.accumulate ? 0 : (a.vocab + kSumBlock - 1) / kSumBlock;
  const dim3 sum_grid(sum_blocks + fill_blocks, a.world, (a.width + lanes * per_lane - 1) / (lanes * per_lane));
  if (a.dy_bf16) {
    if (a.out_bf16) hipLaunchKernelGGL((k_embedding_sum<true, true>), sum_grid, dim3(kSumBlock), 0, s, a, l, lanes, sum_blocks);
    else hipLaunchKernelGGL((k_embedding_sum<true, false>), sum_grid, dim3(kSumBlock), 0, s, a, l, lanes, sum_blocks);
  } else {
    if (a.out_bf16) hipLaunchKernelGGL((k_embedding_sum<false, true>), sum_grid, dim3(kSumBlock), 0, s, a, l, lanes, sum_blocks);
    else hipLaunchKernelGGL((k_embedding_sum<false, false>), sum_grid, dim3(kSumBlock), 0, s, a, l, lanes, sum_blocks);
  }
  e = hipGetLastError();
  if (e != hipSuccess || l.chunks < 2) return e;
  const dim3 join_grid(l.chunks - 1, a.world, (a.width + 255) / 256);
  if (a.out_bf16) hipLaunchKernelGGL((k_embedding_join<true>), join_grid, dim3(64 * kJoinWaves), 0, s, a, l);
  else hipLaunchKernelGGL((k_embedding_join<false>), join_grid, dim3(64 * kJoinWaves), 0, s, a, l);
  return hipGetLastError();
}

}  // namespace caramel
