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
// each, so that four independent loads are in flight per lane.  8 x 4096 tokens of 1024 bf16: 18.9 us back to back, 101 MB at 5.3 TB/s
// (two rows each 20.1, eight 21.0), and 24 with 640 MB of other data read in between (49 MB read, 67 written); fp32 35 us.
constexpr int kLookupRows = 4;

// STREAM: streaming stores, where the output is more than the L2s hold (8 x 4096 tokens of 1024 bf16: 20.3 us with plain
// ones, 18.6); less stays there for the layer that reads it next.
template <bool BF16, bool IDS64, bool STREAM>
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
  if (a.width >= N) {
    for (uint32_t at = lane * N; at < a.width; at += lanes * N) {
      // the last lane takes the last N columns, some of them a second time
      const uint32_t col = min(at, a.width - N);
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
        store_elems<BF16, N, STREAM>(dst + (i * a.out_pitch + col) * ES, x[r]);
      }
    }
  } else if (lane == 0) {
    for (int r = 0; r < kLookupRows; ++r) {
      const uint32_t i = first + r * groups;
      if (i >= n) continue;
      for (uint32_t k = 0; k < a.width; ++k) {
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

// ---- gradient -------------------------------------------------------------------------------

// Up to 64 tokens: one launch, k_embedding_few (below).  Otherwise three.
//   k_embedding_sort   a stable counting sort of the tokens by id.  A workgroup owns a range of ids and reads
//                      all of its worker's ids twice (they are a few ten KiB and stay in the caches), so no
//                      workgroup needs another's counts.
//   k_embedding_sum    the sorted list is cut into chunks of equal length, so that work is even however
//                      often a token occurs; a chunk's lanes walk it and write each row that ends inside.
//                      Rows cut by a chunk's border leave partial sums.  Other workgroups clear the rows that
//                      no token names.
//   k_embedding_join   adds the partial sums of the rows that were cut, in the chunks' order.
// Bound: HBM, most of all the zeros, and the latency of three dependent launches.  8 x 4096 tokens, 30522 x 1024 bf16 (567 MB; by counters
// 506 written and 71 read): 11 + 84 + 6 us back to back, 12 + 107 + 6 with 640 MB of other data read in between; accumulating, without
// the zeros, 44 a call.  All tokens on two rows of 1024 fp32 (134 MB): 6 + 22 + 6 and 7 + 31 + 6.

constexpr int kSortWaves = 16;
constexpr int kSortAhead = 4;          // ids per lane that are fetched at once; up to 4096 tokens they stay in registers
constexpr uint32_t kSortRange = 1008;  // most ids of a workgroup: one per lane in the scan; two workgroups' LDS to a compute unit
constexpr uint32_t kSortHeld = 128;    // tokens that a wavefront gathers before it ranks 64 of them

struct Layout {
  uint64_t start, order, sorted, partial, stride;  // bytes; stride from worker to worker
  uint32_t chunk, chunks;                          // tokens per chunk; chunks of the longest worker
};

constexpr uint32_t kManyTokens = 16384;  // of all workers: longer chunks

// Bytes are laid out for the longest worker, so that offsets are the same for all.
Layout layout(uint32_t world, uint32_t vocab, uint32_t width, uint32_t max_tokens) {
  auto up = [](uint64_t x) { return (x + 255) / 256 * 256; };
  Layout l{};
  // Short chunks give more wavefronts to the sums, long ones cut fewer rows.  Sums and joining, chunks of 8, 16 and 32: 4 x 2050 tokens
  // of 1001 bf16 and fp32 8.3 + 4.4, 9.8 + 3.8 us, -; 8 x 4096 tokens of 1024, bf16, 30522 rows 83 + 10, 86 + 6.4, 91 + 4.9; on two
  // rows (every chunk is cut), fp32 23 + 14, 23 + 9, 22 + 6; 16 x 7400 tokens of 105, bf16, 2759 rows 16 + 12, 15 + 7.7, 22 + 5.4.
  const bool many = uint64_t(world) * max_tokens >= kManyTokens;
  l.chunk = !many ? 8 : max_tokens / 32 < vocab ? 16 : 32;
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

// Bound: latency (a few thousand ids from the caches), with more tokens the instructions of the workgroup whose ids are the most
// frequent.  8 x 4096 tokens of 30522 words 11.0 us; with eight wavefronts 15, and with one round per different id among 64 tokens in
// place of the comparison by bits, and one id in flight per lane, 46.8.  2 x 60000 of 1000 skewed ids 31 us; at least 64 ids to a
// workgroup in place of 16 43; all tokens ranked as they come, in both passes, 80.
template <bool IDS64>
__global__ void __launch_bounds__(64 * kSortWaves) k_embedding_sort(EmbeddingGradientArgs a, Layout l, uint32_t range, uint32_t bits) {
  constexpr uint32_t kLanes = 64 * kSortWaves, kNone = 0xFFFFFFFFu;
  __shared__ uint32_t count[kSortWaves * kSortRange];  // [wave][id - lo]
  __shared__ uint32_t held[kSortWaves][2][kSortHeld];  // ids' places in the range, tokens
  __shared__ uint32_t sums[2][kSortWaves];
  const uint32_t w = blockIdx.y, n = a.w.tokens[w];
  const uint32_t lo = blockIdx.x * range, lane = threadIdx.x % 64;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint64_t ids = a.w.a[w];
  unsigned char* const ws = a.ws + w * l.stride;
  // each wave has a stretch of the tokens
  const uint32_t part = (n + kLanes - 1) / kLanes * 64;
  const uint32_t begin = min(wave * part, n), end = min(begin + part, n);
  // Between lanes of one wavefront, whose accesses to LDS are done in order.  A volatile access through an ordinary pointer
  // would wait for global memory too.
  using Shared = volatile __attribute__((address_space(3))) uint32_t;
  struct Ids {
    uint32_t v[kSortAhead];
  };
  auto fetch = [&](uint32_t i0) {  // begin < end; past the end the last id, so that no branch parts the loads
    Ids r;
#pragma unroll
    for (int j = 0; j < kSortAhead; ++j) r.v[j] = read_id<IDS64>(ids, min(i0 + j * 64 + lane, end - 1), a.vocab);
    return r;
  };
  // One step of a wavefront's walk: every lane's place among the tokens of its id, in order; the counters move on.
  Shared* const next = (Shared*)(count + wave * range);  // one lane moves it on for the others of its wavefront
  const uint64_t lower = (uint64_t(1) << lane) - 1;
  auto rank = [&](uint32_t key) -> uint32_t {
    const bool in = key < range;
    uint64_t same = __ballot(in);
    if (!same) return 0;
    for (uint32_t b = 0; b < bits; ++b) {  // the lanes with the same id
      const bool one = key >> b & 1;
      const uint64_t ones = __ballot(one);
      same &= one ? ones : ~ones;
    }
    uint32_t at = 0;
    if (in) {
      at = next[key] + __popcll(same & lower);
      if ((same >> lane) == 1) next[key] = at + 1;  // the last of them
    }
    return at;
  };
  // A long stretch: the next ids are fetched before these are used.
  auto walk = [&](auto visit) {
    if (begin == end) return;
    Ids id = fetch(begin);
    for (uint32_t i0 = begin; i0 < end; i0 += 64 * kSortAhead) {
      const Ids following = fetch(min(i0 + 64 * kSortAhead, end - 1));
#pragma unroll
      for (int j = 0; j < kSortAhead; ++j) {
        const uint32_t i = i0 + j * 64 + lane;
        visit(i < end ? id.v[j] : kNone, i);
      }
      id = following;
    }
  };
  uint32_t below = 0, place[kSortAhead];
  const bool kept = part <= 64 * kSortAhead;  // ids and places stay in registers
  Ids id;
#pragma unroll
  for (int j = 0; j < kSortAhead; ++j) id.v[j] = kNone;
  if (kept && begin < end) {
    id = fetch(begin);
#pragma unroll
    for (int j = 0; j < kSortAhead; ++j) id.v[j] = begin + j * 64 + lane < end ? id.v[j] : kNone;
  }
  for (uint32_t i = threadIdx.x; i < kSortWaves * range; i += kLanes) count[i] = 0;
  __syncthreads();
  if (kept) {
#pragma unroll
    for (int j = 0; j < kSortAhead; ++j) {
      place[j] = rank(id.v[j] - lo);
      below += id.v[j] < lo;
    }
  } else {
    walk([&](uint32_t v, uint32_t) {
      below += v < lo;
      if (v - lo < range) atomicAdd(count + wave * range + (v - lo), 1u);  // kNone - lo is more than any range
    });
  }
  for (int d = 32; d; d /= 2) below += __shfl_xor(below, d);
  if (lane == 0) sums[0][wave] = below;
  __syncthreads();
  // one id per lane: where its tokens go, wave by wave
  uint32_t mine = 0, before[kSortWaves];
  if (threadIdx.x < range) {
#pragma unroll
    for (int v = 0; v < kSortWaves; ++v) {
      before[v] = mine;
      mine += count[v * range + threadIdx.x];
    }
  }
  uint32_t incl = mine;
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t up = __shfl_up(incl, d);
    if (lane >= uint32_t(d)) incl += up;
  }
  if (lane == 63) sums[1][wave] = incl;
  __syncthreads();
  uint32_t base = incl - mine;
#pragma unroll
  for (uint32_t v = 0; v < kSortWaves; ++v) base += sums[0][v] + (v < wave ? sums[1][v] : 0);
  uint32_t* const start = reinterpret_cast<uint32_t*>(ws + l.start);
  if (threadIdx.x < range) {
#pragma unroll
    for (int v = 0; v < kSortWaves; ++v) count[v * range + threadIdx.x] = base + before[v];
    const uint32_t v = lo + threadIdx.x;
    if (v < a.vocab) {
      start[v] = base;
      if (v == a.vocab - 1) start[a.vocab] = base + mine;
    }
  }
  __syncthreads();
  // each wave deals out its stretch, in order
  uint32_t* const order = reinterpret_cast<uint32_t*>(ws + l.order);
  uint32_t* const sorted = reinterpret_cast<uint32_t*>(ws + l.sorted);
  if (kept) {
#pragma unroll
    for (int j = 0; j < kSortAhead; ++j) {
      const uint32_t key = id.v[j] - lo;
      if (key < range) {
        const uint32_t to = next[key] + place[j];
        order[to] = begin + j * 64 + lane;
        sorted[to] = id.v[j];
      }
    }
  } else {
    // the tokens in the range are gathered first, so that 64 of them are ranked at once
    Shared* const keys = (Shared*)held[wave][0];
    Shared* const tokens = (Shared*)held[wave][1];
    uint32_t total = 0, done = 0;
    auto deal = [&] {
      const uint32_t from = (done + lane) % kSortHeld, key = done + lane < total ? keys[from] : kNone, to = rank(key);
      if (key < range) {
        order[to] = tokens[from];
        sorted[to] = lo + key;
      }
      done += 64;
    };
    walk([&](uint32_t v, uint32_t i) {
      const uint32_t key = v - lo;
      const uint64_t in = __ballot(key < range);
      if (!in) return;
      if (key < range) {
        const uint32_t at = (total + __popcll(in & lower)) % kSortHeld;
        keys[at] = key;
        tokens[at] = i;
      }
      total += __popcll(in);
      if (total - done >= 64) deal();
    });
    if (done < total) deal();
  }
}

// Columns of one lane: N from `col` on, of which the first `twice` belong to the lane before as well (the last lane takes the
// last N columns of the row), or fewer than N where a row is that short.
struct Columns {
  uint32_t col, count, twice;
};
template <int N>
__device__ __forceinline__ Columns columns(uint32_t at, uint32_t width) {
  if (width < N) return {0, width, 0};
  const uint32_t col = min(at, width - N);
  return {col, N, at - col};
}

template <int N>
__device__ __forceinline__ void write_sum(uint64_t at, Columns c, const float* sum) {
  if (c.count == N) store_elems<false, N>(at, sum);
  else
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (uint32_t(j) < c.count) store_elems<false, 1>(at + 4 * j, sum + j);
}

template <bool OUT_BF16, int N>
__device__ __forceinline__ void write_row(const EmbeddingGradientArgs& a, uint64_t out, uint32_t row, Columns c, const float* sum) {
  constexpr int ES = OUT_BF16 ? 2 : 4;
  const uint64_t at = out + (uint64_t(row) * a.width + c.col) * ES;
  // columns that two lanes have are written by both, with the same value, but added to by one
  if (c.count == N && !(a.accumulate && c.twice)) {
    float y[N];
    if (a.accumulate) {
      load_elems<OUT_BF16, N>(at, y);
      for (int j = 0; j < N; ++j) y[j] = __builtin_fmaf(a.scale, sum[j], y[j]);  // one rounding
    } else {
      for (int j = 0; j < N; ++j) y[j] = a.scale * sum[j];
    }
    store_elems<OUT_BF16, N>(at, y);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (uint32_t(j) < c.twice || uint32_t(j) >= c.count) continue;
      float y = a.scale * sum[j];
      if (a.accumulate) {
        float old;
        load_elems<OUT_BF16, 1>(at + j * ES, &old);
        y = __builtin_fmaf(a.scale, sum[j], old);
      }
      store_elems<OUT_BF16, 1>(at + j * ES, &y);
    }
  }
}

constexpr int kSumBlock = 256;
constexpr int kAhead = 8;  // tokens whose rows are fetched at once

// Clears those of the rows [first, first + rows) whose bit in `empty` is set; one wavefront, at most 64 rows.  The rows are taken as
// the one stretch of memory that they are, so that stores are whole and next to each other however wide a row is.  Streaming
// stores: 8 x 30522 x 1024 bf16, 4096 tokens each 90 us, with plain ones 123.
template <bool OUT_BF16>
__device__ __forceinline__ void clear_rows(uint64_t out, uint32_t width, uint32_t first, uint32_t rows, uint64_t empty) {
  constexpr int OS = OUT_BF16 ? 2 : 4, N = 16 / OS;
  if (!empty) return;
  const uint64_t base = out + uint64_t(first) * width * OS;
  const uint32_t total = rows * width, down = 64 * N / width, right = 64 * N % width;
  const float zero[N] = {};
  uint32_t e = threadIdx.x % 64 * N, r = e / width, c = e - r * width;
  for (; e < total; e += 64 * N) {
    // up to two rows, unless a row is narrower than a store
    const bool one = empty >> r & 1, other = c + N <= width ? one : empty >> r >> 1 & 1;
    if (one && other && width >= N && e + N <= total) {
      store_elems<OUT_BF16, N, true>(base + uint64_t(e) * OS, zero);
    } else if (one || other || width < N) {
      uint32_t row = r, col = c;
      for (uint32_t j = 0; j < N && e + j < total; ++j) {
        if (empty >> row & 1) store_elems<OUT_BF16, 1>(base + uint64_t(e + j) * OS, zero);
        if (++col == width) {
          col = 0;
          ++row;
        }
      }
    }
    r += down;
    c += right;
    if (c >= width) {
      c -= width;
      ++r;
    }
  }
}

struct SumShape {
  uint32_t lanes, sum_blocks;  // lanes of a chunk
  uint32_t clear_rows;         // rows that a wavefront looks at, to clear them
};

// FULL: 64 lanes per chunk, so that the walk along the list is the wavefront's own: its tokens are fetched by one load
// and handed round through scalar registers.
template <bool DY_BF16, bool OUT_BF16, bool FULL>
__global__ void __launch_bounds__(kSumBlock) k_embedding_sum(EmbeddingGradientArgs a, Layout l, SumShape h) {
  constexpr int N = DY_BF16 ? 8 : 4, ES = DY_BF16 ? 2 : 4;
  const uint32_t w = blockIdx.y, lanes = FULL ? 64 : h.lanes;
  const unsigned char* const ws = a.ws + w * l.stride;
  const uint32_t* const start = reinterpret_cast<const uint32_t*>(ws + l.start);
  const uint64_t out = a.w.c[w];
  if (blockIdx.x >= h.sum_blocks) {
    const uint32_t wave = ((blockIdx.x - h.sum_blocks) * gridDim.z + blockIdx.z) * (kSumBlock / 64) + threadIdx.x / 64;
    const uint32_t first = wave * h.clear_rows;
    if (first >= a.vocab) return;
    const uint32_t rows = min(h.clear_rows, a.vocab - first), r = first + min(threadIdx.x % 64, rows - 1);
    clear_rows<OUT_BF16>(out, a.width, first, rows, __ballot(start[r] == start[r + 1]));
    return;
  }
  const uint32_t at_col = (blockIdx.z * lanes + threadIdx.x % lanes) * N;
  const uint32_t total = start[a.vocab];
  uint32_t chunk = blockIdx.x * (kSumBlock / lanes) + threadIdx.x / lanes;
  if constexpr (FULL) chunk = __builtin_amdgcn_readfirstlane(chunk);
  const uint32_t c0 = min(chunk, l.chunks) * l.chunk;
  if (c0 >= total) return;
  const uint32_t c1 = min(c0 + l.chunk, total);
  const uint32_t* const order = reinterpret_cast<const uint32_t*>(ws + l.order);
  const uint32_t* const sorted = reinterpret_cast<const uint32_t*>(ws + l.sorted);
  const uint64_t partial = reinterpret_cast<uint64_t>(ws + l.partial);
  const Columns c = columns<N>(at_col, a.width);
  const bool idle = at_col >= a.width;
  const uint64_t dy = a.w.b[w] + uint64_t(c.col) * ES;
  uint32_t list_id = 0, list_token = 0;
  u32x4 ids = 0, tokens = 0;
  if constexpr (FULL) {  // a chunk is at most 64 tokens
    const uint32_t e = min(c0 + threadIdx.x % 64, c1 - 1);
    list_id = sorted[e];
    list_token = order[e];
  } else if (idle) {
    return;
  }
  const uint32_t first_token = FULL ? 0 : order[c0];
  float sum[N] = {};
  uint32_t row = FULL ? __builtin_amdgcn_readlane(list_id, 0) : sorted[c0];
  auto leave = [&](bool cut_end) {
    const bool cut_begin = start[row] < c0;
    if (idle) return;
    if (!cut_begin && !cut_end) {
      write_row<OUT_BF16, N>(a, out, row, c, sum);
    } else {
      // the part of a row that began earlier goes into the chunk's first place, one that begins here into the second
      write_sum<N>(partial + ((uint64_t(chunk) * 2 + (cut_begin ? 0 : 1)) * a.width + c.col) * 4, c, sum);
    }
  };
  auto walk = [&](auto&& fetch) {
    for (uint32_t e = c0; e < c1; e += kAhead) {
      float x[kAhead][N];
      uint32_t id[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        // behind the end: a token again, which is not added
        const uint32_t at = min(e + j, c1 - 1);
        uint32_t token;
        if constexpr (FULL) {
          id[j] = __builtin_amdgcn_readlane(list_id, at - c0);
          token = __builtin_amdgcn_readlane(list_token, at - c0);
        } else {
          if (j % 4 == 0) {  // four of the list at once; the lists' memory goes on to the next 256 bytes
            ids = *reinterpret_cast<const u32x4*>(sorted + e + j);
            tokens = *reinterpret_cast<const u32x4*>(order + e + j);
          }
          id[j] = ids[j % 4];
          token = e + j < c1 ? tokens[j % 4] : first_token;
        }
        fetch(dy + uint64_t(token) * a.dy_pitch * ES, x[j]);
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
  };
  // The choice is made out here: beside each load it would make every load wait for the one before.
  if (a.width >= N) {
    walk([&](uint64_t from, float* x) { load_elems<DY_BF16, N>(from, x); });
  } else {
    walk([&](uint64_t from, float* x) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        x[k] = 0.0f;
        if (uint32_t(k) < a.width) load_elems<DY_BF16, 1>(from + k * ES, x + k);
      }
    });
  }
  leave(start[row + 1] > c1);
}

// Up to 64 tokens per worker: a wavefront owns a few rows, holds all ids in one register, and needs neither a list nor
// partial sums.  64 tokens, and 65 in three launches: 8 x (30522 x 1024) bf16 85.9 and 95.6 us, 2 x (2 x 1024) fp32 9.0 and
// 11.4; 20 tokens of 1000 x 768 fp32 5.9.
constexpr uint32_t kFew = 64;

template <bool IDS64, bool DY_BF16, bool OUT_BF16>
__global__ void __launch_bounds__(kSumBlock) k_embedding_few(EmbeddingGradientArgs a, SumShape h) {
  constexpr int N = DY_BF16 ? 8 : 4, ES = DY_BF16 ? 2 : 4;
  const uint32_t w = blockIdx.y, n = a.w.tokens[w], lane = threadIdx.x % 64;
  const uint32_t row0 = uniform((blockIdx.x * (kSumBlock / 64) + threadIdx.x / 64) * h.clear_rows);
  if (row0 >= a.vocab) return;
  const uint32_t rows = min(h.clear_rows, a.vocab - row0);
  const uint64_t out = a.w.c[w];
  const uint32_t id = lane < n ? read_id<IDS64>(a.w.a[w], lane, a.vocab) : 0xFFFFFFFFu;
  const uint64_t mine = __ballot(id - row0 < rows);
  // rows that no token names; the slices of columns share them
  uint64_t named = 0;
  for (uint64_t left = mine; left; left &= left - 1) named |= uint64_t(1) << (__builtin_amdgcn_readlane(id, __ffsll((unsigned long long)left) - 1) - row0);
  if (!a.accumulate) {
    const uint32_t share = (rows + gridDim.z - 1) / gridDim.z, from = min(blockIdx.z * share, rows);
    if (from < rows) clear_rows<OUT_BF16>(out, a.width, row0 + from, min(share, rows - from), ~named >> from);
  }
  const uint32_t at_col = (blockIdx.z * 64 + lane) * N;
  if (!mine || (blockIdx.z * 64) * N >= a.width) return;
  const Columns c = columns<N>(at_col, a.width);
  const uint64_t dy = a.w.b[w] + uint64_t(c.col) * ES;
  for (uint64_t left = mine; left;) {
    const uint32_t row = __builtin_amdgcn_readlane(id, __ffsll((unsigned long long)left) - 1);
    uint64_t same = __ballot(id == row);
    left &= ~same;
    float sum[N] = {};
    auto walk = [&](auto&& fetch) {
      while (same) {
        float x[kAhead][N];
        bool there[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          there[j] = same != 0;
          // behind the last one: some token again, which is not added
          const uint32_t token = there[j] ? __ffsll((unsigned long long)same) - 1 : 0;
          same &= same - 1;
          fetch(dy + uint64_t(token) * a.dy_pitch * ES, x[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          if (!there[j]) break;
          for (int k = 0; k < N; ++k) sum[k] += x[j][k];
        }
      }
    };
    if (a.width >= N) {
      walk([&](uint64_t from, float* x) { load_elems<DY_BF16, N>(from, x); });
    } else {
      walk([&](uint64_t from, float* x) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
          x[k] = 0.0f;
          if (uint32_t(k) < a.width) load_elems<DY_BF16, 1>(from + k * ES, x + k);
        }
      });
    }
    if (at_col < a.width) write_row<OUT_BF16, N>(a, out, row, c, sum);
  }
}

// Most chunks have nothing to join, so workgroups are small: 8 x 4096 tokens of 30522 words, 32 to a chunk, four wavefronts 4.8 us,
// eight 6.3; all on two rows 5.5 and 5.8, two wavefronts 7.0.
constexpr int kJoinWaves = 4;

// One workgroup per chunk and 256 columns; it works if a row begins in the chunk and runs past its end.  The
// wavefronts take equal stretches of that row's partial sums: however long the row is, one workgroup for 256 of its columns.  2^18 tokens on
// two rows of 128 fp32: sorting 250 us (one workgroup has both ids), sums 22, joining 91; 2^20: 980, 104, 440.
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
  const uint32_t wave = threadIdx.x / 64, at_col = blockIdx.z * 256 + threadIdx.x % 64 * 4;
  const Columns c = columns<4>(at_col, a.width);
  const uint32_t share = (pieces + kJoinWaves - 1) / kJoinWaves;
  const uint32_t p0 = min(wave * share, pieces), p1 = min(p0 + share, pieces);
  const uint64_t partial = reinterpret_cast<uint64_t>(ws + l.partial) + uint64_t(c.col) * 4;
  float sum[4] = {};
#pragma unroll 8
  for (uint32_t p = p0; p < p1; ++p) {
    // the first piece lies in the second place of its chunk, the others in the first
    const uint64_t at = partial + (uint64_t(chunk + p) * 2 + (p == 0 ? 1 : 0)) * a.width * 4;
    float x[4] = {};
    if (a.width >= 4) load_elems<false, 4>(at, x);
    else
      for (int j = 0; j < 4; ++j)
        if (uint32_t(j) < a.width) load_elems<false, 1>(at + 4 * j, x + j);
    for (int j = 0; j < 4; ++j) sum[j] += x[j];
  }
  for (int j = 0; j < 4; ++j) part[wave][threadIdx.x % 64 * 4 + j] = sum[j];
  __syncthreads();
  if (wave || at_col >= a.width) return;
  for (int v = 1; v < kJoinWaves; ++v)
    for (int j = 0; j < 4; ++j) sum[j] += part[v][threadIdx.x * 4 + j];
  write_row<OUT_BF16, 4>(a, a.w.c[w], row, c, sum);
}

uint32_t lanes_for(uint32_t width, uint32_t per_lane, uint32_t most) {
  uint32_t lanes = 1;
  while (lanes < most && lanes * per_lane < width) lanes *= 2;
  return lanes;
}

// `h` has the shape of clearing a row.
hipError_t launch_few(const EmbeddingGradientArgs& a, SumShape h, hipStream_t s) {
  const uint32_t per_lane = a.dy_bf16 ? 8 : 4;
  const uint32_t slices = (a.width + 64 * per_lane - 1) / (64 * per_lane);
  // few rows: one to a wavefront, as long as that gives no more than eight wavefronts per SIMD
  const uint64_t even = (uint64_t(a.vocab) * a.all * slices + 8191) / 8192;
  h.clear_rows = uint32_t(std::min<uint64_t>(h.clear_rows, even));
  const uint32_t rows = h.clear_rows * (kSumBlock / 64);  // of a workgroup
  const dim3 grid((a.vocab + rows - 1) / rows, a.world, slices);
#define CARAMEL_FEW(IDS64, DY, OUT) hipLaunchKernelGGL((k_embedding_few<IDS64, DY, OUT>), grid, dim3(kSumBlock), 0, s, a, h)
  if (a.ids64) {
    if (a.dy_bf16) {
      if (a.out_bf16) CARAMEL_FEW(true, true, true);
      else CARAMEL_FEW(true, true, false);
    } else {
      if (a.out_bf16) CARAMEL_FEW(true, false, true);
      else CARAMEL_FEW(true, false, false);
    }
  } else if (a.dy_bf16) {
    if (a.out_bf16) CARAMEL_FEW(false, true, true);
    else CARAMEL_FEW(false, true, false);
  } else {
    if (a.out_bf16) CARAMEL_FEW(false, false, true);
    else CARAMEL_FEW(false, false, false);
  }
#undef CARAMEL_FEW
  return hipGetLastError();
}

hipError_t launch_sorted(const EmbeddingGradientArgs& a, const Layout& l, SumShape h, hipStream_t s) {
  const uint32_t per_lane = a.dy_bf16 ? 8 : 4;
  // enough workgroups to fill the chip, each with as few ids as that allows
  const uint64_t even = (uint64_t(a.vocab) * a.all + 255) / 256;
  const uint32_t range = uint32_t(std::min<uint64_t>({kSortRange, std::max<uint64_t>(16, even), a.vocab}));
  uint32_t bits = 0;
  while ((1u << bits) < range) ++bits;
  const dim3 sort_grid((a.vocab + range - 1) / range, a.world);
  if (a.ids64) hipLaunchKernelGGL((k_embedding_sort<true>), sort_grid, dim3(64 * kSortWaves), 0, s, a, l, range, bits);
  else hipLaunchKernelGGL((k_embedding_sort<false>), sort_grid, dim3(64 * kSortWaves), 0, s, a, l, range, bits);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  h.lanes = lanes_for(a.width, per_lane, 64);
  const uint32_t groups = kSumBlock / h.lanes, slices = (a.width + h.lanes * per_lane - 1) / (h.lanes * per_lane);
  h.sum_blocks = (l.chunks + groups - 1) / groups;
  const uint32_t cleared = h.clear_rows * (kSumBlock / 64) * slices;  // by the workgroups of one x
  const dim3 sum_grid(h.sum_blocks + (a.accumulate ? 0 : (a.vocab + cleared - 1) / cleared), a.world, slices);
#define CARAMEL_SUM(DY, OUT, FULL) hipLaunchKernelGGL((k_embedding_sum<DY, OUT, FULL>), sum_grid, dim3(kSumBlock), 0, s, a, l, h)
  if (h.lanes == 64) {
    if (a.dy_bf16) {
      if (a.out_bf16) CARAMEL_SUM(true, true, true);
      else CARAMEL_SUM(true, false, true);
    } else {
      if (a.out_bf16) CARAMEL_SUM(false, true, true);
      else CARAMEL_SUM(false, false, true);
    }
  } else {
    if (a.dy_bf16) {
      if (a.out_bf16) CARAMEL_SUM(true, true, false);
      else CARAMEL_SUM(true, false, false);
    } else {
      if (a.out_bf16) CARAMEL_SUM(false, true, false);
      else CARAMEL_SUM(false, false, false);
    }
  }
#undef CARAMEL_SUM
  e = hipGetLastError();
  if (e != hipSuccess || l.chunks < 2) return e;
  const dim3 join_grid(l.chunks - 1, a.world, (a.width + 255) / 256);
  if (a.out_bf16) hipLaunchKernelGGL((k_embedding_join<true>), join_grid, dim3(64 * kJoinWaves), 0, s, a, l);
  else hipLaunchKernelGGL((k_embedding_join<false>), join_grid, dim3(64 * kJoinWaves), 0, s, a, l);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding_lookup(const LookupArgs& args, const AllWorkers& v, hipStream_t s) {
  if (args.max_tokens == 0) return hipSuccess;
  const uint32_t lanes = lanes_for(args.width, args.bf16 ? 8 : 4, 256);
  const uint32_t rows = 256 / lanes * kLookupRows;
  uint64_t bytes = 0;
  for (uint32_t w = 0; w < args.all; ++w) bytes += uint64_t(v.tokens[w]) * args.width * (args.bf16 ? 2 : 4);
  const bool stream = bytes > (uint64_t(32) << 20);
  return in_groups(args, v, [&](const LookupArgs& a, uint32_t) {
    const dim3 grid((a.max_tokens + rows - 1) / rows, a.world);
#define CARAMEL_LOOKUP(BF16, IDS64)                                                                                    \
  if (stream) hipLaunchKernelGGL((k_embedding_lookup<BF16, IDS64, true>), grid, dim3(256), 0, s, a, lanes);            \
  else hipLaunchKernelGGL((k_embedding_lookup<BF16, IDS64, false>), grid, dim3(256), 0, s, a, lanes)
    if (a.bf16) {
      if (a.ids64) {
        CARAMEL_LOOKUP(true, true);
      } else {
        CARAMEL_LOOKUP(true, false);
      }
    } else if (a.ids64) {
      CARAMEL_LOOKUP(false, true);
    } else {
      CARAMEL_LOOKUP(false, false);
    }
#undef CARAMEL_LOOKUP
    return hipGetLastError();
  });
}

// Enough for fewer tokens too: those just below a step to longer chunks have the most of them.
uint64_t embedding_gradient_workspace(uint32_t world, uint32_t vocab, uint32_t width, uint32_t max_tokens) {
  const uint64_t few = (kManyTokens - 1) / world, wide = uint64_t(vocab) * 32 - 1;  // the most tokens with chunks of 8, of 16
  uint64_t most = 0;
  for (uint64_t n : {uint64_t(max_tokens), few, wide})
    if (n <= max_tokens) most = std::max(most, layout(world, vocab, width, uint32_t(n)).stride);
  return most * world;
}

hipError_t launch_embedding_gradient(const EmbeddingGradientArgs& args, const AllWorkers& v, hipStream_t s) {
  if (args.max_tokens == 0 && args.accumulate) return hipSuccess;
  SumShape h{};
  h.clear_rows = std::min(64u, std::max(1u, (32u << 10) / (args.width * (args.out_bf16 ? 2 : 4))));  // 32 KiB
  if (args.max_tokens <= kFew)
    return in_groups(args, v, [&](const EmbeddingGradientArgs& a, uint32_t) { return launch_few(a, h, s); });
  const Layout l = layout(args.all, args.vocab, args.width, args.max_tokens);
  return in_groups(args, v, [&](EmbeddingGradientArgs a, uint32_t first) {
    a.ws += first * l.stride;
    return launch_sorted(a, l, h, s);
  });
}

}  // namespace caramel
