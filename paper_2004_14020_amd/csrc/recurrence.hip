// A gated linear recurrence along packed sequences, and its gradient.
//
//   a_t = 1 / (1 + exp(-gate_t)), b_t = 1 - a_t;   s_t = a_t s_(t-1) + b_t u_t      (u: the input; every channel by itself)
//   gradient, with e_t = dL/ds_t = ds_t + a_(t+1) e_(t+1):   du_t = b_t e_t,   dgate_t = a_t b_t e_t (s_(t-1) - u_t)
//
// A step is an affine map, and two of them in a row are one: (A, B) after (A', B') is (A A', A B' + B).  A workgroup takes a
// span of a worker's tokens for 64 C channels and walks it in tiles; in a tile every wavefront maps its own tokens, all
// exchange what their maps are, and each starts its tokens from the state that the maps before it give.  So every value is read
// and written once.  Where workers and channels are too few for the GPU, the tokens are cut into parts, and where a sequence goes on
// behind a part, a launch before this one leaves the map of its tokens in the part.  The gradient walks the same way from the last token to the first.
//
// A sequence's first token (its last one, in the gradient) takes nothing from what was before: where it stands, the map is replaced
// and not multiplied by zero, so that an infinity or NaN ends with its sequence.  States are fp32.
//
// Bound by memory.  8 workers x 4096 tokens x 1024 bf16 channels in sequences of 512: the walk 40.5 us, 5.0 TB/s (a copy of 1 GiB: 6.08), the maps
// 4.5; the gradient of ragged sequences 73 us, 4.9 TB/s, and 14.8.  One sequence of 16384 tokens x 1000 fp32 channels: gradient 79 us, 5.4 TB/s,
// and 22.8 us for the maps, which read gates and dstates once more.
//
// Sequences of a token or two, as in serving, have a kernel of their own.
#include <algorithm>
#include <type_traits>

#include "layers.hpp"
#include "rows.hpp"

namespace caramel {
namespace {

constexpr int kSteps = 4;            // tokens of a wavefront in a tile
constexpr int kWalkWaves = 8;        // wavefronts of a workgroup
constexpr int kAhead = 8;            // rows of gates that a wavefront asks for at once where it only maps
constexpr uint32_t kTile = kSteps * kWalkWaves;
constexpr uint32_t kLanes = 64 * kWalkWaves;
constexpr uint32_t kDies = 8;
constexpr uint32_t kNone = 0xFFFFFFFFu;

// C neighbouring channels, as they lie in memory, and widened.  Rows are reached through buffer resources: where a wavefront's rows begin, and how
// far a row is from there, are the same for all lanes and stay in scalar registers; `at` is a lane's distance in a row, in bytes.
template <bool BF16, int C>
struct Raw {
  uint32_t w[BF16 && C == 2 ? 1 : C];
};
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(uint64_t first) { return buffer(first, 0xFFFFFFFFu); }
template <bool BF16, int C, bool STREAM = false>
__device__ __forceinline__ Raw<BF16, C> load_raw(const __amdgpu_buffer_rsrc_t& rows, uint32_t at, uint32_t row) {
  Raw<BF16, C> r;
  if constexpr (C == 1 && BF16) {
    r.w[0] = uint32_t(__builtin_amdgcn_raw_buffer_load_b16(rows, int(at), int(row), STREAM ? kStreaming : 0));
  } else if constexpr (C == 1 || BF16) {
    r.w[0] = uint32_t(__builtin_amdgcn_raw_buffer_load_b32(rows, int(at), int(row), STREAM ? kStreaming : 0));
  } else {
    const u32x2 p = __builtin_amdgcn_raw_buffer_load_b64(rows, int(at), int(row), STREAM ? kStreaming : 0);
    r.w[0] = p[0];
    r.w[1] = p[1];
  }
  return r;
}
template <bool BF16, int C>
__device__ __forceinline__ float widen(const Raw<BF16, C>& r, int c) {
  if constexpr (!BF16) return as_float(r.w[c]);
  else return c ? bf16_high(r.w[0]) : bf16_low(r.w[0]);
}
template <bool BF16, int C, bool STREAM = false>
__device__ __forceinline__ void store_channels(const __amdgpu_buffer_rsrc_t& rows, uint32_t at, uint32_t row, const float* v) {
  if constexpr (BF16) {
    const uint32_t p = bf16_pair(v[0], v[C - 1]);
    if constexpr (C == 1) __builtin_amdgcn_raw_buffer_store_b16(uint16_t(p), rows, int(at), int(row), STREAM ? kStreaming : 0);
    else __builtin_amdgcn_raw_buffer_store_b32(p, rows, int(at), int(row), STREAM ? kStreaming : 0);
  } else {
    if constexpr (C == 1) __builtin_amdgcn_raw_buffer_store_b32(as_bits(v[0]), rows, int(at), int(row), STREAM ? kStreaming : 0);
    else __builtin_amdgcn_raw_buffer_store_b64(u32x2{as_bits(v[0]), as_bits(v[1])}, rows, int(at), int(row), STREAM ? kStreaming : 0);
  }
}

// a and b of a gate.  exp(gate) stays below 2^126, which leaves of b what differs from 0 by less than 2^-125.
// fp32 gates: log2(e) is the fp32 number 1.44269504f and 1.926e-8 more, and the product with it is carried in two numbers, so that
// a and b are right to a few last bits; below -150, a is 0.
template <bool BF16>
__device__ __forceinline__ void gates(float g, float* a, float* b) {
  g = g > 87.0f ? 87.0f : g;
  if constexpr (!BF16) g = g < -150.0f ? -150.0f : g;
  const float t = g * 1.44269504f;
  float e = __builtin_amdgcn_exp2f(t);
  if constexpr (!BF16) {
    const float low = __builtin_fmaf(g, 1.92596299e-8f, __builtin_fmaf(g, 1.44269504f, -t));
    e = __builtin_fmaf(e, low * 0.69314718f, e);
  }
  const float s = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(s);
  if constexpr (!BF16) r = __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r);
  *b = r;
  *a = e * r;
}

// ---- where sequences begin ------------------------------------------------------------------

// The list of a worker's starts, in device memory; what is no place among the tokens counts as the nearest one.  A list of up to 64
// numbers is loaded once, one to a lane, and everything is asked of the lanes (a longer one takes a chain of loads for every question, some
// microseconds at the start of a workgroup).
struct Starts {
  uint64_t at;
  uint32_t sequences, tokens;
  bool wide, whole;
  uint32_t mine;  // whole: the lane's entry

  __device__ __forceinline__ Starts(uint64_t list, uint32_t n, uint32_t most, bool is_wide)
      : at(list), sequences(n), tokens(most), wide(is_wide), whole(n < 64), mine(0) {
    if (whole) mine = get(threadIdx.x % 64);
  }
  // two entries alone, `first` and the next
  __device__ __forceinline__ Starts(uint64_t list, uint32_t n, uint32_t most, bool is_wide, uint32_t first)
      : at(list), sequences(n), tokens(most), wide(is_wide), whole(false), mine(get(first + threadIdx.x % 2)) {}
  // lanes ask for entries by themselves; behind the list there is what no token reaches
  __device__ __forceinline__ uint32_t get(uint32_t i) const {
    if (i > sequences) return 0x7FFFFFFFu;
    const int64_t v = wide ? reinterpret_cast<const CARAMEL_GLOBAL int64_t*>(at)[i]
                           : int64_t(reinterpret_cast<const CARAMEL_GLOBAL int32_t*>(at)[i]);
    return v < 0 ? 0u : v > int64_t(tokens) ? tokens : uint32_t(v);
  }
  // an entry that all lanes ask for
  __device__ __forceinline__ uint32_t one(uint32_t i) const {
    if (whole) return i > sequences ? 0x7FFFFFFFu : uint32_t(__builtin_amdgcn_readlane(int(mine), int(i)));
    return uniform(get(i));
  }
  // the first entry that is x or more, by the whole wavefront: 64 probes at a time
  __device__ __forceinline__ uint32_t lower(uint32_t x) const {
    const uint32_t lane = threadIdx.x % 64;
    if (whole) return uint32_t(__builtin_popcountll(__ballot(mine < x)));
    uint32_t lo = 0, len = sequences + 1;
    while (len > 0) {
      const uint32_t step = (len + 63) / 64, probe = lane * step + step - 1;
      const uint32_t below = uint32_t(__builtin_popcountll(__ballot(probe < len && get(lo + probe) < x)));
      lo += below * step;
      len = step == 1 ? 0 : min(step - 1, len - min(len, below * step));
    }
    return uniform(min(lo, sequences + 1));
  }
};

// A wavefront's view of the list: 64 entries from the first one that counts for its tokens.
struct Window {
  uint32_t first;  // index of lane 0's entry
  uint32_t entry;  // a lane's
};
__device__ __forceinline__ Window window(const Starts& s, uint32_t token) {
  Window w;
  w.first = s.whole ? 0 : s.lower(token);
  w.entry = s.whole ? s.mine : s.get(w.first + threadIdx.x % 64);
  return w;
}

// The sequence that begins with a token (kNone: none does), and the one that ends with it.  Of sequences without tokens
// at the same place, neither is one.
struct Marks {
  uint32_t begins[kSteps], ends[kSteps];
  bool any;
};
__device__ __forceinline__ Marks marks(const Starts& s, const Window& v, uint32_t t0) {
  Marks m;
  m.any = __ballot(v.entry >= t0 && v.entry <= t0 + kSteps) != 0;
#pragma unroll
  for (int k = 0; k < kSteps; ++k) m.begins[k] = m.ends[k] = kNone;
  if (!m.any) return m;
  const uint32_t behind = uint32_t(__builtin_amdgcn_readlane(int(v.entry), 63));
  if (behind > t0 + kSteps) {
    uint64_t here = __ballot(v.entry == t0);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const uint64_t next = __ballot(v.entry == t0 + k + 1);
      if (here) m.begins[k] = v.first + 63 - uint32_t(__builtin_clzll(here));
      if (next) m.ends[k] = v.first + uint32_t(__builtin_ctzll(next)) - 1;  // of entry 0: kNone
      here = next;
    }
  } else {  // more than 64 starts here: sequences without tokens
    uint32_t at = s.lower(t0);
#pragma unroll 1
    for (int k = 0; k < kSteps; ++k) {
      const uint32_t next = s.lower(t0 + k + 1);
      const bool begins = next > at, ends = s.one(next) == t0 + k + 1;
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {  // (the index of an array in registers is a constant)
        if (j == k && begins) m.begins[j] = next - 1;
        if (j == k && ends) m.ends[j] = next - 1;
      }
      at = next;
    }
  }
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    if (m.begins[k] >= s.sequences) m.begins[k] = kNone;  // the list's last entry is the end of the last sequence
    if (m.ends[k] >= s.sequences) m.ends[k] = kNone;
  }
  return m;
}

// ---- walking --------------------------------------------------------------------------------

// A workgroup's place: worker w, part, channels.  The last lanes take the last C channels once more: equal values go to equal places.
template <bool BF16, int C, bool BACK>
struct Walk {
  static constexpr int ES = BF16 ? 2 : 4;
  typedef Raw<BF16, C> raw;
  const RecurrenceArgs& r;
  uint32_t w, part, parts;  // parts of the worker
  bool there;               // the grid may have more workgroups than there are parts
  uint32_t at, at32;        // a lane's distance in bytes from the rows of dtype, and from fp32 rows

  __device__ __forceinline__ Walk(const RecurrenceArgs& args) : r(args), w(0) {
    // Workgroups go to the eight dies in turn: all channels of a part go to one of them, whose cache then has whole rows (8 x 4096 tokens of
    // 1000 bf16, whose rows end inside a cache line: gradient 130 us, so 89).
    const uint32_t slabs = (r.channels + 64 * C - 1) / (64 * C), turn = blockIdx.x / kDies, k = turn / slabs * kDies + blockIdx.x % kDies;
    there = k < r.first_part[kGroup];
#pragma unroll
    for (uint32_t i = 1; i < kGroup; ++i) w += there && k >= r.first_part[i] ? 1 : 0;
    part = k - r.first_part[w];
    parts = r.first_part[w + 1] - r.first_part[w];
    place(turn % slabs);
  }
  // by itself: all of the worker's tokens
  __device__ __forceinline__ Walk(const RecurrenceArgs& args, uint32_t worker, uint32_t slab)
      : r(args), w(worker), part(0), parts(1), there(true) {
    place(slab);
  }
  __device__ __forceinline__ void place(uint32_t slab) {
    const uint32_t channel = min((slab * 64 + threadIdx.x % 64) * C, r.channels - C);
    at = channel * ES;
    at32 = channel * 4;
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rows(int which, uint32_t t, uint64_t pitch) const {
    return rows_from(r.w.at[which][w] + t * pitch * ES);
  }

  // fp32 rows of the sequences (zeros, or nothing, where the call has none)
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t row_of(int which, uint32_t sequence) const {
    return rows_from(r.w.at[which][w] + uint64_t(sequence) * r.channels * 4);
  }
  __device__ __forceinline__ void get(int which, uint32_t sequence, float* v) const {
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = 0.0f;
    if (!r.w.at[which][w]) return;
    const raw32 x = load_raw<false, C>(row_of(which, sequence), at32, 0);
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = as_float(x.w[c]);
  }
  __device__ __forceinline__ void put(int which, uint32_t sequence, const float* v) const {
    if (r.w.at[which][w]) store_channels<false, C>(row_of(which, sequence), at32, 0, v);
  }
  typedef Raw<false, C> raw32;
  // what a sequence's walk starts from, and where it leaves what it ends with
  static constexpr int kBegin = BACK ? kRecDafter : kRecBefore, kEnd = BACK ? kRecDbefore : kRecAfter;

  // a part's map in the workspace: two fp32 rows
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t map_of(uint32_t k) const {
    return rows_from(reinterpret_cast<uint64_t>(r.ws) + uint64_t(r.first_part[w] + k) * r.channels * 8);
  }
};

// The sequence that goes on across the border in front of token x: its number, its first token and the one behind its last.
struct Crossing {
  bool there;
  uint32_t sequence, first, behind;
};
__device__ __forceinline__ Crossing crossing(const Starts& s, uint32_t x) {
  const uint32_t next = s.lower(x);  // the first start from x on
  Crossing c;
  c.behind = s.one(next);
  c.there = next > 0 && next <= s.sequences && c.behind != x;
  c.sequence = next - 1;
  c.first = c.there ? s.one(next - 1) : 0;
  return c;
}

// The maps of the parts out of which a sequence goes on: of its tokens there, all of which are inside.  Every wavefront has a stretch of them.
template <bool BF16, int C, bool BACK>
__global__ void __launch_bounds__(kLanes) k_walk_maps(RecurrenceArgs r) {
  __shared__ float maps[kWalkWaves][2][C][64];
  const Walk<BF16, C, BACK> walk(r);
  if (!walk.there) return;
  const uint32_t n = r.w.tokens[walk.w], part = walk.part, span = r.span, lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
  const Starts starts(r.w.at[kRecStarts][walk.w], r.w.more[walk.w], n, r.starts64);
  uint32_t lo = part * span, hi = min(lo + span, n);
  const Crossing x = crossing(starts, BACK ? lo : hi);
  if (!x.there) return;
  const bool begins = BACK ? x.behind <= hi : x.first >= lo;  // inside the part
  if constexpr (BACK) hi = max(min(hi, x.behind), lo + 1);
  else lo = min(max(lo, x.first), hi - 1);
  // stretches in the order of the walk
  const uint32_t each = (hi - lo + kWalkWaves - 1) / kWalkWaves, place = BACK ? kWalkWaves - 1 - wave : wave;
  const uint32_t from = min(lo + place * each, hi), to = min(from + each, hi);
  float A[C], B[C];
#pragma unroll
  for (int c = 0; c < C; ++c) A[c] = 1.0f, B[c] = 0.0f;
  if (begins && wave == 0) walk.get(walk.kBegin, x.sequence, B);
  auto steps = [&](uint32_t done, auto count) {
    constexpr int N = decltype(count)::value;
    typename Walk<BF16, C, BACK>::raw gate[N], add[N];
    const uint32_t t0 = BACK ? to - done - N : from + done;
    const uint64_t add_pitch = BACK ? r.states_pitch : r.pitch;
    const __amdgpu_buffer_rsrc_t gates_at = walk.rows(kRecGate, t0, r.pitch);
    const __amdgpu_buffer_rsrc_t add_at = walk.rows(BACK ? kRecDstates : kRecInput, t0, add_pitch);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint32_t on = BACK ? N - 1 - k : k;
      gate[k] = load_raw<BF16, C>(gates_at, walk.at, on * uint32_t(r.pitch) * walk.ES);
      add[k] = load_raw<BF16, C>(add_at, walk.at, on * uint32_t(add_pitch) * walk.ES);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float a, b;
        gates<BF16>(widen<BF16, C>(gate[k], c), &a, &b);
        const float v = widen<BF16, C>(add[k], c);
        B[c] = BACK ? a * (v + B[c]) : __builtin_fmaf(a, B[c], b * v);
        A[c] *= a;
      }
    }
  };
  uint32_t done = 0;
  for (; done + kAhead <= to - from; done += kAhead) steps(done, std::integral_constant<int, kAhead>{});
  for (; done < to - from; ++done) steps(done, std::integral_constant<int, 1>{});
#pragma unroll
  for (int c = 0; c < C; ++c) {
    maps[wave][0][c][lane] = A[c];
    maps[wave][1][c][lane] = B[c];
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int v = 1; v < kWalkWaves; ++v) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      A[c] *= maps[v][0][c][lane];
      B[c] = __builtin_fmaf(maps[v][0][c][lane], B[c], maps[v][1][c][lane]);
    }
  }
  store_channels<false, C>(walk.map_of(part), walk.at32, 0, A);
  store_channels<false, C>(walk.map_of(part), walk.at32, r.channels * 4, B);
}

// The rows of a wavefront's tokens in a tile, from token t0 on; of those from `stop` on, the last one before it.
template <bool BF16, int C, bool BACK, bool STREAM>
struct TileRows {
  Raw<BF16, C> gate[kSteps], input[kSteps], prior[BACK ? kSteps : 1], ds[BACK ? kSteps : 1];
  __device__ __forceinline__ void load(const Walk<BF16, C, BACK>& walk, uint32_t t0, uint32_t stop) {
    const RecurrenceArgs& r = walk.r;
    const uint32_t base = min(t0, stop - 1), more = stop - 1 - base, before = base ? base - 1 : 0;
    const __amdgpu_buffer_rsrc_t gates_at = walk.rows(kRecGate, base, r.pitch), input_at = walk.rows(kRecInput, base, r.pitch);
    const __amdgpu_buffer_rsrc_t ds_at = walk.rows(kRecDstates, base, r.states_pitch);
    const __amdgpu_buffer_rsrc_t prior_at = walk.rows(kRecStates, before, r.states_pitch);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const uint32_t on = min(uint32_t(k), more), row = on * uint32_t(r.pitch) * walk.ES;
      gate[k] = load_raw<BF16, C, STREAM>(gates_at, walk.at, row);
      if constexpr (BACK) ds[k] = load_raw<BF16, C, STREAM>(ds_at, walk.at, on * uint32_t(r.states_pitch) * walk.ES);
      input[k] = load_raw<BF16, C, STREAM>(input_at, walk.at, row);
      // (the first token of all has no row before it, and needs none)
      if constexpr (BACK) prior[k] = load_raw<BF16, C, STREAM>(prior_at, walk.at, (base || !on ? on : on - 1) * uint32_t(r.states_pitch) * walk.ES);
    }
  }
};

// The walk itself.  STREAM: streaming loads and stores, where every workgroup has whole cache lines of the rows.  (Where two share a line, it had
// better stay in the cache for the other.)
template <bool BF16, int C, bool BACK, bool STREAM>
__global__ void __launch_bounds__(kLanes) k_walk_tokens(RecurrenceArgs r) {
  typedef float Map __attribute__((ext_vector_type(2 * C)));
  __shared__ Map maps[2][kWalkWaves][64];
  __shared__ uint32_t cuts[2][kWalkWaves];
  const Walk<BF16, C, BACK> walk(r);
  if (!walk.there) return;
  const uint32_t n = r.w.tokens[walk.w], part = walk.part, span = r.span, lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
  const Starts starts(r.w.at[kRecStarts][walk.w], r.w.more[walk.w], n, r.starts64);
  const uint32_t lo = part * span, hi = min(lo + span, n);
  // sequences without tokens leave what they start from
  if (r.w.at[walk.kEnd][walk.w]) {
    for (uint32_t s0 = (part * kWalkWaves + wave) * 64; s0 < starts.sequences; s0 += walk.parts * kWalkWaves * 64) {
      uint64_t empty = __ballot(s0 + lane < starts.sequences && starts.get(s0 + lane) >= starts.get(s0 + lane + 1));
      while (empty) {
        const uint32_t one = s0 + uint32_t(__builtin_ctzll(empty));
        float v[C];
        walk.get(walk.kBegin, one, v);
        walk.put(walk.kEnd, one, v);
        empty &= empty - 1;
      }
    }
  }
  const uint32_t none_before = starts.one(0), none_behind = starts.one(starts.sequences);

  // the maps that lead up to this part: of the sequence that comes in, from the part where it begins
  float state[C];
#pragma unroll
  for (int c = 0; c < C; ++c) state[c] = 0.0f;
  const Crossing x = crossing(starts, BACK ? hi : lo);
  if (x.there) {
    uint32_t from = part, to = part;  // parts, without the last one
    if constexpr (BACK) {
      from = part + 1;
      to = min((max(x.behind, 1u) - 1) / span + 1, walk.parts);
    } else {
      from = x.first / span;
    }
    for (uint32_t k = from; k < to; ++k) {
      const __amdgpu_buffer_rsrc_t map = walk.map_of(BACK ? to - 1 - (k - from) : k);
      const Raw<false, C> A = load_raw<false, C>(map, walk.at32, 0), B = load_raw<false, C>(map, walk.at32, r.channels * 4);
#pragma unroll
      for (int c = 0; c < C; ++c)
        state[c] = k == from ? as_float(B.w[c]) : __builtin_fmaf(as_float(A.w[c]), state[c], as_float(B.w[c]));
    }
  }

  const uint32_t tiles = (hi - lo + kTile - 1) / kTile;
  Window view = window(starts, 0);  // the whole list, where it is short
  // the wavefronts' tokens follow each other the way the walk goes
  auto first_token = [&](uint32_t i) {
    return lo + (BACK ? tiles - 1 - i : i) * kTile + (BACK ? kWalkWaves - 1 - wave : wave) * kSteps;
  };
  typedef TileRows<BF16, C, BACK, STREAM> Rows;
  Rows next;
  next.load(walk, first_token(0), hi);
  for (uint32_t i = 0; i < tiles; ++i) {
    const uint32_t t0 = first_token(i);
    const uint32_t count = t0 < hi ? min(hi - t0, uint32_t(kSteps)) : 0;
    const Rows now = next;
    next.load(walk, first_token(min(i + 1, tiles - 1)), hi);  // the next tile's are on their way while this one is worked on
    const auto &gate = now.gate, &input = now.input;
    const auto &prior = now.prior, &ds = now.ds;
    if (!starts.whole) view = window(starts, t0);
    const Marks mark = marks(starts, view, t0);
    const bool plain = !mark.any && count == kSteps && t0 >= none_before && t0 + kSteps <= none_behind;  // all inside one sequence

    // this wavefront's map
    float a[kSteps][C], b[kSteps][C], first[kSteps][C];
    Map map;
    bool cut = false;
#pragma unroll
    for (int c = 0; c < C; ++c) map[c] = 1.0f, map[C + c] = 0.0f;
    auto step = [&](int k) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if constexpr (BACK) map[C + c] = a[k][c] * (widen<BF16, C>(ds[k], c) + map[C + c]);
        else map[C + c] = __builtin_fmaf(a[k][c], map[C + c], b[k][c] * widen<BF16, C>(input[k], c));
        map[c] *= a[k][c];
      }
    };
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int c = 0; c < C; ++c) gates<BF16>(widen<BF16, C>(gate[k], c), &a[k][c], &b[k][c]);
    if (plain) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) step(BACK ? kSteps - 1 - j : j);
    } else {
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const uint32_t s = BACK ? mark.ends[k] : mark.begins[k];
        if (s != kNone && uint32_t(k) < count) walk.get(walk.kBegin, s, first[k]);
      }
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const int k = BACK ? kSteps - 1 - j : j;
        if (uint32_t(k) >= count || t0 + k < none_before || t0 + k >= none_behind) continue;
        if ((BACK ? mark.ends[k] : mark.begins[k]) != kNone) {
          cut = true;
#pragma unroll
          for (int c = 0; c < C; ++c) map[C + c] = first[k][c];
        }
        step(k);
      }
    }
    const uint32_t turn = i % 2;
    maps[turn][wave][lane] = map;
    if (lane == 0) cuts[turn][wave] = cut;
    __syncthreads();
    float s[C];  // the state this wavefront's tokens start from
    const uint64_t cut_by = __ballot(lane < kWalkWaves && cuts[turn][lane % kWalkWaves]);
#pragma unroll
    for (int v = 0; v < kWalkWaves; ++v) {
      const Map m = maps[turn][v][lane];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (uint32_t(v) == wave) s[c] = state[c];
        state[c] = cut_by >> v & 1 ? m[C + c] : __builtin_fmaf(m[c], state[c], m[C + c]);
      }
    }
    const uint32_t base = min(t0, hi - 1);
    const __amdgpu_buffer_rsrc_t to_input = walk.rows(BACK ? kRecDinput : kRecStates, base, BACK ? r.pitch : r.states_pitch);
    const __amdgpu_buffer_rsrc_t to_gate = walk.rows(kRecDgate, base, r.pitch);
    auto out = [&](int k, const float* before) {
      if constexpr (BACK) {
        float du[C], dg[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float e = widen<BF16, C>(ds[k], c) + s[c];
          du[c] = b[k][c] * e;
          dg[c] = (a[k][c] * du[c]) * (before[c] - widen<BF16, C>(input[k], c));
          s[c] = a[k][c] * e;
        }
        store_channels<BF16, C, STREAM>(to_input, walk.at, k * uint32_t(r.pitch) * walk.ES, du);
        store_channels<BF16, C, STREAM>(to_gate, walk.at, k * uint32_t(r.pitch) * walk.ES, dg);
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c) s[c] = __builtin_fmaf(a[k][c], s[c], b[k][c] * widen<BF16, C>(input[k], c));
        store_channels<BF16, C, STREAM>(to_input, walk.at, k * uint32_t(r.states_pitch) * walk.ES, s);
      }
    };
    auto before = [&](int k, float* v) {
#pragma unroll
      for (int c = 0; c < C; ++c) v[c] = BACK ? widen<BF16, C>(prior[BACK ? k : 0], c) : 0.0f;
    };
    if (plain) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const int k = BACK ? kSteps - 1 - j : j;
        float p[C];
        before(k, p);
        out(k, p);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const int k = BACK ? kSteps - 1 - j : j;
        if (uint32_t(k) >= count || t0 + k < none_before || t0 + k >= none_behind) continue;
        if ((BACK ? mark.ends[k] : mark.begins[k]) != kNone) {
#pragma unroll
          for (int c = 0; c < C; ++c) s[c] = first[k][c];
        }
        const uint32_t over = BACK ? mark.begins[k] : mark.ends[k];
        float p[C];
        before(k, p);
        if (BACK && over != kNone) walk.get(kRecBefore, over, p);
        out(k, p);
        if (over != kNone) walk.put(walk.kEnd, over, s);
      }
    }
  }
}

// Short sequences: a wavefront to each, which walks it by itself, four tokens at a time.  What bounds it is how many loads wait for others;
// the sequence's first state, and the tokens that it has where every sequence before it has one, are on their way before its place in
// the list is known.  One token of each of 256 sequences at two workers, 1024 fp32 channels, states in and out: 7.8 us, by the walk in tiles
// 15.4; of 1024 sequences 10.5 and 20.0, their gradient 15.7 and 27.0.
// For up to two tokens a sequence on average, and so many of both that one sequence with all tokens takes no worse than 172 us.
constexpr int kStepWaves = 4;
constexpr uint32_t kFewSteps = 1024;

template <bool BF16, int C, bool BACK>
__global__ void __launch_bounds__(64 * kStepWaves) k_steps(RecurrenceArgs r) {
  const uint32_t w = blockIdx.z, s = blockIdx.y * kStepWaves + uniform(threadIdx.x / 64), n = r.w.tokens[w];
  if (s >= r.w.more[w]) return;
  const Walk<BF16, C, BACK> walk(r, w, blockIdx.x);
  const uint64_t list = r.w.at[kRecStarts][w];
  const Starts starts(list, r.w.more[w], n, r.starts64, s);
  TileRows<BF16, C, BACK, false> rows;
  const uint32_t guess = min(s, n - 1);
  rows.load(walk, guess, min(guess + kSteps, n));
  float state[C], before[C];
  walk.get(walk.kBegin, s, state);
  if constexpr (BACK) walk.get(kRecBefore, s, before);
  const uint32_t lo = uint32_t(__builtin_amdgcn_readlane(int(starts.mine), 0));
  const uint32_t hi = max(uint32_t(__builtin_amdgcn_readlane(int(starts.mine), 1)), lo);
  const uint32_t chunks = (hi - lo + kSteps - 1) / kSteps;
  for (uint32_t i = 0; i < chunks; ++i) {
    const uint32_t t0 = lo + (BACK ? chunks - 1 - i : i) * kSteps, count = min(hi - t0, uint32_t(kSteps));
    if (t0 != guess || i) rows.load(walk, t0, t0 + count);
    const __amdgpu_buffer_rsrc_t to_input = walk.rows(BACK ? kRecDinput : kRecStates, t0, BACK ? r.pitch : r.states_pitch);
    const __amdgpu_buffer_rsrc_t to_gate = walk.rows(kRecDgate, t0, r.pitch);
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int k = BACK ? kSteps - 1 - j : j;
      if (uint32_t(k) >= count) continue;
      float out[C], dgate[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float a, b;
        gates<BF16>(widen<BF16, C>(rows.gate[k], c), &a, &b);
        const float u = widen<BF16, C>(rows.input[k], c);
        if constexpr (BACK) {
          const float e = widen<BF16, C>(rows.ds[k], c) + state[c];
          const float p = t0 + k == lo ? before[c] : widen<BF16, C>(rows.prior[k], c);
          out[c] = b * e;
          dgate[c] = (a * out[c]) * (p - u);
          state[c] = a * e;
        } else {
          out[c] = state[c] = __builtin_fmaf(a, state[c], b * u);
        }
      }
      store_channels<BF16, C>(to_input, walk.at, k * uint32_t(BACK ? r.pitch : r.states_pitch) * walk.ES, out);
      if constexpr (BACK) store_channels<BF16, C>(to_gate, walk.at, k * uint32_t(r.pitch) * walk.ES, dgate);
    }
  }
  walk.put(walk.kEnd, s, state);
}

// Workgroups of a launch that parts are made for: two to a compute unit, which is what the registers of the gradient (81 and 108) leave room for, so
// that all of them run at once.  The forward walk (60 and 73) has room for three, and was measured with two.
constexpr uint32_t kWalkGroups = 512;
constexpr uint32_t kShortest = 2 * kTile;  // tokens of a part, at least

// The most parts that the workers of a launch may have together.
uint32_t most_parts(uint32_t world, uint32_t channels, const uint32_t* tokens) {
  const uint32_t slabs = (channels + 127) / 128, wanted = (kWalkGroups + slabs - 1) / slabs;
  uint64_t could = 0, must = 0;
  for (uint32_t w = 0; w < world; ++w) {
    could += std::max(tokens[w] ? 1u : 0u, tokens[w] / kShortest);
    must += tokens[w] ? 1 : 0;
  }
  return uint32_t(std::max(must, std::min<uint64_t>(could, wanted)));
}
// All workers' parts are equally long, so that they end together: the shortest span that makes no more of them.
uint32_t span_of(uint32_t world, const uint32_t* tokens, uint32_t most, uint32_t max_tokens) {
  uint32_t lo = 1, hi = (max_tokens + kTile - 1) / kTile;  // in tiles
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    uint64_t parts = 0;
    for (uint32_t w = 0; w < world; ++w) parts += (tokens[w] + mid * kTile - 1) / (mid * kTile);
    if (parts <= most) hi = mid;
    else lo = mid + 1;
  }
  return hi * kTile;
}

template <bool BF16, int C, bool BACK>
hipError_t launch_walk(const RecurrenceArgs& a, hipStream_t s) {
  if (a.steps) {
    hipLaunchKernelGGL((k_steps<BF16, C, BACK>),
                       dim3((a.channels + 64 * C - 1) / (64 * C), (a.steps + kStepWaves - 1) / kStepWaves, a.world),
                       dim3(64 * kStepWaves), 0, s, a);
    return hipGetLastError();
  }
  const uint32_t parts = a.first_part[a.world];
  if (!parts) return hipSuccess;
  const dim3 grid((a.channels + 64 * C - 1) / (64 * C) * ((parts + kDies - 1) / kDies * kDies));
  if (a.cut) {
    hipLaunchKernelGGL((k_walk_maps<BF16, C, BACK>), grid, dim3(kLanes), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (C == 2 && a.lines) hipLaunchKernelGGL((k_walk_tokens<BF16, C, BACK, C == 2>), grid, dim3(kLanes), 0, s, a);
  else hipLaunchKernelGGL((k_walk_tokens<BF16, C, BACK, false>), grid, dim3(kLanes), 0, s, a);
  return hipGetLastError();
}

template <bool BACK>
hipError_t launch_any(const RecurrenceArgs& args, const AllBuffers<kRecBuffers>& v, hipStream_t s) {
  if (args.max_tokens == 0) return hipSuccess;
  return in_groups(args, v, [&](RecurrenceArgs a, uint32_t) {
    a.steps = 0;
    for (uint32_t w = 0; w < a.world; ++w) {
      if (a.w.tokens[w] > 2 * uint64_t(a.w.more[w]) || a.w.tokens[w] > kFewSteps || a.w.more[w] > kFewSteps) {
        a.steps = 0;
        break;
      }
      a.steps = std::max(a.steps, a.w.more[w]);
    }
    a.span = span_of(a.world, a.w.tokens, most_parts(a.world, a.channels, a.w.tokens), a.max_tokens);
    a.cut = false;
    // all rows begin on cache lines, and their channels fill them
    const uint64_t es = a.bf16 ? 2 : 4;
    uint64_t ends = a.channels * es | a.pitch * es | a.states_pitch * es;
    for (uint32_t w = 0; w < a.world; ++w)
      for (int which : {kRecGate, kRecInput, kRecStates, kRecDstates, kRecDgate, kRecDinput}) ends |= a.w.tokens[w] ? a.w.at[which][w] : 0;
    a.lines = ends % 128 == 0;
    for (uint32_t w = 0; w < kGroup; ++w) {  // (behind the last worker: its end)
      const uint32_t parts = w < a.world ? (a.w.tokens[w] + a.span - 1) / a.span : 0;
      a.first_part[w + 1] = a.first_part[w] + parts;
      a.cut = a.cut || parts > 1;
    }
    if (a.channels == 1) return a.bf16 ? launch_walk<true, 1, BACK>(a, s) : launch_walk<false, 1, BACK>(a, s);
    return a.bf16 ? launch_walk<true, 2, BACK>(a, s) : launch_walk<false, 2, BACK>(a, s);
  });
}

}  // namespace

// The launches for sixteen workers each follow one another and share it.
uint64_t recurrence_workspace_bytes(uint32_t world, uint32_t channels, const uint32_t* tokens) {
  uint64_t bytes = 0;
  for (uint32_t g = 0; g < world; g += kGroup) {
    const uint32_t n = std::min(world - g, kGroup);
    bool cut = false;
    for (uint32_t w = 0; w < n; ++w) cut = cut || tokens[g + w] / kShortest > 1;
    if (cut) bytes = std::max(bytes, uint64_t(most_parts(n, channels, tokens + g)) * channels * 8);
  }
  return bytes;
}

hipError_t launch_recurrence(const RecurrenceArgs& args, const AllBuffers<kRecBuffers>& v, hipStream_t s) {
  return launch_any<false>(args, v, s);
}

hipError_t launch_recurrence_gradient(const RecurrenceArgs& args, const AllBuffers<kRecBuffers>& v, hipStream_t s) {
  return launch_any<true>(args, v, s);
}

}  // namespace caramel
