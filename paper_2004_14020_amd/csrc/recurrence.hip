// A gated linear recurrence along packed sequences, and its gradient.
//
//   a_t = 1 / (1 + exp(-gate_t)), b_t = 1 - a_t;   s_t = a_t s_(t-1) + b_t u_t      (u: the input; every channel by itself)
//   gradient, with e_t = dL/ds_t = ds_t + a_(t+1) e_(t+1):   du_t = b_t e_t,   dgate_t = a_t b_t e_t (s_(t-1) - u_t)
//
// A step is an affine map, and two of them in a row are one: (A, B) after (A', B') is (A A', A B' + B).  A workgroup takes a
// span of a worker's tokens for 64 C channels and walks it in tiles; in a tile every wavefront maps its own K tokens, all
// exchange what their maps are, and each starts its tokens from the state that the maps before it give.  So every value is read
// and written once.  Where workers and channels are too few for the GPU, the tokens are cut into parts, and a launch
// before this one leaves every part's map; it starts at the last sequence that begins in the part and does nothing where the
// part ends with its sequence.  The gradient walks the same way from the last token to the first.
//
// A sequence's first token (its last one, in the gradient) takes nothing from what was before: where it stands, the map is replaced
// and not multiplied by zero, so that an infinity or NaN ends with its sequence.  States are fp32.
#include <algorithm>

#include "layers.hpp"
#include "vec.hpp"

namespace caramel {
namespace {

constexpr int kSteps = 8;            // tokens of a wavefront in a tile
constexpr int kWalkWaves = 8;        // wavefronts of a workgroup
constexpr uint32_t kTile = kSteps * kWalkWaves;
constexpr uint32_t kLanes = 64 * kWalkWaves;
constexpr uint32_t kNone = 0xFFFFFFFFu;

// C neighbouring channels, as they lie in memory, and widened
template <bool BF16, int C>
struct Raw {
  uint32_t w[BF16 && C == 2 ? 1 : C];
};
template <bool BF16, int C>
__device__ __forceinline__ Raw<BF16, C> load_raw(uint64_t at) {
  Raw<BF16, C> r;
  if constexpr (C == 1) {
    if constexpr (BF16) r.w[0] = *reinterpret_cast<const CARAMEL_GLOBAL uint16_t*>(at);
    else r.w[0] = *reinterpret_cast<const CARAMEL_GLOBAL uint32_t*>(at);
  } else if constexpr (BF16) {
    typedef uint32_t word __attribute__((aligned(2)));
    r.w[0] = *reinterpret_cast<const CARAMEL_GLOBAL word*>(at);
  } else {
    typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(4)));
    const pair p = *reinterpret_cast<const CARAMEL_GLOBAL pair*>(at);
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
template <bool BF16, int C>
__device__ __forceinline__ void store_channels(uint64_t at, const float* v) {
  if constexpr (C == 1) {
    store_elems<BF16, 1>(at, v);
  } else if constexpr (BF16) {
    typedef uint32_t word __attribute__((aligned(2)));
    *reinterpret_cast<CARAMEL_GLOBAL word*>(at) = bf16_pair(v[0], v[1]);
  } else {
    typedef float pair __attribute__((ext_vector_type(2), aligned(4)));
    const pair p = {v[0], v[1]};
    *reinterpret_cast<CARAMEL_GLOBAL pair*>(at) = p;
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

// The list of a worker's starts, in device memory; what is no place among the tokens counts as the nearest one.
struct Starts {
  uint64_t at;
  uint32_t sequences, tokens;
  bool wide;
  // lanes ask for entries by themselves; behind the list there is what no token reaches
  __device__ __forceinline__ uint32_t get(uint32_t i) const {
    if (i > sequences) return 0x7FFFFFFFu;
    const int64_t v = wide ? reinterpret_cast<const CARAMEL_GLOBAL int64_t*>(at)[i]
                           : int64_t(reinterpret_cast<const CARAMEL_GLOBAL int32_t*>(at)[i]);
    return v < 0 ? 0u : v > int64_t(tokens) ? tokens : uint32_t(v);
  }
  // the first entry that is x or more, by the whole wavefront: 64 probes at a time
  __device__ __forceinline__ uint32_t lower(uint32_t x) const {
    const uint32_t lane = threadIdx.x % 64;
    uint32_t lo = 0, len = sequences + 1;
    while (len > 0) {
      const uint32_t step = (len + 63) / 64, probe = lane * step + step - 1;
      const uint32_t below = uint32_t(__builtin_popcountll(__ballot(probe < len && get(lo + probe) < x)));
      lo += below * step;
      len = step == 1 ? 0 : below == 64 ? 0 : min(step - 1, len - min(len, below * step));
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
  w.first = s.sequences < 64 ? 0 : s.lower(token);  // a short list is seen whole
  w.entry = s.get(w.first + threadIdx.x % 64);
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
      const bool begins = next > at, ends = uniform(s.get(next)) == t0 + k + 1;
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

// The buffers of one worker, at the lane's first channel.
struct Columns {
  uint64_t gate, input, states, dstates, dgate, dinput;  // rows
  uint64_t begin, end;  // fp32 rows of the sequences: what their walk starts from, and what it leaves (0: not there)
  uint64_t before;      // gradient: the states before the sequences
};

template <bool BF16, int C, bool BACK>
struct Walk {
  static constexpr int ES = BF16 ? 2 : 4;
  struct Rows {
    Raw<BF16, C> gate[kSteps], input[kSteps];
    Raw<BF16, C> prior[BACK ? kSteps : 1], ds[BACK ? kSteps : 1];
  };

  // The rows of tokens t0 to t0 + kSteps - 1; of those from `stop` on, the last one before it.  (MAPS: only what the maps are made of.)
  template <bool MAPS>
  static __device__ __forceinline__ void load(const RecurrenceArgs& r, const Columns& q, uint32_t t0, uint32_t stop, Rows& x) {
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const uint64_t t = min(t0 + k, stop - 1);
      x.gate[k] = load_raw<BF16, C>(q.gate + t * r.pitch * ES);
      if constexpr (!BACK || !MAPS) x.input[k] = load_raw<BF16, C>(q.input + t * r.pitch * ES);
      if constexpr (BACK) {
        x.ds[k] = load_raw<BF16, C>(q.dstates + t * r.states_pitch * ES);
        if constexpr (!MAPS) x.prior[k] = load_raw<BF16, C>(q.states + (t ? t - 1 : 0) * r.states_pitch * ES);
      }
    }
  }

  // What a sequence's walk starts from.
  static __device__ __forceinline__ void begin(const RecurrenceArgs& r, uint64_t at, uint32_t sequence, float* v) {
#pragma unroll
    for (int c = 0; c < C; ++c) v[c] = 0.0f;
    if (at) {
      const CARAMEL_GLOBAL float* const row =
          reinterpret_cast<const CARAMEL_GLOBAL float*>(at + uint64_t(sequence) * r.channels * 4);
#pragma unroll
      for (int c = 0; c < C; ++c) v[c] = row[c];
    }
  }
  static __device__ __forceinline__ void leave(const RecurrenceArgs& r, uint64_t at, uint32_t sequence, const float* v) {
    if (!at) return;
    CARAMEL_GLOBAL float* const row = reinterpret_cast<CARAMEL_GLOBAL float*>(at + uint64_t(sequence) * r.channels * 4);
#pragma unroll
    for (int c = 0; c < C; ++c) row[c] = v[c];
  }
};

// The tokens of a worker that belong to some sequence
struct Range {
  uint32_t lo, hi;
};

template <bool BF16, int C>
__device__ __forceinline__ Columns columns(const RecurrenceArgs& r, uint32_t w, uint32_t ch, bool back) {
  constexpr int ES = BF16 ? 2 : 4;
  Columns q{};
  auto at = [&](int which, uint32_t es) { return r.w.at[which][w] ? r.w.at[which][w] + uint64_t(ch) * es : 0; };
  q.gate = at(kRecGate, ES);
  q.input = at(kRecInput, ES);
  q.states = at(kRecStates, ES);
  q.before = at(kRecBefore, 4);
  if (back) {
    q.dstates = at(kRecDstates, ES);
    q.dgate = at(kRecDgate, ES);
    q.dinput = at(kRecDinput, ES);
    q.begin = at(kRecDafter, 4);
    q.end = at(kRecDbefore, 4);
  } else {
    q.begin = q.before;
    q.end = at(kRecAfter, 4);
  }
  return q;
}

// MAPS: the parts' maps, left in the workspace; else: the walk itself.  Parts are `span` tokens, a multiple of the tile.
// blockIdx: x channels, y part, z worker.
template <bool BF16, int C, bool BACK, bool MAPS>
__global__ void __launch_bounds__(kLanes) k_walk_tokens(RecurrenceArgs r, uint32_t span, uint32_t parts) {
  using W = Walk<BF16, C, BACK>;
  constexpr int ES = BF16 ? 2 : 4;
  __shared__ float maps[2][kWalkWaves][2][C][64];
  __shared__ uint32_t cuts[2][kWalkWaves];
  const uint32_t w = blockIdx.z, n = r.w.tokens[w], part = blockIdx.y;
  const uint32_t lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
  uint32_t lo = part * span;
  if (lo >= n) return;
  uint32_t hi = min(lo + span, n);
  const Starts starts{r.w.at[kRecStarts][w], r.w.more[w], n, r.starts64};
  // the last lanes take the last C channels once more: equal values go to equal places
  const uint32_t ch = min((blockIdx.x * 64 + lane) * C, r.channels - C);
  const Columns q = columns<BF16, C>(r, w, ch, BACK);
  const uint32_t none_before = uniform(starts.get(0)), none_behind = uniform(starts.get(starts.sequences));

  // the sequence that goes on across the part's border, from the side the walk comes from
  const uint32_t border = BACK ? hi : lo;
  uint32_t from = 0, to = 0;  // parts whose maps lead up to this one
  {
    const uint32_t next = starts.lower(border);                      // the first start at or behind the border
    const bool goes_on = uniform(starts.get(next)) != border && border > none_before && border < none_behind && next > 0;
    if constexpr (MAPS) {
      // the other border: what leaves the part there
      const uint32_t out = BACK ? lo : hi;
      const uint32_t after = starts.lower(out);
      const bool leaves = uniform(starts.get(after)) != out && out > none_before && out < none_behind && after > 0;
      if (!leaves) return;
      const uint32_t cut = uniform(starts.get(BACK ? after : after - 1));
      if constexpr (BACK) hi = min(hi, max(cut, lo + 1));
      else lo = max(lo, min(cut, hi - 1) / kTile * kTile);
    } else if (goes_on) {
      const uint32_t cut = uniform(starts.get(BACK ? next : next - 1));
      if constexpr (BACK) {
        from = part + 1;
        to = min((max(cut, 1u) - 1) / span + 1, parts);
      } else {
        from = cut / span;
        to = part;
      }
    }
  }
  float state[C];
#pragma unroll
  for (int c = 0; c < C; ++c) state[c] = 0.0f;
  if constexpr (!MAPS) {
    const uint64_t stride = uint64_t(r.channels) * 2 * 4;  // bytes of a part's maps
    const uint64_t mine = reinterpret_cast<uint64_t>(r.ws) + uint64_t(w) * parts * stride + uint64_t(ch) * 4;
    for (uint32_t k = from; k < to; ++k) {
      const uint64_t at = mine + uint64_t(BACK ? to - 1 - (k - from) : k) * stride;
      const CARAMEL_GLOBAL float* const A = reinterpret_cast<const CARAMEL_GLOBAL float*>(at);
      const CARAMEL_GLOBAL float* const B = reinterpret_cast<const CARAMEL_GLOBAL float*>(at + uint64_t(r.channels) * 4);
#pragma unroll
      for (int c = 0; c < C; ++c) state[c] = k == from ? B[c] : __builtin_fmaf(A[c], state[c], B[c]);
    }
    // sequences without tokens leave what they start from
    if (q.end) {
      for (uint32_t s0 = (part * kWalkWaves + wave) * 64; s0 < starts.sequences; s0 += parts * kWalkWaves * 64) {
        const uint32_t s = s0 + lane;
        uint64_t empty = __ballot(s < starts.sequences && starts.get(s) >= starts.get(s + 1));
        while (empty) {
          const uint32_t one = s0 + uint32_t(__builtin_ctzll(empty));
          float v[C];
          W::begin(r, q.begin, one, v);
          W::leave(r, q.end, one, v);
          empty &= empty - 1;
        }
      }
    }
  }
  float all_a[C], all_b[C];  // MAPS: the part's map so far
  bool any_cut = false;
#pragma unroll
  for (int c = 0; c < C; ++c) all_a[c] = 1.0f, all_b[c] = 0.0f;

  const uint32_t tiles = (hi - lo + kTile - 1) / kTile;
  const bool whole_list = starts.sequences < 64;
  Window view = window(starts, 0);  // the list, where it is short
  for (uint32_t i = 0; i < tiles; ++i) {
    // the wavefronts' tokens follow each other the way the walk goes
    const uint32_t tile = lo + (BACK ? tiles - 1 - i : i) * kTile;
    const uint32_t t0 = tile + (BACK ? kWalkWaves - 1 - wave : wave) * kSteps;
    const uint32_t count = t0 < hi ? min(hi - t0, uint32_t(kSteps)) : 0;
    typename W::Rows x;
    W::template load<MAPS>(r, q, t0, hi, x);
    if (!whole_list) view = window(starts, t0);
    const Marks mark = marks(starts, view, t0);

    // this wavefront's map
    float a[kSteps][C], b[kSteps][C], A[C], B[C], first[kSteps][C];
    bool cut = false;
#pragma unroll
    for (int c = 0; c < C; ++c) A[c] = 1.0f, B[c] = 0.0f;
    if (mark.any) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const uint32_t s = BACK ? mark.ends[k] : mark.begins[k];
#pragma unroll
        for (int c = 0; c < C; ++c) first[k][c] = 0.0f;
        if (s != kNone && uint32_t(k) < count) W::begin(r, q.begin, s, first[k]);
      }
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int k = BACK ? kSteps - 1 - j : j;
      const uint32_t t = t0 + k;
#pragma unroll
      for (int c = 0; c < C; ++c) gates<BF16>(widen<BF16, C>(x.gate[k], c), &a[k][c], &b[k][c]);
      if (uint32_t(k) >= count || t < none_before || t >= none_behind) continue;
      const bool begins = mark.any && (BACK ? mark.ends[k] : mark.begins[k]) != kNone;
      if (begins) {
        cut = true;
#pragma unroll
        for (int c = 0; c < C; ++c) B[c] = first[k][c];
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if constexpr (BACK) B[c] = a[k][c] * (widen<BF16, C>(x.ds[k], c) + B[c]);
        else B[c] = __builtin_fmaf(a[k][c], B[c], b[k][c] * widen<BF16, C>(x.input[k], c));
        A[c] *= a[k][c];
      }
    }
    const uint32_t turn = i % 2;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      maps[turn][wave][0][c][lane] = A[c];
      maps[turn][wave][1][c][lane] = B[c];
    }
    if (lane == 0) cuts[turn][wave] = cut;
    __syncthreads();
    float s[C];  // the state this wavefront's tokens start from
#pragma unroll
    for (int c = 0; c < C; ++c) s[c] = state[c];
#pragma unroll
    for (int v = 0; v < kWalkWaves; ++v) {
      const bool from_here = uniform(cuts[turn][v]) != 0;
      any_cut = any_cut || from_here;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (uint32_t(v) == wave) s[c] = state[c];
        const float mA = maps[turn][v][0][c][lane], mB = maps[turn][v][1][c][lane];
        if constexpr (MAPS) {
          all_a[c] *= mA;
          all_b[c] = from_here ? mB : __builtin_fmaf(mA, all_b[c], mB);
        } else {
          state[c] = from_here ? mB : __builtin_fmaf(mA, state[c], mB);
        }
      }
    }
    if constexpr (MAPS) continue;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int k = BACK ? kSteps - 1 - j : j;
      const uint32_t t = t0 + k;
      if (uint32_t(k) >= count || t < none_before || t >= none_behind) continue;
      const bool begins = mark.any && (BACK ? mark.ends[k] : mark.begins[k]) != kNone;
      if (begins) {
#pragma unroll
        for (int c = 0; c < C; ++c) s[c] = first[k][c];
      }
      const uint32_t over = !mark.any ? kNone : BACK ? mark.begins[k] : mark.ends[k];
      if constexpr (BACK) {
        float prior[C], du[C], dg[C];
#pragma unroll
        for (int c = 0; c < C; ++c) prior[c] = widen<BF16, C>(x.prior[k], c);
        if (over != kNone) W::begin(r, q.before, over, prior);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float e = widen<BF16, C>(x.ds[k], c) + s[c];
          du[c] = b[k][c] * e;
          dg[c] = (a[k][c] * du[c]) * (prior[c] - widen<BF16, C>(x.input[k], c));
          s[c] = a[k][c] * e;
        }
        store_channels<BF16, C>(q.dinput + t * r.pitch * ES, du);
        store_channels<BF16, C>(q.dgate + t * r.pitch * ES, dg);
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c) s[c] = __builtin_fmaf(a[k][c], s[c], b[k][c] * widen<BF16, C>(x.input[k], c));
        store_channels<BF16, C>(q.states + t * r.states_pitch * ES, s);
      }
      if (over != kNone) W::leave(r, q.end, over, s);
    }
  }
  if constexpr (MAPS) {
    if (wave) return;
    const uint64_t at = reinterpret_cast<uint64_t>(r.ws) + (uint64_t(w) * parts + part) * r.channels * 2 * 4 + uint64_t(ch) * 4;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      reinterpret_cast<CARAMEL_GLOBAL float*>(at)[c] = any_cut ? 0.0f : all_a[c];
      reinterpret_cast<CARAMEL_GLOBAL float*>(at + uint64_t(r.channels) * 4)[c] = all_b[c];
    }
  }
}

constexpr uint32_t kWalkGroups = 512;   // workgroups of a launch that parts are made for
constexpr uint32_t kShortest = 2 * kTile;  // tokens of a part, at least

uint32_t slabs(uint32_t channels) { return (channels + 127) / 128; }

uint32_t walk_parts(uint32_t world, uint32_t channels, uint32_t max_tokens) {
  const uint64_t there = uint64_t(std::min(world, kGroup)) * slabs(channels);
  const uint32_t most = uint32_t((kWalkGroups + there - 1) / there);
  return std::max(1u, std::min(most, max_tokens / kShortest));
}

template <bool BF16, int C, bool BACK>
hipError_t launch_walk(const RecurrenceArgs& a, uint32_t span, uint32_t parts, hipStream_t s) {
  const dim3 grid((a.channels + 64 * C - 1) / (64 * C), parts, a.world);
  if (parts > 1) {
    hipLaunchKernelGGL((k_walk_tokens<BF16, C, BACK, true>), grid, dim3(kLanes), 0, s, a, span, parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_walk_tokens<BF16, C, BACK, false>), grid, dim3(kLanes), 0, s, a, span, parts);
  return hipGetLastError();
}

template <bool BACK>
hipError_t launch_any(const RecurrenceArgs& args, const AllBuffers<kRecBuffers>& v, hipStream_t s) {
  if (args.max_tokens == 0) return hipSuccess;
  const uint32_t most = walk_parts(args.all, args.channels, args.max_tokens);
  const uint32_t span = ((args.max_tokens + most - 1) / most + kTile - 1) / kTile * kTile;
  const uint32_t parts = (args.max_tokens + span - 1) / span;  // no more than `most`
  return in_groups(args, v, [&](RecurrenceArgs a, uint32_t g) {
    a.ws += uint64_t(g) * parts * a.channels * 2 * 4;
    if (a.channels == 1) return a.bf16 ? launch_walk<true, 1, BACK>(a, span, parts, s) : launch_walk<false, 1, BACK>(a, span, parts, s);
    return a.bf16 ? launch_walk<true, 2, BACK>(a, span, parts, s) : launch_walk<false, 2, BACK>(a, span, parts, s);
  });
}

}  // namespace

uint64_t recurrence_workspace_bytes(uint32_t world, uint32_t channels, uint32_t max_tokens) {
  const uint32_t parts = walk_parts(world, channels, max_tokens);
  return parts == 1 ? 0 : uint64_t(world) * parts * channels * 2 * 4;
}

hipError_t launch_recurrence(const RecurrenceArgs& args, const AllBuffers<kRecBuffers>& v, hipStream_t s) {
  return launch_any<false>(args, v, s);
}

hipError_t launch_recurrence_gradient(const RecurrenceArgs& args, const AllBuffers<kRecBuffers>& v, hipStream_t s) {
  return launch_any<true>(args, v, s);
}

}  // namespace caramel
