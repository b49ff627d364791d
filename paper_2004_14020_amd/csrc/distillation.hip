// Distillation from a teacher's best logits, with labels beside them: the loss of every token and the gradient of its logits.
//
//   P = softmax of the teacher's entries over the temperature T, Q = softmax(z / T), q = softmax(z)
//   loss = soft sum_k P_k (ln P_k - ln Q_id(k)) + hard (- ln q_label)
//   dz_j = scale (soft / T (Q_j - sum of P_k with id(k) = j) + hard (q_j - [j = label]))
//
// ln P_k = (t_k - max t) / T - ln sum: no logarithm but of sums, which is taken in 64 bits, as the few products of the loss are.
// All exponentials are 2^(d log2(e) / T) of the distance d <= 0 to the row's largest logit.  Where T is 1, Q and q are one; where it
// is 2 or 4, an exponential of q is that of Q squared, once or twice.
//
// A row is read once: a workgroup holds it in registers, as numbers, then as distances or exponentials.  What does not fit (more than
// 65536 logits) is read again for the gradient.  The gradient is written as if there were no teacher; behind a barrier the few logits
// that the teacher or the label names are written once more.  With few rows, each is cut into parts: one launch leaves every part's
// largest logit and sums, and the next one joins them.
#include <algorithm>

#include "layers.hpp"
#include "rows.hpp"

namespace caramel {
namespace {

enum { kOne, kPower, kTwo };             // exponentials: one for Q and q; those of q are powers of Q's; two
enum { kWhole, kMeasure, kWrite };       // a row at once; a part's largest logit and sums; the gradient of a part

constexpr int kTop = int(kDistillationTop), kEntries = kTop + 1;  // of the teacher; and the label
constexpr uint32_t kNone = 0xFFFFFFFFu;
constexpr uint32_t kGridRows = 1u << 20;  // along x: a grid has less than 2^32 lanes in a direction

struct Sums {
  float largest, warm, cold;  // warm: of 2^(d log2(e) / T); cold: of 2^(d log2(e))
};

__device__ __forceinline__ uint32_t read_id(uint64_t at, uint64_t i, bool wide, uint32_t vocab) {
  const uint64_t id = wide ? reinterpret_cast<const CARAMEL_GLOBAL uint64_t*>(at)[i]
                           : reinterpret_cast<const CARAMEL_GLOBAL uint32_t*>(at)[i];
  return id < vocab ? uint32_t(id) : kNone;  // a negative id is a huge one
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d; d /= 2) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// The exponential of q from that of Q (T = 2 or 4)
__device__ __forceinline__ float power(float e, bool twice) {
  e *= e;
  return twice ? e * e : e;
}

// LANES lanes hold HELD logits each.
template <bool BF16, int KIND, int PHASE, int LANES, int HELD>
__global__ void __launch_bounds__(LANES) k_distillation(DistillationArgs a) {
  constexpr int N = kPiece<BF16>, ES = BF16 ? 2 : 4, V = HELD / N, kWaves = LANES / 64;
  constexpr bool kKeep = KIND != kTwo;  // exponentials stay in registers; else distances
  __shared__ float waves[kWaves][3];
  __shared__ uint32_t ids[kEntries];
  __shared__ float logit[kEntries], weight[kEntries];
  __shared__ double taught;             // the loss without the logarithms of the sums over the vocabulary, and whose it has
  __shared__ uint32_t terms;            // bit 0: the teacher's, bit 1: the label's
  const uint32_t w = blockIdx.z, row = blockIdx.x + (PHASE == kWhole ? blockIdx.y * kGridRows : 0), n = a.w.tokens[w];
  if (row >= n) return;
  const uint32_t lane = threadIdx.x, wave = uniform(threadIdx.x / 64);
  const uint64_t z = a.w.at[kDistLogits][w] + uint64_t(row) * a.pitch * ES;
  // this workgroup's part of the row: whole pieces, and what is left behind the last one
  const uint32_t whole = a.vocab / N, lo = PHASE == kWhole ? 0 : min(blockIdx.y * a.part, whole);
  const uint32_t hi = PHASE == kWhole ? whole : min(lo + a.part, whole);
  const bool last = PHASE == kWhole || blockIdx.y + 1 == a.parts, tells = PHASE == kWhole || blockIdx.y == 0;
  const uint32_t tail = last ? a.vocab - whole * N : 0;
  float* const ws = reinterpret_cast<float*>(a.ws) + (uint64_t(w) * a.max_tokens + row) * a.stride;

  // all loads of the row first
  float x[V][N], odd = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const uint32_t p = lo + i * LANES + lane;
#pragma unroll
    for (int j = 0; j < N; ++j) x[i][j] = -__builtin_inff();
    if (lo + i * LANES < hi && p < hi) load_elems<BF16, N>(z + uint64_t(p) * N * ES, x[i]);
  }
  if (lane < tail) load_elems<BF16, 1>(z + (uint64_t(whole) * N + lane) * ES, &odd);

  // the teacher and the label: the first wavefront, four entries a lane
  constexpr int kEach = kTop / 64;
  if constexpr (PHASE == kMeasure) {
    if (tells && wave == 0) {
#pragma unroll
      for (int i = 0; i <= kEach; ++i) {
        const uint32_t k = i * 64 + lane;
        if (k > a.top) continue;
        uint32_t id = kNone;
        if (k < a.top) id = read_id(a.w.at[kDistIds][w], uint64_t(row) * a.top + k, a.ids64, a.vocab);
        else if (a.has_labels) id = read_id(a.w.at[kDistLabels][w], row, a.ids64, a.vocab);
        float v = 0.0f;
        if (id != kNone) load_elems<BF16, 1>(z + uint64_t(id) * ES, &v);
        ws[3 * a.parts + k] = v;
      }
    }
  } else if (wave == 0) {
    float t[kEach], v[kEach];
    uint32_t id[kEach];
    float most = -__builtin_inff();
    bool bad = false, any = false;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t k = i * 64 + lane;
      id[i] = kNone;
      t[i] = -__builtin_inff();
      v[i] = 0.0f;
      if (uint32_t(i) * 64 >= a.top || k >= a.top) continue;
      id[i] = read_id(a.w.at[kDistIds][w], uint64_t(row) * a.top + k, a.ids64, a.vocab);
      const uint64_t at = a.w.at[kDistTeacher][w] + (uint64_t(row) * a.top + k) * (a.teacher_bf16 ? 2 : 4);
      if (a.teacher_bf16) load_elems<true, 1>(at, &t[i]);
      else load_elems<false, 1>(at, &t[i]);
      if (id[i] == kNone) t[i] = -__builtin_inff();
    }
    uint32_t label = kNone;
    if (a.has_labels) label = uniform(read_id(a.w.at[kDistLabels][w], row, a.ids64, a.vocab));
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t k = i * 64 + lane;
      if (id[i] != kNone) {
        if constexpr (PHASE == kWhole) load_elems<BF16, 1>(z + uint64_t(id[i]) * ES, &v[i]);
        else v[i] = ws[3 * a.parts + k];
      }
      most = fmaxf(most, t[i]);
      bad = bad || t[i] != t[i];
      any = any || t[i] > -__builtin_inff();
    }
    float label_logit = 0.0f;
    if (label != kNone) {
      if constexpr (PHASE == kWhole) load_elems<BF16, 1>(z + uint64_t(label) * ES, &label_logit);
      else label_logit = ws[3 * a.parts + a.top];
    }
    most = wave_max(most);
    const bool has_teacher = a.soft > 0.0f && (__ballot(any) || __ballot(bad));
    float p[kEach], total = 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      p[i] = 0.0f;
      if (id[i] != kNone && has_teacher) p[i] = __builtin_amdgcn_exp2f((t[i] - most) * a.warm_rate);
      if (t[i] == -__builtin_inff()) p[i] = 0.0f;
      total += p[i];
    }
    total = wave_sum(total);
    double part = 0.0;  // sum of P (ln P - z / T), with ln P but for the sum's logarithm
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t k = i * 64 + lane;
      p[i] /= total;
      if (p[i] != 0.0f && has_teacher) part += double(p[i]) * ((double(t[i]) - double(most)) - double(v[i])) * a.inverse;
      if (k < a.top) {
        ids[k] = has_teacher ? id[i] : kNone;
        logit[k] = v[i];
        weight[k] = a.soft * float(a.inverse) * p[i];
      }
    }
    part = wave_sum(part);
    if (lane == 0) {
      const bool has_label = label != kNone;
      ids[a.top] = has_label ? label : kNone;
      logit[a.top] = label_logit;
      weight[a.top] = a.hard;
      terms = (has_teacher ? 1u : 0u) | (has_label ? 2u : 0u);
      taught = has_teacher ? part - log(double(total)) : 0.0;
    }
  }

  // the largest logit
  Sums s{-3.402823466e38f, 0.0f, 0.0f};
  if constexpr (PHASE != kWrite) {
    // pieces that are not held: largest logit and sums together
    for (uint32_t p = lo + V * LANES + lane; p < hi; p += LANES) {
      float y[N], m = s.largest;
      load_elems<BF16, N>(z + uint64_t(p) * N * ES, y);
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, y[j]);
      const float d = s.largest - m;
      s.largest = m;
      s.warm *= __builtin_amdgcn_exp2f(d * a.warm_rate);
      if constexpr (KIND != kOne) s.cold *= __builtin_amdgcn_exp2f(d * a.cold_rate);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float e = __builtin_amdgcn_exp2f((y[j] - m) * a.warm_rate);
        s.warm += e;
        if constexpr (KIND == kPower) s.cold += power(e, a.twice);
        if constexpr (KIND == kTwo) s.cold += __builtin_amdgcn_exp2f((y[j] - m) * a.cold_rate);
      }
    }
    float m = fmaxf(s.largest, odd);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, x[i][j]);
    m = wave_max(m);
    if (lane % 64 == 0) waves[wave][0] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWaves; ++k) m = fmaxf(m, waves[k][0]);
    const float d = s.largest - m;
    s.largest = m;
    s.warm *= __builtin_amdgcn_exp2f(d * a.warm_rate);
    if constexpr (KIND != kOne) s.cold *= __builtin_amdgcn_exp2f(d * a.cold_rate);
  } else {
    __syncthreads();
    // the parts' sums, joined by every wavefront for itself
    Sums mine{-3.402823466e38f, 0.0f, 0.0f};
    for (uint32_t k = lane % 64; k < a.parts; k += 64) {
      const Sums o{ws[3 * k], ws[3 * k + 1], ws[3 * k + 2]};
      const float m = fmaxf(mine.largest, o.largest);
      const float f = __builtin_amdgcn_exp2f((mine.largest - m) * a.warm_rate), g = __builtin_amdgcn_exp2f((o.largest - m) * a.warm_rate);
      const float h = __builtin_amdgcn_exp2f((mine.largest - m) * a.cold_rate), i = __builtin_amdgcn_exp2f((o.largest - m) * a.cold_rate);
      mine = {m, mine.warm * f + o.warm * g, mine.cold * h + o.cold * i};
    }
    s.largest = wave_max(mine.largest);
    const float d = mine.largest - s.largest;
    s.warm = wave_sum(mine.warm * __builtin_amdgcn_exp2f(d * a.warm_rate));
    s.cold = wave_sum(mine.cold * __builtin_amdgcn_exp2f(d * a.cold_rate));
  }

  // distances and exponentials of what is held, and their sums
  float odd_warm = 0.0f, odd_cold = 0.0f;
#pragma unroll
  for (int i = 0; i <= V; ++i) {
    if (i < V && lo + i * LANES >= hi) continue;
#pragma unroll
    for (int j = 0; j < (i < V ? N : 1); ++j) {
      const float d = (i < V ? x[i][j] : odd) - s.largest;
      float warm = 0.0f, cold = 0.0f;
      if (PHASE != kWrite || kKeep || i == V) {
        warm = __builtin_amdgcn_exp2f(d * a.warm_rate);
        if constexpr (KIND == kPower) cold = power(warm, a.twice);
        if constexpr (KIND == kTwo) cold = __builtin_amdgcn_exp2f(d * a.cold_rate);
      }
      if constexpr (PHASE != kWrite) {
        s.warm += warm;
        s.cold += cold;
      }
      if (i < V) x[i][j] = kKeep ? warm : d;
      else odd_warm = warm, odd_cold = cold;
    }
  }
  if constexpr (PHASE != kWrite) {
    const float warm = wave_sum(s.warm), cold = KIND != kOne ? wave_sum(s.cold) : 0.0f;
    if (lane % 64 == 0) waves[wave][1] = warm, waves[wave][2] = cold;
    __syncthreads();
    s.warm = s.cold = 0.0f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      s.warm += waves[k][1];
      s.cold += waves[k][2];
    }
    if constexpr (PHASE == kMeasure) {
      if (lane == 0) {
        ws[3 * blockIdx.y] = s.largest;
        ws[3 * blockIdx.y + 1] = s.warm;
        ws[3 * blockIdx.y + 2] = s.cold;
      }
      return;
    }
  }
  if constexpr (PHASE != kMeasure) {
    if constexpr (KIND == kOne) s.cold = s.warm;
    const bool has_teacher = uniform(terms) & 1, has_label = uniform(terms) & 2;
    if (lane == 0 && tells) {
      double loss = 0.0;
      if (has_teacher) loss += double(a.soft) * (taught + double(s.largest) * a.inverse + log(double(s.warm)));
      if (has_label) loss += double(a.hard) * (log(double(s.cold)) - (double(logit[a.top]) - double(s.largest)));
      reinterpret_cast<CARAMEL_GLOBAL float*>(a.w.at[kDistLoss][w])[row] = float(loss);
    }
    if (!a.gradient) return;
    const uint64_t out = a.w.at[kDistGradient][w] + uint64_t(row) * a.gradient_pitch * ES;
    const float warm = has_teacher ? a.soft * float(a.inverse) / s.warm : 0.0f, cold = has_label ? a.hard / s.cold : 0.0f;
    const bool none = !has_teacher && !has_label;  // zeros, whatever the logits are
    const float kw = a.scale * (KIND == kOne ? warm + cold : warm), kc = a.scale * cold;
    auto gradient = [&](float v) {  // of what is held
      float g;
      if constexpr (KIND == kOne) g = kw * v;
      else if constexpr (KIND == kPower) g = __builtin_fmaf(kw, v, kc * power(v, a.twice));
      else g = __builtin_fmaf(kw, __builtin_amdgcn_exp2f(v * a.warm_rate), kc * __builtin_amdgcn_exp2f(v * a.cold_rate));
      return none ? 0.0f : g;
    };
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t p = lo + i * LANES + lane;
      if (lo + i * LANES >= hi || p >= hi) continue;
#pragma unroll
      for (int j = 0; j < N; ++j) x[i][j] = gradient(x[i][j]);
      store_elems<BF16, N>(out + uint64_t(p) * N * ES, x[i]);
    }
    for (uint32_t p = lo + V * LANES + lane; p < hi; p += LANES) {
      float y[N];
      load_elems<BF16, N>(z + uint64_t(p) * N * ES, y);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float d = y[j] - s.largest;
        y[j] = gradient(kKeep ? __builtin_amdgcn_exp2f(d * a.warm_rate) : d);
      }
      store_elems<BF16, N>(out + uint64_t(p) * N * ES, y);
    }
    if (lane < tail) {
      float g = KIND == kOne ? kw * odd_warm : __builtin_fmaf(kw, odd_warm, kc * odd_cold);
      if (none) g = 0.0f;
      store_elems<BF16, 1>(out + (uint64_t(whole) * N + lane) * ES, &g);
    }
    __syncthreads();
    // the entries' own logits, each written by its first entry
    for (uint32_t k = lane; k <= a.top; k += LANES) {
      const uint32_t id = ids[k];
      if (id == kNone || id / N < lo || (id / N >= hi && !last)) continue;
      float less = 0.0f;
      bool first = true;
      for (uint32_t i = 0; i <= a.top; ++i) {
        const bool same = ids[i] == id;
        less += same ? weight[i] : 0.0f;
        first = first && !(same && i < k);
      }
      if (!first) continue;
      const float d = logit[k] - s.largest, e = __builtin_amdgcn_exp2f(d * a.warm_rate);
      float g = warm * e - less;
      if constexpr (KIND == kOne) g = (warm + cold) * e - less;
      if constexpr (KIND == kPower) g = __builtin_fmaf(cold, power(e, a.twice), warm * e) - less;
      if constexpr (KIND == kTwo) g = __builtin_fmaf(cold, __builtin_amdgcn_exp2f(d * a.cold_rate), warm * e) - less;
      g *= a.scale;
      store_elems<BF16, 1>(out + uint64_t(id) * ES, &g);
    }
  }
}

// Rows in parts: so many of them at most, and parts that make about so many workgroups.
constexpr uint32_t kFewRows = 192, kPartGroups = 512;
constexpr int kPartLanes = 256, kPartHeld = 16;

uint32_t parts_of(uint64_t rows, uint32_t vocab) {
  const uint32_t most = vocab / (kPartLanes * kPartHeld);
  if (rows == 0 || rows > kFewRows || most < 2) return 1;
  return uint32_t(std::min<uint64_t>(most, (kPartGroups + rows - 1) / rows));
}

template <bool BF16, int KIND>
hipError_t launch(const DistillationArgs& a, hipStream_t s) {
  if (a.parts > 1) {
    const dim3 grid(a.max_tokens, a.parts, a.world);
    hipLaunchKernelGGL((k_distillation<BF16, KIND, kMeasure, kPartLanes, kPartHeld>), grid, dim3(kPartLanes), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 write(a.max_tokens, a.gradient ? a.parts : 1, a.world);
    hipLaunchKernelGGL((k_distillation<BF16, KIND, kWrite, kPartLanes, kPartHeld>), write, dim3(kPartLanes), 0, s, a);
    return hipGetLastError();
  }
  const dim3 grid(std::min(a.max_tokens, kGridRows), (a.max_tokens + kGridRows - 1) / kGridRows, a.world);
  if (a.vocab <= 256 * 32) {
    hipLaunchKernelGGL((k_distillation<BF16, KIND, kWhole, 256, 32>), grid, dim3(256), 0, s, a);
  } else if (a.vocab <= 1024 * 32) {
    hipLaunchKernelGGL((k_distillation<BF16, KIND, kWhole, 1024, 32>), grid, dim3(1024), 0, s, a);
  } else {
    hipLaunchKernelGGL((k_distillation<BF16, KIND, kWhole, 1024, 64>), grid, dim3(1024), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace

// Of fewer rows, each may have more parts; all of them together, no more than this.
uint64_t distillation_workspace_bytes(uint32_t world, uint32_t vocab, uint32_t top, uint32_t max_tokens) {
  const uint64_t rows = std::min<uint64_t>(uint64_t(world) * max_tokens, kFewRows);
  if (rows == 0 || parts_of(1, vocab) == 1) return 0;
  return (3 * (kPartGroups + rows) + rows * (top + 1)) * 4;
}

hipError_t launch_distillation(const DistillationArgs& args, const AllBuffers<kDistBuffers>& v, hipStream_t s) {
  if (args.max_tokens == 0) return hipSuccess;
  DistillationArgs all = args;
  all.parts = parts_of(uint64_t(args.all) * args.max_tokens, args.vocab);
  const uint32_t pieces = args.vocab / (args.bf16 ? 8 : 4);
  all.part = (pieces + all.parts - 1) / all.parts;
  all.stride = 3 * all.parts + args.top + 1;
  const bool both = args.soft > 0.0f && args.has_labels;
  const bool squares = args.temperature == 2.0f || args.temperature == 4.0f;
  const int kind = !both || args.temperature == 1.0f ? kOne : squares ? kPower : kTwo;
  const double log2e = 1.4426950408889634;
  // without a teacher's part, all is at temperature 1
  all.warm_rate = float(log2e / (args.soft > 0.0f ? double(args.temperature) : 1.0));
  all.cold_rate = float(log2e);
  all.inverse = 1.0 / double(args.temperature);
  all.twice = args.temperature == 4.0f;
  return in_groups(all, v, [&](DistillationArgs a, uint32_t g) {
    a.ws += uint64_t(g) * a.max_tokens * a.stride * 4;
    if (a.bf16) return kind == kOne ? launch<true, kOne>(a, s) : kind == kPower ? launch<true, kPower>(a, s) : launch<true, kTwo>(a, s);
    return kind == kOne ? launch<false, kOne>(a, s) : kind == kPower ? launch<false, kPower>(a, s) : launch<false, kTwo>(a, s);
  });
}

}  // namespace caramel
