// Distillation from a teacher's best logits, with labels beside them: the loss of every token and the gradient of its logits.
//
//   P = softmax of the teacher's entries over the temperature T, Q = softmax(z / T), q = softmax(z)
//   loss = soft sum_k P_k (ln P_k - ln Q_id(k)) + hard (- ln q_label)
//   dz_j = scale (soft / T (Q_j - sum of P_k with id(k) = j) + hard (q_j - [j = label]))
//
// ln P_k = (t_k - max t) / T - ln sum: no logarithm but of sums, which are fp32, as the exponentials are.  What else the loss is made of is added up
// in 64 bits: distances between logits, never logits, weighted by the teacher's exponentials over their sum, so that the weights add up to 1 and
// nothing hangs on what all logits have in common (with weights rounded to fp32, whose sum is off by 1e-7 or so, the loss was off by as much of the
// largest logit over T: by 0.1 next to logits of 10^6).
// All exponentials are 2^(d log2(e) / T) of the distance d <= 0 to the row's largest logit.  Where T is 1, Q and q are one; where it
// is 2 or 4, an exponential of q is that of Q squared, once or twice.
//
// A row is read once: a workgroup holds it in registers, as numbers, then as distances or exponentials, and a part of a long one in LDS.
// What does not fit (from 115200 bf16 or 130560 fp32 logits on) is read again for the gradient.  The gradient is written as if there were no
// teacher; behind a barrier the few logits that the teacher or the label names are written once more.  Where few rows do not fit registers, each
// is cut into parts: one launch leaves every part's largest logit and sums, and the next one joins them.
//
// Bound by memory and by how much of a workgroup's reading, computing and writing lies beside another's: 8 workers x 512 rows x 30522 bf16
// logits, T = 2 with labels, 106 us, 4.7 TB/s (a copy of 1 GiB: 6.08); the vector units issue in 52 % of that time.
#include <algorithm>

#include "layers.hpp"
#include "rows.hpp"

namespace caramel {
namespace {

enum { kOne, kSquare, kFourth, kTwo };   // exponentials: one for Q and q; those of q are Q's squared, or squared twice; two
enum { kWhole, kMeasure, kWrite };       // a row at once; a part's largest logit and sums; the gradient of a part

constexpr int kTop = int(kDistillationTop), kEntries = kTop + 1;  // of the teacher; and the label
constexpr uint32_t kNone = 0xFFFFFFFFu;
constexpr uint32_t kGridRows = 1u << 20;  // along x: a grid has less than 2^32 lanes in a direction
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ uint64_t load_id(uint64_t at, uint64_t i, bool wide) {
  return wide ? reinterpret_cast<const CARAMEL_GLOBAL uint64_t*>(at)[i] : reinterpret_cast<const CARAMEL_GLOBAL uint32_t*>(at)[i];
}
__device__ __forceinline__ uint32_t known(uint64_t id, uint32_t vocab) { return id < vocab ? uint32_t(id) : kNone; }  // negative: huge

__device__ __forceinline__ float exp2(float v) { return __builtin_amdgcn_exp2f(v); }
// Also far below the smallest fp32 numbers; v is 0 or less, or NaN.
__device__ __forceinline__ double exp2_wide(float v) {
  const float whole = rintf(fmaxf(v, -1100.0f));
  return __builtin_amdgcn_ldexp(double(exp2(v - whole)), int(whole));
}

// The natural logarithm of a sum, whose exponent is taken apart: the rest is in [1/2, 1), and its logarithm off by less than 2^-23 (measured over
// all of these numbers: 1.54 * 2^-24).
__device__ __forceinline__ double ln(float v) {
  return double(__builtin_amdgcn_frexp_expf(v)) * 0.69314718055994531 + double(logf(__builtin_amdgcn_frexp_mantf(v)));
}

// What a row's teacher and label ask for: of entry k (the label: entry `top`) its id, the student's logit there, and what is taken
// from the gradient there; best: the largest logit that the teacher asks for; taught: the loss without the logarithms of sums over the
// vocabulary, as if best were the row's largest logit; terms: bit 0 the teacher's, bit 1 the label's.
struct Lesson {
  uint32_t id[kEntries];
  float logit[kEntries], weight[kEntries];
  uint32_t terms;
  float best;
  double taught;
};

// One wavefront's way to it: ask() begins all loads, learn() waits for them.
template <bool BF16>
struct Student {
  static constexpr int ES = BF16 ? 2 : 4, kEach = kTop / 64;  // entries of a lane
  float t[kEach], v[kEach], label_logit;
  uint32_t id[kEach], label;

  // What needs no id is asked for at once, by all lanes (those without an entry: the last one's).
  __device__ __forceinline__ void ask(const DistillationArgs& a, uint32_t w, uint32_t row, uint64_t z) {
    const uint32_t lane = threadIdx.x % 64;
    uint64_t asked[kEach], asked_label = ~uint64_t(0);
    const uint64_t first = uint64_t(row) * a.top;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      asked[i] = ~uint64_t(0);
      if (uint32_t(i) * 64 >= a.top) continue;
      const uint64_t k = first + min(i * 64 + lane, a.top - 1);
      asked[i] = load_id(a.w.at[kDistIds][w], k, a.ids64);
      if (a.teacher_bf16) load_elems<true, 1>(a.w.at[kDistTeacher][w] + k * 2, &t[i]);
      else load_elems<false, 1>(a.w.at[kDistTeacher][w] + k * 4, &t[i]);
    }
    if (a.has_labels) asked_label = load_id(a.w.at[kDistLabels][w], row, a.ids64);
    label = uniform(known(asked_label, a.vocab));
    load_elems<BF16, 1>(z + uint64_t(label != kNone ? label : 0) * ES, &label_logit);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      id[i] = i * 64 + lane < a.top ? known(asked[i], a.vocab) : kNone;
      if (uint32_t(i) * 64 >= a.top) continue;
      load_elems<BF16, 1>(z + uint64_t(id[i] != kNone ? id[i] : 0) * ES, &v[i]);
    }
  }

  __device__ __forceinline__ void learn(const DistillationArgs& a, Lesson& out) {
    const uint32_t lane = threadIdx.x % 64;
    float most = -__builtin_inff();
    bool bad = false, any = false;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (uint32_t(i) * 64 >= a.top) continue;
      if (id[i] == kNone) t[i] = -__builtin_inff();
      most = fmaxf(most, t[i]);
      bad = bad || t[i] != t[i];
      any = any || t[i] > -__builtin_inff();
    }
    most = wave_max(most);
    const bool has_teacher = a.soft > 0.0f && (__ballot(any) || __ballot(bad));
    float p[kEach], total = 0.0f, best = kLowest;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      p[i] = 0.0f;
      if (uint32_t(i) * 64 >= a.top) continue;
      const bool asks = has_teacher && t[i] != -__builtin_inff();
      if (asks) p[i] = exp2((t[i] - most) * a.warm_rate);
      total += p[i];
      best = fmaxf(best, asks ? v[i] : kLowest);
    }
    total = wave_sum(total);
    best = wave_max(best);
    // sums of the exponentials, and of their products with T (ln P - ln Q) but for the logarithms of sums; best is never -infinity, so a logit
    // of -infinity makes the loss infinite, not NaN.  A P that fp32 has no number for still counts: next to a masked logit, the type's lowest
    // number, 10^-38 of it is a loss of some units
    double part = 0.0, whole = 0.0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const uint32_t k = i * 64 + lane;
      if (uint32_t(i) * 64 >= a.top) continue;
      if (has_teacher && t[i] != -__builtin_inff()) {
        const double e = exp2_wide((t[i] - most) * a.warm_rate);
        if (e != 0.0) part += e * ((double(t[i]) - double(most)) - (double(v[i]) - double(best)));
        whole += e;
      }
      p[i] /= total;
      if (k < a.top) {
        out.id[k] = has_teacher ? id[i] : kNone;
        out.logit[k] = v[i];
        out.weight[k] = a.soft * float(a.inverse) * p[i];
      }
    }
    part = wave_sum(part);
    whole = wave_sum(whole);
    if (lane == 0) {
      out.id[a.top] = label;
      out.logit[a.top] = label_logit;
      out.weight[a.top] = a.hard;
      out.terms = (has_teacher ? 1u : 0u) | (label != kNone ? 2u : 0u);
      out.best = best;
      out.taught = has_teacher ? part / whole * a.inverse - ln(total) : 0.0;
    }
  }
};

// From which number exponents count: 2^(rate (z - base) - shift), where rate (z - base) - shift is one multiply-add.  Next to usual logits base
// is 0 and shift the rounded product of rate and the largest logit; `rest` is what the rounding left, a factor of 2^rest that all
// exponentials share.  Where the product is so large that the factor might overflow, the largest logit is subtracted first.
struct Origin {
  float base, warm_shift, cold_shift, warm_rest, cold_rest;
};
template <int KIND>
__device__ __forceinline__ Origin origin(const DistillationArgs& a, float largest, bool always) {
  const float rate = KIND == kTwo ? fmaxf(a.warm_rate, a.cold_rate) : a.warm_rate;
  const bool near = !always && fabsf(largest * rate) < 1048576.0f;
  const float m = near ? largest : 0.0f;
  Origin o;
  o.base = near ? 0.0f : largest;
  o.warm_shift = m * a.warm_rate;
  o.cold_shift = m * a.cold_rate;
  o.warm_rest = __builtin_fmaf(m, a.warm_rate, -o.warm_shift);
  // a power of Q's exponential has that power of its factor
  o.cold_rest = KIND == kSquare ? 2.0f * o.warm_rest : KIND == kFourth ? 4.0f * o.warm_rest
                : KIND == kOne ? o.warm_rest : __builtin_fmaf(m, a.cold_rate, -o.cold_shift);
  return o;
}

// LANES lanes hold HELD logits each in registers, and EXTRA in LDS.  Of a row at once, one wavefront more learns what the teacher
// and the label ask for, while the others wait for the logits.
template <int PHASE, int LANES>
constexpr int kBlock = LANES + (PHASE == kWhole ? 64 : 0);

template <bool BF16, int KIND, int PHASE, int LANES, int HELD, int EXTRA>
__global__ void __launch_bounds__((kBlock<PHASE, LANES>), HELD <= 32 ? 8 : 4) k_distillation(DistillationArgs a) {
  constexpr int N = kPiece<BF16>, ES = BF16 ? 2 : 4, V = HELD / N, X = EXTRA / N, kWaves = LANES / 64;
  // fp32 rows that are held are read past the caches: 103.7 and 101.0 us at 8 workers x 256 rows x 30522, 73.2 and 68.7 at
  // 8 x 1024 x 5000; bf16 ones (8 x 512 x 30522: 108.4 and 109.0; 8 x 512 x 5000: 23.3 and 25.7) are not
  constexpr bool kPast = !BF16 && PHASE == kWhole;
  constexpr bool kKeep = KIND != kTwo;  // exponentials stay; else distances
  __shared__ float waves[kWaves][3];
  __shared__ Lesson lesson;
  __shared__ f32x4 extra[X > 0 ? X * N / 4 : 1][X > 0 ? LANES : 1];
  const uint32_t w = blockIdx.z, row = blockIdx.x + (PHASE == kWhole ? blockIdx.y * kGridRows : 0), n = a.w.tokens[w];
  if (row >= n) return;
  const uint32_t lane = threadIdx.x, wave = uniform(threadIdx.x / 64);
  const uint64_t z = a.w.at[kDistLogits][w] + uint64_t(row) * a.pitch * ES;
  // of the row in the workspace: three numbers of every part, and the lesson behind them
  float* const ws = reinterpret_cast<float*>(a.ws) + (uint64_t(w) * a.max_tokens + row) * a.stride;
  Lesson* const kept = reinterpret_cast<Lesson*>(ws + (3 * a.parts + 1) / 2 * 2);
  if constexpr (PHASE == kMeasure) {
    if (blockIdx.y == a.parts) {
      if (wave) return;
      Student<BF16> student;
      student.ask(a, w, row, z);
      student.learn(a, *kept);
      return;
    }
  }
  // this workgroup's part of the row
  const uint32_t lo = PHASE == kWhole ? 0 : min(blockIdx.y * a.part, a.vocab);
  const bool last = PHASE == kWhole || blockIdx.y + 1 == a.parts;
  const uint32_t hi = last ? a.vocab : min(lo + a.part, a.vocab), count = (hi - lo) & ~uint32_t(BF16 ? 1 : 0);
  const Row<BF16> in(z + uint64_t(lo) * ES, hi - lo);
  const uint32_t col = lane * N;  // of a lane's first piece; the next one is LANES pieces on
  // what is behind the part counts for nothing
  auto cut = [&](uint32_t at, float* v) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = at + j < count ? v[j] : -__builtin_inff();
  };
  float x[V][N], odd = -__builtin_inff(), largest = kLowest, warm = 0.0f, cold = 0.0f;
  Origin from{};

  if (PHASE == kWhole && wave == kWaves) {
    Student<BF16> student;
    student.ask(a, w, row, z);
    __syncthreads();  // the others' largest logits
    student.learn(a, lesson);
    __syncthreads();  // their sums
  } else {
    // all loads first; what goes to LDS before what stays
    if constexpr (X > 0) {
      constexpr int kBatch = 5;
      static_assert(X % kBatch == 0);
#pragma unroll 1
      for (int i = 0; i < X; i += kBatch) {
        u32x4 raw[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) raw[b] = in.template get<kPast>(col + uint32_t(V + i + b) * LANES * N);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          float y[N];
          widen<BF16>(raw[b], y);
          if (uint32_t(V + i + b + 1) * LANES * N > count) cut(col + uint32_t(V + i + b) * LANES * N, y);
#pragma unroll
          for (int j = 0; j < N; j += 4) {
            extra[((i + b) * N + j) / 4][lane] = f32x4{y[j], y[j + 1], y[j + 2], y[j + 3]};
            largest = fmaxf(largest, fmaxf(fmaxf(y[j], y[j + 1]), fmaxf(y[j + 2], y[j + 3])));
          }
        }
      }
    }
    {
      u32x4 raw[V];
#pragma unroll
      for (int i = 0; i < V; ++i) raw[i] = in.template get<kPast>(col + uint32_t(i) * LANES * N);
      if (in.odd() && lane == 0) odd = bf16_low(in.get_last());
#pragma unroll
      for (int i = 0; i < V; ++i) {
        widen<BF16>(raw[i], x[i]);
        if (uint32_t(i + 1) * LANES * N > count) cut(col + uint32_t(i) * LANES * N, x[i]);
      }
    }

    if constexpr (PHASE != kWrite) {
      // pieces that are not held: largest logit and sums together
      for (uint32_t p = (V + X) * LANES * N; p < count; p += LANES * N) {
        float y[N], m = largest;
        widen<BF16>(in.get(p + col), y);
        cut(p + col, y);
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, y[j]);
        warm *= exp2((largest - m) * a.warm_rate);
        cold *= exp2((largest - m) * a.cold_rate);
        largest = m;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          warm += exp2((y[j] - m) * a.warm_rate);
          if constexpr (KIND != kOne) cold += exp2((y[j] - m) * a.cold_rate);
        }
      }
      float m = fmaxf(largest, odd);
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) m = fmaxf(m, x[i][j]);
      m = wave_max(m);
      if (lane % 64 == 0) waves[wave][0] = m;
      __syncthreads();
      m = across_max<kWaves>(&waves[0][0], 3);
      from = origin<KIND>(a, m, PHASE != kWhole);
      warm *= exp2(__builtin_fmaf(largest - m, a.warm_rate, from.warm_rest));  // (a factor that the held ones have)
      if constexpr (KIND != kOne) cold *= exp2(__builtin_fmaf(largest - m, a.cold_rate, from.cold_rest));
      largest = m;
    } else {
      // the parts' sums, joined by every wavefront for itself; the lesson for all
      float m = kLowest, sum_warm = 0.0f, sum_cold = 0.0f;
      for (uint32_t k = lane % 64; k < a.parts; k += 64) {
        const float its_largest = ws[3 * k], its_warm = ws[3 * k + 1], its_cold = ws[3 * k + 2];
        const float top = fmaxf(m, its_largest), now = m - top, its = its_largest - top;
        sum_warm = sum_warm * exp2(now * a.warm_rate) + its_warm * exp2(its * a.warm_rate);
        sum_cold = sum_cold * exp2(now * a.cold_rate) + its_cold * exp2(its * a.cold_rate);
        m = top;
      }
      for (uint32_t k = lane; k <= a.top; k += LANES) {
        lesson.id[k] = kept->id[k];
        lesson.logit[k] = kept->logit[k];
        lesson.weight[k] = kept->weight[k];
      }
      if (lane == 0) {
        lesson.terms = kept->terms;
        lesson.best = kept->best;
        lesson.taught = kept->taught;
      }
      largest = wave_max(m);
      warm = wave_sum(sum_warm * exp2((m - largest) * a.warm_rate));
      cold = wave_sum(sum_cold * exp2((m - largest) * a.cold_rate));
      from = origin<KIND>(a, largest, true);
      __syncthreads();
    }

    // distances or exponentials in place of what is held, and their sums
    auto measure = [&](float& v) {
      if (kKeep || PHASE != kWrite) {
        const float e = exp2(__builtin_fmaf(v, a.warm_rate, -from.warm_shift));
        if constexpr (PHASE != kWrite) {
          warm += e;
          if constexpr (KIND == kSquare) cold = __builtin_fmaf(e, e, cold);
          if constexpr (KIND == kFourth) cold = __builtin_fmaf(e * e, e * e, cold);
          if constexpr (KIND == kTwo) cold += exp2(__builtin_fmaf(v, a.cold_rate, -from.cold_shift));
        }
        if constexpr (kKeep) v = e;
      }
    };
    if (from.base != 0.0f) {  // also where it is NaN
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) x[i][j] -= from.base;
    }
    odd -= from.base;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (uint32_t(i) * LANES * N >= count) continue;
#pragma unroll
      for (int j = 0; j < N; ++j) measure(x[i][j]);
      __builtin_amdgcn_sched_barrier(0);  // piece by piece: all at once would take as many registers again
    }
    measure(odd);
    if constexpr (X > 0) {
#pragma unroll 1
      for (int i = 0; i < X * N / 4; ++i) {
        if (uint32_t(V + i * 4 / N) * LANES * N >= count) break;
        f32x4 y = extra[i][lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float v = y[j] - from.base;
          measure(v);
          y[j] = v;
        }
        extra[i][lane] = y;
      }
    }
    if constexpr (PHASE != kWrite) {
      warm = wave_sum(warm);
      if constexpr (KIND != kOne) cold = wave_sum(cold);
      if (lane % 64 == 0) waves[wave][1] = warm, waves[wave][2] = cold;
      __syncthreads();
    }
  }
  if constexpr (PHASE != kWrite) {
    if constexpr (PHASE == kWhole) largest = across_max<kWaves>(&waves[0][0], 3);
    warm = across_sum<kWaves>(&waves[0][1], 3);
    cold = KIND != kOne ? across_sum<kWaves>(&waves[0][2], 3) : warm;
  }
  if constexpr (PHASE == kMeasure) {
    if (lane == 0) {
      ws[3 * blockIdx.y] = largest;
      ws[3 * blockIdx.y + 1] = warm;
      ws[3 * blockIdx.y + 2] = cold;
    }
  } else {
    if constexpr (KIND == kOne) cold = warm;
    const bool has_teacher = uniform(lesson.terms) & 1, has_label = uniform(lesson.terms) & 2;
    const float share = has_teacher ? a.soft * float(a.inverse) / warm : 0.0f, label_share = has_label ? a.hard / cold : 0.0f;
    const uint64_t out = a.w.at[kDistGradient][w] + uint64_t(row) * a.gradient_pitch * ES;
    const bool holds = PHASE != kWhole || wave < kWaves;
    if (a.gradient && holds) {
      const Row<BF16> to(out + uint64_t(lo) * ES, hi - lo);
      const float kw = a.scale * (KIND == kOne ? share + label_share : share), kc = a.scale * label_share;
      const bool none = !has_teacher && !has_label;  // zeros, whatever the logits are
      if (none) {
        from = Origin{};
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int j = 0; j < N; ++j) x[i][j] = 0.0f;
      }
      auto gradient = [&](float v) {  // of what is held
        if constexpr (KIND == kOne) return kw * v;
        else if constexpr (KIND == kSquare) return v * __builtin_fmaf(kc, v, kw);
        else if constexpr (KIND == kFourth) return v * __builtin_fmaf(kc, v * (v * v), kw);
        else return __builtin_fmaf(kw, exp2(__builtin_fmaf(v, a.warm_rate, -from.warm_shift)),
                                   kc * exp2(__builtin_fmaf(v, a.cold_rate, -from.cold_shift)));
      };
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (uint32_t(i) * LANES * N >= count) continue;
        float g[N];
#pragma unroll
        for (int j = 0; j < N; ++j) g[j] = gradient(x[i][j]);
        to.template put<true>(col + uint32_t(i) * LANES * N, narrow<BF16>(g));
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (X > 0) {
#pragma unroll 1
        for (int i = 0; i < X; ++i) {
          if (uint32_t(V + i) * LANES * N >= count) break;
          float y[N];
#pragma unroll
          for (int j = 0; j < N; j += 4) {
            const f32x4 e = extra[(i * N + j) / 4][lane];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[j + k] = none ? 0.0f : gradient(e[k]);
          }
          to.template put<true>(col + uint32_t(V + i) * LANES * N, narrow<BF16>(y));
        }
      }
      for (uint32_t p = (V + X) * LANES * N; p < count; p += LANES * N) {
        float y[N];
        widen<BF16>(in.get(p + col), y);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          float v = y[j] - from.base;
          if constexpr (kKeep) v = exp2(__builtin_fmaf(v, a.warm_rate, -from.warm_shift));
          y[j] = none ? 0.0f : gradient(v);
        }
        to.template put<true>(p + col, narrow<BF16>(y));
      }
      if (in.odd() && lane == 0) {
        const float g = none ? 0.0f : gradient(odd);
        store_elems<BF16, 1>(out + uint64_t(hi - 1) * ES, &g);
      }
    }
    if (PHASE == kWhole) from = origin<KIND>(a, largest, false);  // (the wavefront that learned has none)
    if (PHASE == kWhole ? lane == LANES : lane == 0 && blockIdx.y == 0) {
      double loss = 0.0;
      if (has_teacher)
        loss += double(a.soft) * (lesson.taught + (double(largest) - double(lesson.best)) * a.inverse +
                                  (ln(warm) - double(from.warm_rest) * 0.69314718055994531));
      if (has_label)
        loss += double(a.hard) *
                ((ln(cold) - double(from.cold_rest) * 0.69314718055994531) - (double(lesson.logit[a.top]) - double(largest)));
      reinterpret_cast<CARAMEL_GLOBAL float*>(a.w.at[kDistLoss][w])[row] = float(loss);
    }
    if (!a.gradient) return;
    __syncthreads();
    // the entries' own logits, each written by its first entry
    for (uint32_t k = lane; k <= a.top; k += kBlock<PHASE, LANES>) {
      const uint32_t id = lesson.id[k];
      if (id == kNone || id < lo || id >= hi) continue;
      float less = 0.0f;
      bool first = true;
      for (uint32_t i = 0; i <= a.top; ++i) {
        const bool same = lesson.id[i] == id;
        less += same ? lesson.weight[i] : 0.0f;
        first = first && !(same && i < k);
      }
      if (!first) continue;
      const float d = lesson.logit[k] - from.base, e = exp2(__builtin_fmaf(d, a.warm_rate, -from.warm_shift));
      float g = share * e;
      if constexpr (KIND == kOne) g = (share + label_share) * e;
      if constexpr (KIND == kSquare) g = __builtin_fmaf(label_share, e * e, g);
      if constexpr (KIND == kFourth) g = __builtin_fmaf(label_share, (e * e) * (e * e), g);
      if constexpr (KIND == kTwo) g = __builtin_fmaf(label_share, exp2(__builtin_fmaf(d, a.cold_rate, -from.cold_shift)), g);
      g = a.scale * (g - less);
      store_elems<BF16, 1>(out + uint64_t(id) * ES, &g);
    }
  }
}

// Rows that registers do not hold are cut into parts, so many rows at most, into about so many workgroups.  20 rows of 400000 fp32
// logits: 21 us, one workgroup to a row 67; 100 of 129999: 32 and 32; 192 of them 62 and 47.  A row in registers is quicker whole, which
// is one launch instead of two: 3 rows of 30522 logits 7.9 us, in parts 11.0.
constexpr uint32_t kFewRows = 96, kPartGroups = 512;
constexpr int kPartLanes = 256, kPartHeld = 16;

uint32_t parts_of(uint64_t rows, uint32_t vocab) {
  const uint32_t most = vocab / (kPartLanes * kPartHeld);
  if (rows == 0 || rows > kFewRows || vocab <= 960 * 64) return 1;
  return uint32_t(std::min<uint64_t>(most, (kPartGroups + rows - 1) / rows));
}

template <int LANES, int HELD, int EXTRA>
struct Shape {
  static constexpr int kLanes = LANES, kHeld = HELD, kExtra = EXTRA;
};

template <bool BF16, int KIND>
hipError_t launch(const DistillationArgs& a, hipStream_t s) {
  if (a.parts > 1) {
    const dim3 grid(a.max_tokens, a.parts + 1, a.world);  // one more learns the lesson
    hipLaunchKernelGGL((k_distillation<BF16, KIND, kMeasure, kPartLanes, kPartHeld, 0>), grid, dim3(kPartLanes), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 write(a.max_tokens, a.gradient ? a.parts : 1, a.world);
    hipLaunchKernelGGL((k_distillation<BF16, KIND, kWrite, kPartLanes, kPartHeld, 0>), write, dim3(kPartLanes), 0, s, a);
    return hipGetLastError();
  }
  const dim3 grid(std::min(a.max_tokens, kGridRows), (a.max_tokens + kGridRows - 1) / kGridRows, a.world);
  // the smallest that holds a row
  auto fits = [&](auto shape) {
    constexpr int LANES = decltype(shape)::kLanes, HELD = decltype(shape)::kHeld, EXTRA = decltype(shape)::kExtra;
    hipLaunchKernelGGL((k_distillation<BF16, KIND, kWhole, LANES, HELD, EXTRA>), grid, dim3(kBlock<kWhole, LANES>), 0, s, a);
  };
  if (a.vocab <= 192 * 32) fits(Shape<192, 32, 0>{});
  else if (a.vocab <= 448 * 32) fits(Shape<448, 32, 0>{});
  else if (a.vocab <= 960 * 32) fits(Shape<960, 32, 0>{});
  else if (a.vocab <= 960 * 64) fits(Shape<960, 64, 0>{});
  else fits(Shape<960, BF16 ? 80 : 96, 40>{});  // (two wavefronts' registers; with 96 numbers as bf16 the compiler would spill)
  return hipGetLastError();
}

}  // namespace

// Of fewer rows, each may have more parts; all of them together, no more than this.
uint64_t distillation_workspace_bytes(uint32_t world, uint32_t vocab, uint32_t max_tokens) {
  const uint64_t rows = std::min<uint64_t>(uint64_t(world) * max_tokens, kFewRows);
  if (rows == 0 || parts_of(1, vocab) == 1) return 0;
  return (3 * (kPartGroups + rows) + rows * (1 + sizeof(Lesson) / 4)) * 4;
}

hipError_t launch_distillation(const DistillationArgs& args, const AllBuffers<kDistBuffers>& v, hipStream_t s) {
  if (args.max_tokens == 0) return hipSuccess;
  DistillationArgs all = args;
  all.parts = parts_of(uint64_t(args.all) * args.max_tokens, args.vocab);
  all.part = ((args.vocab + all.parts - 1) / all.parts + 7) / 8 * 8;
  all.stride = (3 * all.parts + 1) / 2 * 2 + sizeof(Lesson) / 4;
  const bool both = args.soft > 0.0f && args.has_labels;
  const int kind = !both || args.temperature == 1.0f ? kOne : args.temperature == 2.0f ? kSquare : args.temperature == 4.0f ? kFourth : kTwo;
  const double log2e = 1.4426950408889634;
  // without a teacher's part, all is at temperature 1
  all.warm_rate = float(log2e / (args.soft > 0.0f ? double(args.temperature) : 1.0));
  all.cold_rate = float(log2e);
  all.inverse = 1.0 / double(args.temperature);
  return in_groups(all, v, [&](DistillationArgs a, uint32_t g) {
    a.ws += uint64_t(g) * a.max_tokens * a.stride * 4;
    const bool b = a.bf16;
    if (kind == kOne) return b ? launch<true, kOne>(a, s) : launch<false, kOne>(a, s);
    if (kind == kSquare) return b ? launch<true, kSquare>(a, s) : launch<false, kSquare>(a, s);
    if (kind == kFourth) return b ? launch<true, kFourth>(a, s) : launch<false, kFourth>(a, s);
    return b ? launch<true, kTwo>(a, s) : launch<false, kTwo>(a, s);
  });
}

}  // namespace caramel
