// Kernels that fill a plan's gradient tensors, and those of a training step before and between them: the
// embedding lookup and its gradient, activation checkpoints in 8 bits, the weight and bias gradients that
// read them, the residual norm and the gated recurrence with their gradients, distillation.  Launch wrappers; the arguments have been checked by the entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "caramel.h"

namespace caramel {

// Addresses and lengths of the workers' buffers.
struct AllWorkers {
  uint64_t a[CARAMEL_MAX_WORLD];
  uint64_t b[CARAMEL_MAX_WORLD];
  uint64_t c[CARAMEL_MAX_WORLD];
  uint64_t d[CARAMEL_MAX_WORLD];
  uint32_t tokens[CARAMEL_MAX_WORLD];
};

// Those of one launch, passed by value: nothing is uploaded, so a call can be captured, and two calls never share a table.  More
// workers than this go out in several launches: arguments for 64 take 2 KiB, which costs every launch 0.2 to 0.5 us of 5.
constexpr uint32_t kGroup = 16;
struct Workers {
  uint64_t a[kGroup];
  uint64_t b[kGroup];
  uint64_t c[kGroup];
  uint64_t d[kGroup];
  uint32_t tokens[kGroup];
};

// Calls launch(arguments of the group, first worker of the group) for all workers, sixteen at a time.
template <typename ARGS, typename LAUNCH>
hipError_t in_groups(ARGS a, const AllWorkers& v, LAUNCH&& launch) {
  for (uint32_t g = 0; g < a.all; g += kGroup) {
    a.world = a.all - g < kGroup ? a.all - g : kGroup;
    for (uint32_t w = 0; w < a.world; ++w) {
      a.w.a[w] = v.a[g + w];
      a.w.b[w] = v.b[g + w];
      a.w.c[w] = v.c[g + w];
      a.w.d[w] = v.d[g + w];
      a.w.tokens[w] = v.tokens[g + w];
    }
    const hipError_t e = launch(a, g);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// The same for calls with more buffers, or with another count per worker.  A buffer that a call goes without has address 0.
template <int N>
struct AllBuffers {
  uint64_t at[N][CARAMEL_MAX_WORLD];
  uint32_t tokens[CARAMEL_MAX_WORLD];
  uint32_t more[CARAMEL_MAX_WORLD];
};
template <int N>
struct Buffers {
  uint64_t at[N][kGroup];
  uint32_t tokens[kGroup];
  uint32_t more[kGroup];
};

template <typename ARGS, int N, typename LAUNCH>
hipError_t in_groups(ARGS a, const AllBuffers<N>& v, LAUNCH&& launch) {
  for (uint32_t g = 0; g < a.all; g += kGroup) {
    a.world = a.all - g < kGroup ? a.all - g : kGroup;
    for (uint32_t w = 0; w < a.world; ++w) {
      for (int i = 0; i < N; ++i) a.w.at[i][w] = v.at[i][g + w];
      a.w.tokens[w] = v.tokens[g + w];
      a.w.more[w] = v.more[g + w];
    }
    const hipError_t e = launch(a, g);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

constexpr uint32_t kCheckpointBlock = 32;  // tokens that share a scale

inline uint64_t checkpoint_blocks(uint64_t tokens) { return (tokens + kCheckpointBlock - 1) / kCheckpointBlock; }

struct LookupArgs {
  Workers w;  // a: tables, b: ids, c: out
  uint32_t world, all;  // workers of the launch, of the call
  uint32_t max_tokens;  // of all workers
  uint32_t vocab, width;
  uint64_t out_pitch;  // elements
  float scale;
  bool ids64, bf16;
};
hipError_t launch_embedding_lookup(const LookupArgs& args, const AllWorkers& v, hipStream_t s);

struct EmbeddingGradientArgs {
  Workers w;  // a: ids, b: dy, c: gradient
  uint32_t world, all;  // workers of the launch, of the call
  uint32_t max_tokens;  // of all workers
  uint32_t vocab, width;
  uint64_t dy_pitch;
  float scale;
  bool ids64, dy_bf16, out_bf16, accumulate;
  unsigned char* ws;
};
uint64_t embedding_gradient_workspace(uint32_t world, uint32_t vocab, uint32_t width, uint32_t max_tokens);
hipError_t launch_embedding_gradient(const EmbeddingGradientArgs& args, const AllWorkers& v, hipStream_t s);

struct CheckpointArgs {
  Workers w;  // a: activations, b: checkpoints
  uint32_t world, all;  // workers of the launch, of the call
  uint32_t max_tokens;  // of all workers
  uint32_t features;
  uint64_t pitch;  // of the activations, elements
  bool bf16;
};
hipError_t launch_checkpoint_store(const CheckpointArgs& args, const AllWorkers& v, hipStream_t s);
hipError_t launch_checkpoint_load(const CheckpointArgs& args, const AllWorkers& v, hipStream_t s);

struct WeightGradientArgs {
  Workers w;  // a: checkpoints, b: dy, c: weight gradients, d: bias gradients
  uint32_t world, all;  // workers of the launch, of the call
  uint32_t max_tokens;  // of all workers
  uint32_t features, outputs;
  uint64_t dy_pitch;
  bool dy_bf16, out_bf16, accumulate, has_bias;
  unsigned char* ws;
};
uint64_t weight_gradient_workspace(uint32_t world, uint32_t features, uint32_t outputs, uint32_t max_tokens);
hipError_t launch_weight_gradient(const WeightGradientArgs& args, const AllWorkers& v, hipStream_t s);

constexpr uint32_t kNormWidth = 32768;  // most columns: a row stays in the registers of one workgroup

enum { kNormX, kNormResidual, kNormSum, kNormY, kNormRstd, kNormGain, kNormCheckpoint, kNormBuffers };
struct NormArgs {
  Buffers<kNormBuffers> w;
  uint32_t world, all;  // workers of the launch, of the call
  uint32_t max_tokens;  // of all workers
  uint32_t width;
  uint64_t pitch;  // of all rows, elements
  float eps;
  double inverse_width;  // made by the launch, as is
  bool stream;           // matrices are larger than the caches near the compute units
  bool bf16, gain_bf16, residual, checkpoint;
};
hipError_t launch_norm(const NormArgs& args, const AllBuffers<kNormBuffers>& v, hipStream_t s);

enum { kNormGradX, kNormGradRstd, kNormGradDy, kNormGradDsum, kNormGradDx, kNormGradGain, kNormGradOut, kNormGradBuffers };
struct NormGradientArgs {
  Buffers<kNormGradBuffers> w;
  uint32_t world, all;  // workers of the launch, of the call
  uint32_t max_tokens;  // of all workers
  uint32_t width;
  uint64_t pitch;
  bool bf16, gain_bf16, dsum, accumulate;  // gain_bf16: the plan's dtype, of gain and its gradient
  bool stream;  // made by the launch
  unsigned char* ws;
};
uint64_t norm_gradient_workspace(uint32_t world, uint32_t width, uint32_t max_tokens);
hipError_t launch_norm_gradient(const NormGradientArgs& args, const AllBuffers<kNormGradBuffers>& v, hipStream_t s);

enum {
  kRecStarts, kRecGate, kRecInput, kRecBefore, kRecStates, kRecAfter,   // after: forward
  kRecDstates, kRecDafter, kRecDgate, kRecDinput, kRecDbefore, kRecBuffers  // gradient
};
struct RecurrenceArgs {
  Buffers<kRecBuffers> w;  // more: sequences
  uint32_t world, all;     // workers of the launch, of the call
  uint32_t max_tokens;     // of all workers
  uint32_t channels;
  uint64_t pitch, states_pitch;  // of gates, inputs and their gradients; of states and theirs; elements
  bool bf16, starts64;
  unsigned char* ws;
  // made by the launch: tokens are cut into parts of `span`, and the parts are counted through all workers
  uint32_t span, first_part[kGroup + 1];
  bool cut;    // a worker has more than one
  bool lines;  // rows are whole cache lines
  uint32_t steps;  // not 0: sequences are short, and there are so many at a worker at most
};
uint64_t recurrence_workspace_bytes(uint32_t world, uint32_t channels, const uint32_t* tokens);
hipError_t launch_recurrence(const RecurrenceArgs& args, const AllBuffers<kRecBuffers>& v, hipStream_t s);
hipError_t launch_recurrence_gradient(const RecurrenceArgs& args, const AllBuffers<kRecBuffers>& v, hipStream_t s);

constexpr uint32_t kDistillationTop = 256;  // most entries of the teacher per token

enum { kDistLogits, kDistIds, kDistTeacher, kDistLabels, kDistLoss, kDistGradient, kDistBuffers };
struct DistillationArgs {
  Buffers<kDistBuffers> w;
  uint32_t world, all;  // workers of the launch, of the call
  uint32_t max_tokens;  // of all workers
  uint32_t vocab, top;
  uint64_t pitch, gradient_pitch;  // elements
  float temperature, soft, hard, scale;
  bool bf16, teacher_bf16, ids64, has_labels, gradient;
  unsigned char* ws;
  // made by the launch
  uint32_t parts, part, stride;  // of a row; logits of a part; floats of a row in the workspace
  float warm_rate, cold_rate;  // log2(e) / temperature, log2(e)
  double inverse;              // 1 / temperature
};
uint64_t distillation_workspace_bytes(uint32_t world, uint32_t vocab, uint32_t max_tokens);
hipError_t launch_distillation(const DistillationArgs& args, const AllBuffers<kDistBuffers>& v, hipStream_t s);

}  // namespace caramel
