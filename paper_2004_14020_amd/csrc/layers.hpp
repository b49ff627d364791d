// Kernels that fill a plan's gradient tensors: the embedding lookup and its gradient, activation
// checkpoints in 8 bits, and the weight and bias gradients that read them.  Launch wrappers; the
// arguments have been checked by the entry points.
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

}  // namespace caramel
