// Kernels that fill a plan's gradient tensors: the embedding lookup and its gradient, activation
// checkpoints in 8 bits, and the weight and bias gradients that read them.  Launch wrappers; the
// arguments have been checked by the entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "caramel.h"

namespace caramel {

// Addresses and lengths of the workers' buffers, passed by value: nothing is uploaded, so a call can be
// captured, and two calls never share a table.
struct Workers {
  uint64_t a[CARAMEL_MAX_WORLD];
  uint64_t b[CARAMEL_MAX_WORLD];
  uint64_t c[CARAMEL_MAX_WORLD];
  uint32_t tokens[CARAMEL_MAX_WORLD];
};

constexpr uint32_t kCheckpointBlock = 32;  // tokens that share a scale

inline uint64_t checkpoint_blocks(uint64_t tokens) { return (tokens + kCheckpointBlock - 1) / kCheckpointBlock; }

struct LookupArgs {
  Workers w;  // a: tables, b: ids, c: out
  uint32_t world, max_tokens;
  uint32_t vocab, width;
  uint64_t out_pitch;  // elements
  float scale;
  bool ids64, bf16;
};
hipError_t launch_embedding_lookup(const LookupArgs& a, hipStream_t s);

struct EmbeddingGradientArgs {
  Workers w;  // a: ids, b: dy, c: gradient
  uint32_t world, max_tokens;
  uint32_t vocab, width;
  uint64_t dy_pitch;
  float scale;
  bool ids64, dy_bf16, out_bf16, accumulate;
  unsigned char* ws;
};
uint64_t embedding_gradient_workspace(uint32_t world, uint32_t vocab, uint32_t width, uint32_t max_tokens);
hipError_t launch_embedding_gradient(const EmbeddingGradientArgs& a, hipStream_t s);

struct CheckpointArgs {
  Workers w;  // a: activations, b: checkpoints
  uint32_t world, max_tokens;
  uint32_t features;
  uint64_t pitch;  // of the activations, elements
  bool bf16;
};
hipError_t launch_checkpoint_store(const CheckpointArgs& a, hipStream_t s);
hipError_t launch_checkpoint_load(const CheckpointArgs& a, hipStream_t s);

struct WeightGradientArgs {
  Workers w;                          // a: checkpoints, b: dy, c: weight gradients
  uint64_t bias[CARAMEL_MAX_WORLD];   // bias gradients, or 0
  uint32_t world, max_tokens;
  uint32_t features, outputs;
  uint64_t dy_pitch;
  bool dy_bf16, out_bf16, accumulate, has_bias;
  unsigned char* ws;
};
uint64_t weight_gradient_workspace(uint32_t world, uint32_t features, uint32_t outputs, uint32_t max_tokens);
hipError_t launch_weight_gradient(const WeightGradientArgs& a, hipStream_t s);

}  // namespace caramel
