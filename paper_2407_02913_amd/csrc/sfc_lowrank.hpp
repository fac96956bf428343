// Low-rank adapters of many requests: arguments of the kernels.
#pragma once
#include "sfc_values.hpp"

namespace sfc {

struct LowrankArgs {
  const void* x;         // [tokens][inputs]
  const void* dy;        // [tokens][outputs], backward
  const int32_t* ids;    // [tokens]
  const void* down;      // [adapters][rank][inputs]
  const void* up;        // [adapters][outputs][rank]
  const float* scale;    // [adapters] or null: ones
  const void* base;      // [tokens][outputs] or null: zeros; backward: [tokens][inputs]
  void* y;               // [tokens][outputs]; backward: dx
  void* d_down;          // backward, as down
  void* d_up;            // backward, as up
  char* space;           // workspace
  int64_t x_stride, base_stride, y_stride, dy_stride;
  int tokens, inputs, outputs, rank, adapters;
};

size_t lowrank_bytes(const LowrankArgs& a, int size);
size_t lowrank_backward_bytes(const LowrankArgs& a, int size);
// type: sfc_type
hipError_t launch_lowrank(const LowrankArgs& a, int type, hipStream_t s);
// the factors' gradients without any token: zeros
hipError_t launch_lowrank_no_tokens(const LowrankArgs& a, int type, hipStream_t s);
hipError_t launch_lowrank_backward(const LowrankArgs& a, int type, hipStream_t s);

}  // namespace sfc
