// Distillation from a teacher's top logits: arguments of the kernels.
#pragma once
#include "sfc_values.hpp"

namespace sfc {

struct DistillArgs {
  const void* logits;      // [rows][classes]
  const float* values;     // [rows][top]
  const void* index;       // [rows][top], int32 or int64
  const float* row_scale;  // [rows] or null: ones
  float* loss;             // [rows] or null
  float* stats;            // [rows][4]: written with the loss (or null), read by the gradient alone
  void* grad;              // [rows][classes] or null
  int64_t rows;
  int classes, top;
  int64_t logits_stride, grad_stride, values_stride, index_stride;
  bool wide, tail;         // int64 places; the rest of the mass as one more outcome
  float temperature;
  bool stream;             // the gradient is stored past the caches
};

// loss: from the logits (with stats if given); grad alone: from stats.  type: sfc_type.
hipError_t launch_distill(const DistillArgs& a, int type, hipStream_t s);

}  // namespace sfc
