// C entry points of the distillation loss: checks.
#include "sfc.h"
#include "sfc_distill.hpp"

namespace {

bool aligned(const void* p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) == 0; }

sfc_status run(const sfc_distill_desc* d, const void* logits, const float* values, const void* index,
               const float* row_scale, float* loss, const float* stats, void* grad, void* stream) {
  if (!d) return SFC_EINVAL;
  if (d->rows < 0 || d->classes <= 0 || d->top <= 0) return SFC_EINVAL;
  if (d->type < SFC_TYPE_F32 || d->type > SFC_TYPE_BF16) return SFC_EINVAL;
  if ((d->index_wide & ~1) != 0 || (d->tail & ~1) != 0) return SFC_EINVAL;
  if (!(d->temperature > 0.0f) || d->temperature > 1e30f || d->temperature < 1e-30f) return SFC_EINVAL;
  if (d->classes > 1 << 18 || d->top > 1024 || d->rows > 0x7fffffff) return SFC_EUNSUPPORTED;
  sfc::DistillArgs a = {};
  a.logits_stride = d->logits_stride ? d->logits_stride : d->classes;
  a.grad_stride = d->grad_stride ? d->grad_stride : d->classes;
  a.values_stride = d->values_stride ? d->values_stride : d->top;
  a.index_stride = d->index_stride ? d->index_stride : d->top;
  if (a.logits_stride < d->classes || a.grad_stride < d->classes || a.values_stride < d->top || a.index_stride < d->top)
    return SFC_EINVAL;
  if (d->rows == 0) return SFC_OK;
  const int size = d->type == SFC_TYPE_F32 ? 4 : 2;
  if (!logits || !values || !index || (!loss && !stats) || (!loss && !grad)) return SFC_EINVAL;
  if (!aligned(logits, size) || !aligned(grad, size) || !aligned(values, 4) || !aligned(index, d->index_wide ? 8 : 4) ||
      !aligned(row_scale, 4) || !aligned(loss, 4) || !aligned(stats, 16))
    return SFC_EINVAL;
  a.logits = logits;
  a.values = values;
  a.index = index;
  a.row_scale = row_scale;
  a.loss = loss;
  a.stats = const_cast<float*>(stats);
  a.grad = grad;
  a.rows = d->rows;
  a.classes = d->classes;
  a.top = d->top;
  a.wide = d->index_wide != 0;
  a.tail = d->tail != 0;
  a.temperature = d->temperature;
  a.stream = d->rows * d->classes * size >= sfc::kStreamBytes;
  return sfc::launch_distill(a, d->type, static_cast<hipStream_t>(stream)) == hipSuccess ? SFC_OK : SFC_EHIP;
}

}  // namespace

extern "C" {

sfc_status sfc_distill_loss(const sfc_distill_desc* desc, const void* logits_dev, const float* values_dev,
                            const void* index_dev, const float* row_scale_dev, float* loss_dev,
                            float* stats_dev, void* stream) {
  if (desc && desc->rows > 0 && !loss_dev) return SFC_EINVAL;
  return run(desc, logits_dev, values_dev, index_dev, row_scale_dev, loss_dev, stats_dev, nullptr, stream);
}

sfc_status sfc_distill_grad(const sfc_distill_desc* desc, const void* logits_dev, const float* values_dev,
                            const void* index_dev, const float* row_scale_dev, const float* stats_dev,
                            void* grad_dev, void* stream) {
  return run(desc, logits_dev, values_dev, index_dev, row_scale_dev, nullptr, stats_dev, grad_dev, stream);
}

sfc_status sfc_distill_loss_grad(const sfc_distill_desc* desc, const void* logits_dev, const float* values_dev,
                                 const void* index_dev, const float* row_scale_dev, float* loss_dev,
                                 void* grad_dev, void* stream) {
  if (desc && desc->rows > 0 && (!loss_dev || !grad_dev)) return SFC_EINVAL;
  return run(desc, logits_dev, values_dev, index_dev, row_scale_dev, loss_dev, nullptr, grad_dev, stream);
}

}  // extern "C"
