// Host-side description of a call of the distillation operators, and their launchers.
#pragma once
#include <hip/hip_runtime.h>
#include "../../include/bpc.h"

namespace bpc {

// A call of the distillation operators (bpc_logits_topk, bpc_distill_*), as the kernels take it.
struct DistillCall {
  const void *logits;
  int dtype;
  uint64_t row_stride, rows;
  uint32_t vocab, k;
  const uint8_t *messages;
  uint64_t message_stride;
  bool half, rest_too;      // values of the messages in half precision; TAIL_REST
  float temperature, soft, hard;
  const int64_t *labels;    // or NULL
  const float *weight;      // or NULL
  float *loss;
  void *stats;              // or NULL
  void *grad;
  uint64_t grad_stride;
};
enum class DistillRole { loss, grad, step };
hipError_t distill_run_f32(const DistillCall &call, DistillRole role, uint8_t *ws, hipStream_t stream);
hipError_t distill_run_f16(const DistillCall &call, DistillRole role, uint8_t *ws, hipStream_t stream);
hipError_t distill_run_bf16(const DistillCall &call, DistillRole role, uint8_t *ws, hipStream_t stream);
inline hipError_t distill_run(const DistillCall &call, DistillRole role, uint8_t *ws, hipStream_t stream) {
  return call.dtype == BPC_F32 ? distill_run_f32(call, role, ws, stream)
         : call.dtype == BPC_F16 ? distill_run_f16(call, role, ws, stream)
                                 : distill_run_bf16(call, role, ws, stream);
}
hipError_t logits_topk(const DistillCall &call, uint8_t *out, uint8_t *ws, hipStream_t stream);

}  // namespace bpc
