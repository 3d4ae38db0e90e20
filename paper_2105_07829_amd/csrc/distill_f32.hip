// The student's kernels for logits of one type (a file a type, so that they are compiled side by side).
#include "distill_student.hpp"

namespace bpc {

hipError_t distill_run_f32(const DistillCall &call, DistillRole role, uint8_t *ws, hipStream_t stream) {
  return run_hard<BPC_F32>(call, role, ws, stream);
}

}  // namespace bpc
