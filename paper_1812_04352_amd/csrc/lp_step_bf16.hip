// Layer steps of any width, 8-bit checkpoints and heads over large vocabularies: bf16.
#include <algorithm>

#include "lp_labels_impl.h"
#include "lp_step_impl.h"

namespace lp {

hipError_t step_forward_bf16(const StepArgs& a, hipStream_t st) { return wide::step_forward_t<__bf16>(a, st); }
hipError_t step_backward_bf16(const StepArgs& a, hipStream_t st) { return wide::step_backward_t<__bf16>(a, st); }
hipError_t ck_store_bf16(const void* x, int8_t* x8, uint8_t* xe, long B, int q, hipStream_t st) {
  return wide::ck_store_t<__bf16>(x, x8, xe, B, q, st);
}
hipError_t ck_load_bf16(const int8_t* x8, const uint8_t* xe, void* x, long B, int q, hipStream_t st) {
  return wide::ck_load_t<__bf16>(x8, xe, x, B, q, q, st);
}
hipError_t loss_labels_bf16(const LabelArgs& a, hipStream_t st) { return wide::loss_labels_t<__bf16>(a, st); }

}  // namespace lp
