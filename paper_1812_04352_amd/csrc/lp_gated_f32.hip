// Gated layers: f32.
#include "lp_gated_impl.h"

namespace lp {

hipError_t gated_forward_f32(const GatedArgs& a, hipStream_t st) { return gated::forward_t<float>(a, st); }
hipError_t gated_backward_f32(const GatedArgs& a, hipStream_t st) { return gated::backward_t<float>(a, st); }

}  // namespace lp
