// Gated layers: bf16.
#include "lp_gated_impl.h"

namespace lp {

hipError_t gated_forward_bf16(const GatedArgs& a, hipStream_t st) { return gated::forward_t<__bf16>(a, st); }
hipError_t gated_backward_bf16(const GatedArgs& a, hipStream_t st) { return gated::backward_t<__bf16>(a, st); }

}  // namespace lp
