// Gated layers: f16.
#include "lp_gated_impl.h"

namespace lp {

hipError_t gated_forward_f16(const GatedArgs& a, hipStream_t st) { return gated::forward_t<_Float16>(a, st); }
hipError_t gated_backward_f16(const GatedArgs& a, hipStream_t st) { return gated::backward_t<_Float16>(a, st); }

}  // namespace lp
