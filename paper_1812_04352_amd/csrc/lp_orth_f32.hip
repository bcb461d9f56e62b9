// Orthogonalised updates of fp32 gradients: products of values in two f16 parts.
#include "lp_orth_impl.h"

namespace lp {

hipError_t orth_update_f32(const OrthArgs& a, hipStream_t st) { return orth::update_t<float, mm::Duo>(a, st); }

}  // namespace lp
