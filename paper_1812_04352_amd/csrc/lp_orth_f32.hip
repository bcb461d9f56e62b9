// Orthogonalised updates of fp32 gradients: products of floats (split bf16 products).
#include "lp_orth_impl.h"

namespace lp {

hipError_t orth_update_f32(const OrthArgs& a, hipStream_t st) { return orth::update_t<float, float>(a, st); }

}  // namespace lp
