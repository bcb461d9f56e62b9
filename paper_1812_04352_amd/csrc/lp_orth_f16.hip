// Orthogonalised updates of 16-bit gradients: products of f16 values.
#include "lp_orth_impl.h"

namespace lp {

hipError_t orth_update_bf16(const OrthArgs& a, hipStream_t st) { return orth::update_t<__bf16, _Float16>(a, st); }
hipError_t orth_update_f16(const OrthArgs& a, hipStream_t st) { return orth::update_t<_Float16, _Float16>(a, st); }

}  // namespace lp
