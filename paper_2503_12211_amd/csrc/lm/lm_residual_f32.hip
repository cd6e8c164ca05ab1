// The residual step for fp32 storage (a file of its own: the two storage types compile side by side).
#include "lm_residual.h"

namespace stl {
namespace lm {

hipError_t residual_forward_f32(const ResidualArgs &a, void *Xout, void *Z, hipStream_t s) { return residual_forward<float>(a, Xout, Z, s); }

hipError_t residual_backward_f32(const ResidualArgs &a, const ResidualGrads &g, const ResidualItems &it, int grid, hipStream_t s)
{
    return residual_backward<float>(a, g, it, grid, s);
}

}  // namespace lm
}  // namespace stl
