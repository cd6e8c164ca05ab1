// Internal launcher interface between the C ABI (lm_api.hip) and the kernels of the residual step and the vocabulary loss.
#pragma once
#include "../stl_kernels.h"

namespace stl {
namespace lm {

// fills with zero bits (a kernel: memset nodes in a captured graph are avoided); bytes a multiple of 4, p aligned to 4
hipError_t launch_zero(void *p, size_t bytes, hipStream_t s);

// ---- residual step (lm_residual.h) -------------------------------------------------------------------------------------------
struct ResidualArgs {
    int rows, n;
    int per_gate;                            // rows that share a row of the gate
    float skip, scale, eps;
    bool post, pre, center;
    const void *X, *H, *gate, *w_post, *b_post, *w_pre, *b_pre;      // storage type; gate, weights and offsets may be NULL
};
struct ResidualGrads {                       // what the backward pass reads besides (X is the stream behind the sum) and writes; any may be NULL
    const void *dXout, *dZ;
    void *dX, *dH;
    float *dgate, *dw_post, *db_post, *dw_pre, *db_pre;
    int accumulate;
};
constexpr int kResidualWidest = 32768;       // a row is held in the registers of one workgroup
size_t residual_workspace_bytes(int rows, int n, int per_gate);
hipError_t launch_residual_forward(int dtype, const ResidualArgs &a, void *Xout, void *Z, hipStream_t s);
hipError_t launch_residual_backward(int dtype, const ResidualArgs &a, const ResidualGrads &g, void *ws, hipStream_t s);

}  // namespace lm
}  // namespace stl
