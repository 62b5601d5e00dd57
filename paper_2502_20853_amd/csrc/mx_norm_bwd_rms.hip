// Backward pass of the gated residual, RMS norms.
#include "mx_norm_bwd.hpp"

namespace mxl {

hipError_t launch_norm_bwd_rms(const NormGradArgs& a, bool x_bf16, bool u_bf16, bool eight, RowEnd end, int v, BwdPart part, dim3 grid, uint32_t threads, size_t lds, hipStream_t st)
{
    return launch_norm_bwd<false>(a, x_bf16, u_bf16, eight, end, v, part, grid, threads, lds, st);
}

}  // namespace mxl
