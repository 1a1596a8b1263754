// The encoder layer's products on 256 x 256 tiles: instances of the kernel of gemm_wide.h.
#include "gemm_wide.h"

namespace mtgr {

hipError_t launch_gemm_wide(const GemmArgs& a, hipStream_t s) {
    TileArgs g{};
    (GemmArgs&)g = a;
    if (g.layout == GEMM_TN)
        return g.colsum ? wide_launch<GEMM_TN, GEMM_EPI_NONE, true>(g, s)
                        : wide_launch<GEMM_TN, GEMM_EPI_NONE, false>(g, s);
    if (g.layout == GEMM_NN) {
        if (g.epilogue == GEMM_EPI_BIAS_SILU) return wide_launch<GEMM_NN, GEMM_EPI_BIAS_SILU, false>(g, s);
        if (g.epilogue == GEMM_EPI_BIAS_RESIDUAL) return wide_launch<GEMM_NN, GEMM_EPI_BIAS_RESIDUAL, false>(g, s);
        return wide_launch<GEMM_NN, GEMM_EPI_NONE, false>(g, s);
    }
    if (g.epilogue == GEMM_EPI_BIAS_SILU) return wide_launch<GEMM_NT, GEMM_EPI_BIAS_SILU, false>(g, s);
    if (g.epilogue == GEMM_EPI_BIAS_RESIDUAL) return wide_launch<GEMM_NT, GEMM_EPI_BIAS_RESIDUAL, false>(g, s);
    return wide_launch<GEMM_NT, GEMM_EPI_NONE, false>(g, s);
}

}  // namespace mtgr
