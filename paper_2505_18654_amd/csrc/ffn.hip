// Gated feed-forward block (bf16):
//   pre = x W_in              W_in [d, 2f]: gate columns, then up columns
//   h   = silu(gate) * up     [T, f]
//   y   = h W_out (+ r)       W_out [f, d]
// and its backward pass
//   dgate = dh up silu'(gate), dup = dh silu(gate) with dh = dy W_out^T
//   dx = dpre W_in^T, dW_in = x^T dpre, dW_out = h^T dy.
// Both projections, the activation and the product are one kernel (a tile holds the gate and the up
// columns of the same numbers, in the same lanes), and so are dh and dpre: neither the pre-activations
// (in serving) nor dh go through memory.  Roundings to bf16: h and dpre, as operands of the next product;
// pre, which the forward keeps for the backward (its tensors of the kind are bf16).
#include "gemm_wide.h"

namespace mtgr {

constexpr int FEW_ROWS = 1024;

static void tiles_of(GemmArgs* g, int ntile) {
    g->mblocks = (int)((g->M + WBM - 1) / WBM);
    g->nblocks = (int)((g->N + ntile - 1) / ntile);
    g->splits = 1;
    g->ks_per_split = (int)((g->K + WBK - 1) / WBK);
    g->wide = true;
}

hipError_t launch_ffn_fwd(const FfnArgs& a, hipStream_t s) {
    if (a.T <= FEW_ROWS) return launch_ffn_rows(a, s);
    GemmArgs g{};
    g.layout = GEMM_NN;
    g.M = a.T;
    g.N = a.f;
    g.K = a.d;
    g.A = a.x;
    g.lda = a.ld_x;
    g.B = a.w_in;
    g.ldb = a.ld_win;
    g.C = a.pre;
    g.ldc = a.ld_pre;
    g.C2 = a.h;
    g.ldc2 = a.ld_h;
    tiles_of(&g, WBN / 2);
    hipError_t e = a.pre ? wide_launch<GEMM_NN, GEMM_EPI_GATED_SAVE, false>(g, s)
                         : wide_launch<GEMM_NN, GEMM_EPI_GATED, false>(g, s);
    if (e != hipSuccess) return e;
    g = GemmArgs{};
    g.layout = GEMM_NN;
    g.M = a.T;
    g.N = a.d;
    g.K = a.f;
    g.A = a.h;
    g.lda = a.ld_h;
    g.B = a.w_out;
    g.ldb = a.ld_wout;
    g.C = a.y;
    g.ldc = a.ld_y;
    g.R = a.residual;
    g.ldr = a.ld_r;
    if (a.residual) {
        tiles_of(&g, WBN);
        return wide_launch<GEMM_NN, GEMM_EPI_RESIDUAL, false>(g, s);
    }
    gemm_plan(&g);
    return launch_gemm_bf16(g, s);
}

// Workspace of the backward: dpre [T, 2f] bf16, then the larger of the weight gradients' partials.
static size_t dpre_bytes(long long T, int f) { return ((size_t)T * 2 * f * 2 + 255) & ~(size_t)255; }

size_t ffn_bwd_workspace_bytes(long long T, int d, int f) {
    return dpre_bytes(T, f) + std::max(gemm_workspace_bytes(GEMM_TN, d, 2ll * f, T), gemm_workspace_bytes(GEMM_TN, f, d, T));
}

hipError_t launch_ffn_bwd(const FfnArgs& a, void* workspace, hipStream_t s) {
    if (a.T == 0) {
        const hipError_t z = launch_zero_rows(a.d, a.f / 4, a.dw_in, a.ld_win / 8, s);
        return z != hipSuccess ? z : launch_zero_rows(a.f, a.d / 8, a.dw_out, a.ld_wout / 8, s);
    }
    char* dpre = (char*)workspace;
    float* partial = (float*)(dpre + dpre_bytes(a.T, a.f));
    GemmArgs g{};
    g.layout = GEMM_NT;
    g.M = a.T;
    g.N = a.f;
    g.K = a.d;
    g.A = a.dy;
    g.lda = a.ld_y;
    g.B = a.w_out;
    g.ldb = a.ld_wout;
    g.C = dpre;
    g.ldc = 2ll * a.f;
    g.R = a.pre;
    g.ldr = a.ld_pre;
    tiles_of(&g, WBN);
    hipError_t e = wide_launch<GEMM_NT, GEMM_EPI_GATED_BWD, false>(g, s);
    if (e != hipSuccess) return e;
    auto product = [&](int layout, long long M, long long N, long long K, const void* A, long long lda, const void* B,
                       long long ldb, void* C, long long ldc) {
        GemmArgs p{};
        p.layout = layout;
        p.M = M;
        p.N = N;
        p.K = K;
        p.A = A;
        p.lda = lda;
        p.B = B;
        p.ldb = ldb;
        p.C = C;
        p.ldc = ldc;
        gemm_plan(&p);
        p.partial = partial;
        return launch_gemm_bf16(p, s);
    };
    const long long f2 = 2ll * a.f;
    if ((e = product(GEMM_NT, a.T, a.d, f2, dpre, f2, a.w_in, a.ld_win, a.dx, a.ld_x)) != hipSuccess) return e;
    if ((e = product(GEMM_TN, a.d, f2, a.T, a.x, a.ld_x, dpre, f2, a.dw_in, a.ld_win)) != hipSuccess) return e;
    return product(GEMM_TN, a.f, a.d, a.T, a.h, a.ld_h, a.dy, a.ld_y, a.dw_out, a.ld_wout);
}

}  // namespace mtgr
