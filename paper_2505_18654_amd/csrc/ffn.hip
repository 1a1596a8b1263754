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
#include "gemm_mid.h"

namespace mtgr {

namespace {

// out = sum of the K splits' partials (+ residual), rounded once.
__global__ __launch_bounds__(256) void ffn_sum_kernel(const float* partial, int splits, long long rows, int cols, uint16_t* out,
                                                      long long ld_out, const uint16_t* residual, long long ld_r) {
    const int ch = cols / 4;
    const long long n = rows * ch;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const long long r = i / ch;
        const int c = (int)(i % ch) * 4;
        floatx4 s = ((const floatx4*)partial)[i];
#pragma unroll 4
        for (int k = 1; k < splits; k++) s += ((const floatx4*)partial)[k * n + i];
        if (residual) {
            const uint2 v = *(const uint2*)(residual + r * ld_r + c);
            s += floatx4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                         __uint_as_float(v.y & 0xffff0000u)};
        }
        *(uint2*)(out + r * ld_out + c) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
    }
}

GemmArgs product(int layout, long long M, long long N, long long K, const void* A, long long lda, const void* B,
                 long long ldb, void* C, long long ldc) {
    GemmArgs g{};
    g.layout = layout;
    g.M = M;
    g.N = N;
    g.K = K;
    g.A = A;
    g.lda = lda;
    g.B = B;
    g.ldb = ldb;
    g.C = C;
    g.ldc = ldc;
    return g;
}

}  // namespace

// C = A B (NN) or A B^T (NT), plus the residual R where there is one; `partial` holds the K splits' sums.
template <int LAYOUT>
static hipError_t deep_product(GemmArgs g, float* partial, hipStream_t s) {
    const Tiles t = plan_deep(g.M, g.N, g.K);
    if (!t.mid && (LAYOUT == GEMM_NT || !g.R)) {
        gemm_plan(&g);
        return launch_gemm_bf16(g, s);
    }
    set_tiles(&g, t);
    if constexpr (LAYOUT == GEMM_NN) {
        if (!t.mid) return wide_launch<GEMM_NN, GEMM_EPI_RESIDUAL, false>(g, s);
        if (t.splits == 1 && g.R) return mid_launch<GEMM_NN, GEMM_EPI_RESIDUAL>(g, s);
    }
    if (t.splits == 1) return mid_launch<LAYOUT, GEMM_EPI_NONE>(g, s);
    g.partial = partial;
    const hipError_t e = mid_launch<LAYOUT, GEMM_EPI_PART>(g, s);
    if (e != hipSuccess) return e;
    const int grid = (int)std::min((g.M * (g.N / 4) + 255) / 256, 8192ll);
    ffn_sum_kernel<<<grid, 256, 0, s>>>(partial, g.splits, g.M, (int)g.N, (uint16_t*)g.C, g.ldc, (const uint16_t*)g.R, g.ldr);
    return hipGetLastError();
}

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Workspace of the forward: h, where the caller does not keep it, and the second product's partials.
size_t ffn_fwd_workspace_bytes(long long T, int d, int f, bool save) {
    const bool few = ffn_rows_fit(T, d, FFN_OUT_COLUMNS);
    return (save ? 0 : align256((size_t)T * f * 2)) + (few ? 0 : partial_bytes(plan_deep(T, d, f), T, d));
}

hipError_t launch_ffn_fwd(const FfnArgs& f, void* workspace, hipStream_t s) {
    FfnArgs a = f;
    float* partial = (float*)workspace;
    if (!a.pre) {
        a.h = workspace;
        a.ld_h = a.f;
        partial = (float*)((char*)workspace + align256((size_t)a.T * a.f * 2));
    }
    hipError_t e;
    if (ffn_rows_fit(a.T, a.f, FFN_HIDDEN_COLUMNS)) {
        e = launch_ffn_rows_hidden(a, s);
    } else {
        GemmArgs g = product(GEMM_NN, a.T, a.f, a.d, a.x, a.ld_x, a.w_in, a.ld_win, a.pre, a.ld_pre);
        g.C2 = a.h;
        g.ldc2 = a.ld_h;
        const Tiles t = plan(a.T, a.f, a.d, 2);
        set_tiles(&g, t);
        if (t.mid) e = a.pre ? mid_launch<GEMM_NN, GEMM_EPI_GATED_SAVE>(g, s) : mid_launch<GEMM_NN, GEMM_EPI_GATED>(g, s);
        else e = a.pre ? wide_launch<GEMM_NN, GEMM_EPI_GATED_SAVE, false>(g, s) : wide_launch<GEMM_NN, GEMM_EPI_GATED, false>(g, s);
    }
    if (e != hipSuccess) return e;
    if (ffn_rows_fit(a.T, a.d, FFN_OUT_COLUMNS)) return launch_ffn_rows_out(a, s);
    GemmArgs g = product(GEMM_NN, a.T, a.d, a.f, a.h, a.ld_h, a.w_out, a.ld_wout, a.y, a.ld_y);
    g.R = a.residual;
    g.ldr = a.ld_r;
    return deep_product<GEMM_NN>(g, partial, s);
}

// Workspace of the backward: dpre [T, 2f] bf16, then the largest of the three products' partials.
size_t ffn_bwd_workspace_bytes(long long T, int d, int f) {
    const size_t weights = (size_t)d * f * sizeof(float);
    return align256((size_t)T * 2 * f * 2) +
           std::max({plan_split(d, 2ll * f, T, true).splits * 2 * weights, plan_split(f, d, T, true).splits * weights,
                     partial_bytes(plan_deep(T, d, 2ll * f), T, d)});
}

hipError_t launch_ffn_bwd(const FfnArgs& a, void* workspace, hipStream_t s) {
    if (a.T == 0) {
        const hipError_t z = launch_zero_rows(a.d, a.f / 4, a.dw_in, a.ld_win / 8, s);
        return z != hipSuccess ? z : launch_zero_rows(a.f, a.d / 8, a.dw_out, a.ld_wout / 8, s);
    }
    const long long f2 = 2ll * a.f;
    char* dpre = (char*)workspace;
    float* partial = (float*)(dpre + align256((size_t)a.T * f2 * 2));
    GemmArgs g = product(GEMM_NT, a.T, a.f, a.d, a.dy, a.ld_y, a.w_out, a.ld_wout, dpre, f2);
    g.R = a.pre;
    g.ldr = a.ld_pre;
    const Tiles t = plan(a.T, a.f, a.d, 1);
    set_tiles(&g, t);
    hipError_t e = t.mid ? mid_launch<GEMM_NT, GEMM_EPI_GATED_BWD>(g, s) : wide_launch<GEMM_NT, GEMM_EPI_GATED_BWD, false>(g, s);
    if (e != hipSuccess) return e;
    e = deep_product<GEMM_NT>(product(GEMM_NT, a.T, a.d, f2, dpre, f2, a.w_in, a.ld_win, a.dx, a.ld_x), partial, s);
    if (e != hipSuccess) return e;
    auto gradient = [&](GemmArgs w) {
        const Tiles q = plan_split(w.M, w.N, w.K, true);
        set_tiles(&w, q);
        w.partial = partial;
        const hipError_t r = q.mid ? mid_launch<GEMM_TN, GEMM_EPI_NONE>(w, s) : wide_launch<GEMM_TN, GEMM_EPI_NONE, false>(w, s);
        return r != hipSuccess ? r : launch_split_reduce(w, s);
    };
    if ((e = gradient(product(GEMM_TN, a.d, f2, a.T, a.x, a.ld_x, dpre, f2, a.dw_in, a.ld_win))) != hipSuccess) return e;
    return gradient(product(GEMM_TN, a.f, a.d, a.T, a.h, a.ld_h, a.dy, a.ld_y, a.dw_out, a.ld_wout));
}

}  // namespace mtgr
