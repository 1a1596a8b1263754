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
//
// h and dpre are rounded to bf16 because the next product's matrix instructions take bf16 operands (split into two bf16
// numbers each they would double that product); every sum is fp32, and h and dpre are formed from unrounded sums.
//
// Bound by the matrix cores (power) and, beside them, by what the epilogues read and write and compute.
// Large products run on 256 x 256 tiles (the second one of a training forward partly on the 256 x 128 tiles of gemm.hip),
// fewer tiles than CUs on 128 x 128 ones (gemm_mid.h), deep ones of them split over k; few tokens on a kernel of their
// own (ffn_rows.hip).  Measured in a kernel trace of ten calls in a row (in short bursts, as the rules' figures below were
// taken, the clock is up to a fifth higher):
// - 75,132 tokens, 512 / 1408, training: first product 292 us (0.74 PFLOP/s; 635 MB written), second 132 (0.82);
// - 69,563 tokens, 1024 / 2816, training: 915 (0.88) and 449 us (0.89); backward: dpre 555 us (0.72; 1.6 GB of
//   pre read and dpre written), dx 734 (1.09), the weight gradients 763 and 401 (1.05, 1.00), their splits' sums 43;
// - 6,418 tokens, 256 / 704, backward: dpre 16.7 us, the three products behind it in one launch 27.1, the sums 7.1.
#include <stdio.h>

#include "gemm_mid.h"

namespace mtgr {

namespace {

// out = sum of the K splits' partials (+ residual), rounded once.
struct SumArgs {
    const float* partial;
    int splits, cols;
    long long rows;
    uint16_t* out;
    long long ld_out;
    const uint16_t* residual;
    long long ld_r;
};

__device__ __forceinline__ void sum_splits(const SumArgs& a, int block, int blocks) {
    const int ch = a.cols / 4;
    const long long n = a.rows * ch;
    for (long long i = (long long)block * 256 + threadIdx.x; i < n; i += (long long)blocks * 256) {
        const long long r = i / ch;
        const int c = (int)(i % ch) * 4;
        floatx4 s = ((const floatx4*)a.partial)[i];
#pragma unroll 4
        for (int k = 1; k < a.splits; k++) s += ((const floatx4*)a.partial)[k * n + i];
        if (a.residual) {
            const uint2 v = *(const uint2*)(a.residual + r * a.ld_r + c);
            s += floatx4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                         __uint_as_float(v.y & 0xffff0000u)};
        }
        *(uint2*)(a.out + r * a.ld_out + c) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
    }
}

// Up to three products' sums; the second one's workgroups from `first` on, the third one's from `second` on.
__global__ __launch_bounds__(256) void ffn_sum_kernel(SumArgs a, SumArgs b, SumArgs c, int first, int second) {
    if ((int)blockIdx.x < first) sum_splits(a, blockIdx.x, first);
    else if ((int)blockIdx.x < second) sum_splits(b, blockIdx.x - first, second - first);
    else sum_splits(c, blockIdx.x - second, gridDim.x - second);
}

SumArgs sum_of(const TileArgs& g) {
    return {g.partial, g.splits, (int)g.N, g.M, (uint16_t*)g.C, g.ldc, (const uint16_t*)g.R, g.ldr};
}

int sum_grid(const TileArgs& g) { return (int)std::min((g.M * (g.N / 4) + 255) / 256, 4096ll); }

TileArgs product(int layout, long long M, long long N, long long K, const void* A, long long lda, const void* B,
                 long long ldb, void* C, long long ldc) {
    TileArgs g{};
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

// What the epilogues of the gated products take beside the figures of tiles_of, us: storing pre, and reading it with
// silu' in the backward.  On 256 x 256 tiles nothing runs beside them (6,418 tokens, 1024 / 2816, dpre: 79 us on 256 x 256
// tiles, 68 on 128 x 128; 75,132, 512 / 1408: 219, 233; 8,000, 512 / 1408, training forward: 38, 36; 20,000: 74, 78).
constexpr double WIDE_SAVE = 3.0, WIDE_BWD = 14.0, MID_BWD = 6.0;

// C = A B (NN) or A B^T (NT), plus the residual R where there is one; `partial` holds the K splits' sums.
// Where 256 x 256 tiles are estimated to end before 128 x 128 ones, an NN product without a residual goes by gemm_plan,
// which may take 256 x 128 tiles (us on 256 x 128, 256 x 256 and 128 x 128 tiles: 33,001 tokens, 512 / 1408: 67, 76, 71;
// 40,001: 73, 76, 81; 75,132: 120, 120, 133; 17,001, 1024 / 2816: 122, 136, 126; 20,001: 132, 138, 138); those have no
// epilogue for a residual.  NT products stay on 256 x 256 tiles (33,001, 512 / 1408: 126, 128, 117; 40,001: 148, 136,
// 152; 45,001: 150, 134, 166; 17,001, 1024 / 2816: 259, 250, 262; 22,001: 283, 257, 286; 70,001, 256 / 704: 78, 74, 76).
template <int LAYOUT>
static hipError_t deep_product(TileArgs g, const Tiles& t, float* partial, hipStream_t s) {
    if constexpr (LAYOUT == GEMM_NN) {
        if (!t.mid && !g.R) {
            gemm_plan(&g);
            return launch_gemm_bf16(g, s);
        }
    }
    set_tiles(&g, t);
    if (!t.mid) return wide_launch<LAYOUT, LAYOUT == GEMM_NN ? GEMM_EPI_RESIDUAL : GEMM_EPI_NONE, false>(g, s);
    if constexpr (LAYOUT == GEMM_NN) {
        if (t.splits == 1 && g.R) return mid_launch<GEMM_NN, GEMM_EPI_RESIDUAL>(g, s);
    }
    if (t.splits == 1) return mid_launch<LAYOUT, GEMM_EPI_NONE>(g, s);
    g.partial = partial;
    const hipError_t e = mid_launch<LAYOUT, GEMM_EPI_PART>(g, s);
    if (e != hipSuccess) return e;
    ffn_sum_kernel<<<sum_grid(g), 256, 0, s>>>(sum_of(g), SumArgs{}, SumArgs{}, sum_grid(g), sum_grid(g));
    return hipGetLastError();
}

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

namespace {

// The kernels of the forward's two products: the one for few rows, or tiles.
struct ForwardPlan {
    bool rows_hidden, rows_out;
    Tiles hidden, out;
};

// The second product on the kernel for few rows: its waves go through k alone (no launch adds partials), so that a
// deep k favours the tiles split over k: 64 .. 128 tokens, f = 1408: 8.7 us, 11.2 there; f = 2816: 15, 11.3; up to
// 32 tokens, f = 2816: 7.5 .. 10.8, 9.6 .. 10.1; 312 tokens, f = 2048: 11.5, 14.4.
ForwardPlan plan_forward(long long T, int d, int f, bool save) {
    ForwardPlan p{};
    p.rows_hidden = ffn_rows_fit(T, f, FFN_HIDDEN_COLUMNS);
    if (!p.rows_hidden) p.hidden = plan(T, f, d, WBN / 2, save ? WIDE_SAVE : 0.0);
    p.out = plan_deep(T, d, f);
    const double us = T <= 16 ? 1.0 + 1.4 * f / 512 : 1.5 + (T <= 32 ? 0.85 : 1.25) * f / 256;
    p.rows_out = ffn_rows_fit(T, d, FFN_OUT_COLUMNS) && us < p.out.us;
    return p;
}

}  // namespace

// Workspace of the forward: h, where the caller does not keep it, and the second product's partials.
size_t ffn_fwd_workspace_bytes(long long T, int d, int f, bool save) {
    const ForwardPlan p = plan_forward(T, d, f, save);
    return (save ? 0 : align256((size_t)T * f * 2)) + (p.rows_out ? 0 : partial_bytes(p.out, T, d));
}

hipError_t launch_ffn_fwd(const FfnArgs& f, void* workspace, hipStream_t s) {
    FfnArgs a = f;
    float* partial = (float*)workspace;
    if (!a.pre) {
        a.h = workspace;
        a.ld_h = a.f;
        partial = (float*)((char*)workspace + align256((size_t)a.T * a.f * 2));
    }
    const ForwardPlan p = plan_forward(a.T, a.d, a.f, a.pre != nullptr);
    hipError_t e;
    if (p.rows_hidden) {
        e = launch_ffn_rows_hidden(a, s);
    } else {
        TileArgs g = product(GEMM_NN, a.T, a.f, a.d, a.x, a.ld_x, a.w_in, a.ld_win, a.pre, a.ld_pre);
        g.C2 = a.h;
        g.ldc2 = a.ld_h;
        set_tiles(&g, p.hidden);
        if (p.hidden.mid) e = a.pre ? mid_launch<GEMM_NN, GEMM_EPI_GATED_SAVE>(g, s) : mid_launch<GEMM_NN, GEMM_EPI_GATED>(g, s);
        else e = a.pre ? wide_launch<GEMM_NN, GEMM_EPI_GATED_SAVE, false>(g, s) : wide_launch<GEMM_NN, GEMM_EPI_GATED, false>(g, s);
    }
    if (e != hipSuccess) return e;
    if (p.rows_out) return launch_ffn_rows_out(a, s);
    TileArgs g = product(GEMM_NN, a.T, a.d, a.f, a.h, a.ld_h, a.w_out, a.ld_wout, a.y, a.ld_y);
    g.R = a.residual;
    g.ldr = a.ld_r;
    return deep_product<GEMM_NN>(g, p.out, partial, s);
}

namespace {

// The backward's products: dpre, and the three behind it: dx, dW_in and dW_out, one after the other, or in one launch on
// 128 x 128 tiles, their k cut into about equal numbers of steps, and one launch that adds up all partials.
struct BackwardPlan {
    bool together;
    Tiles dpre;               // of dh = dy W_out^T with the gradient of the activation
    Tiles dx, in, out;
    size_t bytes;             // of the partials
};

BackwardPlan plan_backward(long long T, int d, int f) {
    BackwardPlan p{};
    p.dpre = plan(T, f, d, WBN, WIDE_BWD, MID_BWD);
    p.dx = plan_deep(T, d, 2ll * f);
    p.in = plan_split(d, 2ll * f, T, true);
    p.out = plan_split(f, d, T, true);
    const Tiles x = tiles_of(true, T, d, 2ll * f, WBN, 1, false), i = tiles_of(true, d, 2ll * f, T, WBN, 1, false),
                o = tiles_of(true, f, d, T, WBN, 1, false);
    const double tx = (double)x.mblocks * x.nblocks, tg = (double)i.mblocks * i.nblocks + (double)o.mblocks * o.nblocks;
    const unsigned nx = (2u * f + WBK - 1) / WBK, ng = (unsigned)((T + WBK - 1) / WBK);
    double best = p.dx.us + p.in.us + p.out.us;
    int sx = 0, sg = 0;
    for (unsigned steps = 4; steps <= 128; steps += steps / 2 < 4 ? 2 : steps / 4) {
        const unsigned a = (nx + steps - 1) / steps, b = (ng + steps - 1) / steps;
        const double qx = (nx + a - 1) / a, qg = (ng + b - 1) / b, items = tx * a + tg * b, top = std::max(qx, qg);
        // (beyond one round a workgroup follows another as soon as it can: the mean, and half of a last one)
        const double us = (items <= MID_WORKGROUPS ? MID_START + (items > WIDE_WORKGROUPS ? MID_STEP : MID_STEP_ALONE) * top
                           : (tx * a * (MID_START + MID_STEP * qx) + tg * b * (MID_START + MID_STEP * qg)) / MID_WORKGROUPS +
                                 0.5 * (MID_START + MID_STEP * top)) +
                          partials_us((double)a * T * d + 3.0 * b * d * f);
        if (us < best && a <= 64 && b <= 64) {
            best = us;
            sx = (int)a;
            sg = (int)b;
        }
    }
    const size_t weights = (size_t)d * f * sizeof(float);
    p.together = sx > 0;
    if (p.together) {
        p.dx = x;
        p.in = i;
        p.out = o;
        p.dx.splits = sx;
        p.in.splits = p.out.splits = sg;
        p.bytes = (size_t)sx * T * d * sizeof(float) + 3 * sg * weights;
    } else {
        p.bytes = std::max({partial_bytes(p.dx, T, d), 2 * p.in.splits * weights, p.out.splits * weights});
    }
    return p;
}

}  // namespace

// Workspace of the backward: dpre [T, 2f] bf16, then the partials.
size_t ffn_bwd_workspace_bytes(long long T, int d, int f) {
    return align256((size_t)T * 2 * f * 2) + plan_backward(T, d, f).bytes;
}

hipError_t launch_ffn_bwd(const FfnArgs& a, void* workspace, hipStream_t s) {
    if (a.T == 0) {
        const hipError_t z = launch_zero_rows(a.d, a.f / 4, a.dw_in, a.ld_win / 8, s);
        return z != hipSuccess ? z : launch_zero_rows(a.f, a.d / 8, a.dw_out, a.ld_wout / 8, s);
    }
    const long long f2 = 2ll * a.f;
    char* dpre = (char*)workspace;
    float* partial = (float*)(dpre + align256((size_t)a.T * f2 * 2));
    TileArgs g = product(GEMM_NT, a.T, a.f, a.d, a.dy, a.ld_y, a.w_out, a.ld_wout, dpre, f2);
    g.R = a.pre;
    g.ldr = a.ld_pre;
    const BackwardPlan p = plan_backward(a.T, a.d, a.f);
    set_tiles(&g, p.dpre);
    hipError_t e = p.dpre.mid ? mid_launch<GEMM_NT, GEMM_EPI_GATED_BWD>(g, s) : wide_launch<GEMM_NT, GEMM_EPI_GATED_BWD, false>(g, s);
    if (e != hipSuccess) return e;
    TileArgs x = product(GEMM_NT, a.T, a.d, f2, dpre, f2, a.w_in, a.ld_win, a.dx, a.ld_x);
    TileArgs wi = product(GEMM_TN, a.d, f2, a.T, a.x, a.ld_x, dpre, f2, a.dw_in, a.ld_win);
    TileArgs wo = product(GEMM_TN, a.f, a.d, a.T, a.h, a.ld_h, a.dy, a.ld_y, a.dw_out, a.ld_wout);
    set_tiles(&wi, p.in);
    set_tiles(&wo, p.out);
    if (p.together) {
        set_tiles(&x, p.dx);
        x.partial = partial;
        wi.partial = x.partial + (size_t)x.splits * a.T * a.d;
        wo.partial = wi.partial + (size_t)wi.splits * a.d * f2;
        const int first = mid_grid(x), second = first + mid_grid(wi), sx = sum_grid(x), si = sx + sum_grid(wi);
        gemm_mid_trio_kernel<GEMM_NT, GEMM_EPI_PART, GEMM_TN, GEMM_EPI_PART><<<second + mid_grid(wo), 256, 0, s>>>(x, wi, wo, first, second);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        ffn_sum_kernel<<<si + sum_grid(wo), 256, 0, s>>>(sum_of(x), sum_of(wi), sum_of(wo), sx, si);
        return hipGetLastError();
    }
    if ((e = deep_product<GEMM_NT>(x, p.dx, partial, s)) != hipSuccess) return e;
    wi.partial = wo.partial = partial;
    auto gradient = [&](const TileArgs& w) {
        const hipError_t r = w.wide ? wide_launch<GEMM_TN, GEMM_EPI_NONE, false>(w, s) : mid_launch<GEMM_TN, GEMM_EPI_PART>(w, s);
        return r != hipSuccess ? r : launch_split_reduce(w, s);
    };
    e = gradient(wi);
    return e != hipSuccess ? e : gradient(wo);
}

// As deep_product chooses, for the text below.
static TilesName deep_name(int layout, const Tiles& t, bool residual, long long M, long long N, long long K) {
    if (t.mid || layout == GEMM_NT || residual) return tiles_name(t);
    TileArgs g = product(layout, M, N, K, nullptr, K, nullptr, N, nullptr, N);
    gemm_plan(&g);
    return tiles_name(g.wide ? "256x256" : "256x128", 1);
}

int ffn_fwd_kernels(long long T, int d, int f, bool save, bool residual, char* text, size_t n) {
    const ForwardPlan p = plan_forward(T, d, f, save);
    return snprintf(text, n, "hidden=%s h=%s out=%s", p.rows_hidden ? "rows" : tiles_name(p.hidden).text,
                    p.rows_hidden || p.hidden.mid || h_stays(T, f) ? "cached" : "streamed",
                    p.rows_out ? "rows" : deep_name(GEMM_NN, p.out, residual, T, d, f).text);
}

int ffn_bwd_kernels(long long T, int d, int f, char* text, size_t n) {
    const BackwardPlan p = plan_backward(T, d, f);
    return snprintf(text, n, "dpre=%s store=%s together=%d dx=%s dw_in=%s dw_out=%s", tiles_name(p.dpre).text,
                    p.dpre.mid || dpre_stays(T, f) ? "cached" : "streamed", p.together,
                    p.together ? tiles_name(p.dx).text : deep_name(GEMM_NT, p.dx, false, T, d, 2ll * f).text,
                    tiles_name(p.in).text, tiles_name(p.out).text);
}

}  // namespace mtgr
