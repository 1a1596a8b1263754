// Host-side argument structs and launch entry points behind include/mtgr_block.h, and the arguments of the
// tile kernels that its operators share with the encoder layer's products.
#pragma once

#include <algorithm>

#include "mtgr_internal.h"

namespace mtgr {

// Epilogues of gemm_wide.h alone (ffn.hip, softmax_loss.hip): C = acc + R; the gated products; softmax
// statistics and gradient of a class tile; fp32 partials that add up over calls; a weight gradient
// over rows counted on the device, as fp32 partials or finished; fp32 partials of an NN or NT product.
constexpr int GEMM_EPI_RESIDUAL = 3, GEMM_EPI_GATED = 4, GEMM_EPI_GATED_SAVE = 5, GEMM_EPI_GATED_BWD = 6,
              GEMM_EPI_SM_STATS = 7, GEMM_EPI_SM_GRAD = 8, GEMM_EPI_ACC = 9, GEMM_EPI_ROWS = 10, GEMM_EPI_ROWS_DIRECT = 11,
              GEMM_EPI_PART = 12;
struct TileArgs : GemmArgs {
    // The products of the softmax loss:
    const int* rows;          // number of token rows on the device (at most M, or K of TN); behind it a float, the
                              // largest gradient of a row's loss (SM_GRAD), and tile_run's number (softmax_tiles.h)
    int b_rows;               // rows of B (classes), where they are fewer than N or K
    int class0;               // first class of the piece
    int group_m;              // m blocks that an XCD's workgroups share
    int accumulate;           // ACC: add to the partials of the calls before; ks_per_split is the k steps of the first
                              // call, by which all of them are split (256 x 256 tiles)
    float scale;              // z = scale acc + bias, in units of log 2; ROWS_DIRECT: C = scale max |g| acc
    float2* stats;            // SM_STATS: (reference, sum) per row and wave, [4 chunks][M] (128 x 128 tiles: [2 nblocks][M])
    const int4* row_info;     // SM_GRAD: per row (lse, gradient of its loss, label, factor 2^-low of lse), whole m blocks
    float* col_partial;       // SM_GRAD: [2 mblocks][N] column sums, or NULL
};
hipError_t launch_split_reduce(const GemmArgs& g, hipStream_t s);   // C and colsum from a TN product's partials (gemm.hip)

// Zero rows of `chunks` 16-byte chunks, `ld` chunks apart.
hipError_t launch_zero_rows(long long rows, int chunks, void* p, long long ld, hipStream_t s);

// Dropout (dropout.hip).
struct DropoutArgs {
    long long rows;
    int cols;
    const void* x;
    long long ld_x;
    const void* residual;     // or NULL
    long long ld_r;
    void* out;
    long long ld_out;
    const unsigned long long* rng;   // device: seed, step
    uint32_t site;
    uint32_t threshold;       // kept: word >= threshold
    float scale;              // 1 / (1 - p)
};
hipError_t launch_dropout(const DropoutArgs& a, bool bf16, hipStream_t s);

// Gated feed-forward block (ffn.hip).
struct FfnArgs {
    long long T;
    int d, f;
    const void *x, *w_in, *w_out, *residual, *dy;
    void *y, *pre, *h;        // pre NULL: not kept
    void *dx, *dw_in, *dw_out;
    long long ld_x, ld_win, ld_wout, ld_y, ld_r, ld_pre, ld_h;
};
size_t ffn_fwd_workspace_bytes(long long T, int d, int f, bool save);
hipError_t launch_ffn_fwd(const FfnArgs& a, void* workspace, hipStream_t s);
// Its two products for few tokens (ffn_rows.hip), of so many columns per workgroup.
constexpr int FFN_HIDDEN_COLUMNS = 32, FFN_OUT_COLUMNS = 32;
bool ffn_rows_fit(long long T, int N, int columns);
hipError_t launch_ffn_rows_hidden(const FfnArgs& a, hipStream_t s);
hipError_t launch_ffn_rows_out(const FfnArgs& a, hipStream_t s);
size_t ffn_bwd_workspace_bytes(long long T, int d, int f);
hipError_t launch_ffn_bwd(const FfnArgs& a, void* workspace, hipStream_t s);
// The kernels that a pass runs on, as text (snprintf's result).
int ffn_fwd_kernels(long long T, int d, int f, bool save, bool residual, char* text, size_t n);
int ffn_bwd_kernels(long long T, int d, int f, char* text, size_t n);

// Softmax loss over a class set (softmax_loss.hip).
struct SoftmaxLossArgs {
    long long N;
    int V, d;
    const void *x, *w;
    long long ld_x, ld_w;
    const void* targets;
    bool targets64;
    const float* bias;        // [V] or NULL
    float scale;
    float *loss, *lse;        // forward: written; backward: lse read
    const float* dloss;
    void *dx, *dw;            // layouts of x, w
    float* dbias;             // or NULL
};
size_t softmax_loss_workspace_bytes(long long N, int V, int d, bool backward);
hipError_t launch_softmax_loss_fwd(const SoftmaxLossArgs& a, void* workspace, hipStream_t s);
hipError_t launch_softmax_loss_bwd(const SoftmaxLossArgs& a, void* workspace, hipStream_t s);
int softmax_loss_kernels(long long N, int V, int d, bool backward, long long labels, char* text, size_t n);

}  // namespace mtgr
