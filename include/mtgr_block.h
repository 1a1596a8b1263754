/*
 * mtgr_block.h — C ABI of the operators around the encoder layer of include/mtgr_hstu.h: the gated
 * feed-forward block, dropout and the softmax loss over a class set.
 *
 * The conventions are those of include/mtgr_hstu.h: caller-owned device memory, calls asynchronous on
 * `stream`, no allocation, no synchronisation, outputs overwritten, arguments checked on the host before
 * any launch.  Matrices are row-major with a row stride (ld, in elements) of at least their columns, a
 * multiple of 16 bytes, below 2^22; their base is 16-byte aligned.  Outputs do not overlap inputs unless stated.  A
 * workspace may hold anything before a call and belongs to it until it has ended on its stream: calls
 * that can run at the same time (captured graphs too) take one each.
 */
#ifndef MTGR_BLOCK_H
#define MTGR_BLOCK_H

#include "mtgr_hstu.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- gated feed-forward block (bf16)
 *
 *   pre = x W_in               x [T, d], W_in [d, 2 f]: gate columns 0 .. f-1, up columns f .. 2 f-1
 *   h   = silu(gate) * up      [T, f]
 *   y   = h W_out (+ r)        W_out [f, d], r [T, d]
 *
 * d and f are multiples of 32, below 2^20; ceil(T / 256) ceil(2 max(d, f) / 128) is below 2^24.  Sums are fp32; h, pre
 * and the gradients of pre are rounded to bf16. */
typedef struct {
    int64_t num_tokens;       /* T, 0 .. 2^31 - 1 */
    int32_t dim;              /* d */
    int32_t hidden;           /* f */
    int64_t ld_x;             /* row strides: of x and dx */
    int64_t ld_w_in;          /* W_in and dW_in */
    int64_t ld_w_out;         /* W_out and dW_out */
    int64_t ld_y;             /* y (forward), dy (backward) */
    int64_t ld_r;             /* the residual */
    int64_t ld_pre;           /* pre */
    int64_t ld_h;             /* h */
} mtgr_gated_ffn_problem_t;

typedef enum {
    MTGR_FFN_SERVING = 0,     /* forward, pre and h not kept */
    MTGR_FFN_BACKWARD = 1,
    MTGR_FFN_TRAINING = 2     /* forward that keeps pre and h */
} mtgr_ffn_pass_t;

/* Workspace bytes of a pass. */
mtgr_status_t mtgr_gated_ffn_workspace_size(const mtgr_gated_ffn_problem_t* p, mtgr_ffn_pass_t pass, size_t* bytes);

/* Forward.  residual may be NULL, and may be y itself.  For the backward pass, pre and h are kept: both
 * given.  For serving, both NULL: h then lives in the workspace. */
mtgr_status_t mtgr_gated_ffn_fwd(const mtgr_gated_ffn_problem_t* p, const void* x, const void* w_in,
                                 const void* w_out, const void* residual, void* y, void* pre, void* h,
                                 void* workspace, size_t workspace_bytes, mtgr_stream_t stream);

/* Backward: gradients of y = h W_out with respect to x, W_in and W_out (the residual's gradient is dy).
 * T = 0: the weight gradients are zero-filled. */
mtgr_status_t mtgr_gated_ffn_bwd(const mtgr_gated_ffn_problem_t* p, const void* dy, const void* x, const void* pre,
                                 const void* h, const void* w_in, const void* w_out, void* dx, void* dw_in,
                                 void* dw_out, void* workspace, size_t workspace_bytes, mtgr_stream_t stream);

/* Debugging aid (host only): the kernels that a pass of these sizes runs on, as "name=kernel" pairs separated by
 * blanks, for profiles and for tests that mean to reach a certain kernel; the names may change.  Forward: hidden
 * (rows, or tiles with their K splits), h (cached or streamed stores), out; residual: whether there is one.
 * Backward: dpre, store, together (one launch behind dpre), dx, dw_in, dw_out.  128 bytes are enough. */
mtgr_status_t mtgr_debug_gated_ffn_kernels(const mtgr_gated_ffn_problem_t* p, mtgr_ffn_pass_t pass, int residual, char* text,
                                           size_t text_bytes);

/* ---------------------------------------------------------------- dropout
 *
 *   out = [residual +] (keep ? x / (1 - prob) : 0)         [rows, cols] of bf16 or fp32
 *
 * The mask is a function of (seed, step, site, row * cols + column) and is never stored: the backward
 * pass is the same call on the gradient, without the residual.  rng [2] uint64 on the device holds
 * (seed, step); a program advances the step between its training steps on the device, also under a
 * captured graph.  site numbers the places of a model that drop, so that their masks differ; the step
 * counts modulo 2^32.  Element e is kept when word e % 4 of Philox4x32-7 with the key seed and the counter
 * (e / 4 low, e / 4 high, site, step) is at least floor(prob 2^32).  0 <= prob < 1.  cols is a multiple of
 * 16 bytes, rows * cols below 2^50; dense rows (ld = cols) may be of any width.  A dropped element counts as 0
 * whatever x holds.  out may be x or the residual. */
mtgr_status_t mtgr_dropout(int64_t rows, int32_t cols, mtgr_dtype_t dtype, const void* x, int64_t ld_x, double prob,
                           const uint64_t* rng, uint32_t site, const void* residual, int64_t ld_residual, void* out,
                           int64_t ld_out, mtgr_stream_t stream);

/* ---------------------------------------------------------------- softmax loss over a class set
 *
 *   z_nc = scale x_n . w_c + bias_c        x [N, d] bf16, w [V, d] bf16, bias [V] fp32 or NULL
 *   lse_n = log sum_c exp z_nc             [N] fp32
 *   loss_n = lse_n - z_n,t(n)              [N] fp32, t = targets[n]
 *
 * The logits are never kept.  A row whose target lies outside 0 .. V-1 has no label: its loss, lse and
 * gradient are 0, its x may hold anything, and it costs next to nothing.  A bias of -inf takes a class
 * out (its row of w still has to be finite), and so does one below -2.36e38, which is -inf in the units of
 * log 2 that it is kept in; a row for which no class is left has the loss 0, lse -inf and no gradient; a
 * label whose class is out has the loss +inf.  bias below 2.36e38; d is a multiple of 32, at most 2048; N
 * below 2^24, V below 2^30.
 */
typedef struct {
    int64_t num_rows;         /* N */
    int64_t num_classes;      /* V */
    int32_t dim;              /* d */
    int32_t target_bits;      /* targets are int32 (32) or int64 (64) */
    float scale;              /* absolute value below 2.358e38 (finite in units of log 2) */
    int64_t ld_x;             /* x and dx */
    int64_t ld_w;             /* w and dw */
} mtgr_softmax_loss_problem_t;

mtgr_status_t mtgr_softmax_loss_workspace_size(const mtgr_softmax_loss_problem_t* p, int backward, size_t* bytes);

mtgr_status_t mtgr_softmax_loss_fwd(const mtgr_softmax_loss_problem_t* p, const void* x, const void* w,
                                    const void* targets, const float* bias, float* loss, float* lse, void* workspace,
                                    size_t workspace_bytes, mtgr_stream_t stream);

/* Gradients for dloss [N] fp32 (that of a mean: 1 / count), with lse of the forward pass on the same
 * inputs: dx [N, d] bf16, dw [V, d] bf16, dbias [V] fp32 or NULL.  N = 0: dw and dbias are zero-filled.  The gradient of
 * the logits, dz, is rounded to bf16 relative to the largest |dloss| of a row with a label, as operand of the products
 * that form dx and dw; their sums are fp32, dbias is summed from unrounded dz.  The workspace holds dz of a piece of the
 * classes: 2 N V bytes (all rows count, with a label or not) up to 4 GB, beyond which there are more pieces. */
mtgr_status_t mtgr_softmax_loss_bwd(const mtgr_softmax_loss_problem_t* p, const float* dloss, const void* x,
                                    const void* w, const void* targets, const float* bias, const float* lse, void* dx,
                                    void* dw, float* dbias, void* workspace, size_t workspace_bytes,
                                    mtgr_stream_t stream);

/* Debugging aid (host only), as mtgr_debug_gated_ffn_kernels, for `labels` rows with a label: logits, run (class tiles
 * that an item goes through), pieces and piece (of classes), and for the backward dz (cached or streamed stores), dx, dw. */
mtgr_status_t mtgr_debug_softmax_loss_kernels(const mtgr_softmax_loss_problem_t* p, int backward, int64_t labels, char* text,
                                              size_t text_bytes);

#ifdef __cplusplus
}
#endif
#endif /* MTGR_BLOCK_H */
