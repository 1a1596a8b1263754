// C entry points of include/mtgr_block.h: argument validation (host code, before any HIP call), workspace
// checks and launches.
#include <cmath>

#include "../../include/mtgr_block.h"
#include "api_util.h"
#include "block_internal.h"

namespace {

using namespace mtgr_api;

constexpr long long MAX_LD = 1ll << 22;        // 32-bit copy offsets over 256 rows

// A matrix of `cols` columns of `esize` bytes per element; dense_any: of any width where its rows are dense.
mtgr_status_t check_matrix(const void* p, const char* name, int64_t ld, int64_t cols, int esize = 2, bool dense_any = false) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "%s is NULL", name);
    if (!aligned16(p)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "%s is not 16-byte aligned", name);
    if (ld < cols || ld % (16 / esize) != 0)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "row stride of %s = %lld (needs at least %lld and 16-byte rows)", name,
                    (long long)ld, (long long)cols);
    if (ld >= MAX_LD && !(dense_any && ld == cols))
        return fail(MTGR_ERROR_UNSUPPORTED, "row stride of %s = %lld is not below %lld", name, (long long)ld, MAX_LD);
    return MTGR_SUCCESS;
}

mtgr_status_t check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (need == 0) return MTGR_SUCCESS;
    if (bytes < need) return fail(MTGR_ERROR_WORKSPACE_TOO_SMALL, "workspace %zu bytes, need %zu", bytes, need);
    if (!workspace) return fail(MTGR_ERROR_NULL_POINTER, "workspace is NULL");
    if (((uintptr_t)workspace & 255u) != 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "workspace is not 256-byte aligned");
    return MTGR_SUCCESS;
}

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

#define CHECK(call)                                  \
    do {                                             \
        const mtgr_status_t st_ = (call);            \
        if (st_ != MTGR_SUCCESS) return st_;         \
    } while (0)

mtgr_status_t check_ffn(const mtgr_gated_ffn_problem_t* p) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "problem is NULL");
    if (p->num_tokens < 0 || p->num_tokens >= (1ll << 31))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_tokens %lld outside [0, 2^31)", (long long)p->num_tokens);
    if (p->dim <= 0 || p->hidden <= 0)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "dim = %d, hidden = %d", p->dim, p->hidden);
    if (p->dim % 32 != 0 || p->hidden % 32 != 0)
        return fail(MTGR_ERROR_UNSUPPORTED, "dim = %d and hidden = %d are not multiples of 32", p->dim, p->hidden);
    if (p->dim >= (1 << 20) || p->hidden >= (1 << 20))
        return fail(MTGR_ERROR_UNSUPPORTED, "dim = %d, hidden = %d: below 2^20 each", p->dim, p->hidden);
    // work items of one launch (the tiles of the widest product)
    const long long tiles = (p->num_tokens + 255) / 256 * ((2ll * std::max(p->hidden, p->dim) + 127) / 128);
    if (tiles >= (1ll << 24)) return fail(MTGR_ERROR_UNSUPPORTED, "problem too large for one launch");
    return MTGR_SUCCESS;
}

size_t ffn_fwd_workspace(const mtgr_gated_ffn_problem_t* p, bool save) {
    return align256(mtgr::ffn_fwd_workspace_bytes(p->num_tokens, p->dim, p->hidden, save));
}

mtgr_status_t check_loss(const mtgr_softmax_loss_problem_t* p) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "problem is NULL");
    if (p->num_rows < 0 || p->num_rows >= (1ll << 24))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_rows %lld outside [0, 2^24)", (long long)p->num_rows);
    if (p->num_classes < 0 || p->num_classes >= (1ll << 30))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_classes %lld outside [0, 2^30)", (long long)p->num_classes);
    if (p->dim <= 0 || p->dim % 32 != 0 || p->dim > 2048)
        return fail(MTGR_ERROR_UNSUPPORTED, "dim = %d is not a multiple of 32 up to 2048", p->dim);
    if (p->target_bits != 32 && p->target_bits != 64)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "target_bits = %d is not 32 or 64", p->target_bits);
    // (the logits are formed in units of log 2)
    if (!std::isfinite(p->scale * 1.4426950408889634f))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "scale = %g is not below 2.358e38", p->scale);
    if (p->num_rows > 0 && p->num_classes == 0)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_classes is 0 with rows present");
    // tiles of a piece's products in one launch
    if ((p->num_rows + 255) / 256 * ((p->num_classes + 255) / 256) >= (1ll << 31))
        return fail(MTGR_ERROR_UNSUPPORTED, "problem too large");
    return MTGR_SUCCESS;
}

mtgr_status_t loss_inputs(const mtgr_softmax_loss_problem_t* p, const void* x, const void* w, const void* targets,
                          const float* bias) {
    CHECK(check_matrix(x, "x", p->ld_x, p->dim));
    CHECK(check_matrix(w, "w", p->ld_w, p->dim));
    if (!targets) return fail(MTGR_ERROR_NULL_POINTER, "targets is NULL");
    if (!aligned(targets, p->target_bits / 8)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "targets is not aligned to its type");
    if (bias && !aligned(bias, 4)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "bias is not 4-byte aligned");
    return MTGR_SUCCESS;
}

mtgr_status_t check_floats(const void* v, const char* name) {
    if (!v) return fail(MTGR_ERROR_NULL_POINTER, "%s is NULL", name);
    if (!aligned(v, 4)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "%s is not 4-byte aligned", name);
    return MTGR_SUCCESS;
}

mtgr::SoftmaxLossArgs loss_args(const mtgr_softmax_loss_problem_t* p, const void* x, const void* w, const void* targets,
                                const float* bias) {
    mtgr::SoftmaxLossArgs a{};
    a.N = p->num_rows;
    a.V = (int)p->num_classes;
    a.d = p->dim;
    a.x = x;
    a.w = w;
    a.ld_x = p->ld_x;
    a.ld_w = p->ld_w;
    a.targets = targets;
    a.targets64 = p->target_bits == 64;
    a.bias = bias;
    a.scale = p->scale;
    return a;
}

// What snprintf returned for a caller's buffer.
mtgr_status_t text_fits(int length, size_t bytes) {
    if (length < 0 || (size_t)length >= bytes)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "text of %d bytes does not fit into %zu", length + 1, bytes);
    return ok();
}

size_t loss_workspace(const mtgr_softmax_loss_problem_t* p, bool backward) {
    return mtgr::softmax_loss_workspace_bytes(p->num_rows, (int)p->num_classes, p->dim, backward);
}

}  // namespace

extern "C" {

mtgr_status_t mtgr_gated_ffn_workspace_size(const mtgr_gated_ffn_problem_t* p, mtgr_ffn_pass_t pass, size_t* bytes) {
    if (!bytes) return fail(MTGR_ERROR_NULL_POINTER, "bytes is NULL");
    CHECK(check_ffn(p));
    if (pass != MTGR_FFN_SERVING && pass != MTGR_FFN_BACKWARD && pass != MTGR_FFN_TRAINING)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "pass %d unknown", (int)pass);
    *bytes = p->num_tokens == 0 ? 0
             : pass == MTGR_FFN_BACKWARD
                 ? align256(mtgr::ffn_bwd_workspace_bytes(p->num_tokens, p->dim, p->hidden))
                 : ffn_fwd_workspace(p, pass == MTGR_FFN_TRAINING);
    return ok();
}

mtgr_status_t mtgr_gated_ffn_fwd(const mtgr_gated_ffn_problem_t* p, const void* x, const void* w_in, const void* w_out,
                                 const void* residual, void* y, void* pre, void* h, void* workspace,
                                 size_t workspace_bytes, mtgr_stream_t stream) {
    CHECK(check_ffn(p));
    if (p->num_tokens == 0) return ok();
    CHECK(check_matrix(x, "x", p->ld_x, p->dim));
    CHECK(check_matrix(w_in, "w_in", p->ld_w_in, 2ll * p->hidden));
    CHECK(check_matrix(w_out, "w_out", p->ld_w_out, p->dim));
    CHECK(check_matrix(y, "y", p->ld_y, p->dim));
    if (residual) CHECK(check_matrix(residual, "residual", p->ld_r, p->dim));
    if ((pre == nullptr) != (h == nullptr))
        return fail(MTGR_ERROR_NULL_POINTER, "pre and h are kept together: %s is NULL", pre ? "h" : "pre");
    if (pre) {
        CHECK(check_matrix(pre, "pre", p->ld_pre, 2ll * p->hidden));
        CHECK(check_matrix(h, "h", p->ld_h, p->hidden));
    }
    CHECK(check_workspace(workspace, workspace_bytes, ffn_fwd_workspace(p, pre != nullptr)));
    mtgr::FfnArgs a{};
    a.ld_h = p->ld_h;
    a.T = p->num_tokens;
    a.d = p->dim;
    a.f = p->hidden;
    a.x = x;
    a.w_in = w_in;
    a.w_out = w_out;
    a.residual = residual;
    a.y = y;
    a.pre = pre;
    a.h = h;
    a.ld_x = p->ld_x;
    a.ld_win = p->ld_w_in;
    a.ld_wout = p->ld_w_out;
    a.ld_y = p->ld_y;
    a.ld_r = p->ld_r;
    a.ld_pre = p->ld_pre;
    const hipError_t e = mtgr::launch_ffn_fwd(a, workspace, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "gated feed-forward");
    return ok();
}

mtgr_status_t mtgr_gated_ffn_bwd(const mtgr_gated_ffn_problem_t* p, const void* dy, const void* x, const void* pre,
                                 const void* h, const void* w_in, const void* w_out, void* dx, void* dw_in,
                                 void* dw_out, void* workspace, size_t workspace_bytes, mtgr_stream_t stream) {
    CHECK(check_ffn(p));
    CHECK(check_matrix(dw_in, "dw_in", p->ld_w_in, 2ll * p->hidden));
    CHECK(check_matrix(dw_out, "dw_out", p->ld_w_out, p->dim));
    mtgr::FfnArgs a{};
    a.T = p->num_tokens;
    a.d = p->dim;
    a.f = p->hidden;
    a.dw_in = dw_in;
    a.dw_out = dw_out;
    a.ld_win = p->ld_w_in;
    a.ld_wout = p->ld_w_out;
    if (p->num_tokens > 0) {
        CHECK(check_matrix(dy, "dy", p->ld_y, p->dim));
        CHECK(check_matrix(x, "x", p->ld_x, p->dim));
        CHECK(check_matrix(pre, "pre", p->ld_pre, 2ll * p->hidden));
        CHECK(check_matrix(h, "h", p->ld_h, p->hidden));
        CHECK(check_matrix(w_in, "w_in", p->ld_w_in, 2ll * p->hidden));
        CHECK(check_matrix(w_out, "w_out", p->ld_w_out, p->dim));
        CHECK(check_matrix(dx, "dx", p->ld_x, p->dim));
        CHECK(check_workspace(workspace, workspace_bytes,
                              align256(mtgr::ffn_bwd_workspace_bytes(p->num_tokens, p->dim, p->hidden))));
        a.dy = dy;
        a.x = x;
        a.pre = (void*)pre;
        a.h = (void*)h;
        a.w_in = w_in;
        a.w_out = w_out;
        a.dx = dx;
        a.ld_x = p->ld_x;
        a.ld_y = p->ld_y;
        a.ld_pre = p->ld_pre;
        a.ld_h = p->ld_h;
    }
    const hipError_t e = mtgr::launch_ffn_bwd(a, workspace, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "gated feed-forward backward");
    return ok();
}

mtgr_status_t mtgr_debug_gated_ffn_kernels(const mtgr_gated_ffn_problem_t* p, mtgr_ffn_pass_t pass, int residual, char* text,
                                           size_t text_bytes) {
    if (!text) return fail(MTGR_ERROR_NULL_POINTER, "text is NULL");
    CHECK(check_ffn(p));
    if (pass != MTGR_FFN_SERVING && pass != MTGR_FFN_BACKWARD && pass != MTGR_FFN_TRAINING)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "pass %d unknown", (int)pass);
    if (p->num_tokens == 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "no tokens, no kernels");
    const long long T = p->num_tokens;
    return text_fits(pass == MTGR_FFN_BACKWARD
                         ? mtgr::ffn_bwd_kernels(T, p->dim, p->hidden, text, text_bytes)
                         : mtgr::ffn_fwd_kernels(T, p->dim, p->hidden, pass == MTGR_FFN_TRAINING, residual != 0, text, text_bytes),
                     text_bytes);
}

mtgr_status_t mtgr_dropout(int64_t rows, int32_t cols, mtgr_dtype_t dtype, const void* x, int64_t ld_x, double prob,
                           const uint64_t* rng, uint32_t site, const void* residual, int64_t ld_residual, void* out,
                           int64_t ld_out, mtgr_stream_t stream) {
    if (dtype != MTGR_DTYPE_BF16 && dtype != MTGR_DTYPE_FP32) return fail(MTGR_ERROR_UNSUPPORTED, "dtype %d", (int)dtype);
    const int esize = dtype == MTGR_DTYPE_BF16 ? 2 : 4, per = 16 / esize;
    if (rows < 0 || cols <= 0 || rows >= (1ll << 50) / cols)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "rows = %lld, cols = %d", (long long)rows, cols);
    if (cols % per != 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "cols = %d is not a multiple of %d", cols, per);
    if (!(prob >= 0.0 && prob < 1.0)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "prob = %g outside [0, 1)", prob);
    if (rows == 0) return ok();
    CHECK(check_matrix(x, "x", ld_x, cols, esize, true));
    CHECK(check_matrix(out, "out", ld_out, cols, esize, true));
    if (residual) CHECK(check_matrix(residual, "residual", ld_residual, cols, esize, true));
    if (!rng) return fail(MTGR_ERROR_NULL_POINTER, "rng is NULL");
    if (!aligned(rng, 8)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "rng is not 8-byte aligned");
    mtgr::DropoutArgs a{};
    a.rows = rows;
    a.cols = cols;
    a.x = x;
    a.ld_x = ld_x;
    a.residual = residual;
    a.ld_r = ld_residual;
    a.out = out;
    a.ld_out = ld_out;
    a.rng = (const unsigned long long*)rng;
    a.site = site;
    a.threshold = (uint32_t)std::floor(prob * 4294967296.0);      // (below 2^32: prob < 1)
    a.scale = (float)(1.0 / (1.0 - prob));
    const hipError_t e = mtgr::launch_dropout(a, dtype == MTGR_DTYPE_BF16, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "dropout");
    return ok();
}

mtgr_status_t mtgr_softmax_loss_workspace_size(const mtgr_softmax_loss_problem_t* p, int backward, size_t* bytes) {
    if (!bytes) return fail(MTGR_ERROR_NULL_POINTER, "bytes is NULL");
    CHECK(check_loss(p));
    *bytes = loss_workspace(p, backward != 0);
    return ok();
}

mtgr_status_t mtgr_debug_softmax_loss_kernels(const mtgr_softmax_loss_problem_t* p, int backward, int64_t labels, char* text,
                                              size_t text_bytes) {
    if (!text) return fail(MTGR_ERROR_NULL_POINTER, "text is NULL");
    CHECK(check_loss(p));
    if (labels < 0 || labels > p->num_rows)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "labels = %lld of %lld rows", (long long)labels, (long long)p->num_rows);
    if (p->num_rows == 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "no rows, no kernels");
    return text_fits(mtgr::softmax_loss_kernels(p->num_rows, (int)p->num_classes, p->dim, backward != 0, labels, text, text_bytes),
                     text_bytes);
}

mtgr_status_t mtgr_softmax_loss_fwd(const mtgr_softmax_loss_problem_t* p, const void* x, const void* w,
                                    const void* targets, const float* bias, float* loss, float* lse, void* workspace,
                                    size_t workspace_bytes, mtgr_stream_t stream) {
    CHECK(check_loss(p));
    if (p->num_rows == 0) return ok();
    CHECK(loss_inputs(p, x, w, targets, bias));
    CHECK(check_floats(loss, "loss"));
    CHECK(check_floats(lse, "lse"));
    CHECK(check_workspace(workspace, workspace_bytes, loss_workspace(p, false)));
    mtgr::SoftmaxLossArgs a = loss_args(p, x, w, targets, bias);
    a.loss = loss;
    a.lse = lse;
    const hipError_t e = mtgr::launch_softmax_loss_fwd(a, workspace, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "softmax loss");
    return ok();
}

mtgr_status_t mtgr_softmax_loss_bwd(const mtgr_softmax_loss_problem_t* p, const float* dloss, const void* x,
                                    const void* w, const void* targets, const float* bias, const float* lse, void* dx,
                                    void* dw, float* dbias, void* workspace, size_t workspace_bytes,
                                    mtgr_stream_t stream) {
    CHECK(check_loss(p));
    if (p->num_classes == 0) return ok();
    CHECK(check_matrix(dw, "dw", p->ld_w, p->dim));
    if (dbias) CHECK(check_floats(dbias, "dbias"));
    if (p->num_rows > 0) {
        CHECK(loss_inputs(p, x, w, targets, bias));
        CHECK(check_matrix(dx, "dx", p->ld_x, p->dim));
        CHECK(check_floats(dloss, "dloss"));
        CHECK(check_floats(lse, "lse"));
        CHECK(check_workspace(workspace, workspace_bytes, loss_workspace(p, true)));
    }
    mtgr::SoftmaxLossArgs a = loss_args(p, x, w, targets, bias);
    a.dloss = dloss;
    a.lse = (float*)lse;
    a.dx = dx;
    a.dw = dw;
    a.dbias = dbias;
    const hipError_t e = mtgr::launch_softmax_loss_bwd(a, workspace, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "softmax loss backward");
    return ok();
}

}  // extern "C"
