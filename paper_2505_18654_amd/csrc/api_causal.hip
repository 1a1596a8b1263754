// C entry points of include/mtgr_causal.h: argument validation (host code, before any HIP call), workspace checks and
// launches.
#include <cmath>

#include "../../include/mtgr_causal.h"
#include "api_util.h"
#include "causal_internal.h"

namespace {

using namespace mtgr_api;

constexpr long long MAX_LD = 1ll << 22;        // 32-bit copy offsets over a tile's rows
// A launch has fewer than 2^32 threads: 2^24 workgroups of 256.  (The dK / dV kernel takes up to 1,024 + kv_heads more than tiles.)
constexpr long long MAX_THREADS = (1ll << 32) - 256, MAX_TILES = (1ll << 24) - (1ll << 17);

#define CHECK(call)                                  \
    do {                                             \
        const mtgr_status_t st_ = (call);            \
        if (st_ != MTGR_SUCCESS) return st_;         \
    } while (0)

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// [rows, heads, head_dim] with dense heads.
mtgr_status_t check_heads(const void* p, const char* name, int64_t ld, int64_t heads, int64_t head_dim, int esize = 2) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "%s is NULL", name);
    if (!aligned16(p)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "%s is not 16-byte aligned", name);
    if (ld < heads * head_dim || ld % (16 / esize) != 0)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "token stride of %s = %lld (needs at least %lld and 16-byte rows)", name,
                    (long long)ld, (long long)(heads * head_dim));
    if (ld >= MAX_LD) return fail(MTGR_ERROR_UNSUPPORTED, "token stride of %s = %lld is not below %lld", name, (long long)ld, MAX_LD);
    return MTGR_SUCCESS;
}

// An output that is its input has its stride too: with another one, rows would be read after others were written over them.
mtgr_status_t check_in_place(const void* in, int64_t ld_in, const void* out, int64_t ld_out, const char* name) {
    if (in == out && ld_in != ld_out)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "%s in place with token strides %lld and %lld", name, (long long)ld_in, (long long)ld_out);
    return MTGR_SUCCESS;
}

mtgr_status_t check_array(const void* p, const char* name, size_t align) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "%s is NULL", name);
    if (!aligned(p, align)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "%s is not aligned to its type", name);
    return MTGR_SUCCESS;
}

mtgr_status_t check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (need == 0) return MTGR_SUCCESS;
    if (bytes < need) return fail(MTGR_ERROR_WORKSPACE_TOO_SMALL, "workspace %zu bytes, need %zu", bytes, need);
    if (!workspace) return fail(MTGR_ERROR_NULL_POINTER, "workspace is NULL");
    if (!aligned(workspace, 256)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "workspace is not 256-byte aligned");
    return MTGR_SUCCESS;
}

mtgr_status_t check_tokens(int64_t n, const char* name) {
    if (n < 0 || n >= (1ll << 31)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "%s = %lld outside [0, 2^31)", name, (long long)n);
    return MTGR_SUCCESS;
}

mtgr_status_t check_rotation(int32_t head_dim, int32_t rot_dim, int32_t layout, float amplitude) {
    if (rot_dim < 16 || rot_dim % 16 != 0 || rot_dim > head_dim)
        return fail(MTGR_ERROR_UNSUPPORTED, "rot_dim = %d is not a multiple of 16 in 16 .. head_dim = %d", rot_dim, head_dim);
    if (layout != MTGR_ROPE_HALF && layout != MTGR_ROPE_INTERLEAVED)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "layout %d unknown", layout);
    if (!std::isfinite(amplitude)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "amplitude = %g", amplitude);
    return MTGR_SUCCESS;
}

mtgr_status_t check_head_dim(int32_t head_dim) {
    if (head_dim <= 0 || head_dim % 8 != 0 || head_dim > 1024)
        return fail(MTGR_ERROR_UNSUPPORTED, "head_dim = %d is not a multiple of 8 up to 1024", head_dim);
    return MTGR_SUCCESS;
}

// A thread takes 32 bytes of a token's heads.
mtgr_status_t check_threads(int64_t tokens, int32_t head_dim, int esize) {
    if (tokens * ((head_dim * esize + 31) / 32) >= MAX_THREADS)
        return fail(MTGR_ERROR_UNSUPPORTED, "problem too large for one launch");
    return MTGR_SUCCESS;
}

mtgr_status_t check_attn(int32_t heads, int32_t kv_heads, int32_t head_dim, float scale) {
    if (heads <= 0 || kv_heads <= 0 || heads % kv_heads != 0 || heads > 65535)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "heads = %d, kv_heads = %d", heads, kv_heads);
    if (head_dim != 32 && head_dim != 64 && head_dim != 128)
        return fail(MTGR_ERROR_UNSUPPORTED, "head_dim = %d is not 32, 64 or 128", head_dim);
    // (the scores are formed in units of log 2)
    if (!(scale > 0.0f) || !std::isfinite(scale * 1.4426950408889634f))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "scale = %g is not positive and below 2.358e38", scale);
    return MTGR_SUCCESS;
}

long long causal_slots(const mtgr_causal_problem_t* p) { return p->total_tokens / 128 + p->num_seqs; }

mtgr_status_t check_causal(const mtgr_causal_problem_t* p) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "problem is NULL");
    if (p->num_seqs < 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_seqs = %d", p->num_seqs);
    if (p->reserved != 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "reserved = %d", p->reserved);
    if (p->total_tokens < 0 || p->total_tokens >= (1ll << 30))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "total_tokens = %lld outside [0, 2^30)", (long long)p->total_tokens);
    CHECK(check_attn(p->heads, p->kv_heads, p->head_dim, p->scale));
    if (causal_slots(p) * p->heads >= MAX_TILES) return fail(MTGR_ERROR_UNSUPPORTED, "problem too large for one launch");
    return MTGR_SUCCESS;
}

// The backward's workspace: - lse / ln 2 and - delta, then the plan with its sums.
size_t rows_bytes(const mtgr_causal_problem_t* p) { return align256((size_t)p->heads * (size_t)p->total_tokens * 4); }

mtgr::CausalPlan plan_of(const mtgr_causal_problem_t* p) {
    return mtgr::causal_plan(p->total_tokens, p->num_seqs, p->heads, p->kv_heads, p->head_dim);
}

size_t causal_workspace(const mtgr_causal_problem_t* p) {
    if (p->total_tokens == 0 || p->num_seqs == 0) return 0;
    return 2 * rows_bytes(p) + plan_of(p).bytes;
}

mtgr::CausalArgs causal_args(const mtgr_causal_problem_t* p, const int32_t* offsets, const void* q, const void* k, const void* v) {
    mtgr::CausalArgs a{};
    a.B = p->num_seqs;
    a.H = p->heads;
    a.Hk = p->kv_heads;
    a.group = p->heads / p->kv_heads;
    a.T = p->total_tokens;
    a.slots = (int)causal_slots(p);
    a.scale = p->scale;
    a.c = p->scale * 1.4426950408889634f;
    a.least = mtgr::least_score(a.c);
    a.offsets = offsets;
    a.q = q;
    a.k = k;
    a.v = v;
    a.ld_q = p->ld_q;
    a.ld_k = p->ld_k;
    a.ld_v = p->ld_v;
    a.ld_o = p->ld_o;
    a.ld_do = p->ld_do;
    return a;
}

mtgr_status_t check_qkv(const mtgr_causal_problem_t* p, const int32_t* offsets, const void* q, const void* k, const void* v) {
    CHECK(check_array(offsets, "offsets", 4));
    CHECK(check_heads(q, "q", p->ld_q, p->heads, p->head_dim));
    CHECK(check_heads(k, "k", p->ld_k, p->kv_heads, p->head_dim));
    CHECK(check_heads(v, "v", p->ld_v, p->kv_heads, p->head_dim));
    return MTGR_SUCCESS;
}

int page_shift(int32_t page_size) { return __builtin_ctz((unsigned)page_size); }

mtgr_status_t check_cache(const mtgr_kv_cache_t* c, bool pointers) {
    if (!c) return fail(MTGR_ERROR_NULL_POINTER, "cache is NULL");
    if (c->num_pages < 1 || c->num_pages >= (1ll << 31))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_pages = %lld outside [1, 2^31)", (long long)c->num_pages);
    if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0)
        return fail(MTGR_ERROR_UNSUPPORTED, "page_size = %d is not a power of two in 16 .. 4096", c->page_size);
    if (c->kv_heads <= 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "kv_heads = %d", c->kv_heads);
    if (c->reserved != 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "reserved = %d", c->reserved);
    if (!pointers) return MTGR_SUCCESS;
    if (!c->keys || !c->values) return fail(MTGR_ERROR_NULL_POINTER, "%s of the cache is NULL", c->keys ? "values" : "keys");
    if (!aligned16(c->keys) || !aligned16(c->values))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "keys and values of the cache are 16-byte aligned");
    return MTGR_SUCCESS;
}

mtgr_status_t check_table(const int32_t* table, int64_t ld, int32_t max_pages) {
    CHECK(check_array(table, "page_table", 4));
    if (ld < max_pages || ld >= (1ll << 31))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "row stride of page_table = %lld, max_pages = %d", (long long)ld, max_pages);
    return MTGR_SUCCESS;
}

mtgr::CacheArgs cache_args(const mtgr_kv_cache_t* c, const int32_t* table, int64_t ld, int32_t max_pages) {
    mtgr::CacheArgs a{};
    a.keys = c->keys;
    a.values = c->values;
    a.num_pages = c->num_pages;
    a.page_shift = page_shift(c->page_size);
    a.kv_heads = c->kv_heads;
    a.table = table;
    a.ld_table = ld;
    a.max_pages = max_pages;
    return a;
}

mtgr_status_t check_cache_attn(const mtgr_cache_attn_problem_t* p, const mtgr_kv_cache_t* cache, bool pointers) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "problem is NULL");
    CHECK(check_cache(cache, pointers));
    if (p->num_seqs < 0 || p->num_seqs > 65535)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_seqs = %d outside [0, 65535]", p->num_seqs);
    CHECK(check_attn(p->heads, cache->kv_heads, cache->head_dim, p->scale));
    if ((int64_t)p->num_seqs * p->heads >= (1ll << 23)) return fail(MTGR_ERROR_UNSUPPORTED, "num_seqs heads is not below 2^23");
    if (p->max_pages < 1) return fail(MTGR_ERROR_INVALID_ARGUMENT, "max_pages = %d", p->max_pages);
    if (p->max_len < 0 || p->max_len > (int64_t)p->max_pages * cache->page_size || p->max_len >= (1ll << 31) - 4096)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "max_len = %lld outside [0, max_pages page_size = %lld] or not below 2^31 - 4096",
                    (long long)p->max_len, (long long)p->max_pages * cache->page_size);
    return MTGR_SUCCESS;
}

mtgr::CacheAttnPlan plan_of(const mtgr_cache_attn_problem_t* p, const mtgr_kv_cache_t* cache) {
    return mtgr::cache_attn_plan(std::max(p->num_seqs, 1), p->heads, cache->kv_heads, cache->head_dim, p->max_len);
}

}  // namespace

extern "C" {

mtgr_status_t mtgr_rope_frequencies(int32_t rot_dim, double base, mtgr_rope_scaling_t scaling, double factor,
                                    int64_t trained_len, double slow, double fast, double* freqs, float* amplitude) {
    if (!freqs || !amplitude) return fail(MTGR_ERROR_NULL_POINTER, "%s is NULL", freqs ? "amplitude" : "freqs");
    CHECK(check_rotation(1024, rot_dim, MTGR_ROPE_HALF, 1.0f));
    if (!(base > 1.0) || !std::isfinite(base)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "base = %g", base);
    if (scaling < MTGR_ROPE_NONE || scaling > MTGR_ROPE_PARTS)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "scaling %d unknown", (int)scaling);
    if (scaling != MTGR_ROPE_NONE && (!(factor >= 1.0) || !std::isfinite(factor)))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "factor = %g", factor);
    if (scaling == MTGR_ROPE_PARTS && (trained_len <= 0 || !(slow >= 0.0) || !(fast > slow) || !std::isfinite(fast)))
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "trained_len = %lld, slow = %g, fast = %g", (long long)trained_len, slow, fast);
    if (scaling == MTGR_ROPE_BASE) {
        base *= std::pow(factor, rot_dim / (rot_dim - 2.0));
        if (!std::isfinite(base)) return fail(MTGR_ERROR_INVALID_ARGUMENT, "factor = %g", factor);
    }
    for (int i = 0; i < rot_dim / 2; i++) {
        double f = std::pow(base, -2.0 * i / rot_dim);
        if (scaling == MTGR_ROPE_LINEAR) f /= factor;
        if (scaling == MTGR_ROPE_PARTS) {
            const double turns = (double)trained_len * f / 6.283185307179586;
            const double keep = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
            f *= keep + (1.0 - keep) / factor;
        }
        freqs[i] = f;
    }
    *amplitude = scaling == MTGR_ROPE_PARTS ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
    return ok();
}

mtgr_status_t mtgr_rope(const mtgr_rope_problem_t* p, const void* x, const int32_t* positions, const int32_t* offsets,
                        const double* freqs, void* out, mtgr_stream_t stream) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "problem is NULL");
    CHECK(check_tokens(p->num_tokens, "num_tokens"));
    if (p->dtype != MTGR_DTYPE_BF16 && p->dtype != MTGR_DTYPE_FP32) return fail(MTGR_ERROR_UNSUPPORTED, "dtype %d", p->dtype);
    if (p->num_seqs < 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_seqs = %d", p->num_seqs);
    if (p->heads <= 0 || p->heads > 65535) return fail(MTGR_ERROR_INVALID_ARGUMENT, "heads = %d", p->heads);
    CHECK(check_head_dim(p->head_dim));
    CHECK(check_rotation(p->head_dim, p->rot_dim, p->layout, p->amplitude));
    if (p->num_tokens == 0) return ok();
    const int esize = p->dtype == MTGR_DTYPE_BF16 ? 2 : 4;
    CHECK(check_threads(p->num_tokens, p->head_dim, esize));
    CHECK(check_heads(x, "x", p->ld_x, p->heads, p->head_dim, esize));
    CHECK(check_heads(out, "out", p->ld_out, p->heads, p->head_dim, esize));
    CHECK(check_in_place(x, p->ld_x, out, p->ld_out, "x"));
    if ((positions == nullptr) == (offsets == nullptr))
        return fail(positions ? MTGR_ERROR_INVALID_ARGUMENT : MTGR_ERROR_NULL_POINTER, "either positions or offsets is given");
    CHECK(positions ? check_array(positions, "positions", 4) : check_array(offsets, "offsets", 4));
    CHECK(check_array(freqs, "freqs", 8));
    if (offsets && p->num_seqs == 0) return ok();
    mtgr::RopeArgs a{};
    a.T = p->num_tokens;
    a.B = p->num_seqs;
    a.heads = p->heads;
    a.dh = p->head_dim;
    a.rot = p->rot_dim;
    a.interleaved = p->layout == MTGR_ROPE_INTERLEAVED;
    a.inverse = p->inverse != 0;
    a.amplitude = p->amplitude;
    a.freqs = freqs;
    a.x = x;
    a.out = out;
    a.ld_x = p->ld_x;
    a.ld_out = p->ld_out;
    a.positions = positions;
    a.offsets = offsets;
    const hipError_t e = mtgr::launch_rope(a, p->dtype == MTGR_DTYPE_BF16, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "rotary positions");
    return ok();
}

mtgr_status_t mtgr_causal_attn_workspace_size(const mtgr_causal_problem_t* p, size_t* bytes) {
    if (!bytes) return fail(MTGR_ERROR_NULL_POINTER, "bytes is NULL");
    CHECK(check_causal(p));
    *bytes = causal_workspace(p);
    return ok();
}

mtgr_status_t mtgr_causal_attn_fwd(const mtgr_causal_problem_t* p, const int32_t* offsets, const void* q, const void* k,
                                   const void* v, void* out, float* lse, mtgr_stream_t stream) {
    CHECK(check_causal(p));
    if (p->total_tokens == 0 || p->num_seqs == 0) return ok();
    CHECK(check_qkv(p, offsets, q, k, v));
    CHECK(check_heads(out, "out", p->ld_o, p->heads, p->head_dim));
    if (lse) CHECK(check_array(lse, "lse", 4));
    mtgr::CausalArgs a = causal_args(p, offsets, q, k, v);
    a.out = out;
    a.lse = lse;
    const hipError_t e = mtgr::launch_causal_fwd(a, p->head_dim, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "causal attention");
    return ok();
}

mtgr_status_t mtgr_causal_attn_bwd(const mtgr_causal_problem_t* p, const int32_t* offsets, const void* q, const void* k,
                                   const void* v, const void* out, const float* lse, const void* dout, void* dq, void* dk,
                                   void* dv, void* workspace, size_t workspace_bytes, mtgr_stream_t stream) {
    CHECK(check_causal(p));
    if (p->total_tokens == 0 || p->num_seqs == 0) return ok();
    CHECK(check_qkv(p, offsets, q, k, v));
    CHECK(check_heads(out, "out", p->ld_o, p->heads, p->head_dim));
    CHECK(check_heads(dout, "dout", p->ld_do, p->heads, p->head_dim));
    CHECK(check_array(lse, "lse", 4));
    CHECK(check_heads(dq, "dq", p->ld_q, p->heads, p->head_dim));
    CHECK(check_heads(dk, "dk", p->ld_k, p->kv_heads, p->head_dim));
    CHECK(check_heads(dv, "dv", p->ld_v, p->kv_heads, p->head_dim));
    CHECK(check_workspace(workspace, workspace_bytes, causal_workspace(p)));
    mtgr::CausalArgs a = causal_args(p, offsets, q, k, v);
    a.out = (void*)out;
    a.lse = (float*)lse;
    a.dout = dout;
    a.dq = dq;
    a.dk = dk;
    a.dv = dv;
    char* ws = (char*)workspace;
    a.rows_l = (float*)ws;
    a.rows_d = (float*)(ws + rows_bytes(p));
    ws += 2 * rows_bytes(p);
    const mtgr::CausalPlan plan = plan_of(p);
    a.items = (mtgr::CausalItem*)ws;
    a.joins = (mtgr::CausalItem*)(ws + plan.joins_ofs);
    a.parts = (float*)(ws + plan.parts_ofs);
    const hipStream_t s = (hipStream_t)stream;
    hipError_t e = mtgr::launch_causal_dq(a, plan, p->head_dim, s);
    if (e == hipSuccess) e = mtgr::launch_causal_dkdv(a, plan, p->head_dim, s);
    if (e != hipSuccess) return device_fail(e, "causal attention backward");
    return ok();
}

mtgr_status_t mtgr_kv_append(const mtgr_kv_append_problem_t* p, const mtgr_kv_cache_t* cache, const int32_t* page_table,
                             const int32_t* past, const int32_t* offsets, const void* q, const void* k, const void* v,
                             const double* freqs, void* q_out, mtgr_stream_t stream) {
    if (!p) return fail(MTGR_ERROR_NULL_POINTER, "problem is NULL");
    CHECK(check_cache(cache, true));
    CHECK(check_head_dim(cache->head_dim));
    CHECK(check_tokens(p->num_tokens, "num_tokens"));
    if (p->num_seqs < 0) return fail(MTGR_ERROR_INVALID_ARGUMENT, "num_seqs = %d", p->num_seqs);
    if (p->max_pages < 1) return fail(MTGR_ERROR_INVALID_ARGUMENT, "max_pages = %d", p->max_pages);
    if (p->heads < 0 || p->heads > 65535 || cache->kv_heads > 65535)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "heads = %d, kv_heads = %d", p->heads, cache->kv_heads);
    if (p->rot_dim != 0) CHECK(check_rotation(cache->head_dim, p->rot_dim, p->layout, p->amplitude));
    if (!offsets && p->num_tokens != p->num_seqs)
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "without offsets, num_tokens = %lld is num_seqs = %d", (long long)p->num_tokens,
                    p->num_seqs);
    if (p->num_tokens == 0 || p->num_seqs == 0) return ok();
    CHECK(check_threads(p->num_tokens, cache->head_dim, 2));
    CHECK(check_table(page_table, p->ld_table, p->max_pages));
    CHECK(check_array(past, "past", 4));
    if (offsets) CHECK(check_array(offsets, "offsets", 4));
    CHECK(check_heads(k, "k", p->ld_k, cache->kv_heads, cache->head_dim));
    CHECK(check_heads(v, "v", p->ld_v, cache->kv_heads, cache->head_dim));
    if (p->heads > 0) {
        CHECK(check_heads(q, "q", p->ld_q, p->heads, cache->head_dim));
        CHECK(check_heads(q_out, "q_out", p->ld_q_out, p->heads, cache->head_dim));
        CHECK(check_in_place(q, p->ld_q, q_out, p->ld_q_out, "q"));
    } else if (q || q_out) {
        return fail(MTGR_ERROR_INVALID_ARGUMENT, "q of 0 heads is given");
    }
    if (p->rot_dim != 0) CHECK(check_array(freqs, "freqs", 8));
    mtgr::AppendArgs a{};
    a.rope.T = p->num_tokens;
    a.rope.B = p->num_seqs;
    a.rope.heads = p->heads;
    a.rope.dh = cache->head_dim;
    a.rope.rot = p->rot_dim;
    a.rope.interleaved = p->layout == MTGR_ROPE_INTERLEAVED;
    a.rope.amplitude = p->amplitude;
    a.rope.freqs = freqs;
    a.rope.x = q;
    a.rope.out = q_out;
    a.rope.ld_x = p->ld_q;
    a.rope.ld_out = p->ld_q_out;
    a.rope.offsets = offsets;
    a.cache = cache_args(cache, page_table, p->ld_table, p->max_pages);
    a.past = past;
    a.k = k;
    a.v = v;
    a.ld_k = p->ld_k;
    a.ld_v = p->ld_v;
    const hipError_t e = mtgr::launch_kv_append(a, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "append to the cache");
    return ok();
}

mtgr_status_t mtgr_cache_attn_workspace_size(const mtgr_cache_attn_problem_t* p, const mtgr_kv_cache_t* cache,
                                             size_t* bytes) {
    if (!bytes) return fail(MTGR_ERROR_NULL_POINTER, "bytes is NULL");
    CHECK(check_cache_attn(p, cache, false));
    *bytes = p->num_seqs == 0 ? 0 : plan_of(p, cache).bytes;
    return ok();
}

mtgr_status_t mtgr_cache_attn(const mtgr_cache_attn_problem_t* p, const mtgr_kv_cache_t* cache, const int32_t* page_table,
                              const int32_t* lens, const void* q, void* out, float* lse, void* workspace,
                              size_t workspace_bytes, mtgr_stream_t stream) {
    CHECK(check_cache_attn(p, cache, true));
    if (p->num_seqs == 0) return ok();
    CHECK(check_table(page_table, p->ld_table, p->max_pages));
    CHECK(check_array(lens, "lens", 4));
    CHECK(check_heads(q, "q", p->ld_q, p->heads, cache->head_dim));
    CHECK(check_heads(out, "out", p->ld_o, p->heads, cache->head_dim));
    if (lse) CHECK(check_array(lse, "lse", 4));
    const mtgr::CacheAttnPlan plan = plan_of(p, cache);
    CHECK(check_workspace(workspace, workspace_bytes, plan.need));
    mtgr::CacheAttnArgs a{};
    a.cache = cache_args(cache, page_table, p->ld_table, p->max_pages);
    a.B = p->num_seqs;
    a.H = p->heads;
    a.group = p->heads / cache->kv_heads;
    a.chunk = plan.chunk;
    a.splits = plan.splits;
    a.waves = plan.waves;
    a.max_len = (int)p->max_len;
    a.scale = p->scale;
    a.c = p->scale * 1.4426950408889634f;
    a.least = mtgr::least_score(a.c);
    a.lens = lens;
    a.q = q;
    a.ld_q = p->ld_q;
    a.ld_o = p->ld_o;
    a.out = out;
    a.lse = lse;
    a.part = (float*)workspace;
    a.part_ml = (float2*)((char*)workspace + plan.part_bytes);
    const hipError_t e = mtgr::launch_cache_attn(a, cache->head_dim, (hipStream_t)stream);
    if (e != hipSuccess) return device_fail(e, "attention over the cache");
    return ok();
}

}  // extern "C"
