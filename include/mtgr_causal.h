/*
 * mtgr_causal.h — C ABI of softmax attention over a user's own past: rotary positions, causal attention of packed
 * sequences (forward, backward), a paged cache of keys and values, and single tokens against it.  It stands beside
 * the SiLU attention of mtgr_hstu.h: the same jagged batches (offsets [B + 1] int32 on the device, offsets[0] = 0,
 * ascending), with each token seeing itself and the tokens before it.
 *
 * The conventions are those of mtgr_hstu.h: caller-owned device memory, calls asynchronous on `stream`, no allocation,
 * no synchronisation, outputs overwritten, arguments checked on the host before any launch.  Tensors of heads,
 * [T, heads, head_dim], have dense heads and a token stride (ld, in elements) of at least heads head_dim, a multiple of
 * 16 bytes, below 2^22, so that they can be columns of one projection; their base is 16-byte aligned.  Outputs do
 * not overlap inputs unless stated.  A workspace may hold anything before a call and belongs to it until it has ended
 * on its stream: calls that can run at the same time (captured graphs too) take one each.
 *
 * Query head h uses key and value head h / (heads / kv_heads).
 *
 * The attention's products and sums have to stay in fp32's range: |q . k|, and |v| times 2^8 times the tokens that a token sees,
 * below 2^127 (the sums of v are divided by those of the probabilities, which reach 2^8, at the end).
 */
#ifndef MTGR_CAUSAL_H
#define MTGR_CAUSAL_H

#include "mtgr_hstu.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- rotary positions
 *
 * Features 0 .. rot_dim-1 of a head form rot_dim / 2 pairs; pair i of a token at position p turns by the angle p f_i:
 *   (a, b) -> amplitude (a cos - b sin, a sin + b cos)
 * HALF pairs feature i with i + rot_dim / 2, INTERLEAVED 2 i with 2 i + 1; the features behind rot_dim are kept.  The
 * angles are formed in 64 bits (p f_i modulo whole turns), sines, cosines and products in fp32, results are rounded once.
 * `inverse` turns the other way: the gradient of x from that of the output. */
typedef enum { MTGR_ROPE_HALF = 0, MTGR_ROPE_INTERLEAVED = 1 } mtgr_rope_layout_t;

/* How the frequencies f_i = base^(-2 i / rot_dim) change for contexts `factor` times as long as the trained ones:
 *   NONE    not at all
 *   LINEAR  f_i / factor
 *   BASE    base factor^(rot_dim / (rot_dim - 2)) in place of base: the slowest pair stretched, the fastest kept
 *   PARTS   f_i (g + (1 - g) / factor), g rising from 0 to 1 as the pair's turns over trained_len positions rise from
 *           `slow` to `fast`; the amplitude is 0.1 ln(factor) + 1 (1 with the others) */
typedef enum { MTGR_ROPE_NONE = 0, MTGR_ROPE_LINEAR = 1, MTGR_ROPE_BASE = 2, MTGR_ROPE_PARTS = 3 } mtgr_rope_scaling_t;

/* Host only: writes rot_dim / 2 frequencies (radians per position) and the amplitude to host memory.  base > 1, factor >= 1
 * (BASE: rot_dim > 2); PARTS: trained_len > 0, 0 <= slow < fast. */
mtgr_status_t mtgr_rope_frequencies(int32_t rot_dim, double base, mtgr_rope_scaling_t scaling, double factor,
                                    int64_t trained_len, double slow, double fast, double* freqs, float* amplitude);

typedef struct {
    int64_t num_tokens;       /* T, 0 .. 2^31 - 1; T times the 32-byte pieces of a head below 2^32 - 256 */
    int32_t num_seqs;         /* B, used with offsets */
    int32_t heads;            /* 1 .. 65535, here and below */
    int32_t head_dim;         /* a multiple of 8, at most 1024 */
    int32_t rot_dim;          /* a multiple of 16, 16 .. head_dim */
    int32_t layout;           /* mtgr_rope_layout_t */
    int32_t dtype;            /* mtgr_dtype_t */
    int32_t inverse;
    float amplitude;          /* finite */
    int64_t ld_x;
    int64_t ld_out;
} mtgr_rope_problem_t;

/* x, out [T, heads, head_dim]; out may be x, with the same stride.  freqs [rot_dim / 2] fp64 on the device.  The positions
 * are given [T] int32 (of any sign), or, where positions is NULL, follow from offsets: those inside each sequence; rows
 * behind the last sequence are then left as they were.  Exactly one of the two is given. */
mtgr_status_t mtgr_rope(const mtgr_rope_problem_t* p, const void* x, const int32_t* positions, const int32_t* offsets,
                        const double* freqs, void* out, mtgr_stream_t stream);

/* ---------------------------------------------------------------- causal softmax attention (bf16)
 *
 *   z_ij = scale q_i . k_j,  j <= i in the same sequence
 *   lse_i = log sum_j exp z_ij                       [heads, T] fp32
 *   o_i = sum_j exp(z_ij - lse_i) v_j
 *
 * head_dim 32, 64 or 128; heads a multiple of kv_heads.  Sums are fp32; probabilities, their gradients and the results are
 * rounded to bf16.  A sequence's results depend on its own tokens alone, and a token's output on tokens up to it alone,
 * whatever the others hold (infinities and NaN too).  Up to rounding, that is: total_tokens, num_seqs and heads choose the
 * kernels, all lengths the pieces that the backward's sums are formed in, and an infinity or NaN up to 31 tokens behind a
 * token the way that its feature is summed.  But for that, the forward of these sizes gives a token the same bits whatever
 * the other sequences and later tokens are.  Rows of outputs behind the last sequence are left as they were. */
typedef struct {
    int32_t num_seqs;         /* B >= 0 */
    int32_t heads;
    int32_t kv_heads;
    int32_t head_dim;
    int64_t total_tokens;     /* T, 0 .. 2^30 - 1: rows of the tensors, at least offsets[B]; (T / 128 + B) heads below
                                 2^24 - 2^17 */
    float scale;              /* positive and finite, in units of log 2 too */
    int32_t reserved;         /* 0 */
    int64_t ld_q;             /* q and dq */
    int64_t ld_k;             /* k and dk */
    int64_t ld_v;             /* v and dv */
    int64_t ld_o;             /* out */
    int64_t ld_do;            /* dout (backward) */
} mtgr_causal_problem_t;

/* lse may be NULL (serving). */
mtgr_status_t mtgr_causal_attn_fwd(const mtgr_causal_problem_t* p, const int32_t* offsets, const void* q, const void* k,
                                   const void* v, void* out, float* lse, mtgr_stream_t stream);

/* Workspace bytes of the backward pass; as many or fewer for fewer tokens or sequences. */
mtgr_status_t mtgr_causal_attn_workspace_size(const mtgr_causal_problem_t* p, size_t* bytes);

/* Gradients for dout [T, heads, head_dim], with out and lse of the forward pass on the same inputs.  The gradients of
 * shared key and value heads are summed in fp32 over their query heads, in a fixed order.  Infinities and NaN in a sequence
 * may spread over that sequence's gradients, and no further. */
mtgr_status_t mtgr_causal_attn_bwd(const mtgr_causal_problem_t* p, const int32_t* offsets, const void* q, const void* k,
                                   const void* v, const void* out, const float* lse, const void* dout, void* dq, void* dk,
                                   void* dv, void* workspace, size_t workspace_bytes, mtgr_stream_t stream);

/* ---------------------------------------------------------------- paged cache of keys and values (bf16)
 *
 * keys, values [num_pages, kv_heads, page_size, head_dim], dense: token p of a sequence lies in row p % page_size of page
 * page_table[sequence][p / page_size].  page_size is a power of two, 16 .. 4096.  The page table is int32
 * [num_seqs, max_pages] with a row stride ld_table; entries past a sequence's length are not used, and an entry outside
 * 0 .. num_pages-1 is no page: nothing is written through it, and its tokens count as absent. */
typedef struct {
    int64_t num_pages;        /* 1 .. 2^31 - 1 */
    int32_t page_size;
    int32_t kv_heads;
    int32_t head_dim;         /* append: a multiple of 8, at most 1024; attention: 32, 64 or 128 */
    int32_t reserved;         /* 0 */
    void* keys;
    void* values;
} mtgr_kv_cache_t;

typedef struct {
    int64_t num_tokens;       /* N, rows of q, k, v, limited as T of mtgr_rope */
    int32_t num_seqs;         /* B */
    int32_t heads;            /* of q; 0 without q */
    int32_t max_pages;        /* columns of the page table, >= 1 */
    int32_t rot_dim;          /* 0: nothing is rotated; else as in mtgr_rope */
    int32_t layout;
    float amplitude;
    int64_t ld_table;
    int64_t ld_q;
    int64_t ld_q_out;
    int64_t ld_k;
    int64_t ld_v;
} mtgr_kv_append_problem_t;

/* Appends new tokens to their sequences: rows offsets[b] .. offsets[b+1]-1 of k and v [N, kv_heads, head_dim] become tokens
 * past[b], past[b] + 1, .. of sequence b; offsets NULL: one token per sequence, N = B.  k is rotated on the way by its
 * token's position in the sequence, and q [N, heads, head_dim] is rotated by the same into q_out (which may be q, with the
 * same stride; both NULL without q).  past [B] int32; a sequence whose past is negative is left alone (q_out too), as are
 * tokens past the page table's columns and rows behind the last sequence.  Sequences must not share a page that they write. */
mtgr_status_t mtgr_kv_append(const mtgr_kv_append_problem_t* p, const mtgr_kv_cache_t* cache, const int32_t* page_table,
                             const int32_t* past, const int32_t* offsets, const void* q, const void* k, const void* v,
                             const double* freqs, void* q_out, mtgr_stream_t stream);

typedef struct {
    int32_t num_seqs;         /* B, 0 .. 65535; B heads below 2^23 */
    int32_t heads;
    int32_t max_pages;        /* columns of the page table, >= 1 */
    float scale;              /* as in mtgr_causal_problem_t */
    int64_t max_len;          /* bound of the lengths, known to the host: 0 .. max_pages page_size, below 2^31 - 4096 */
    int64_t ld_table;
    int64_t ld_q;
    int64_t ld_o;
} mtgr_cache_attn_problem_t;

/* Workspace bytes of a call.  They never fall where num_seqs or max_len rises and the heads stay the same: a workspace for the
 * largest batch and the longest history serves every smaller one. */
mtgr_status_t mtgr_cache_attn_workspace_size(const mtgr_cache_attn_problem_t* p, const mtgr_kv_cache_t* cache,
                                             size_t* bytes);

/* One query token of each sequence, q [B, heads, head_dim], against tokens 0 .. lens[b]-1 of its cache (itself among them,
 * once appended): out [B, heads, head_dim] bf16 and, unless NULL, lse [B, heads] fp32.  lens [B] int32 counts as at most
 * max_len, which should be tight: the keys are split over the chip by it.  A sequence without tokens (lens <= 0, or no
 * page) gets zeros and an lse of -inf. */
mtgr_status_t mtgr_cache_attn(const mtgr_cache_attn_problem_t* p, const mtgr_kv_cache_t* cache, const int32_t* page_table,
                              const int32_t* lens, const void* q, void* out, float* lse, void* workspace,
                              size_t workspace_bytes, mtgr_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* MTGR_CAUSAL_H */
