// Host-side argument structs and launch entry points behind include/mtgr_causal.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace mtgr {

// Rotary positions, and the append that applies them (rope.hip).
struct RopeArgs {
    long long T;
    int B;
    int heads;                // heads of x; append: of q
    int dh, rot;
    bool interleaved, inverse;
    float amplitude;
    const double* freqs;
    const void* x;            // append: q or NULL
    void* out;                // append: q_out
    long long ld_x, ld_out;
    const int* positions;     // or NULL
    const int* offsets;       // or NULL
};
hipError_t launch_rope(const RopeArgs& a, bool bf16, hipStream_t s);

struct CacheArgs {
    void *keys, *values;
    long long num_pages;
    int page_shift, kv_heads;
    const int* table;
    long long ld_table;
    int max_pages;
};
struct AppendArgs {
    RopeArgs rope;            // of q and k; rot 0: none
    CacheArgs cache;
    const int* past;
    const void *k, *v;
    long long ld_k, ld_v;
};
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t s);

// The reference that scores start from, below all that count: 3e38 in units of log 2, so that least c is finite (an infinite
// one met scores of minus infinity as NaN).
inline float least_score(float c) { return -3.0e38f / std::max(c, 1.0f); }

// Work of the dK / dV kernel (causal_plan.h).  An item is a range of the 32-query units that read a tile of 128 keys; a
// tile of many units is cut into several, which leave fp32 sums that a second kernel adds up.
struct CausalItem {
    int o, n, tile;           // the sequence's first row and length, the tile in it; tile < 0: no item
    int first, last;          // units first .. last-1 of group ceil((n - 128 tile) / 32)
    int part;                 // where the sums go; < 0: the tile is whole
    int parts, pad;           // of a tile to join: its sums are part .. part + parts - 1
};
// Causal attention (causal_fwd.hip, causal_bwd_dq.hip, causal_bwd_dkdv.hip).
struct CausalArgs {
    int B, H, Hk, group;      // group: query heads of a key head
    long long T;
    int slots;                // tiles of 128 rows, at most
    float scale, c;           // c = scale / ln 2
    float least;              // least_score(c)
    const int* offsets;
    const void *q, *k, *v, *dout;
    void* out;                // backward: read
    float* lse;               // [H, T], or NULL in the forward
    float *rows_l, *rows_d;   // [H, T] each: - lse / ln 2 and - delta, from the dQ kernel to the dK / dV kernel
    void *dq, *dk, *dv;
    CausalItem *items, *joins;       // the dK / dV kernel's plan, from the dQ kernel; behind the joins' bound, their number as parts
    float* parts;
    long long ld_q, ld_k, ld_v, ld_o, ld_do;
};

struct CausalPlan {
    int items, joins, parts;  // bounds of the items, the tiles to join and the sums of each key head
    size_t joins_ofs, parts_ofs, bytes;
};
CausalPlan causal_plan(long long T, int B, int H, int Hk, int head_dim);
hipError_t launch_causal_fwd(const CausalArgs& a, int head_dim, hipStream_t s);
hipError_t launch_causal_dq(const CausalArgs& a, const CausalPlan& p, int head_dim, hipStream_t s);
hipError_t launch_causal_dkdv(const CausalArgs& a, const CausalPlan& p, int head_dim, hipStream_t s);

// Single tokens against the cache (cache_attn.hip).
struct CacheAttnArgs {
    CacheArgs cache;
    int B, H, group;
    int chunk, splits;        // keys of a workgroup, and how many of them a sequence has at most
    int waves;                // of a workgroup: 4 or 8
    int max_len;
    float scale, c, least;    // as in CausalArgs
    const int* lens;
    const void* q;
    long long ld_q, ld_o;
    void* out;
    float* lse;               // or NULL
    float* part;              // [B H][splits][dh] sums, splits > 1
    float2* part_ml;          // [B H][splits] their maxima and totals
};
struct CacheAttnPlan {
    int chunk, splits, waves;
    size_t part_bytes;        // of the chunks' sums
    size_t need;              // with their maxima and totals
    size_t bytes;             // of a workspace, at least `need`
};
CacheAttnPlan cache_attn_plan(int B, int H, int Hk, int head_dim, long long max_len);
hipError_t launch_cache_attn(const CacheAttnArgs& a, int head_dim, hipStream_t s);

}  // namespace mtgr
