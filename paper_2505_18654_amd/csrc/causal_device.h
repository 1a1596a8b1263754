// Device-side pieces shared by the kernels behind include/mtgr_causal.h.
#pragma once

#include "causal_internal.h"
#include "mtgr_device.h"

namespace mtgr {
namespace causal {

constexpr int BM = 128;       // query rows (dK, dV: keys) of a workgroup

// Up to so many 32-row tiles (of all heads) the kernels for few are taken.  They win by far wherever a sequence is long, and
// lose less where all are short, which the host does not know.  Forward, few and other kernel: one of 700 tokens, 6 / 2 heads of
// 128, 9.9 and 17.8 us; one of 3,000, 8 heads of 128 (752 tiles), 41 and 59; one of 3,000 beside 31 of 10, 4 heads of 64 (540),
// 19 and 45; 32 of up to 320 (540), 9.5 and 9.0; 20 of 150, 4 / 2 heads of 128 (452), 11.1 and 8.1.  Above: 32 of 320, 4 heads of
// 64 (1,408), 21.7 and 10.3.
constexpr long long FEW_TILES = 1024;

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// Sequence of a slot.  The tiles (of R rows) of sequence b take slots floor(o_b / R) + b on (o: the offsets): at least
// ceil(n_b / R) of them lie before those of sequence b + 1, so that a tile's sequence follows from the offsets alone,
// without a plan, and T / R + B slots hold every tile.  The search takes the first entries of 64 ranges at once, a range per
// lane: two loads one after another for 4,096 sequences.  All lanes get the same result.  B >= 1.
struct Tile {
    int o, n, tile;           // the sequence's first row and length, the tile inside it; no tile: tile < 0
};
// begin, end: the sequence's offsets.
template <int R = BM>
__device__ __forceinline__ Tile tile_at(int begin, int end, long long T, int b, int slot) {
    // rows outside 0 .. T-1 are never touched, whatever the offsets hold
    const int o = (int)min(max((long long)begin, 0ll), T), e = (int)min((long long)end, T);
    Tile t;
    t.o = o;
    t.n = max(e - o, 0);
    t.tile = slot - begin / R - b;
    if (t.tile >= (t.n + R - 1) / R) t.tile = -1;
    return t;
}
template <int R = BM>
__device__ __forceinline__ Tile tile_of_slot(const int* offsets, int B, long long T, int slot) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = B;
    for (;;) {
        const int step = (hi - lo + 63) >> 6, i = lo + lane * step, o = offsets[min(i, B)];
        const bool before = i < hi && o / R + i <= slot;
        // (offsets that do not ascend leave the range too, as does a slot before the first sequence's)
        const int k = max(__builtin_popcountll(__ballot(before)), 1) - 1, b = min(lo + k * step, hi - 1);
        if (step == 1) {
            // the next lane holds the sequence's end, but for the last one
            const int j = b - lo, end = j < 63 ? __builtin_amdgcn_readlane(o, min(j + 1, 63)) : offsets[b + 1];
            return tile_at<R>(__builtin_amdgcn_readlane(o, j), end, T, b, slot);
        }
        lo = __builtin_amdgcn_readfirstlane(b);
        hi = min(lo + step, hi);
    }
}

// Larger (sum) of this lane's value and that of lane ^ 32, in both.
__device__ __forceinline__ float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A wave's transposed outputs (as in store_rows) as [query][feature] fp32 into its LDS tiles, 16-byte pieces swizzled by the
// query, of the first `queries` alone.
template <int DH>
__device__ __forceinline__ int part_chunk(int q, int chunk) { return q * (DH / 4) + (chunk ^ (q & (DH / 4 - 1))); }
template <int DH>
__device__ __forceinline__ void write_part(const floatx16 (&acc)[DH / 32], float* part, int lane, int queries) {
    const int col = lane & 31, hh = lane >> 5;
    if (col >= queries) return;
#pragma unroll
    for (int d = 0; d < DH / 32; d++)
#pragma unroll
        for (int g = 0; g < 4; g++)
            *(float4*)&part[4 * part_chunk<DH>(col, 8 * d + 2 * g + hh)] =
                make_float4(acc[d][4 * g], acc[d][4 * g + 1], acc[d][4 * g + 2], acc[d][4 * g + 3]);
}
// Features 4 f .. 4 f + 3 of query q over the waves' parts, relative to their largest reference score `top`, and their sum.
template <int DH, int WAVES>
__device__ __forceinline__ float4 join_parts(const uint16_t (*tiles)[2][32 * DH], const float (*ml)[2][32], int q, int f, float c,
                                             float& top, float& total) {
    top = ml[0][0][q];
#pragma unroll
    for (int j = 1; j < WAVES; j++) top = fmaxf(top, ml[j][0][q]);
    total = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int j = 0; j < WAVES; j++) {
        const float e = __builtin_amdgcn_exp2f((ml[j][0][q] - top) * c);
        const float4 v = *(const float4*)&((const float*)tiles[j])[4 * part_chunk<DH>(q, f)];
        total = __builtin_fmaf(e, ml[j][1][q], total);
        o.x = __builtin_fmaf(e, v.x, o.x);
        o.y = __builtin_fmaf(e, v.y, o.y);
        o.z = __builtin_fmaf(e, v.z, o.z);
        o.w = __builtin_fmaf(e, v.w, o.w);
    }
    return o;
}

// A wave's 32 x DH results, transposed in the accumulators (lane: row lane % 32; element 4 g + e of block d: feature
// 32 d + 8 g + 4 (lane / 32) + e), times `scale`, as bf16 rows row0 .. of dst, through 32 swizzled LDS rows of the wave.
template <int DH>
__device__ __forceinline__ void store_rows(const floatx16 (&acc)[DH / 32], float scale, uint16_t* sO, uint16_t* dst,
                                           long long ld, int row0, int n, int lane) {
    constexpr int CPR = DH / 8;
    const int col = lane & 31, hh = lane >> 5;
#pragma unroll
    for (int d = 0; d < DH / 32; d++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const int f = 32 * d + 8 * g + 4 * hh;
            *(uint2*)&sO[8 * tile_chunk<CPR>(col, f >> 3) + (f & 7)] =
                make_uint2(pack_bf16x2(acc[d][4 * g] * scale, acc[d][4 * g + 1] * scale),
                           pack_bf16x2(acc[d][4 * g + 2] * scale, acc[d][4 * g + 3] * scale));
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (each wave reads only the rows it staged)
#pragma unroll
    for (int i = 0; i < 32 * CPR / 64; i++) {
        const int c = lane + 64 * i, row = c / CPR, cc = c % CPR;
        if (row0 + row < n) store_nt16(dst + (long long)(row0 + row) * ld + cc * 8, &sO[8 * tile_chunk<CPR>(row, cc)]);
    }
}

}  // namespace causal
}  // namespace mtgr
