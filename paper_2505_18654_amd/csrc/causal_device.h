// Device-side pieces shared by the kernels behind include/mtgr_causal.h.
#pragma once

#include "causal_internal.h"
#include "mtgr_device.h"

namespace mtgr {
namespace causal {

constexpr int BM = 128;       // query rows (dK, dV: keys) of a workgroup

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// Sequence of a slot.  The tiles of sequence b take slots floor(o_b / 128) + b on (o: the offsets): at least
// ceil(n_b / 128) of them lie before those of sequence b + 1, so that a tile's sequence follows from the offsets alone,
// without a plan, and T / 128 + B slots hold every tile.  The search takes the first entries of 64 ranges at once, a range per
// lane: two loads one after another for 4,096 sequences.  All lanes get the same result.
struct Tile {
    int o, n, tile;           // the sequence's first row and length, the tile inside it; no tile: tile < 0
};
__device__ __forceinline__ Tile tile_at(const int* offsets, long long T, int b, int slot) {
    // rows outside 0 .. T-1 are never touched, whatever the offsets hold
    const int o = (int)min(max((long long)offsets[b], 0ll), T), e = (int)min((long long)offsets[b + 1], T);
    Tile t;
    t.o = o;
    t.n = max(e - o, 0);
    t.tile = slot - (offsets[b] >> 7) - b;
    if (t.tile >= (t.n + BM - 1) / BM) t.tile = -1;
    return t;
}
__device__ __forceinline__ Tile tile_of_slot(const int* offsets, int B, long long T, int slot) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, i = lo + lane * step;
        const bool before = i < hi && (offsets[min(i, B)] >> 7) + i <= slot;
        // (offsets that do not ascend leave the range too, as does a slot before the first sequence's)
        const int k = max(__builtin_popcountll(__ballot(before)), 1) - 1;
        lo = min(lo + k * step, hi - 1);
        hi = min(lo + step, hi);
    }
    return tile_at(offsets, T, __builtin_amdgcn_readfirstlane(lo), slot);
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
