// The large dense products of the encoder layer (the same layouts and epilogues as gemm.hip), of the
// feed-forward block (ffn.hip) and of the softmax loss (softmax_loss.hip): a 256 x 256 tile of C per
// workgroup of 8 waves, one workgroup per CU.
//
// What bounds the 256 x 128 tiles of gemm.hip on large products is the path into LDS, not the
// matrix cores: per 32 k a tile copies 24 KB for 512 cycles of MFMA work, and the path delivers
// 1 KB per 13.2 ns and CU when a copy instruction's rows are 64 bytes long (32 k of a
// k-contiguous operand), 9.2 ns when they are 128 bytes or more (measured, operands in L2).  A
// 256 x 256 tile copies a third less per MFMA, and k steps of 64 make every row 128 bytes:
// 64 KB x 9.2 ns = 0.59 us of copies under 2048 cycles = 0.89 us of MFMAs.
//
// Wave w computes the 128 x 64 part (m half w % 2, n quarter w / 2; in the gated products 64 x 128, so that
// its 64 gate and 64 up columns leave as whole 128-byte lines) as 8 x 4 blocks of 16 x 16, transposed
// (C^T = B^T A^T), with v_mfma_f32_16x16x32_bf16.  On random data the card is bound by
// its power, not by issue: the clock falls to 1.3 - 1.8 GHz, and a loop of nothing but MFMAs on
// N(0, 1) operands in registers reaches 2.02 PFLOP/s with 16 x 16 x 32 and 1.82 with 32 x 32 x 16
// (both 2.45 on zeros).
//
// LDS (160 KB) holds three stages of A and two of B, 32 KB each: A streams from HBM and is copied
// two k steps ahead, B (weights, shared by all m blocks) comes from the XCD's L2 and is copied one
// step ahead.  One barrier per k step, half way through its second k32 part: behind it the step's
// slots are free and the next stage is visible, and the part's other MFMAs cover the first reads
// of the next stage.  Operands are read four blocks (16 MFMAs) ahead of their use, and the copies
// are spread between the MFMAs.
//
// NN / NT run persistently: a workgroup walks tiles, and the first two stages of its next tile are
// copied under the epilogue of the current one, whose stores nothing waits for.
//
// Measured against the 256 x 128 tiles, M = 79,372 rows, d = 1024: [d, 4d] product with bias + SiLU
// 1,045 -> 850 us, without 723 -> 615 us, its input gradient 702 -> 541 us (1.23 PFLOP/s; hipBLASLt
// 616 us), its weight gradient 654 -> 612 us, the d x d products 193 -> 170, 173 -> 150 and
// 190 -> 170 us.
//
// A k step takes about 1.27 us.  The epilogues of the gated product and of the softmax come on top: their
// vector work (about 28 cycles per logit and 50 per hidden value, of which transcendentals 16 and 32) fills a
// SIMD while its matrix cores rest, and both waves of a SIMD are in it at once (counters, loss of 1,900 rows,
// 400,003 classes, d = 256: MFMA 35 % busy, VALU 46 %, both at once 2 %).  Starting the workgroups at
// different times changed nothing (-1 to +2 %); two workgroups of 128 x 256 tiles per CU, which do overlap,
// have room for k steps of 32 only, whose half lines make the copies as slow as that gained (statistics,
// d = 256: 502 -> 430 us; d = 512: 1,124 -> 1,184).  Up to 256 columns the loss has softmax_tiles.h instead.
#pragma once

#include <type_traits>

#include "block_internal.h"
#include "mtgr_device.h"

namespace mtgr {

namespace {

constexpr int WBM = 256, WBN = 256, WBK = 64;
constexpr int WNM = 8, WNN = 4;                 // 16 x 16 blocks per wave (m, n)
constexpr uint32_t WSLOT = WBM * WBK * 2;       // bytes of one operand's stage
constexpr int ACC_ROUNDS = 4, ACC_SPLITS = 64;  // see acc_splits
constexpr int WQ = 4;                           // copy instructions per wave, operand and stage
// Slots: A 0, A 1, B 0, B 1 and the third stage of the deep operand; the epilogue stages in the last one.
constexpr uint32_t WSTAGING = 4 * WSLOT;

template <int V>
using IC = std::integral_constant<int, V>;

__device__ __forceinline__ uint32_t slot_a(int r) { return r == 2 ? 4u * WSLOT : (uint32_t)r * WSLOT; }
__device__ __forceinline__ uint32_t slot_b(int r) { return (2u + (uint32_t)r) * WSLOT; }      // (4: the third stage)

__device__ __forceinline__ float silu(float z) {
    return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}

// The same value, opaque to the compiler: what is derived from it is computed where it is used
// and not kept in registers across the k loop.
__device__ __forceinline__ int once(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Low or high bf16 of a packed pair.
__device__ __forceinline__ float bf16_half(uint32_t w, int hi) {
    return __uint_as_float(hi ? w & 0xffff0000u : w << 16);
}

// K splits of a product of `tiles` tiles and `steps` k steps whose rows are counted on the device: the number that
// fills one to four rounds of the chip and ends first, by the figures of tiles_of in gemm_mid.h in 64ths of a step,
// in integers, because the kernel that adds the splits has to come to the same number (188 tiles, 391 steps: four
// splits, 752 items in three rounds, 566 us; one, on 188 of the 256 CUs, 630; 130 tiles, 782 steps: 786 and 1,120).
__host__ __device__ __forceinline__ int acc_splits(int tiles, int steps) {
    constexpr int START = 346, STEP = 64, PARTIAL = 5;      // an item, its steps, its partials written and read
    if (tiles > 256 * ACC_ROUNDS) return 1;
    int best = 1, cost = (tiles + 255) / 256 * (START + STEP * steps) + PARTIAL * tiles;
#pragma unroll
    for (int k = 1; k <= ACC_ROUNDS; k++) {
        const int s = max(min(min(256 * k / max(tiles, 1), ACC_SPLITS), steps), 1);
        const int c = (s * tiles + 255) / 256 * (START + STEP * ((steps + s - 1) / s)) + PARTIAL * s * tiles;
        if (c < cost) {
            best = s;
            cost = c;
        }
    }
    return best;
}

// Columns of items of the softmax statistics: about 16 items per CU, so that the last round of them is short,
// each of as many class tiles as that leaves (their statistics stay in registers in between).
__host__ __device__ __forceinline__ int stat_chunks(int mblocks, int nblocks) {
    const int per_item = min(max(mblocks * nblocks / 4096, 1), 32);
    return (nblocks + per_item - 1) / per_item;
}

// 16 bytes that are read once: they leave the operands of the next k steps in the L2 (backward of the gated
// product, 69,563 tokens, 1024 / 2816: 551 -> 535 us).
__device__ __forceinline__ uint4 load_nt16(const void* p) {
    const u32x4_nt v = __builtin_nontemporal_load((const u32x4_nt*)p);
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// Whether a result is left in the last-level cache of 256 MB for the next product, or stored past the caches, by its
// bytes.  Measured with plain stores and with stores past the caches, us (products that write and read it, in turn):
// dz, up to 192 MiB: 2,900 rows, 20,011 classes, 120 MB, backward 171 and 186; 8,000 rows, 320 MB: 266 and 247.
// h, up to 176 MiB (training forward, 512 / 1408): 56 MB 109 and 114; 85 MB 147 and 152; 113 MB 190 and 204; 155 MB
// 263 and 273; 189 MB 317 and 329, 335 and 331 on another card; 203 MB 367 and 349; 212 MB 386 and 371.  1024 / 2816:
// 141 MB 406 and 417, 169 MB 476 and 486, 197 MB 590 and 595, 225 MB 654 and 657, 392 MB 1,210 and 1,204.
// dpre, up to 256 MiB (backward, 512 / 1408): 113 MB 243 and 250; 169 MB 317 and 323; 225 MB 448 and 467; 282 MB 553 and
// 555; 338 MB 605 and 606.  1024 / 2816: 135 MB 473 and 483, 191 MB 725 and 735, 225 MB 801 and 822, 248 MB 884 and 896.
__host__ __device__ __forceinline__ bool dz_stays(long long rows, long long ld) { return rows * ld * 2 <= 192ll << 20; }
__host__ __device__ __forceinline__ bool h_stays(long long rows, long long hidden) { return rows * hidden * 2 <= 176ll << 20; }
__host__ __device__ __forceinline__ bool dpre_stays(long long rows, long long hidden) { return rows * hidden * 4 <= 256ll << 20; }

// A plain store beside a non-temporal one of the same value: merged by the compiler, both would be plain.
__device__ __forceinline__ void store_plain16(void* p, const uint4& v) {
    asm volatile("" ::: "memory");
    *(uint4*)p = v;
    asm volatile("" ::: "memory");
}

// dgate = dh up silu'(gate) and dup = dh silu(gate) of eight columns (dh: x0, x1), each rounded once: dpre is an operand of
// the next products.
__device__ __forceinline__ void gated_gradient(const floatx4& x0, const floatx4& x1, const uint4& gate, const uint4& up,
                                               uint4* dgate, uint4* dup) {
    const uint32_t gw[4] = {gate.x, gate.y, gate.z, gate.w}, uw[4] = {up.x, up.y, up.z, up.w};
    float dg[8], du[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const float dh = e < 4 ? x0[e & 3] : x1[e & 3], z = bf16_half(gw[e >> 1], e & 1);
        const float sg = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
        const float s = dh * sg;
        du[e] = s * z;
        dg[e] = s * bf16_half(uw[e >> 1], e & 1) * (1.0f + z * (1.0f - sg));
    }
    *dgate = make_uint4(pack_bf16x2(dg[0], dg[1]), pack_bf16x2(dg[2], dg[3]), pack_bf16x2(dg[4], dg[5]), pack_bf16x2(dg[6], dg[7]));
    *dup = make_uint4(pack_bf16x2(du[0], du[1]), pack_bf16x2(du[2], du[3]), pack_bf16x2(du[4], du[5]), pack_bf16x2(du[6], du[7]));
}

// LDS hand-off between the lanes of one wave (its LDS operations run in order).
__device__ __forceinline__ void wave_lds_fence() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

}  // namespace

template <int LAYOUT, int EPI, bool COLSUM>
__global__ __launch_bounds__(512, 2) void gemm_wide_kernel(TileArgs g) {
    constexpr bool A_KR = LAYOUT == GEMM_TN;      // A stored [K][M]
    constexpr bool B_KR = LAYOUT != GEMM_NT;      // B stored [K][N]
    constexpr bool ACC = EPI == GEMM_EPI_ACC;     // fp32 partials added up over calls
    constexpr bool DIRECT = EPI == GEMM_EPI_ROWS_DIRECT;
    constexpr bool SPLIT = (LAYOUT == GEMM_TN && !DIRECT) || ACC;     // fp32 partials per K split, one tile per workgroup
    constexpr bool GATED = EPI == GEMM_EPI_GATED || EPI == GEMM_EPI_GATED_SAVE;
    constexpr bool RESIDUAL = EPI == GEMM_EPI_BIAS_RESIDUAL || EPI == GEMM_EPI_RESIDUAL;
    constexpr bool STATS = EPI == GEMM_EPI_SM_STATS, GRAD = EPI == GEMM_EPI_SM_GRAD;
    // The number of token rows is on the device (g.rows): M, or K of a weight gradient.
    constexpr bool DYN = STATS || GRAD || ACC || EPI == GEMM_EPI_ROWS || DIRECT;
    // The rows of B end before N (its last columns of C are formed from copies of the last row).
    constexpr bool B_SHORT = STATS || GRAD;
    // Which operand is copied two k steps ahead, into three stages: A, which streams while B (weights) stays
    // in the XCD's L2; the softmax products stream the classes (B) past a few m blocks of rows.
    constexpr bool DEEP_B = B_SHORT;
    constexpr int NTILE = GATED ? WBN / 2 : WBN;  // columns of C per tile
    constexpr int WAVE_M = GATED ? 64 : 128, WAVE_N = GATED ? 128 : 64;      // a wave's part of a tile
    __shared__ __align__(1024) char sm[5 * WSLOT];

    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int wm = GATED ? w & 3 : w & 1, wn = GATED ? w >> 2 : w >> 1;
    int M = (int)g.M, K = (int)g.K, mblocks = g.mblocks;
    const int N = (int)g.N;
    if constexpr (DYN) {
        if constexpr (LAYOUT == GEMM_TN) {
            K = min(*g.rows, K);
        } else {
            M = min(*g.rows, M);
            mblocks = (M + WBM - 1) / WBM;
        }
    }
    // Items (split, m block, n block), an equal share of consecutive ones per XCD (workgroup % 8):
    // an XCD's 32 workgroups share a few m blocks' rows (NN / NT) or few k ranges (TN) in its L2.
    const int x = blockIdx.x % XCDS, tiles = mblocks * g.nblocks;
    const int splits = ACC ? acc_splits(tiles, g.ks_per_split) : g.splits;
    // SM_STATS: an item is an m block and every chunks-th n block
    const int chunks = STATS ? stat_chunks(mblocks, g.nblocks) : g.nblocks;
    const int items = STATS ? mblocks * chunks : tiles * splits;
    const int share = (items + XCDS - 1) / XCDS;
    int j = blockIdx.x / XCDS, mb, nb;            // j: item within the share
    auto tile_of = [&](int jj) {
        const int it = x * share + jj;
        if (DYN && it >= items) return false;     // (no rows, no tiles)
        if constexpr (B_SHORT) {
            // Groups of g.group_m m blocks, m fastest: an XCD's workgroups share the rows of a few m
            // blocks and of a few n blocks (a class set is far larger than an L2).
            const int per = g.group_m * chunks, r = it % per, m = it / per * g.group_m;
            const int in_group = min(g.group_m, mblocks - m);
            mb = m + r % in_group;
            nb = r / in_group;
        } else {
            mb = it % tiles / g.nblocks;
            nb = it % g.nblocks;
        }
        return jj < share && it < items;
    };
    if (!tile_of(j)) return;
    const int split = SPLIT ? (x * share + j) / tiles : 0;
    const int nks = (int)(((DYN ? (long long)K : g.K) + WBK - 1) / WBK);
    const int per_split = DYN && SPLIT ? (nks + splits - 1) / splits : g.ks_per_split;
    const int ks_begin = SPLIT ? split * per_split : 0;
    const int nk = (SPLIT ? min(nks, ks_begin + per_split) : nks) - ks_begin;     // >= 1 by the plan
    if constexpr (DYN && SPLIT) {
        if (nk <= 0) {                            // a split without k
            for (int c = tid; c < WBM * WBN / 4 && !(ACC && g.accumulate); c += 512) {
                const int gm = mb * WBM + c / (WBN / 4), gn = nb * WBN + 4 * (c % (WBN / 4));
                if (gm < M && gn < N) *(floatx4*)(g.partial + ((long long)split * M + gm) * N + gn) = floatx4{};
            }
            return;
        }
    }
    if constexpr (DIRECT) {
        if (nk <= 0) {                            // no rows: no gradient
            do {
                for (int c = tid; c < WBM * WBN / 8; c += 512) {
                    const int gm = mb * WBM + c / (WBN / 8), gn = nb * WBN + 8 * (c % (WBN / 8));
                    if (gm < M && gn < N) *(uint4*)((uint16_t*)g.C + gm * g.ldc + gn) = make_uint4(0, 0, 0, 0);
                }
                j += gridDim.x / XCDS;
            } while (tile_of(j));
            return;
        }
    }
    const bool ragged = (long long)(ks_begin + nk) * WBK > K;     // the last step holds fewer than 64 k

    const uint32_t lds0 = lds_address(sm);
    const uint32_t ldsw = lds0 + __builtin_amdgcn_readfirstlane((uint32_t)w * 1024u);

    // ---- copies: instruction q of wave w fills the 1 KB block 8 q + w of a slot
    // [256 rows][64 k] (8 chunks per row, 8 rows per instruction): rows past `rvalid` and chunks
    // past `kvalid` clamp
    auto kc_offsets = [&](uint32_t* vo, long long ld, int rvalid, int kvalid) {
        const int ln = once(lane), r = 8 * w + (ln >> 3);
        const int c = min((ln & 7) ^ swz<8>(r), (kvalid >> 3) - 1);
#pragma unroll
        for (int q = 0; q < WQ; q++) vo[q] = (uint32_t)(min(64 * q + r, rvalid - 1) * ld + 8 * c) * 2u;
    };
    // [64 k][256 cols] (32 chunks per row, 2 rows per instruction)
    auto kr_offsets = [&](uint32_t* vo, long long ld, int cvalid, int kvalid) {
        const int ln = once(lane), r = 2 * w + (ln >> 5);
        const int c = min((ln & 31) ^ swz<32>(r), ((DYN ? cvalid + 7 : cvalid) >> 3) - 1);
#pragma unroll
        for (int q = 0; q < WQ; q++) vo[q] = (uint32_t)(min(16 * q + r, kvalid - 1) * ld + 8 * c) * 2u;
    };
    // The gated product's B: half q of a stage's columns holds gate columns 64 q .. + 63 of the tile, then the
    // up columns of the same numbers (hidden columns past `hvalid` clamp)
    auto gated_offsets = [&](uint32_t* vo, long long ld, int h0, int hvalid, int kvalid) {
        const int ln = once(lane), r = 2 * w + (ln >> 5), c = (ln & 31) ^ swz<32>(r);
        const int col = 8 * min(8 * (c >> 4) + (c & 7), (hvalid >> 3) - 1) + h0 + ((c & 8) ? N : 0);
#pragma unroll
        for (int q = 0; q < WQ; q++) vo[q] = (uint32_t)(min(16 * q + r, kvalid - 1) * ld + col) * 2u;
    };
    uint32_t voA[WQ], voB[WQ];
    const char *pa, *pb;
    int m0, n0;
    const long long stepA = 2ll * (A_KR ? WBK * g.lda : WBK), stepB = 2ll * (B_KR ? WBK * g.ldb : WBK);
    auto offsets_a = [&](uint32_t* vo, int kvalid) {
        if constexpr (A_KR) kr_offsets(vo, g.lda, M - m0, kvalid);
        else kc_offsets(vo, g.lda, min(WBM, M - m0), kvalid);
    };
    auto offsets_b = [&](uint32_t* vo, int kvalid) {
        if constexpr (GATED) gated_offsets(vo, g.ldb, n0, N - n0, kvalid);
        else if constexpr (B_KR) kr_offsets(vo, g.ldb, N - n0, kvalid);
        else kc_offsets(vo, g.ldb, min(WBN, (B_SHORT ? g.b_rows : N) - n0), kvalid);
    };
    auto start_tile = [&]() {
        m0 = mb * WBM;
        n0 = nb * NTILE;
        offsets_a(voA, WBK);
        offsets_b(voB, WBK);
        pa = (const char*)g.A + 2 * (A_KR ? (long long)m0 : (long long)m0 * g.lda) + ks_begin * stepA;
        pb = (const char*)g.B + 2 * (GATED ? 0ll : B_KR ? (long long)n0 : (long long)n0 * g.ldb) + ks_begin * stepB;
    };
    // copies [Q0, Q1) of stage i of one operand; stages are issued in order, the source moves on
    // after the last copy of each
    auto copy = [&](auto q0c, auto q1c, auto is_a, uint32_t slot, int i) {
        constexpr int Q0 = decltype(q0c)::value, Q1 = decltype(q1c)::value;
        constexpr bool IS_A = decltype(is_a)::value;
        uint32_t vo[WQ];
#pragma unroll
        for (int q = 0; q < WQ; q++) vo[q] = IS_A ? voA[q] : voB[q];
        if (ragged && i == nk - 1) {
            if constexpr (IS_A) offsets_a(vo, K - (ks_begin + i) * WBK);
            else offsets_b(vo, K - (ks_begin + i) * WBK);
        }
        // (the A of these products is padded with zeros in k: only the rows of B end early)
        if constexpr (ACC && !IS_A) {
            if ((ks_begin + i + 1) * WBK > g.b_rows) offsets_b(vo, g.b_rows - (ks_begin + i) * WBK);
        }
#pragma unroll
        for (int q = Q0; q < Q1; q++) lds_dma16(ldsw + slot + 8192u * q, IS_A ? pa : pb, vo[q]);
        if constexpr (Q1 == WQ) {
            if constexpr (IS_A) pa += stepA;
            else pb += stepB;
        }
    };
    using A_ = std::true_type;
    using B_ = std::false_type;
    using X_ = std::integral_constant<bool, !DEEP_B>;      // the deep operand, and the other one
    using Y_ = std::integral_constant<bool, DEEP_B>;
    auto copy_a = [&](int i, int r) { copy(IC<0>{}, IC<WQ>{}, A_{}, slot_a(r), i); };
    auto copy_b = [&](int i, int r) { copy(IC<0>{}, IC<WQ>{}, B_{}, slot_b(r), i); };
    // The k past K of a ragged last stage hold copies of valid values; zeros in both operands add
    // nothing.  Ends with a barrier.
    auto zero_tail = [&](uint32_t sa, uint32_t sb) {
        const int valid = K - (ks_begin + nk - 1) * WBK;
        auto clear = [&](bool kr, char* t) {
            if (kr) {
                for (int c = valid * 32 + tid; c < WBK * 32; c += 512) ((uint4*)t)[c] = make_uint4(0, 0, 0, 0);
            } else {
                for (int c = tid; c < WBM * 8; c += 512)
                    if (((c & 7) ^ swz<8>(c >> 3)) >= (valid >> 3)) ((uint4*)t)[c] = make_uint4(0, 0, 0, 0);
            }
        };
        clear(A_KR, sm + sa);
        clear(B_KR, sm + sb);
        lds_barrier();
    };

    // ---- operand reads: per-lane byte offsets within a slot; lane l of an operand of
    // v_mfma_f32_16x16x32_bf16 holds row (or column) l % 16 and k 8 (l / 16) .. + 7.
    // k-contiguous rows r0 + 16 b: chunk (4 p + l / 16) ^ swz(r0) for k32 part p, i.e. the offset of
    // part 0 XOR 64 p, block b at + 2048 b.
    // k-row column block c0 + 16 b: supplier rows of the two halves (k + 0..3, + 4..7) of part 0;
    // part 1 is 16384 bytes further, block b the offset XOR 32 b (c0 is a multiple of its 64 or 128 columns).
    const int lr = lane & 15, lg = lane >> 4;
    auto kc_base = [&](int r0) { return lds0 + 16u * (uint32_t)((r0 + lr) * 8 + (lg ^ swz<8>(lr))); };
    auto kr_base = [&](int c0, int half) {
        const int row = 8 * lg + 4 * half + (lr >> 2), colx = c0 + 4 * (lr & 3);
        return lds0 + 16u * (uint32_t)tile_chunk<32>(row, colx >> 3) + 2u * (uint32_t)(colx & 7);
    };
    uint32_t rm[2], rn[2];
    rm[0] = A_KR ? kr_base(WAVE_M * wm, 0) : kc_base(WAVE_M * wm);
    rm[1] = A_KR ? kr_base(WAVE_M * wm, 1) : 0;
    rn[0] = B_KR ? kr_base(WAVE_N * wn, 0) : kc_base(WAVE_N * wn);
    rn[1] = B_KR ? kr_base(WAVE_N * wn, 1) : 0;
    typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
    auto read_frag = [&](auto kr, const uint32_t (&r)[2], uint32_t slot, auto pc, auto bc) {
        constexpr uint32_t P = decltype(pc)::value, BL = decltype(bc)::value;
        if constexpr (decltype(kr)::value) {
            const uint32_t o0 = ((r[0] + slot) ^ (32u * BL)) + 16384u * P, o1 = ((r[1] + slot) ^ (32u * BL)) + 16384u * P;
            const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)o0);
            const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)o1);
            const short __attribute__((ext_vector_type(8))) v = {lo[0], lo[1], lo[2], lo[3],
                                                                 hi[0], hi[1], hi[2], hi[3]};
            return __builtin_bit_cast(bf16x8, v);
        } else {
            return *(const lds_bf16x8*)(uintptr_t)(((r[0] + slot) ^ (64u * P)) + 2048u * BL);
        }
    };
    auto read_a = [&](uint32_t slot, auto pc, auto bc) { return read_frag(std::integral_constant<bool, A_KR>{}, rm, slot, pc, bc); };
    auto read_b = [&](uint32_t slot, auto pc, auto bc) { return read_frag(std::integral_constant<bool, B_KR>{}, rn, slot, pc, bc); };
    // the operand of the wave's eight blocks (A; B in the gated products) and that of its four
    auto read_m = [&](uint32_t slot, auto pc, auto bc) { if constexpr (GATED) return read_b(slot, pc, bc); else return read_a(slot, pc, bc); };
    auto read_n = [&](uint32_t slot, auto pc, auto bc) { if constexpr (GATED) return read_a(slot, pc, bc); else return read_b(slot, pc, bc); };

    floatx4 acc[WNN][WNM];
    bf16x8 fm[WNM], fn[2][WNN];       // operands: the eight blocks (four ahead), the four blocks of both k32 parts
    float csum[8];
    const bool colsum = COLSUM && mb == 0;
    auto colsum_step = [&](uint32_t sb) {
        if (COLSUM && colsum) {
            // bias gradient: column sums of B over this K split, 8 columns x 4 rows per thread
            const int c = tid & 31, rg = tid >> 5;
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const bf16x8 v = tile_read8<32>((const uint16_t*)(sm + sb), 4 * rg + r, c);
#pragma unroll
                for (int e = 0; e < 8; e++) csum[e] += (float)v[e];
            }
        }
    };
    // Slot b of k32 part P: the four MFMAs of m block b (gated: n block b), block b + 4 read ahead (from part NP in
    // slot nsm once past the part's end), and in slots 4 and 5 the other operand's blocks of the next part.
    auto slot = [&](auto pc, auto bc, uint32_t csm, uint32_t nsm, uint32_t nsn) {
        constexpr int P = decltype(pc)::value, b = decltype(bc)::value, NP = P ^ 1;
        if constexpr (b < 4) {
            fm[b + 4] = read_m(csm, IC<P>{}, IC<b + 4>{});
        } else {
            if constexpr (b < 6) {
                fn[NP][2 * (b - 4)] = read_n(nsn, IC<NP>{}, IC<2 * (b - 4)>{});
                fn[NP][2 * (b - 4) + 1] = read_n(nsn, IC<NP>{}, IC<2 * (b - 4) + 1>{});
            }
            fm[b - 4] = read_m(nsm, IC<NP>{}, IC<b - 4>{});
        }
#pragma unroll
        for (int a = 0; a < WNN; a++)
            acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(GATED ? fm[b] : fn[P][a], GATED ? fn[P][a] : fm[b], acc[a][b], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };

    // Stores of a full tile's epilogue per wave.  The waits below count on at least as many memory
    // operations behind the copies of stage 1 (more only make them stricter).
    constexpr int NOUT = EPI == GEMM_EPI_BIAS_SILU ? 2 : 1;
    constexpr int NSTORE = STATS ? 0 : EPI == GEMM_EPI_GATED ? 8 : EPI == GEMM_EPI_GATED_SAVE ? 24
                           : EPI == GEMM_EPI_GATED_BWD ? 32 : 16 * NOUT;
    constexpr int NBIAS = B_SHORT ? WNN : 0;     // loads of a tile's class bias
    start_tile();
    copy_b(0, 0);
    copy_a(0, 0);
    if (nk > 1) {
        copy_b(1, 1);
        copy_a(1, 1);
    }
    bool counted = false;      // the previous tile of this workgroup was a full one
    float ref[STATS ? WNM : 1], sum[STATS ? WNM : 1];      // this lane's columns of an item's rows
    bool fresh = true;
    for (;;) {
        floatx4 cbias[B_SHORT ? WNN : 1];
        if constexpr (B_SHORT) {
            const char* cb = (const char*)(g.bias + n0);
            const uint32_t off = 256u * (uint32_t)wn + 16u * (uint32_t)(once(lane) >> 4);
#pragma unroll
            for (int a = 0; a < WNN; a++) cbias[a] = *(const floatx4*)(cb + (off + 64u * a));
        }
        // Stage 0 has landed (a full tile's NSTORE stores and the copies of stage 1 may be in
        // flight behind it), and the fifth slot, where the epilogue staged, is free.
        if (counted && nk > 1) wait_vmcnt<NSTORE + 2 * WQ + NBIAS>();
        else wait_vmem();
        lds_barrier();
        if (nk > 2) copy(IC<0>{}, IC<WQ>{}, X_{}, slot_a(2), 2);
        if (ragged && nk == 1) zero_tail(slot_a(0), slot_b(0));
#pragma unroll
        for (int a = 0; a < WNN; a++)
#pragma unroll
            for (int b = 0; b < WNM; b++)
#pragma unroll
                for (int r = 0; r < 4; r++) acc[a][b][r] = 0.f;
        if (COLSUM) {
#pragma unroll
            for (int e = 0; e < 8; e++) csum[e] = 0.f;
        }
        const uint32_t first_m = GATED ? slot_b(0) : slot_a(0), first_n = GATED ? slot_a(0) : slot_b(0);
        fn[0][0] = read_n(first_n, IC<0>{}, IC<0>{});
        fm[0] = read_m(first_m, IC<0>{}, IC<0>{});
        fn[0][1] = read_n(first_n, IC<0>{}, IC<1>{});
        fn[0][2] = read_n(first_n, IC<0>{}, IC<2>{});
        fn[0][3] = read_n(first_n, IC<0>{}, IC<3>{});
        fm[1] = read_m(first_m, IC<0>{}, IC<1>{});
        fm[2] = read_m(first_m, IC<0>{}, IC<2>{});
        fm[3] = read_m(first_m, IC<0>{}, IC<3>{});
        // Step i, with X the deep operand (A) and Y the other one: copies of the second half of Y(i+1), then
        // X(i+2), then, behind the barrier that frees its slot, the first half of Y(i+2).
        uint32_t sa = slot_a(0), sb = slot_b(0), sa1 = slot_a(1), sb1 = slot_b(1), sx2 = slot_a(2);
        for (int i = 0; i < nk; i++) {
            const bool cb = i > 0 && i + 1 < nk, ca = i > 0 && i + 2 < nk, cn = i + 2 < nk;
            const uint32_t cm = GATED ? sb : sa, cf = GATED ? sa : sb, nm = GATED ? sb1 : sa1, nf = GATED ? sa1 : sb1;
            colsum_step(sb);
            slot(IC<0>{}, IC<0>{}, cm, cm, cf);
            if (cb) copy(IC<2>{}, IC<3>{}, Y_{}, DEEP_B ? sa1 : sb1, i + 1);
            slot(IC<0>{}, IC<1>{}, cm, cm, cf);
            slot(IC<0>{}, IC<2>{}, cm, cm, cf);
            if (cb) copy(IC<3>{}, IC<4>{}, Y_{}, DEEP_B ? sa1 : sb1, i + 1);
            slot(IC<0>{}, IC<3>{}, cm, cm, cf);
            slot(IC<0>{}, IC<4>{}, cm, cm, cf);
            if (ca) copy(IC<0>{}, IC<1>{}, X_{}, sx2, i + 2);
            slot(IC<0>{}, IC<5>{}, cm, cm, cf);
            slot(IC<0>{}, IC<6>{}, cm, cm, cf);
            if (ca) copy(IC<1>{}, IC<2>{}, X_{}, sx2, i + 2);
            slot(IC<0>{}, IC<7>{}, cm, cm, cf);
            slot(IC<1>{}, IC<0>{}, cm, nm, nf);
            if (ca) copy(IC<2>{}, IC<3>{}, X_{}, sx2, i + 2);
            slot(IC<1>{}, IC<1>{}, cm, nm, nf);
            slot(IC<1>{}, IC<2>{}, cm, nm, nf);
            if (ca) copy(IC<3>{}, IC<4>{}, X_{}, sx2, i + 2);
            slot(IC<1>{}, IC<3>{}, cm, nm, nf);
            // stage i + 1 has landed; X(i+2) may still be in flight, in step 0 also the previous
            // tile's stores (and the class bias), which were issued between the copies of stage 1 and X(2)
            if (cn) {
                if (i == 0) wait_vmcnt<NSTORE + WQ + NBIAS>();
                else wait_vmcnt<WQ>();
            } else if (i + 1 < nk) {
                wait_vmem();
            }
            lds_barrier_seen();                 // ... everywhere, and stage i is no longer read
            if (ragged && i + 2 == nk) zero_tail(sa1, sb1);
            // (after the last step the reads touch a slot that may be changing and are not used)
            slot(IC<1>{}, IC<4>{}, cm, nm, nf);
            slot(IC<1>{}, IC<5>{}, cm, nm, nf);
            if (cn) copy(IC<0>{}, IC<1>{}, Y_{}, DEEP_B ? sa : sb, i + 2);
            slot(IC<1>{}, IC<6>{}, cm, nm, nf);
            if (cn) copy(IC<1>{}, IC<2>{}, Y_{}, DEEP_B ? sa : sb, i + 2);
            slot(IC<1>{}, IC<7>{}, cm, nm, nf);
            const uint32_t t = sa, u = sb;
            sa = sa1;
            sb = sb1;
            sa1 = DEEP_B ? t : sx2;
            sb1 = DEEP_B ? sx2 : u;
            sx2 = DEEP_B ? u : t;
        }

        // ---- epilogue.  acc[a][b] holds C of row m0 + 128 wm + 16 b + l % 16, columns
        // n0 + 64 wn + 16 a + 4 (l / 16) + 0..3 (gated: row m0 + 64 wm + 16 a + l % 16, stage columns
        // 128 wn + 16 b + 4 (l / 16) + 0..3).  Each wave passes its part through 4 KB of its own
        // in the fifth slot (no barrier), so that a store instruction writes whole 128-byte lines (or
        // 256-byte rows of fp32 partials), and the first stages of the workgroup's next tile are
        // copied meanwhile.
        const int el = once(lane), er = el & 15, eg = el >> 4;
        const int em = m0 + WAVE_M * wm, en = n0 + 64 * wn;
        const int tile_mb = mb, tile_nb = nb;          // (mb, nb, m0 and n0 move on to the next tile below)
        char* stg = sm + WSTAGING + 4096 * w;
        // fp32 rows of block b: 16-byte chunk c (of 16) of row r at chunk c ^ r
        auto stage_f32 = [&](int b) {
#pragma unroll
            for (int a = 0; a < WNN; a++)
                *(floatx4*)(stg + 256 * er + 16 * ((4 * a + eg) ^ er)) = acc[a][b];
            wave_lds_fence();
        };
        if constexpr (SPLIT) {
#pragma unroll
            for (int b = 0; b < WNM; b++) {
                stage_f32(b);
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const int row = 4 * q + eg, gm = em + 16 * b + row, gn = en + 4 * er;
                    floatx4 v = *(const floatx4*)(stg + 256 * row + 16 * (er ^ row));
                    floatx4* dst = (floatx4*)(g.partial + ((long long)split * M + gm) * N + gn);
                    if (gm < M && gn < N) {
                        if (ACC && g.accumulate) v += *dst;
                        *dst = v;
                    }
                }
                wave_lds_fence();
            }
            if (COLSUM && colsum) {
                float* red = (float*)sm;               // [16 row groups][256 columns]
                const int c = tid & 31, rg = tid >> 5;
#pragma unroll
                for (int e = 0; e < 8; e++) red[rg * WBN + 8 * c + e] = csum[e];
                lds_barrier();
                if (tid < WBN && n0 + tid < N) {
                    float s = 0.f;
#pragma unroll
                    for (int r = 0; r < 16; r++) s += red[r * WBN + tid];
                    g.colsum_partial[(long long)split * N + n0 + tid] = s;
                }
            }
            return;
        }
        const bool full = m0 + WBM <= M && n0 + NTILE <= N;
        floatx4 bi[WNN];                               // bias of this lane's columns
        if constexpr (EPI == GEMM_EPI_BIAS_SILU) {
#pragma unroll
            for (int a = 0; a < WNN; a++) {
                const int gn = en + 16 * a + 4 * eg;
                bi[a] = gn < N ? *(const floatx4*)(g.bias + gn) : floatx4{};
            }
            wait_vmcnt_seen<0>();                      // (before the copies, which it would wait for)
        }
        int4 ri[GRAD ? WNM : 1];                       // the rows of this lane
        if constexpr (GRAD) {
#pragma unroll
            for (int b = 0; b < WNM; b++) ri[b] = g.row_info[em + 16 * b + er];
        }
        // gate and up values of row 8 q + l / 8 of block b, chunk l % 8, four blocks ahead
        uint4 pg[EPI == GEMM_EPI_GATED_BWD ? 4 : 1][2], pu[EPI == GEMM_EPI_GATED_BWD ? 4 : 1][2];
        auto load_pre = [&](int b) {
            const uint16_t* R = (const uint16_t*)g.R + min(en + 8 * (el & 7), N - 8);
#pragma unroll
            for (int q = 0; q < 2; q++) {
                const uint16_t* r = R + min(em + 16 * b + 8 * q + (el >> 3), M - 1) * g.ldr;
                pg[b & 3][q] = load_nt16(r);
                pu[b & 3][q] = load_nt16(r + N);
            }
        };
        if constexpr (EPI == GEMM_EPI_GATED_BWD) {
#pragma unroll
            for (int b = 0; b < 4; b++) load_pre(b);
        }
        // residual rows (row 8 q + l / 8 of block b, chunk l % 8), four blocks ahead, and their
        // columns' bias
        uint4 rr[RESIDUAL ? 4 : 1][2];
        floatx4 rb[2];
        auto load_residual = [&](int b) {
            const uint16_t* R = (const uint16_t*)g.R + min(en + 8 * (el & 7), N - 8);
#pragma unroll
            for (int q = 0; q < 2; q++)
                rr[b & 3][q] = *(const uint4*)(R + min(em + 16 * b + 8 * q + (el >> 3), M - 1) * g.ldr);
        };
        if constexpr (RESIDUAL) {
            const int gn = min(en + 8 * (el & 7), N - 8);
            rb[0] = rb[1] = floatx4{};
            if constexpr (EPI == GEMM_EPI_BIAS_RESIDUAL) {
                rb[0] = *(const floatx4*)(g.bias + gn);
                rb[1] = *(const floatx4*)(g.bias + gn + 4);
            }
#pragma unroll
            for (int b = 0; b < 4; b++) load_residual(b);
        }
        bool more, last_of_item = true;
        if (STATS && nb + chunks < g.nblocks) {
            nb += chunks;
            more = true;
            last_of_item = false;
        } else {
            j += gridDim.x / XCDS;
            more = tile_of(j);
        }
        if (more) start_tile();
        if constexpr (B_SHORT) wait_vmcnt_seen<0>();   // (before the copies, which it would wait for)
        if (more) {
            copy_b(0, 0);
            copy_a(0, 0);
            if (nk > 1) {
                copy_b(1, 1);
                copy_a(1, 1);
            }
        }
        counted = full;
        if constexpr (STATS) {
            // Softmax statistics in units of log 2, z = scale log2(e) x.w + bias: sum of 2^(z - ref) over the
            // columns of a row that this lane has seen in the item.  ref is the lane's maximum in the item's
            // first tile.  Later tiles cost no maximum: terms far below ref do not count beside it, and
            // terms far above are noticed in their sum, which the float range holds up to 2^127 times ref.
            // It starts at the lowest number, so that columns of -inf alone leave a sum of 0.
            bool high = fresh;
            float part[WNM];
            if (fresh) {
#pragma unroll
                for (int b = 0; b < WNM; b++) {
                    ref[b] = -3.402823466e38f;
                    sum[b] = 0.f;
                }
            } else {
#pragma unroll
                for (int b = 0; b < WNM; b++) {
                    float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int a = 0; a < WNN; a++)
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            s4[e] += __builtin_amdgcn_exp2f(fmaf(acc[a][b][e], g.scale, cbias[a][e]) - ref[b]);
                    part[b] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
                    high |= !(part[b] < 0x1p100f);
                }
            }
            if (__any(high)) {
#pragma unroll
                for (int b = 0; b < WNM; b++) {
                    float top = ref[b];
#pragma unroll
                    for (int a = 0; a < WNN; a++)
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            acc[a][b][e] = fmaf(acc[a][b][e], g.scale, cbias[a][e]);
                            top = fmaxf(top, acc[a][b][e]);
                        }
                    float s = sum[b] * __builtin_amdgcn_exp2f(ref[b] - top);
#pragma unroll
                    for (int a = 0; a < WNN; a++)
#pragma unroll
                        for (int e = 0; e < 4; e++) s += __builtin_amdgcn_exp2f(acc[a][b][e] - top);
                    sum[b] = s;
                    ref[b] = top;
                }
            } else {
#pragma unroll
                for (int b = 0; b < WNM; b++) sum[b] += part[b];
            }
            fresh = last_of_item;
            if (last_of_item) {
                // the four lanes of a row together, to slot (chunk, wave)
#pragma unroll
                for (int b = 0; b < WNM; b++) {
                    float top = fmaxf(ref[b], __shfl_xor(ref[b], 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    float s = sum[b] * __builtin_amdgcn_exp2f(ref[b] - top);
                    s += __shfl_xor(s, 16, 64);
                    s += __shfl_xor(s, 32, 64);
                    const int gm = em + 16 * b + er;
                    if (eg == 0 && gm < M) g.stats[(long long)(4 * (tile_nb % chunks) + wn) * g.M + gm] = make_float2(top, s);
                }
            }
        } else if constexpr (EPI == GEMM_EPI_GATED_BWD) {
            const bool keep = dpre_stays(M, N);
            // dh passes through LDS in fp32, one block at a time, so that a lane has 8 columns of a row:
            // dgate = dh up silu'(gate), dup = dh silu(gate), rounded once
#pragma unroll
            for (int b = 0; b < WNM; b++) {
                stage_f32(b);
#pragma unroll
                for (int q = 0; q < 2; q++) {
                    const int row = 8 * q + (el >> 3), ch = el & 7, gm = em + 16 * b + row, gn = en + 8 * ch;
                    const floatx4 x0 = *(const floatx4*)(stg + 256 * row + 16 * ((2 * ch) ^ row));
                    const floatx4 x1 = *(const floatx4*)(stg + 256 * row + 16 * ((2 * ch + 1) ^ row));
                    uint4 og, ou;
                    gated_gradient(x0, x1, pg[b & 3][q], pu[b & 3][q], &og, &ou);
                    if (full || (gm < M && gn < N)) {
                        uint16_t* dst = (uint16_t*)g.C + gm * g.ldc + gn;
                        if (keep) {
                            store_plain16(dst, og);
                            store_plain16(dst + N, ou);
                        } else {
                            store_nt16(dst, &og);
                            store_nt16(dst + N, &ou);
                        }
                    }
                }
                if (b < 4) load_pre(b + 4);
                wave_lds_fence();
            }
        } else if constexpr (GATED) {
            const bool keep_h = h_stays(M, N);
            // acc[a][0..3] hold gate columns en + 16 b + 4 (l / 16) + 0..3, acc[a][4..7] the up columns of the same
            // numbers; h is rounded as an operand of the second product, from unrounded values.  32 rows at a time:
            // 16-byte chunk c (of 8) of row r at c ^ (r & 7)
            auto rows_out = [&](int rd, uint16_t* base, long long ld, bool keep, auto value) {
#pragma unroll
                for (int aa = 0; aa < 2; aa++)
#pragma unroll
                    for (int b = 0; b < 4; b++) {
                        const floatx4 v = value(2 * rd + aa, b);
                        *(uint2*)(stg + 128 * (16 * aa + er) + 16 * ((2 * b + (eg >> 1)) ^ (er & 7)) + 8 * (eg & 1)) =
                            make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                    }
                wave_lds_fence();
                const int gm = em + 32 * rd + (el >> 3), gn = en + 8 * (el & 7);
                uint16_t* dst = base + gm * ld + gn;
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const uint4 v = *(const uint4*)(stg + 128 * (8 * q + (el >> 3)) + 16 * ((el & 7) ^ (el >> 3)));
                    if (full || (gm + 8 * q < M && gn < N)) {
                        if (keep) store_plain16(dst + 8 * q * ld, v);
                        else store_nt16(dst + 8 * q * ld, &v);
                    }
                }
                wave_lds_fence();
            };
#pragma unroll
            for (int rd = 0; rd < 2; rd++) {
                if constexpr (EPI == GEMM_EPI_GATED_SAVE) {
                    rows_out(rd, (uint16_t*)g.C, g.ldc, false, [&](int a, int b) { return acc[a][b]; });
                    rows_out(rd, (uint16_t*)g.C + N, g.ldc, false, [&](int a, int b) { return acc[a][b + 4]; });
                }
                rows_out(rd, (uint16_t*)g.C2, g.ldc2, keep_h, [&](int a, int b) {
                    const floatx4 ga = acc[a][b], up = acc[a][b + 4];
                    return floatx4{silu(ga[0]) * up[0], silu(ga[1]) * up[1], silu(ga[2]) * up[2], silu(ga[3]) * up[3]};
                });
            }
        } else if constexpr (!RESIDUAL) {
            if constexpr (GRAD) {
                // dz = g (exp(z - lse) - [column = label]) / max |g| in place of the products, and its column sums
                const float top = ((const float*)g.rows)[1];     // the largest |g|
                floatx4 cs[WNN];
#pragma unroll
                for (int a = 0; a < WNN; a++) cs[a] = floatx4{};
#pragma unroll
                for (int b = 0; b < WNM; b++) {
                    const float lse = __int_as_float(ri[b].x), gr = __int_as_float(ri[b].y) / top;
                    const float gp = gr * __int_as_float(ri[b].w);
                    const int label = ri[b].z - g.class0 - en;
#pragma unroll
                    for (int a = 0; a < WNN; a++)
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            acc[a][b][e] = gp * __builtin_amdgcn_exp2f(fmaf(acc[a][b][e], g.scale, cbias[a][e]) - lse);
                    if (__any((unsigned)label < 64u)) {
#pragma unroll
                        for (int a = 0; a < WNN; a++)
#pragma unroll
                            for (int e = 0; e < 4; e++)
                                if (label == 16 * a + 4 * eg + e) acc[a][b][e] -= gr;
                    }
                    if (g.col_partial != nullptr) {
#pragma unroll
                        for (int a = 0; a < WNN; a++) cs[a] += acc[a][b];
                    }
                }
                if (g.col_partial != nullptr) {
#pragma unroll
                    for (int a = 0; a < WNN; a++) {
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            float v = dpp_add<0xB1>(cs[a][e]);
                            v = dpp_add<0x4E>(v);
                            v = dpp_add<0x141>(v);
                            cs[a][e] = dpp_add<0x140>(v);
                        }
                        if (er == 0)
                            *(floatx4*)(g.col_partial + (long long)(2 * tile_mb + wm) * g.N + en + 16 * a + 4 * eg) = cs[a];
                    }
                }
            }
            // (scale and the largest |g| one after the other: their product alone may leave the float range)
            const float largest = DIRECT ? ((const float*)g.rows)[1] : 0.f;
            const bool plain = GRAD && dz_stays(M, g.ldc);
            // bf16 (dz: an operand of the next two products; its column sums above take it unrounded), 32 rows (two blocks) at
            // a time: 16-byte chunk c (of 8) of row r at c ^ (r & 7)
#pragma unroll
            for (int rd = 0; rd < WNM / 2; rd++)
#pragma unroll
                for (int out = 0; out < NOUT; out++) {
#pragma unroll
                    for (int bb = 0; bb < 2; bb++)
#pragma unroll
                        for (int a = 0; a < WNN; a++) {
                            floatx4 v = acc[a][2 * rd + bb];
                            if constexpr (DIRECT) v = v * g.scale * largest;
                            if (out == 1) {
#pragma unroll
                                for (int e = 0; e < 4; e++) v[e] = silu(v[e] + bi[a][e]);
                            }
                            *(uint2*)(stg + 128 * (16 * bb + er) + 16 * ((2 * a + (eg >> 1)) ^ (er & 7)) + 8 * (eg & 1)) =
                                make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                        }
                    wave_lds_fence();
                    uint16_t* Cout = (uint16_t*)(out == 0 ? g.C : g.C2);
                    const long long ldo = out == 0 ? g.ldc : g.ldc2;
                    uint4 v[4];
#pragma unroll
                    for (int q = 0; q < 4; q++)
                        v[q] = *(const uint4*)(stg + 128 * (8 * q + (el >> 3)) + 16 * ((el & 7) ^ (el >> 3)));
                    const int gm = em + 32 * rd + (el >> 3), gn = en + 8 * (el & 7);
                    uint16_t* dst = Cout + gm * ldo + gn;
                    if (plain) {
#pragma unroll
                        for (int q = 0; q < 4; q++)
                            if (full || (gm + 8 * q < M && gn < N)) store_plain16(dst + 8 * q * ldo, v[q]);
                    } else if (full) {
#pragma unroll
                        for (int q = 0; q < 4; q++) store_nt16(dst + 8 * q * ldo, &v[q]);
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; q++)
                            if (gm + 8 * q < M && gn < N) store_nt16(dst + 8 * q * ldo, &v[q]);
                    }
                    wave_lds_fence();
                }
        } else {
            // bias + residual: the fp32 products of one block at a time, so that
            // acc + (bias + residual) is formed in fp32 and rounded once
#pragma unroll
            for (int b = 0; b < WNM; b++) {
                stage_f32(b);
#pragma unroll
                for (int q = 0; q < 2; q++) {
                    const int row = 8 * q + (el >> 3), ch = el & 7, gm = em + 16 * b + row, gn = en + 8 * ch;
                    const floatx4 x0 = *(const floatx4*)(stg + 256 * row + 16 * ((2 * ch) ^ row));
                    const floatx4 x1 = *(const floatx4*)(stg + 256 * row + 16 * ((2 * ch + 1) ^ row));
                    const uint32_t rw[4] = {rr[b & 3][q].x, rr[b & 3][q].y, rr[b & 3][q].z, rr[b & 3][q].w};
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        v[e] = x0[e] + (rb[0][e] + bf16_half(rw[e >> 1], e & 1));
                        v[4 + e] = x1[e] + (rb[1][e] + bf16_half(rw[2 + (e >> 1)], e & 1));
                    }
                    const uint4 o = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                               pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
                    if (full || (gm < M && gn < N)) store_nt16((uint16_t*)g.C + gm * g.ldc + gn, &o);
                }
                if (b < 4) load_residual(b + 4);
                wave_lds_fence();
            }
        }
        if (!more) return;
    }
}

template <int LAYOUT, int EPI, bool COLSUM>
static hipError_t wide_launch(const TileArgs& g, hipStream_t s) {
    // NN / NT: one workgroup per CU (those without a tile end at once); TN: one per (split, tile)
    const int items = g.mblocks * g.nblocks * g.splits;
    const int gx = LAYOUT == GEMM_TN && EPI != GEMM_EPI_ROWS_DIRECT ? XCDS * ((items + XCDS - 1) / XCDS) : WIDE_WORKGROUPS;
    gemm_wide_kernel<LAYOUT, EPI, COLSUM><<<gx, 512, 0, s>>>(g);
    return hipGetLastError();
}

}  // namespace mtgr
