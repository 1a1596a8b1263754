// The class logits of the softmax loss for rows of up to 256 columns: x W^T with the rows in registers.
//
// A workgroup of 4 waves has 256 rows, each wave 64 of them, whose operands stay in its registers (KP / 2 of
// them) while tiles of 64 classes pass through LDS, all their columns at a time: two stages, one barrier per
// tile.  Per matrix instruction that is half the LDS reads and a quarter of the copies of 128 x 128 tiles with
// both operands in LDS, and 80 KB at the most, so that two workgroups share a CU: the epilogue of one (the
// exponentials of a tile take about as long as its products) runs beside the matrix instructions of the other.
// In turn, in short bursts: 1,900 rows, 400,003 classes, d = 256: statistics 513 us on 256 x 256 tiles, 312 here (1.25
// PFLOP/s: power); dz 700 and 560 (1.5 GB written).  7,900 rows, 50,021 classes, d = 128: 190 and 109, 237 and 204.  4,800, d = 64: 98
// and 60, 118 and 118 (writes).  Wave priorities and a later start of every other workgroup changed nothing.
// Transposed as in gemm_wide.h: a lane holds rows l % 16 of each block of 16, four consecutive classes each.
#pragma once

#include "gemm_wide.h"

namespace mtgr {

namespace {

constexpr int CT_ROWS = 256, CT_CLASSES = 64, CT_MAX_D = 256;

// Class tiles of an item (256 rows; the number of rows is on the device): as many items as fill one to four rounds
// of two workgroups per CU, whichever ends first, an item's start being about CT_START tiles.  `cost`: in tiles.
constexpr int CT_SLOTS = 512, CT_ROUNDS = 4, CT_START = 2;
__host__ __device__ inline int tile_run(int mblocks, int nblocks, int* cost) {
    int best = nblocks;
    *cost = 0x7fffffff;
#pragma unroll
    for (int k = 1; k <= CT_ROUNDS; k++) {
        const int most = CT_SLOTS * k / (mblocks > 0 ? mblocks : 1), runs = most < 1 ? 1 : most < nblocks ? most : nblocks;
        const int run = (nblocks + runs - 1) / runs;
        const int c = (mblocks * ((nblocks + run - 1) / run) + CT_SLOTS - 1) / CT_SLOTS * (CT_START + run);
        if (c < *cost) {
            best = run;
            *cost = c;
        }
    }
    return best;
}

// Microseconds of the statistics (measured: a tile of two workgroups on a CU takes 1.8 us at 64 columns, 3.2 at 256).
inline double sm_tiles_us(long long rows, long long classes, int d) {
    int cost;
    tile_run((int)((rows + CT_ROWS - 1) / CT_ROWS), (int)((classes + CT_CLASSES - 1) / CT_CLASSES), &cost);
    return 5.0 + cost * (1.35 + 0.46 * ((d + 63) / 64));
}

// The lane's number, formed where it is used: no register holds it across the tiles.
__device__ __forceinline__ int lane_now() { return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, once(0))); }

}  // namespace

// KP: columns of x and w, rounded up to 64.  GRAD: dz and its column sums; otherwise the statistics of every
// run of tiles, [runs][M].
template <int KP, bool GRAD>
__global__ __launch_bounds__(256, 2) void sm_tile_kernel(TileArgs g) {
    constexpr int PARTS = KP / 32;
    constexpr uint32_t STAGE = 128u * KP;                     // 64 classes, as blocks of [64 classes][64 columns]
    __shared__ __align__(1024) char sm[2 * STAGE + (GRAD ? 4 * 2048 + CT_ROWS * 16 : 0)];
    __shared__ __align__(256) float sm_bias[2][CT_CLASSES];
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int M = min(*g.rows, (int)g.M), d = (int)g.K, mblocks = (M + CT_ROWS - 1) / CT_ROWS;
    // items (run of class tiles, m block) as in gemm_wide.h: groups of g.group_m m blocks, m fastest
    const int run = g.rows[2], runs = (g.nblocks + run - 1) / run, items = mblocks * runs;
    const int share = (items + XCDS - 1) / XCDS, it = blockIdx.x % XCDS * share + blockIdx.x / XCDS;
    if ((int)blockIdx.x / XCDS >= share || it >= items) return;
    const int per = g.group_m * runs, first_m = it / per * g.group_m, in_group = min(g.group_m, mblocks - first_m);
    const int mb = first_m + it % per % in_group, r = it % per / in_group;
    const int t0 = r * run, nt = min(g.nblocks - t0, run), m0 = mb * CT_ROWS, em = m0 + 64 * w;
    const bool full = m0 + CT_ROWS <= M, plain = GRAD && dz_stays(M, g.ldc);

    const uint32_t lds0 = lds_address(sm), ldsw = lds0 + (uint32_t)w * 1024u;
    // copies: instruction q of wave w fills the 1 KB block 4 q + w of a [64][64] block
    auto copy = [&](int t) {
        const int ln = lane_now(), cr = 8 * w + (ln >> 3), cc = (ln & 7) ^ swz<8>(cr);
        const int n0 = (t0 + t) * CT_CLASSES, last = g.b_rows - n0 - 1;
        const char* src = (const char*)g.B + 2ll * n0 * g.ldb;
        const uint32_t stage = (t & 1) ? STAGE : 0u;
#pragma unroll
        for (int q = 0; q < 2; q++) {
            const uint32_t row = (uint32_t)min(32 * q + cr, last) * (uint32_t)g.ldb;
#pragma unroll
            for (int s = 0; s < KP / 64; s++) {
                // (the last block's columns past d clamp: the rows' operands are zero there)
                const int c = s == KP / 64 - 1 ? min(cc, ((d - 64 * s) >> 3) - 1) : cc;
                lds_dma16(ldsw + stage + 8192u * s + 4096u * q, src + 128 * s, (row + 8u * c) * 2u);
            }
        }
        if (w == 0) lds_dma4(lds_address(sm_bias[t & 1]), g.bias + n0, 4u * ln);
    };
    copy(0);
    bf16x8 fm[PARTS][4];
    const int fl = lane_now(), fr = fl & 15, fg = fl >> 4;
#pragma unroll
    for (int b = 0; b < 4; b++) {
        const uint16_t* x = (const uint16_t*)g.A + (long long)min(em + 16 * b + fr, M - 1) * d + 8 * fg;
#pragma unroll
        for (int p = 0; p < PARTS; p++)
            fm[p][b] = 32 * p + 8 * fg < d ? *(const bf16x8*)(x + 32 * p) : bf16x8{};
    }
    char* stg = sm + 2 * STAGE + 2048 * w;                    // GRAD: 16 rows of a wave's results
    int4* info = (int4*)(sm + 2 * STAGE + 8192);              // GRAD: the rows' info
    float top = 1.f;
    if constexpr (GRAD) {
        top = ((const float*)g.rows)[1];
        int4 v = g.row_info[em + fl];
        v.y = __float_as_int(__int_as_float(v.y) / top);
        v.w = __float_as_int(__int_as_float(v.y) * __int_as_float(v.w));
        info[64 * w + fl] = v;
    }
    typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
    wait_vmcnt_seen<0>();
    float ref[4], sum[4];
    for (int t = 0; t < nt; t++) {
        // the tile has landed (the stores of a full block of the tile before it may be in flight behind it), and the
        // other stage is free
        if (GRAD && full && t > 0) wait_vmcnt<8>();
        else wait_vmem();
        lds_barrier();
        if (t + 1 < nt) copy(t + 1);
        const int rl = lane_now(), rr = rl & 15;
        const uint32_t rn = lds0 + ((t & 1) ? STAGE : 0u) + 16u * (uint32_t)(rr * 8 + ((rl >> 4) ^ swz<8>(rr)));
        auto read_n = [&](int p, int a) {
            return *(const lds_bf16x8*)(uintptr_t)((rn ^ (64u * (p & 1))) + 8192u * (p >> 1) + 2048u * a);
        };
        floatx4 acc[4][4];
        bf16x8 fn[4];
#pragma unroll
        for (int a = 0; a < 4; a++) fn[a] = read_n(0, a);
#pragma unroll
        for (int p = 0; p < PARTS; p++) {
#pragma unroll
            for (int a = 0; a < 4; a++) {
#pragma unroll
                for (int b = 0; b < 4; b++)
                    acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fn[a], fm[p][b], p ? acc[a][b] : floatx4{}, 0, 0, 0);
                if (p + 1 < PARTS) fn[a] = read_n(p + 1, a);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // acc[a][b]: row em + 16 b + l % 16, classes n0 + 16 a + 4 (l / 16) + 0..3
        const int n0 = (t0 + t) * CT_CLASSES, el = lane_now(), lr = el & 15, lg = el >> 4;
        floatx4 bias[4];
#pragma unroll
        for (int a = 0; a < 4; a++) bias[a] = *(const floatx4*)(sm_bias[t & 1] + 16 * a + 4 * lg);
        if constexpr (!GRAD) {
            // as in gemm_wide.h: ref is the lane's maximum of a row in the first tile
            bool high = t == 0;
            float part[4];
            if (t == 0) {
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    ref[b] = -3.402823466e38f;
                    sum[b] = 0.f;
                }
            } else {
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    float s2[2] = {0.f, 0.f};
#pragma unroll
                    for (int a = 0; a < 4; a++)
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            s2[e & 1] += __builtin_amdgcn_exp2f(fmaf(acc[a][b][e], g.scale, bias[a][e]) - ref[b]);
                    part[b] = s2[0] + s2[1];
                    high |= !(part[b] < 0x1p100f);
                }
            }
            if (__any(high)) {
#pragma unroll
                for (int b = 0; b < 4; b++) {
                    float m = ref[b];
#pragma unroll
                    for (int a = 0; a < 4; a++)
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            acc[a][b][e] = fmaf(acc[a][b][e], g.scale, bias[a][e]);
                            m = fmaxf(m, acc[a][b][e]);
                        }
                    float s = sum[b] * __builtin_amdgcn_exp2f(ref[b] - m);
#pragma unroll
                    for (int a = 0; a < 4; a++)
#pragma unroll
                        for (int e = 0; e < 4; e++) s += __builtin_amdgcn_exp2f(acc[a][b][e] - m);
                    sum[b] = s;
                    ref[b] = m;
                }
            } else {
#pragma unroll
                for (int b = 0; b < 4; b++) sum[b] += part[b];
            }
        } else {
            floatx4 cs[4];
#pragma unroll
            for (int a = 0; a < 4; a++) cs[a] = floatx4{};
#pragma unroll
            for (int b = 0; b < 4; b++) {
                const int4 ri = info[64 * w + 16 * b + lr];
                const float lse = __int_as_float(ri.x), gp = __int_as_float(ri.w);
                const int label = ri.z - g.class0 - n0;
                floatx4 v[4];
#pragma unroll
                for (int a = 0; a < 4; a++)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        v[a][e] = gp * __builtin_amdgcn_exp2f(fmaf(acc[a][b][e], g.scale, bias[a][e]) - lse);
                if (__any((unsigned)label < (unsigned)CT_CLASSES)) {
#pragma unroll
                    for (int a = 0; a < 4; a++)
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            if (label == 16 * a + 4 * lg + e) v[a][e] -= __int_as_float(ri.y);
                }
                // rounded (an operand of the next two products; the column sums above take it unrounded); 16-byte chunk c
                // (of 8) of row r at c ^ (r & 7), so that a store writes whole lines
#pragma unroll
                for (int a = 0; a < 4; a++) {
                    cs[a] += v[a];
                    *(uint2*)(stg + 128 * lr + 16 * ((2 * a + (lg >> 1)) ^ (lr & 7)) + 8 * (lg & 1)) =
                        make_uint2(pack_bf16x2(v[a][0], v[a][1]), pack_bf16x2(v[a][2], v[a][3]));
                }
                wave_lds_fence();
#pragma unroll
                for (int q = 0; q < 2; q++) {
                    const uint4 o = *(const uint4*)(stg + 128 * (8 * q + (el >> 3)) + 16 * ((el & 7) ^ (el >> 3)));
                    const int gm = em + 16 * b + 8 * q + (el >> 3);
                    if (full || gm < M) {
                        uint16_t* dst = (uint16_t*)g.C + gm * g.ldc + n0 + 8 * (el & 7);
                        if (plain) store_plain16(dst, o);
                        else store_nt16(dst, &o);
                    }
                }
                wave_lds_fence();
            }
            if (g.col_partial != nullptr) {
#pragma unroll
                for (int a = 0; a < 4; a++) {
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        float s = dpp_add<0xB1>(cs[a][e]);
                        s = dpp_add<0x4E>(s);
                        s = dpp_add<0x141>(s);
                        cs[a][e] = dpp_add<0x140>(s);
                    }
                    if (lr == 0) *(floatx4*)(g.col_partial + (long long)(4 * mb + w) * g.N + n0 + 16 * a + 4 * lg) = cs[a];
                }
            }
        }
    }
    if constexpr (!GRAD) {
        // the four lanes of a row together
        const int el = lane_now(), lr = el & 15, lg = el >> 4;
#pragma unroll
        for (int b = 0; b < 4; b++) {
            float m = fmaxf(ref[b], __shfl_xor(ref[b], 16, 64));
            m = fmaxf(m, __shfl_xor(m, 32, 64));
            float s = sum[b] * __builtin_amdgcn_exp2f(ref[b] - m);
            s += __shfl_xor(s, 16, 64);
            s += __shfl_xor(s, 32, 64);
            const int gm = em + 16 * b + lr;
            if (lg == 0 && gm < M) g.stats[(long long)r * g.M + gm] = make_float2(m, s);
        }
    }
}

template <bool GRAD>
static hipError_t sm_tile_launch(const TileArgs& g, hipStream_t s) {
    // (the rows are counted on the device)
    const long long mblocks = (g.M + CT_ROWS - 1) / CT_ROWS;
    const long long items = std::max((long long)CT_SLOTS * CT_ROUNDS, mblocks);
    const int grid = (int)(XCDS * ((items + XCDS - 1) / XCDS));
    if (g.K <= 64) sm_tile_kernel<64, GRAD><<<grid, 256, 0, s>>>(g);
    else if (g.K <= 128) sm_tile_kernel<128, GRAD><<<grid, 256, 0, s>>>(g);
    else if (g.K <= 192) sm_tile_kernel<192, GRAD><<<grid, 256, 0, s>>>(g);
    else sm_tile_kernel<256, GRAD><<<grid, 256, 0, s>>>(g);
    return hipGetLastError();
}

}  // namespace mtgr
