// dK and dV of the causal softmax attention.
//
// With P = exp(z - lse) recomputed from q, k and lse:  dV = P^T dO,  dP = dO V^T,  dS = P (dP - delta),  dK = scale dS^T Q.
// A workgroup owns 128 keys (32 per wave) of one (sequence, key head), K in LDS and V in registers, and goes over an item's
// units: 32 queries of one of the query heads that share the key head.  A shared head's gradients are so summed in the
// accumulators, in a fixed order.  Rounded to bf16 are P and dS (matrix operands) and the results.
//
// Four products of 60.4 million pairs of 8 heads of 128: 500 .. 550 us, 900 .. 990 TFLOP/s, bound by the matrix cores at the
// clock that the power limit leaves (busy 53 %).  - delta starts dP's accumulators, so that dS costs one multiplication.
#include <type_traits>

#include "causal_device.h"

namespace mtgr {
namespace {

using namespace causal;

constexpr int JOIN_GROUPS = 2048;                            // 8 of a CU

// A wave's sums in the order of its registers, 16 bytes per lane.
template <int DBLK>
__device__ __forceinline__ float4* part_of(float* parts, long long part, int which, int w, int lane) {
    return (float4*)parts + ((part * 2 + which) * 4 + w) * (DBLK * 4 * 64) + lane;
}

template <int DH>
__global__ __launch_bounds__(256, 2) void causal_dkdv_kernel(CausalArgs a) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, UNIT = 32 * DH;
    __shared__ __align__(16) uint16_t sK[BM * DH];
    __shared__ __align__(16) uint16_t sQG[2][2 * UNIT];          // Q, then dO, of a unit
    __shared__ __align__(16) float sL[2][32], sD[2][32];         // - lse / ln 2 and - delta of its rows
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    const int hk = blockIdx.x % a.Hk;
    const CausalItem it = a.items[blockIdx.x / a.Hk];
    if (it.tile < 0) return;
    const int k0 = it.tile * BM, n = it.n, kw = k0 + 32 * w;
    bf16x8 vreg[KSTEPS];
    {
        const uint16_t* V = (const uint16_t*)a.v + (long long)(it.o + min(kw + col, n - 1)) * a.ld_v + hk * DH + 8 * hh;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++) vreg[kk] = as_bf16x8(*(const uint4*)(V + 16 * kk));
    }
    floatx16 dk[DBLK], dv[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) dk[d] = dv[d] = floatx16{};
    const uint16_t* Qb = (const uint16_t*)a.q + (long long)it.o * a.ld_q;
    const uint16_t* Gb = (const uint16_t*)a.dout + (long long)it.o * a.ld_do;
    // the unit that is copied next: head and first row
    int h = hk * a.group + it.first / ((n - k0 + 31) / 32), row = k0 + 32 * (it.first % ((n - k0 + 31) / 32));
    auto issue = [&](int buf) {
        tile_dma_pair<DH, 32>(sQG[buf], Qb, a.ld_q, sQG[buf] + UNIT, Gb, a.ld_do, row, n, h * DH, tid);
        if (tid < 32) {
            const uint32_t voff = (uint32_t)min(tid, n - 1 - row) * 4u;
            lds_dma4(lds_address(sL[buf]), uniform_ptr(a.rows_l + h * a.T + it.o + row), voff);
            lds_dma4(lds_address(sD[buf]), uniform_ptr(a.rows_d + h * a.T + it.o + row), voff);
        }
        row += 32;
        if (row >= n) {
            row = k0;
            h++;
        }
    };
    wait_vmcnt_seen<0>();
    tile_dma<DH, BM>(sK, (const uint16_t*)a.k + (long long)it.o * a.ld_k, a.ld_k, k0, n, hk * DH, tid);
    int r0 = row;
    issue(0);
    for (int i = it.first; i < it.last; i++) {
        const int buf = (i - it.first) & 1;
        wait_vmem();
        // rows behind the sequence are copies of its last one: their probabilities are 2^-inf = 0
        if (tid < 32 && r0 + tid >= n) sL[buf][tid] = neg_inf(), sD[buf][tid] = 0.f;
        lds_barrier();
        const int q0 = r0;
        r0 = row;
        if (i + 1 < it.last) issue(buf ^ 1);
        if (q0 < kw) continue;                                   // before all of the wave's keys
        const uint16_t* sQ = sQG[buf];
        const uint16_t* sG = sQ + UNIT;
        // S and dP - delta (32 queries x 32 keys): lane = key, element 4 g + e = query 8 g + 4 hh + e
        floatx16 s{}, dp;
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const floatx4 D = *(const floatx4*)&sD[buf][8 * g + 4 * hh];
#pragma unroll
            for (int e = 0; e < 4; e++) dp[4 * g + e] = D[e];
        }
        bf16x8 qa[KSTEPS], ga[KSTEPS], kb[KSTEPS];
        auto load_s = [&](int kk) {
            qa[kk] = tile_read8<CPR>(sQ, col, 2 * kk + hh);
            kb[kk] = tile_read8<CPR>(sK, 32 * w + col, 2 * kk + hh);
            ga[kk] = tile_read8<CPR>(sG, col, 2 * kk + hh);
        };
        load_s(0);
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++) {
            if (kk + 1 < KSTEPS) load_s(kk + 1);
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qa[kk], kb[kk], s, 0, 0, 0);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ga[kk], vreg[kk], dp, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (q0 == kw) {                                          // on the diagonal
#pragma unroll
            for (int e = 0; e < 16; e++) s[e] = 8 * (e >> 2) + 4 * hh + (e & 3) < col ? neg_inf() : s[e];
        }
        uint32_t pk[8], dsk[8];
        auto elements = [&](int e) {                             // e, e + 1
            const float2_t L = *(const float2_t*)&sL[buf][8 * (e >> 2) + 4 * hh + (e & 3)];
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c, L[0]));
            const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], a.c, L[1]));
            pk[e >> 1] = pack_bf16x2(p0, p1);
            dsk[e >> 1] = pack_bf16x2(p0 * dp[e], p1 * dp[e + 1]);
        };
        constexpr int NJ = 2 * DBLK;
        bf16x8 gt[NJ], qt[NJ];
        auto load_d = [&](int j) {
            gt[j] = tile_read_tr<CPR>(sG, 16 * (j / DBLK), 32 * (j % DBLK), lane);
            qt[j] = tile_read_tr<CPR>(sQ, 16 * (j / DBLK), 32 * (j % DBLK), lane);
        };
        auto product = [&](int j) {
            const int kq = j / DBLK, d = j % DBLK;
            const bf16x8 pa = as_bf16x8(make_uint4(pk[4 * kq], pk[4 * kq + 1], pk[4 * kq + 2], pk[4 * kq + 3]));
            const bf16x8 da = as_bf16x8(make_uint4(dsk[4 * kq], dsk[4 * kq + 1], dsk[4 * kq + 2], dsk[4 * kq + 3]));
            dv[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gt[j], pa, dv[d], 0, 0, 0);
            dk[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qt[j], da, dk[d], 0, 0, 0);
        };
        // The elements of queries 0 .. 15, then those of 16 .. 31 beside the products of the first
#pragma unroll
        for (int e = 0; e < 8; e += 2) elements(e);
        load_d(0);
#pragma unroll
        for (int j = 0; j < NJ; j++) {
            if (j + 1 < NJ) load_d(j + 1);
            product(j);
            if (j < DBLK) {
#pragma unroll
                for (int e = 8 + 8 * j / DBLK; e < 8 + 8 * (j + 1) / DBLK; e += 2) elements(e);
                asm volatile("" : "+v"(dv[j % DBLK]), "+v"(dk[j % DBLK]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (it.part >= 0) {
#pragma unroll
        for (int which = 0; which < 2; which++) {
            float4* dst = part_of<DBLK>(a.parts, (long long)it.part * a.Hk + hk, which, w, lane);
            const floatx16* x = which ? dv : dk;
#pragma unroll
            for (int d = 0; d < DBLK; d++)
#pragma unroll
                for (int g = 0; g < 4; g++)
                    dst[(4 * d + g) * 64] = make_float4(x[d][4 * g], x[d][4 * g + 1], x[d][4 * g + 2], x[d][4 * g + 3]);
        }
        return;
    }
    __syncthreads();                                             // K's LDS is reused below
    uint16_t* sO = sK + w * 32 * DH;
    store_rows<DH>(dk, a.scale, sO, (uint16_t*)a.dk + (long long)it.o * a.ld_k + hk * DH, a.ld_k, kw, n, lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    store_rows<DH>(dv, 1.0f, sO, (uint16_t*)a.dv + (long long)it.o * a.ld_v + hk * DH, a.ld_v, kw, n, lane);
}

// The sums of a tile's items, added in their order.  A wave takes 32 keys' 32 features of dK or dV, four items' sums at a time, so
// that a long sequence's first tiles, whose items are many, do not hold up the rest (one of 4,000 tokens, 8 / 1 heads of 128, up
// to 63 items: the backward 174 us, with 128 keys' 128 features per workgroup 228, 79 of them here).  The workgroups go over what the plan counted.
template <int DH>
__global__ __launch_bounds__(256) void causal_dkdv_join_kernel(CausalArgs a, int most) {
    constexpr int DBLK = DH / 32, AHEAD = 4;
    const int lane = threadIdx.x & 63, units = 8 * DBLK * a.Hk;
    const int all = min(a.joins[most].parts, most) * units;
    for (int u = 4 * blockIdx.x + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); u < all; u += 4 * gridDim.x) {
        const int d = u % DBLK, w = u / DBLK % 4, which = u / (4 * DBLK) % 2, hk = u / (8 * DBLK) % a.Hk;
        const CausalItem it = a.joins[u / units];
        if (it.tile < 0) continue;
        float4 x[4] = {};
        auto add = [&](int i, auto n_tag) {                      // items i .. i + N - 1, all loads before the first sum
            constexpr int N = decltype(n_tag)::value;
            float4 v[N][4];
#pragma unroll
            for (int p = 0; p < N; p++) {
                const float4* src = part_of<DBLK>(a.parts, (long long)(it.part + i + p) * a.Hk + hk, which, w, lane);
#pragma unroll
                for (int g = 0; g < 4; g++) v[p][g] = src[(4 * d + g) * 64];
            }
#pragma unroll
            for (int p = 0; p < N; p++)
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    x[g].x += v[p][g].x;
                    x[g].y += v[p][g].y;
                    x[g].z += v[p][g].z;
                    x[g].w += v[p][g].w;
                }
        };
        int i = 0;
        for (; i + AHEAD <= it.parts; i += AHEAD) add(i, std::integral_constant<int, AHEAD>{});
        if (it.parts - i == 3) add(i, std::integral_constant<int, 3>{});
        else if (it.parts - i == 2) add(i, std::integral_constant<int, 2>{});
        else if (it.parts - i == 1) add(i, std::integral_constant<int, 1>{});
        // A lane of the lower half takes features 0 .. 15 of its row from both halves, one of the upper half 16 .. 31.
        const float scale = which ? 1.0f : a.scale;
        const int row = it.tile * BM + 32 * w + (lane & 31);
        uint32_t pk[8];
#pragma unroll
        for (int g = 0; g < 4; g++) {
            pk[2 * g] = pack_bf16x2(x[g].x * scale, x[g].y * scale);
            pk[2 * g + 1] = pack_bf16x2(x[g].z * scale, x[g].w * scale);
        }
        uint4 out[2];
#pragma unroll
        for (int g = 0; g < 2; g++) {
            const auto lo = __builtin_amdgcn_permlane32_swap(pk[2 * g], pk[2 * g + 4], false, false);
            const auto hi = __builtin_amdgcn_permlane32_swap(pk[2 * g + 1], pk[2 * g + 5], false, false);
            out[g] = make_uint4(lo[0], hi[0], lo[1], hi[1]);
        }
        if (row >= it.n) continue;
        uint16_t* dst = (uint16_t*)(which ? a.dv : a.dk) + (it.o + row) * (which ? a.ld_v : a.ld_k) + hk * DH + 32 * d + 16 * (lane >> 5);
        *(uint4*)dst = out[0];
        *(uint4*)(dst + 8) = out[1];
    }
}

template <int DH>
hipError_t dkdv(const CausalArgs& a, const CausalPlan& p, hipStream_t s) {
    causal_dkdv_kernel<DH><<<p.items * a.Hk, 256, 0, s>>>(a);
    causal_dkdv_join_kernel<DH><<<std::min(p.joins * a.Hk * (DH / 16), JOIN_GROUPS), 256, 0, s>>>(a, p.joins);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_causal_dkdv(const CausalArgs& a, const CausalPlan& p, int head_dim, hipStream_t s) {
    switch (head_dim) {
        case 32: return dkdv<32>(a, p, s);
        case 64: return dkdv<64>(a, p, s);
        case 128: return dkdv<128>(a, p, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace mtgr
