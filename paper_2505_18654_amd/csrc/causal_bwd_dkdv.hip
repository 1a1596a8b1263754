// dK and dV of the causal softmax attention, and the row sums delta = sum_d dO O that both backward kernels need.
//
// With P = exp(z - lse) recomputed from q, k and lse:  dV = P^T dO,  dP = dO V^T,  dS = P (dP - delta),  dK = scale dS^T Q.
// A workgroup owns 128 keys (32 per wave) of one (sequence, key head) and goes over the query heads that share it and
// over their queries from its first key on, 32 at a time, so that a shared head's gradients are summed in its
// accumulators in a fixed order.
#include "causal_device.h"

namespace mtgr {
namespace {

using namespace causal;

template <int DH>
__global__ __launch_bounds__(256, 2) void causal_dkdv_kernel(CausalArgs a) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, UNIT = 32 * DH;
    __shared__ __align__(16) uint16_t sK[BM * DH];
    __shared__ __align__(16) uint16_t sQG[2][2 * UNIT];          // Q, then dO, of a unit
    __shared__ __align__(16) float sL[2][32], sD[2][32];         // lse and delta of its rows
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    const int hk = blockIdx.x % a.Hk;
    const Tile at = tile_of_slot(a.offsets, a.B, a.T, blockIdx.x / a.Hk);
    const int k0 = at.tile * BM, n = at.n;
    if (at.tile < 0 || k0 >= n) return;
    const int kw = k0 + 32 * w, kj = kw + col;
    bf16x8 vreg[KSTEPS];
    {
        const uint16_t* V = (const uint16_t*)a.v + (long long)(at.o + min(kj, n - 1)) * a.ld_v + hk * DH + 8 * hh;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++) vreg[kk] = as_bf16x8(*(const uint4*)(V + 16 * kk));
    }
    floatx16 dk[DBLK], dv[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) dk[d] = dv[d] = floatx16{};
    const uint16_t* Qb = (const uint16_t*)a.q + (long long)at.o * a.ld_q;
    const uint16_t* Gb = (const uint16_t*)a.dout + (long long)at.o * a.ld_do;
    const int units = (n - k0 + 31) / 32, all = units * a.group;
    auto issue = [&](int i, int buf) {
        const int h = hk * a.group + i / units, r0 = k0 + 32 * (i % units);
        tile_dma_pair<DH, 32>(sQG[buf], Qb, a.ld_q, sQG[buf] + UNIT, Gb, a.ld_do, r0, n, h * DH, tid);
        if (tid < 32) {
            const uint32_t voff = (uint32_t)min(tid, n - 1 - r0) * 4u;
            lds_dma4(lds_address(sL[buf]), uniform_ptr(a.lse + h * a.T + at.o + r0), voff);
            lds_dma4(lds_address(sD[buf]), uniform_ptr(a.delta + h * a.T + at.o + r0), voff);
        }
    };
    wait_vmcnt_seen<0>();
    tile_dma<DH, BM>(sK, (const uint16_t*)a.k + (long long)at.o * a.ld_k, a.ld_k, k0, n, hk * DH, tid);
    issue(0, 0);
    for (int i = 0; i < all; i++) {
        const int buf = i & 1, r0 = k0 + 32 * (i % units);
        wait_vmem();
        // rows behind the sequence are copies of its last one: an lse of +inf makes their probabilities 0
        if (tid < 32 && r0 + tid >= n) sL[buf][tid] = -neg_inf(), sD[buf][tid] = 0.f;
        lds_barrier();
        if (i + 1 < all) issue(i + 1, buf ^ 1);
        if (r0 < kw) continue;                                   // before all of the wave's keys
        const uint16_t* sQ = sQG[buf];
        const uint16_t* sG = sQ + UNIT;
        floatx16 s{}, dp{};
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sQ, col, 2 * kk + hh),
                                                        tile_read8<CPR>(sK, 32 * w + col, 2 * kk + hh), s, 0, 0, 0);
            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sG, col, 2 * kk + hh), vreg[kk], dp, 0, 0, 0);
        }
        const bool diagonal = r0 == kw;
        uint32_t pk[8], dsk[8];
#pragma unroll
        for (int g = 0; g < 4; g++) {                            // element 4 g + e is query 8 g + 4 hh + e
            const floatx4 L = *(const floatx4*)&sL[buf][8 * g + 4 * hh], D = *(const floatx4*)&sD[buf][8 * g + 4 * hh];
            float p[4], ds[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * g + e], a.c, L[e] * NEG_LOG2E));
                ds[e] = p[e] * (dp[4 * g + e] - D[e]);
                if (diagonal && 8 * g + 4 * hh + e < col) p[e] = ds[e] = 0.f;
            }
            pk[2 * g] = pack_bf16x2(p[0], p[1]);
            pk[2 * g + 1] = pack_bf16x2(p[2], p[3]);
            dsk[2 * g] = pack_bf16x2(ds[0], ds[1]);
            dsk[2 * g + 1] = pack_bf16x2(ds[2], ds[3]);
        }
#pragma unroll
        for (int kq = 0; kq < 2; kq++) {
            const bf16x8 pa = as_bf16x8(make_uint4(pk[4 * kq], pk[4 * kq + 1], pk[4 * kq + 2], pk[4 * kq + 3]));
            const bf16x8 da = as_bf16x8(make_uint4(dsk[4 * kq], dsk[4 * kq + 1], dsk[4 * kq + 2], dsk[4 * kq + 3]));
#pragma unroll
            for (int d = 0; d < DBLK; d++) {
                dv[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read_tr<CPR>(sG, 16 * kq, 32 * d, lane), pa, dv[d], 0, 0, 0);
                dk[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read_tr<CPR>(sQ, 16 * kq, 32 * d, lane), da, dk[d], 0, 0, 0);
            }
        }
    }
    __syncthreads();                                             // K's LDS is reused below
    uint16_t* sO = sK + w * 32 * DH;
    store_rows<DH>(dk, a.scale, sO, (uint16_t*)a.dk + (long long)at.o * a.ld_k + hk * DH, a.ld_k, kw, n, lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    store_rows<DH>(dv, 1.0f, sO, (uint16_t*)a.dv + (long long)at.o * a.ld_v + hk * DH, a.ld_v, kw, n, lane);
}

// A head's row per DH / 8 lanes.
template <int DH>
__global__ __launch_bounds__(256) void causal_delta_kernel(CausalArgs a, float* delta) {
    constexpr int L = DH / 8;
    const long long i = (blockIdx.x * 256ll + threadIdx.x) / L;
    const int c = threadIdx.x % L;
    if (i >= a.T * a.H) return;
    const long long t = i / a.H;
    const int h = (int)(i % a.H);
    float v = 0.f;
    if (t < a.offsets[a.B]) {
        const uint4 o = *(const uint4*)((const uint16_t*)a.out + t * a.ld_o + h * DH + 8 * c);
        const uint4 g = *(const uint4*)((const uint16_t*)a.dout + t * a.ld_do + h * DH + 8 * c);
        const uint32_t ow[4] = {o.x, o.y, o.z, o.w}, gw[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            v = __builtin_fmaf(__uint_as_float(ow[j] << 16), __uint_as_float(gw[j] << 16), v);
            v = __builtin_fmaf(__uint_as_float(ow[j] & 0xffff0000u), __uint_as_float(gw[j] & 0xffff0000u), v);
        }
    }
#pragma unroll
    for (int off = L / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    if (c == 0) delta[h * a.T + t] = v;
}

}  // namespace

hipError_t launch_causal_dkdv(const CausalArgs& a, int head_dim, hipStream_t s) {
    const int grid = a.slots * a.Hk;
    switch (head_dim) {
        case 32: causal_dkdv_kernel<32><<<grid, 256, 0, s>>>(a); break;
        case 64: causal_dkdv_kernel<64><<<grid, 256, 0, s>>>(a); break;
        case 128: causal_dkdv_kernel<128><<<grid, 256, 0, s>>>(a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_causal_delta(const CausalArgs& a, int head_dim, float* delta, hipStream_t s) {
    const long long rows = a.T * a.H;
    const int grid = (int)((rows * (head_dim / 8) + 255) / 256);
    switch (head_dim) {
        case 32: causal_delta_kernel<32><<<grid, 256, 0, s>>>(a, delta); break;
        case 64: causal_delta_kernel<64><<<grid, 256, 0, s>>>(a, delta); break;
        case 128: causal_delta_kernel<128><<<grid, 256, 0, s>>>(a, delta); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace mtgr
