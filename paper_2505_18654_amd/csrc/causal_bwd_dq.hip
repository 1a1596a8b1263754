// dQ of the causal softmax attention: dQ = scale dS K with dS = P (dP - delta) recomputed.  As the forward, a workgroup
// takes 128 query rows of one (sequence, head), 32 per wave, over the 64-key tiles up to its last row; a lane holds one
// query's scores, so its lse and delta are one value each.
#include "causal_device.h"

namespace mtgr {
namespace {

using namespace causal;
constexpr int BN = 64;

template <int DH>
__global__ __launch_bounds__(256, 2) void causal_dq_kernel(CausalArgs a) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, TILE = BN * DH;
    __shared__ __align__(16) uint16_t sKV[4][TILE];              // K 0, K 1, V 0, V 1
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    int id = blockIdx.x;
    const int hk = id % a.Hk;
    id /= a.Hk;
    const int h = hk * a.group + id % a.group;
    const Tile at = tile_of_slot(a.offsets, a.B, a.T, a.slots - 1 - id / a.group);
    const int q0 = at.tile * BM, n = at.n;
    if (at.tile < 0 || q0 >= n) return;
    const uint16_t* Kb = (const uint16_t*)a.k + (long long)at.o * a.ld_k;
    const uint16_t* Vb = (const uint16_t*)a.v + (long long)at.o * a.ld_v;
    const int qw = q0 + 32 * w, qr = min(qw + col, n - 1);
    bf16x8 qreg[KSTEPS], greg[KSTEPS];
    {
        const uint16_t* Q = (const uint16_t*)a.q + (long long)(at.o + qr) * a.ld_q + h * DH + 8 * hh;
        const uint16_t* G = (const uint16_t*)a.dout + (long long)(at.o + qr) * a.ld_do + h * DH + 8 * hh;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++) {
            qreg[kk] = as_bf16x8(*(const uint4*)(Q + 16 * kk));
            greg[kk] = as_bf16x8(*(const uint4*)(G + 16 * kk));
        }
    }
    const float lse = a.lse[h * a.T + at.o + qr] * NEG_LOG2E, delta = a.delta[h * a.T + at.o + qr];
    floatx16 dq[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) dq[d] = floatx16{};
    const int ntk = (min(q0 + BM, n) + BN - 1) / BN;
    auto issue = [&](int t, int buf) {
        tile_dma<DH>(sKV[buf], Kb, a.ld_k, t * BN, n, hk * DH, tid);
        tile_dma<DH>(sKV[2 + buf], Vb, a.ld_v, t * BN, n, hk * DH, tid);
    };
    wait_vmcnt_seen<0>();
    issue(0, 0);
    for (int t = 0; t < ntk; t++) {
        wait_vmem();
        lds_barrier();
        if (t + 1 < ntk) issue(t + 1, (t + 1) & 1);
        const uint16_t* sK = sKV[t & 1];
        const uint16_t* sV = sKV[2 + (t & 1)];
#pragma unroll
        for (int half = 0; half < 2; half++) {
            const int k0 = t * BN + 32 * half;
            if (k0 > qw) continue;
            floatx16 s{}, dp{};
#pragma unroll
            for (int kk = 0; kk < KSTEPS; kk++) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sK, 32 * half + col, 2 * kk + hh), qreg[kk], s, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sV, 32 * half + col, 2 * kk + hh), greg[kk], dp, 0, 0, 0);
            }
            float ds[16];
#pragma unroll
            for (int e = 0; e < 16; e++) {
                ds[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c, lse)) * (dp[e] - delta);
                if (k0 == qw && 8 * (e >> 2) + 4 * hh + (e & 3) > col) ds[e] = 0.f;
            }
#pragma unroll
            for (int kq = 0; kq < 2; kq++) {
                const float* x = ds + 8 * kq;
                const bf16x8 db = as_bf16x8(make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                                       pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])));
#pragma unroll
                for (int d = 0; d < DBLK; d++)
                    dq[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        tile_read_tr<CPR>(sK, 32 * half + 16 * kq, 32 * d, lane), db, dq[d], 0, 0, 0);
            }
        }
    }
    __syncthreads();                                             // the tiles' LDS is reused below
    store_rows<DH>(dq, a.scale, sKV[0] + w * 32 * DH, (uint16_t*)a.dq + (long long)at.o * a.ld_q + h * DH, a.ld_q, qw, n, lane);
}

}  // namespace

hipError_t launch_causal_dq(const CausalArgs& a, int head_dim, hipStream_t s) {
    const int grid = a.slots * a.H;
    switch (head_dim) {
        case 32: causal_dq_kernel<32><<<grid, 256, 0, s>>>(a); break;
        case 64: causal_dq_kernel<64><<<grid, 256, 0, s>>>(a); break;
        case 128: causal_dq_kernel<128><<<grid, 256, 0, s>>>(a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace mtgr
