// Forward of the causal softmax attention.
//
// One workgroup = 4 waves = 128 query rows of one (sequence, head), 32 rows per wave, over the 64-key tiles up to its last
// row.  A wave computes the transposed products: S^T (32 keys x 32 queries) = K Q^T, so that a lane holds 16 scores of one
// query (lane % 32) and the packed probabilities serve directly as the operand of O^T += V^T P^T, whose columns, again a
// query per lane, are rescaled by one multiplication per lane where the running maximum grows.
#include "causal_device.h"

namespace mtgr {
namespace {

using namespace causal;
constexpr int BN = 64;        // keys of a tile

// Output rows with infinities or NaN once more, a key after the other: P = 0 of the keys behind a query, times an infinite or
// NaN value there, is NaN in the products.  Such rows are rare, so that this path is slow (about 0.2 us per row and
// thousand keys) and costs the others one look at their results.  A lane holds features lane, lane + 64 of the row; finite
// ones keep what the products gave.
template <int DH>
__device__ void redo_rows(const CausalArgs& a, const Tile& at, const uint16_t* sO, int qw, int h, int hk, float m, float inv,
                          unsigned long long rows, int lane) {
    constexpr int CPR = DH / 8, F = (DH + 63) / 64;
    const bool has = lane < DH;
    wait_vmem();                                                 // the rows as they are have been written
    while (rows) {
        const int r = __builtin_ctzll(rows), i = qw + r;
        rows &= rows - 1;
        const float mc = __shfl(m, r, 64) * a.c, scale = __shfl(inv, r, 64);
        const uint16_t* Q = (const uint16_t*)a.q + (long long)(at.o + i) * a.ld_q + h * DH;
        float q[F], o[F];
#pragma unroll
        for (int f = 0; f < F; f++) {
            q[f] = has ? bf16_to_f32(Q[lane + 64 * f]) : 0.f;
            o[f] = 0.f;
        }
        for (int j = 0; j <= i; j++) {
            const uint16_t* K = (const uint16_t*)a.k + (long long)(at.o + j) * a.ld_k + hk * DH;
            const uint16_t* V = (const uint16_t*)a.v + (long long)(at.o + j) * a.ld_v + hk * DH;
            float s = 0.f;
#pragma unroll
            for (int f = 0; f < F; f++) s = __builtin_fmaf(q[f], has ? bf16_to_f32(K[lane + 64 * f]) : 0.f, s);
            const float p = bf16_to_f32((uint16_t)f32_to_bf16_bits(__builtin_amdgcn_exp2f(__builtin_fmaf(wave_sum(s), a.c, -mc))));
#pragma unroll
            for (int f = 0; f < F; f++) o[f] = __builtin_fmaf(p, has ? bf16_to_f32(V[lane + 64 * f]) : 0.f, o[f]);
        }
#pragma unroll
        for (int f = 0; f < F; f++) {
            const int d = lane + 64 * f;
            if (has && (sO[8 * tile_chunk<CPR>(r, d >> 3) + (d & 7)] & 0x7f80) == 0x7f80)
                ((uint16_t*)a.out)[(long long)(at.o + i) * a.ld_o + h * DH + d] = (uint16_t)f32_to_bf16_bits(o[f] * scale);
        }
    }
}

template <int DH>
__global__ __launch_bounds__(256, 2) void causal_fwd_kernel(CausalArgs a) {
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
    const int qw = q0 + 32 * w, qi = qw + col;
    bf16x8 qreg[KSTEPS];
    {
        const uint16_t* Q = (const uint16_t*)a.q + (long long)(at.o + min(qi, n - 1)) * a.ld_q + h * DH + 8 * hh;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++) qreg[kk] = as_bf16x8(*(const uint4*)(Q + 16 * kk));
    }
    floatx16 oacc[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) oacc[d] = floatx16{};
    float m = -3.0e38f, l = 0.f;                                 // running maximum of the scores, sum of 2^(c (s - m))
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
            if (k0 > qw) continue;                               // behind all of the wave's rows
            floatx16 s{};
#pragma unroll
            for (int kk = 0; kk < KSTEPS; kk++)
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sK, 32 * half + col, 2 * kk + hh), qreg[kk], s, 0, 0, 0);
            if (k0 == qw) {                                      // on the diagonal: element e is key 8 (e / 4) + 4 hh + e % 4
#pragma unroll
                for (int e = 0; e < 16; e++) s[e] = 8 * (e >> 2) + 4 * hh + (e & 3) > col ? neg_inf() : s[e];
            }
            float top = s[0];
#pragma unroll
            for (int e = 1; e < 16; e++) top = fmaxf(top, s[e]);
            top = fmaxf(max_halves(top), m);
            if (__any(top > m)) {
                const float f = __builtin_amdgcn_exp2f((m - top) * a.c);
                l *= f;
#pragma unroll
                for (int d = 0; d < DBLK; d++) oacc[d] *= f;
                m = top;
            }
            const float mc = m * a.c;
            uint32_t pk[8];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c, -mc));
                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], a.c, -mc));
                l += p0 + p1;
                pk[e >> 1] = pack_bf16x2(p0, p1);
            }
#pragma unroll
            for (int kq = 0; kq < 2; kq++) {
                const bf16x8 pb = as_bf16x8(make_uint4(pk[4 * kq], pk[4 * kq + 1], pk[4 * kq + 2], pk[4 * kq + 3]));
#pragma unroll
                for (int d = 0; d < DBLK; d++)
                    oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        tile_read_tr<CPR>(sV, 32 * half + 16 * kq, 32 * d, lane), pb, oacc[d], 0, 0, 0);
            }
        }
    }
    __syncthreads();                                             // the tiles' LDS is reused below
    l = sum_halves(l);
    if (a.lse && hh == 0 && qi < n) a.lse[h * a.T + at.o + qi] = m * a.scale + logf(l);
    // (0 times an infinity or NaN is NaN)
    float zero = 0.f;
#pragma unroll
    for (int d = 0; d < DBLK; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) zero = __builtin_fmaf(oacc[d][e], 0.f, zero);
    const unsigned long long bad = __ballot(zero != 0.f && qi < n);
    const float inv = 1.0f / l;
    uint16_t* sO = sKV[0] + w * 32 * DH;
    store_rows<DH>(oacc, inv, sO, (uint16_t*)a.out + (long long)at.o * a.ld_o + h * DH, a.ld_o, qw, n, lane);
    if (bad) redo_rows<DH>(a, at, sO, qw, h, hk, m, inv, (bad | (bad >> 32)) & 0xffffffffull, lane);
}

}  // namespace

hipError_t launch_causal_fwd(const CausalArgs& a, int head_dim, hipStream_t s) {
    const int grid = a.slots * a.H;
    switch (head_dim) {
        case 32: causal_fwd_kernel<32><<<grid, 256, 0, s>>>(a); break;
        case 64: causal_fwd_kernel<64><<<grid, 256, 0, s>>>(a); break;
        case 128: causal_fwd_kernel<128><<<grid, 256, 0, s>>>(a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace mtgr
