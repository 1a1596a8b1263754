// Forward of the causal softmax attention.
//
// One workgroup = 4 waves = 128 query rows of one (sequence, head), 32 rows per wave, over the 64-key tiles up to its last
// row.  A wave computes the transposed products: S^T (32 keys x 32 queries) = K Q^T, so that a lane holds 16 scores of one
// query (lane % 32) and the packed probabilities serve directly as the operand of O^T += V^T P^T, whose columns, again a
// query per lane, are rescaled by one multiplication per lane where the running maximum grows.
#include <type_traits>

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
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, TILE = BN * DH, NK = DH / 32;
    constexpr int NM = KSTEPS + 2 * DBLK, PF = 3;                // products of a step; how far ahead operands are read
    __shared__ __align__(16) uint16_t sKV[4][TILE];              // K 0, K 1, V 0, V 1
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    int id = blockIdx.x;
    const int hk = id % a.Hk;
    id /= a.Hk;
    const int h = hk * a.group + id % a.group;
    const Tile at = tile_of_slot(a.offsets, a.B, a.T, a.slots - 1 - id / a.group);
    const int q0 = at.tile * BM, n = at.n;
    if (at.tile < 0) return;
    const uint16_t* Qb = (const uint16_t*)a.q + (long long)at.o * a.ld_q;
    const uint16_t* Kb = (const uint16_t*)a.k + (long long)at.o * a.ld_k;
    const uint16_t* Vb = (const uint16_t*)a.v + (long long)at.o * a.ld_v;
    const int qw = q0 + 32 * w, qi = qw + col;
    const int nh = qw < n ? qw / 32 + 1 : 0;                     // halves that this wave's rows see, the last on the diagonal
    const int ntk = (min(q0 + BM, n) + BN - 1) / BN;
    auto issue_k = [&](int t, int buf) { tile_dma<DH, 64, false, true>(sKV[buf], Kb, a.ld_k, t * BN, n, hk * DH, tid); };
    auto issue_v = [&](int t, int buf) { tile_dma<DH, 64, false, true>(sKV[2 + buf], Vb, a.ld_v, t * BN, n, hk * DH, tid); };
    // The workgroup's query rows come in as two tiles, through the second buffers.
    tile_dma<DH>(sKV[1], Qb, a.ld_q, q0, n, h * DH, tid);
    if (q0 + BN < n) tile_dma<DH>(sKV[3], Qb, a.ld_q, q0 + BN, n, h * DH, tid);
    issue_k(0, 0);
    issue_v(0, 0);
    wait_vmcnt_seen<0>();
    lds_barrier();
    bf16x8 qreg[KSTEPS];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) qreg[kk] = tile_read8<CPR>(sKV[w < 2 ? 1 : 3], 32 * (w & 1) + col, 2 * kk + hh);
    wait_lgkm_seen();
    lds_barrier();                                               // every wave holds its Q
    if (ntk > 1) issue_k(1, 1);

    const uint32_t kofs0 = tile_ofs<CPR>(col, hh);
    uint32_t vofs0, vofs1;
    tile_ofs_tr<CPR>(0, lane, vofs0, vofs1);
    constexpr uint32_t ROW16 = 16u * CPR * 16u;                  // bytes of 16 tile rows

    floatx16 oacc[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) oacc[d] = floatx16{};
    // Scores are taken relative to m, a score that is at most 8 / c below the largest so far: outputs and sums are rescaled
    // only where a score passes it by more, so that probabilities reach 2^8, which bf16 and fp32 hold as well as 1.
    float m = -3.0e38f, mc = m * a.c, l0 = 0.f, l1 = 0.f;
    auto mask = [&](floatx16& s) {                               // on the diagonal: element e is key 8 (e / 4) + 4 hh + e % 4
#pragma unroll
        for (int e = 0; e < 16; e++) s[e] = 8 * (e >> 2) + 4 * hh + (e & 3) > col ? neg_inf() : s[e];
    };
    auto raise = [&](float top) {
        top = max_halves(top);
        if (__any(__builtin_fmaf(top, a.c, -mc) > 8.f)) {
            top = fmaxf(top, m);
            const float f = __builtin_amdgcn_exp2f((m - top) * a.c);
            l0 *= f;
            l1 *= f;
#pragma unroll
            for (int d = 0; d < DBLK; d++) oacc[d] *= f;
            m = top;
            mc = m * a.c;
        }
    };
    // A step: probabilities and their products with V for half HC of the tile in buffer VB, whose scores are `cur`; beside
    // them the next half's scores from half HN of K buffer KB, masked if it is the diagonal one.  The products are issued one
    // by one between the elements' arithmetic, since a wave's matrix and vector instructions run side by side: scores beside
    // elements 0 .. 11, keys 0 .. 15 beside the rest, keys 16 .. 31 beside the next scores' maximum.  The last step forms
    // scores that nothing uses: a second form without them made the compiler copy the accumulators between the two.
    auto step = [&](auto vb_tag, auto hc_tag, auto kb_tag, auto hn_tag, const floatx16& cur, floatx16& nxt, int j) {
        constexpr int VB = decltype(vb_tag)::value, HC = decltype(hc_tag)::value, KB = decltype(kb_tag)::value,
                      HN = decltype(hn_tag)::value;
        const uint16_t* Vc = sKV[2 + VB];
        const uint16_t* Kn = sKV[KB];
        auto operand = [&](int i) {
            if (i < KSTEPS) return lds_read16(Kn, (kofs0 ^ (32u * i)) + 2 * HN * ROW16);
            const uint32_t d = (i - KSTEPS) % DBLK, kq = (i - KSTEPS) / DBLK;
            return lds_read_tr(Vc, (vofs0 ^ (64u * d)) + (2 * HC + kq) * ROW16, (vofs1 ^ (64u * d)) + (2 * HC + kq) * ROW16);
        };
        bf16x8 op[NM];
#pragma unroll
        for (int i = 0; i < PF && i < NM; i++) op[i] = operand(i);
        float p[16];
        uint32_t pk[8];
        auto element = [&](int e) {
            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[e], a.c, -mc));
            if (e & 1) {
                l0 += p[e - 1];
                l1 += p[e];
                pk[e >> 1] = pack_bf16x2(p[e - 1], p[e]);
                // (kept here: the compiler otherwise sinks them behind the branch below)
                asm volatile("" : "+v"(pk[e >> 1]), "+v"(l0), "+v"(l1));
            }
        };
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < NM; i++) {
            if (i + PF < NM) op[i + PF] = operand(i + PF);
            if (i < KSTEPS) {
                nxt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i], qreg[i], i == 0 ? floatx16{} : nxt, 0, 0, 0);
#pragma unroll
                for (int e = 12 * i / KSTEPS; e < 12 * (i + 1) / KSTEPS; e++) element(e);
            } else {
                const int d = (i - KSTEPS) % DBLK, kq = (i - KSTEPS) / DBLK;
                if (kq == 1 && d == 0) {
                    if (j + 2 == nh) mask(nxt);
                    top = nxt[0];
                }
                const bf16x8 pb = as_bf16x8(make_uint4(pk[4 * kq], pk[4 * kq + 1], pk[4 * kq + 2], pk[4 * kq + 3]));
                oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i], pb, oacc[d], 0, 0, 0);
                if (kq == 0) {
#pragma unroll
                    for (int e = 12 + 4 * d / DBLK; e < 12 + 4 * (d + 1) / DBLK; e++) element(e);
                } else {
#pragma unroll
                    for (int e = 16 * d / DBLK; e < 16 * (d + 1) / DBLK; e++) top = fmaxf(top, nxt[e]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (j + 1 < nh) raise(top);
    };
    using C0 = std::integral_constant<int, 0>;
    using C1 = std::integral_constant<int, 1>;

    floatx16 sA, sB;                                             // scores of the tile's halves 0 and 1
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++)
        sA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(sKV[0], kofs0 ^ (32u * kk)), qreg[kk], kk == 0 ? floatx16{} : sA, 0, 0, 0);
    if (nh == 1) mask(sA);
    {
        float top = sA[0];
#pragma unroll
        for (int e = 1; e < 16; e++) top = fmaxf(top, sA[e]);
        raise(top);
    }
    // Tile t in buffers P.  K runs half a tile ahead of V.
    auto tile = [&](auto par, int t) {
        constexpr int P = decltype(par)::value;
        using CP = std::integral_constant<int, P>;
        using CQ = std::integral_constant<int, P ^ 1>;
        const bool more = t + 1 < ntk;
        // V(t) has landed; K(t + 1) may be in flight
        if (more) wait_vmcnt<NK>(); else wait_vmem();
        lds_barrier();
        if (more) issue_v(t + 1, P ^ 1);
        if (2 * t < nh) step(CP{}, C0{}, CP{}, C1{}, sA, sB, 2 * t);
        if (more) {
            // K(t + 1) has landed everywhere, and K(t) is no longer read
            wait_vmcnt<NK>();
            lds_barrier();
            if (t + 2 < ntk) issue_k(t + 2, P);
        }
        if (2 * t + 1 < nh) step(CP{}, C1{}, CQ{}, C0{}, sB, sA, 2 * t + 1);
    };
    for (int t = 0; t < ntk; t += 2) {
        tile(C0{}, t);
        if (t + 1 < ntk) tile(C1{}, t + 1);
    }
    __syncthreads();                                             // the tiles' LDS is reused below
    const float l = sum_halves(l0 + l1);
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
