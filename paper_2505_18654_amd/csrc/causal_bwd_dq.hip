// dQ of the causal softmax attention: dQ = scale dS K with dS = P (dP - delta) recomputed, delta = sum_d dO O.
//
// As the forward, a workgroup takes 128 query rows of one (sequence, head), 32 per wave, over the 64-key tiles up to its last
// row; a lane holds one query's scores, so its lse and delta are one value each.  It forms delta from the rows of dO that it
// holds anyway and leaves it, and the lse in units of log 2, both negative, for the dK / dV kernel behind it: a kernel of
// its own read dO and O once more (50 us for 68,000 tokens, 8 heads of 128).  Rounded to bf16 are dS (a matrix operand) and
// the result; delta is formed from the rounded O that the forward left, but for a sequence's first 128 rows.  These attend to
// few keys, so that O's rounding is not small beside dP - delta; they form their scores once before, and delta as the sum of P dP
// (relative errors of dQ and dK of 32 sequences of up to 320 tokens 2.4e-3, with O's rounding 2.5e-3, of shorter ones 3e-3; 500 of
// up to 100 tokens, 8 / 2 heads of 128: the backward 96 -> 107 us, 64 of up to 3,200: 968 -> 974).
//
// S and dP are formed again here, two products beside dQ's own: 440 .. 490 us for 60.4 million pairs of 8 heads of 128 (760 ..
// 840 TFLOP/s).  The matrix cores are busy 42 % of that and the vector units 33 %, and 29 % of the waves' cycles are waits; the
// forward and the dK / dV kernel, at the power limit's clock, keep the matrix cores busy 53 % and more.  Each operand from LDS
// feeds one product here: 24 reads for the 24 products of 32 keys.  With heads of 32 and 64 the elements' arithmetic, which does
// not shrink with the head, outweighs the products: vector units busy 42 and 41 %, matrix cores 16 and 32 (256 sequences of up to
// 1,000 tokens, 4 / 1 heads of 32; 8 of up to 4,096, 16 / 2 of 64).  With dS stored by the dK / dV kernel (2 bytes a pair, up to
// 2 GB) and dQ from it, the backward took 915 us instead of 947 there, with heads of 64 (8 sequences of 4,096 tokens, 16 / 2
// heads) 1,205 instead of 1,021.  A third buffer of keys, copied a tile and a half ahead, changed 1 % for the worse.
#include <type_traits>

#include "causal_plan.h"

namespace mtgr {
namespace {

using namespace causal;
constexpr int BN = 64;

// What a lane's 16 keys add to delta = sum_j P dP (of one query): g = dP - delta from the rounded O, and the sum of P (g) is
// what that delta lacks.
__device__ __forceinline__ float missing(const floatx16& s, const floatx16& g, float c, float nl) {
    float more = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) more = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, nl)), g[e], more);
    return more;
}

template <int DH>
__global__ __launch_bounds__(256, 2) void causal_dq_kernel(CausalArgs a, CausalPlan p) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, TILE = BN * DH;
    constexpr int NM = 2 * KSTEPS + 2 * DBLK, PF = 3;            // products of a step; how far ahead operands are read
    __shared__ __align__(16) uint16_t sKV[4][TILE];              // K 0, K 1, V 0, V 1
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    if (blockIdx.x == 0) {
        static_assert(PLAN_LDS * 4 <= 4 * TILE * 2, "the plan fits the tiles");
        make_plan<256>(a, p, (int*)sKV);
        return;
    }
    int id = blockIdx.x - 1;
    const int hk = id % a.Hk;
    id /= a.Hk;
    const int h = hk * a.group + id % a.group;
    const Tile at = tile_of_slot(a.offsets, a.B, a.T, a.slots - 1 - id / a.group);
    const int q0 = at.tile * BM, n = at.n;
    if (at.tile < 0) return;
    const uint16_t* Kb = (const uint16_t*)a.k + (long long)at.o * a.ld_k;
    const uint16_t* Vb = (const uint16_t*)a.v + (long long)at.o * a.ld_v;
    const int qw = q0 + 32 * w, qr = min(qw + col, n - 1);
    const int nh = qw < n ? qw / 32 + 1 : 0;                     // halves that this wave's rows see, the last on the diagonal
    const int ntk = (min(q0 + BM, n) + BN - 1) / BN;
    // The thread's number, counted afresh for each copy: kept in a register it spilled, and its reload waits for the copies
    // under way.
    auto thread = [&] {
        uint32_t none = 0;
        asm volatile("" : "+v"(none));
        return 64 * w + (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
    };
    auto issue_k = [&](int t, int buf) { tile_dma<DH>(sKV[buf], Kb, a.ld_k, t * BN, n, hk * DH, thread()); };
    auto issue_v = [&](int t, int buf) { tile_dma<DH>(sKV[2 + buf], Vb, a.ld_v, t * BN, n, hk * DH, thread()); };
    issue_k(0, 0);
    issue_v(0, 0);
    if (ntk > 1) {
        issue_v(1, 1);
        if (q0 == 0) issue_k(1, 1);
    }
    bf16x8 qreg[KSTEPS], greg[KSTEPS];
    float nl, nd;                                                // - lse / ln 2 and - delta of the lane's query
    {
        const uint16_t* Q = (const uint16_t*)a.q + (long long)(at.o + qr) * a.ld_q + h * DH + 8 * hh;
        const uint16_t* G = (const uint16_t*)a.dout + (long long)(at.o + qr) * a.ld_do + h * DH + 8 * hh;
        const uint16_t* O = (const uint16_t*)a.out + (long long)(at.o + qr) * a.ld_o + h * DH + 8 * hh;
        nl = a.lse[h * a.T + at.o + qr] * NEG_LOG2E;
        float d = 0.f;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++) {
            qreg[kk] = as_bf16x8(*(const uint4*)(Q + 16 * kk));
            const uint4 g = *(const uint4*)(G + 16 * kk), o = *(const uint4*)(O + 16 * kk);
            greg[kk] = as_bf16x8(g);
            const uint32_t gw[4] = {g.x, g.y, g.z, g.w}, ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                d = __builtin_fmaf(__uint_as_float(gw[i] << 16), __uint_as_float(ow[i] << 16), d);
                d = __builtin_fmaf(__uint_as_float(gw[i] & 0xffff0000u), __uint_as_float(ow[i] & 0xffff0000u), d);
            }
        }
        nd = -sum_halves(d);
    }
    floatx16 dq[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) dq[d] = floatx16{};
    const uint32_t kofs0 = tile_ofs<CPR>(col, hh);
    uint32_t tofs0, tofs1;
    tile_ofs_tr<CPR>(0, lane, tofs0, tofs1);
    constexpr uint32_t ROW16 = 16u * CPR * 16u;                  // bytes of 16 tile rows

    auto mask = [&](floatx16& s) {                               // on the diagonal: element e is key 8 (e / 4) + 4 hh + e % 4
#pragma unroll
        for (int e = 0; e < 16; e++) s[e] = 8 * (e >> 2) + 4 * hh + (e & 3) > col ? neg_inf() : s[e];
    };
    // A step: dS and its product with K for half HC of the tile in buffer KB, whose scores and dP - delta are s and g; beside
    // them those of the next half, half HN of the tile in buffers NB, product by product between the elements' arithmetic.
    auto step = [&](auto kb_tag, auto hc_tag, auto nb_tag, auto hn_tag, const floatx16& s, const floatx16& g, floatx16& sn,
                    floatx16& gn, int j) {
        constexpr int KB = decltype(kb_tag)::value, HC = decltype(hc_tag)::value, NB = decltype(nb_tag)::value,
                      HN = decltype(hn_tag)::value;
        // (the transposed reads' offsets afresh in each step: kept in registers, at 256 of them, one fragment of Q spilled,
        // whose reload waits for the copies under way)
        uint32_t t0 = tofs0, t1 = tofs1;
        if constexpr (DH == 128) asm volatile("" : "+v"(t0), "+v"(t1));
        auto operand = [&](int i) {
            if (i < 2 * KSTEPS) return lds_read16(sKV[NB + 2 * (i & 1)], (kofs0 ^ (32u * (i >> 1))) + 2 * HN * ROW16);
            const uint32_t d = (i - 2 * KSTEPS) % DBLK, kq = (i - 2 * KSTEPS) / DBLK;
            return lds_read_tr(sKV[KB], (t0 ^ (64u * d)) + (2 * HC + kq) * ROW16, (t1 ^ (64u * d)) + (2 * HC + kq) * ROW16);
        };
        bf16x8 op[NM];
#pragma unroll
        for (int i = 0; i < PF; i++) op[i] = operand(i);
        uint32_t pk[8];
        float ds[16];
        auto element = [&](int e) {
            ds[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c, nl)) * g[e];
            if (e & 1) {
                pk[e >> 1] = pack_bf16x2(ds[e - 1], ds[e]);
                asm volatile("" : "+v"(pk[e >> 1]));
            }
        };
#pragma unroll
        for (int i = 0; i < NM; i++) {
            if (i + PF < NM) op[i + PF] = operand(i + PF);
            if (i < 2 * KSTEPS) {
                const int kk = i >> 1;
                if ((i & 1) == 0) {
                    sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i], qreg[kk], kk == 0 ? floatx16{} : sn, 0, 0, 0);
                } else {
                    if (kk == 0) {
#pragma unroll
                        for (int e = 0; e < 16; e++) gn[e] = nd;
                    }
                    gn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i], greg[kk], gn, 0, 0, 0);
                }
#pragma unroll
                for (int e = 16 * i / (2 * KSTEPS); e < 16 * (i + 1) / (2 * KSTEPS); e++) element(e);
            } else {
                const int d = (i - 2 * KSTEPS) % DBLK, kq = (i - 2 * KSTEPS) / DBLK;
                const bf16x8 b = as_bf16x8(make_uint4(pk[4 * kq], pk[4 * kq + 1], pk[4 * kq + 2], pk[4 * kq + 3]));
                dq[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i], b, dq[d], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (j + 2 == nh) mask(sn);
    };
    using C0 = std::integral_constant<int, 0>;
    using C1 = std::integral_constant<int, 1>;

    floatx16 sA{}, pA, sB, pB;                                   // of the tile's halves 0 and 1
    wait_vmcnt_seen<0>();
    lds_barrier();
    if (q0 == 0) {
        float more = 0.f;
        for (int j = 0; j < nh; j++) {
            const uint32_t row = 2 * (j & 1) * ROW16;
            const uint16_t* Kc = sKV[j >> 1];
            const uint16_t* Vc = sKV[2 + (j >> 1)];
            floatx16 s{}, g;
#pragma unroll
            for (int e = 0; e < 16; e++) g[e] = nd;
#pragma unroll
            for (int kk = 0; kk < KSTEPS; kk++) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(Kc, (kofs0 ^ (32u * kk)) + row), qreg[kk], s, 0, 0, 0);
                g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(Vc, (kofs0 ^ (32u * kk)) + row), greg[kk], g, 0, 0, 0);
            }
            if (j + 1 == nh) mask(s);
            more += missing(s, g, a.c, nl);
        }
        nd -= sum_halves(more);
    }
    if (hh == 0 && qw + col < n) {
        a.rows_l[h * a.T + at.o + qr] = nl;
        a.rows_d[h * a.T + at.o + qr] = nd;
    }
#pragma unroll
    for (int e = 0; e < 16; e++) pA[e] = nd;
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) {
        sA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(sKV[0], kofs0 ^ (32u * kk)), qreg[kk], sA, 0, 0, 0);
        pA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_read16(sKV[2], kofs0 ^ (32u * kk)), greg[kk], pA, 0, 0, 0);
    }
    if (nh == 1) mask(sA);
    // Tile t in buffers P; its first half's scores are formed.  V(t + 1) is on its way or here.
    auto tile = [&](auto par, int t) {
        constexpr int P = decltype(par)::value;
        using CP = std::integral_constant<int, P>;
        using CQ = std::integral_constant<int, P ^ 1>;
        const bool more = t + 1 < ntk;
        if (t > 0) lds_barrier();                                // K(t - 1) is no longer read
        if (more && (t > 0 || q0 > 0)) issue_k(t + 1, P ^ 1);
        if (2 * t < nh) step(CP{}, C0{}, CP{}, C1{}, sA, pA, sB, pB, 2 * t);
        if (more) {
            wait_vmem();                                         // K(t + 1), V(t + 1)
            lds_barrier();                                       // everywhere, and V(t) is no longer read
            if (t + 2 < ntk) issue_v(t + 2, P);
        }
        if (2 * t + 1 < nh) step(CP{}, C1{}, CQ{}, C0{}, sB, pB, sA, pA, 2 * t + 1);
    };
    for (int t = 0; t < ntk; t += 2) {
        tile(C0{}, t);
        if (t + 1 < ntk) tile(C1{}, t + 1);
    }
    __syncthreads();                                             // the tiles' LDS is reused below
    store_rows<DH>(dq, a.scale, sKV[0] + w * 32 * DH, (uint16_t*)a.dq + (long long)at.o * a.ld_q + h * DH, a.ld_q, qw, n, lane);
}

// Few query tiles, as in the forward: a workgroup takes 32 query rows of one (sequence, head), and its 8 waves their halves
// of 32 keys in turn, each with its own LDS tiles; their sums are added at the end, in the order of the waves.
template <int DH>
__global__ __launch_bounds__(512, 2) void causal_dq_few_kernel(CausalArgs a, CausalPlan p) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, TILE = 32 * DH, NI = CPR / 2, WAVES = 8;
    __shared__ __align__(16) uint16_t sT[WAVES][2][TILE];        // K and V of each wave; then its sums
    __shared__ float sMore[BM / 32][32], sD[32];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    if (blockIdx.x == 0) {
        static_assert(PLAN_LDS * 4 <= WAVES * 2 * TILE * 2, "the plan fits the tiles");
        make_plan<512>(a, p, (int*)sT);
        return;
    }
    int id = blockIdx.x - 1;
    const int hk = id % a.Hk;
    id /= a.Hk;
    const int h = hk * a.group + id % a.group;
    const Tile at = tile_of_slot<32>(a.offsets, a.B, a.T, (int)(a.T / 32) + a.B - 1 - id / a.group);
    if (at.tile < 0) return;
    const int q0 = 32 * at.tile, n = at.n, qr = min(q0 + col, n - 1);
    // 32 rows from row0 on of columns of a matrix; rows behind the sequence are copies of its last one
    auto copy = [&](const void* src, long long ld, int col0, int row0, int which) {
        const uint16_t* base = (const uint16_t*)src + (long long)(at.o + row0) * ld + col0;
        const int last = n - 1 - row0;
#pragma unroll
        for (int i = 0; i < NI; i++) {
            const int row = i * (64 / CPR) + lane / CPR;
            lds_dma16(lds_address(sT[w][which]) + i * 1024u, uniform_ptr(base),
                      (uint32_t)(min(row, last) * ld + ((lane % CPR) ^ swz<CPR>(row)) * 8) * 2u);
        }
    };
    auto issue_k = [&](int j) { copy(a.k, a.ld_k, hk * DH, 32 * j, 0); };
    auto issue_v = [&](int j) { copy(a.v, a.ld_v, hk * DH, 32 * j, 1); };
    copy(a.q, a.ld_q, h * DH, q0, 0);
    copy(a.dout, a.ld_do, h * DH, q0, 1);
    // delta of four rows, CPR lanes for each (of all rows in each wave, from the pieces that the products take: the backward of 700
    // tokens, 6 / 2 heads of 128, 33.1 us instead of 31.7)
    const int dr = 4 * w + lane / CPR % 4;
    uint4 o, g0;
    {
        const long long row = at.o + min(q0 + dr, n - 1);
        o = *(const uint4*)((const uint16_t*)a.out + row * a.ld_o + h * DH + 8 * (lane % CPR));
        g0 = *(const uint4*)((const uint16_t*)a.dout + row * a.ld_do + h * DH + 8 * (lane % CPR));
    }
    const float nl = a.lse[h * a.T + at.o + qr] * NEG_LOG2E;
    wait_vmcnt_seen<0>();
    bf16x8 qreg[KSTEPS], greg[KSTEPS];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) {
        qreg[kk] = tile_read8<CPR>(sT[w][0], col, 2 * kk + hh);
        greg[kk] = tile_read8<CPR>(sT[w][1], col, 2 * kk + hh);
    }
    wait_lgkm_seen();
    const bool any = w <= at.tile;
    if (any) {
        issue_k(w);
        issue_v(w);
    }
    {
        const uint32_t gw[4] = {g0.x, g0.y, g0.z, g0.w}, ow[4] = {o.x, o.y, o.z, o.w};
        float d = 0.f;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            d = __builtin_fmaf(__uint_as_float(gw[i] << 16), __uint_as_float(ow[i] << 16), d);
            d = __builtin_fmaf(__uint_as_float(gw[i] & 0xffff0000u), __uint_as_float(ow[i] & 0xffff0000u), d);
        }
#pragma unroll
        for (int off = CPR / 2; off >= 1; off >>= 1) d += __shfl_xor(d, off, 64);
        if (lane < 4 * CPR && lane % CPR == 0) sD[dr] = -d;
    }
    lds_barrier();
    float nd = sD[col];
    floatx16 dq[DBLK];
#pragma unroll
    for (int i = 0; i < DBLK; i++) dq[i] = floatx16{};
    floatx16 s, g;                                               // scores and dP - delta of a half
    auto scores = [&](int j, bool more) {
        wait_vmem();                                             // K(j), V(j)
        s = floatx16{};
#pragma unroll
        for (int e = 0; e < 16; e++) g[e] = nd;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++) {
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sT[w][0], col, 2 * kk + hh), qreg[kk], s, 0, 0, 0);
            g = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sT[w][1], col, 2 * kk + hh), greg[kk], g, 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // V(j) is read
        if (more) issue_v(j + WAVES);
        if (j == at.tile) {
#pragma unroll
            for (int e = 0; e < 16; e++) s[e] = 8 * (e >> 2) + 4 * hh + (e & 3) > col ? neg_inf() : s[e];
        }
    };
    auto products = [&](int j, bool more) {
        uint32_t pk[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2)
            pk[e >> 1] = pack_bf16x2(__builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.c, nl)) * g[e],
                                     __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], a.c, nl)) * g[e + 1]);
#pragma unroll
        for (int kq = 0; kq < 2; kq++) {
            const bf16x8 b = as_bf16x8(make_uint4(pk[4 * kq], pk[4 * kq + 1], pk[4 * kq + 2], pk[4 * kq + 3]));
#pragma unroll
            for (int i = 0; i < DBLK; i++)
                dq[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read_tr<CPR>(sT[w][0], 16 * kq, 32 * i, lane), b, dq[i], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) issue_k(j + WAVES);
    };
    if (q0 < BM) {                                               // one half at most for each of the first waves
        static_assert(BM / 32 <= WAVES, "a wave has no second half");
        if (any) {
            scores(w, false);
            const float more = sum_halves(missing(s, g, a.c, nl));
            if (hh == 0) sMore[w][col] = more;
        }
        __syncthreads();
        float all = 0.f;
        for (int i = 0; i <= at.tile; i++) all += sMore[i][col];
        nd -= all;
        if (any) {
            g -= all;
            products(w, false);
        }
    } else {
        for (int j = w; j <= at.tile; j += WAVES) {
            const bool more = j + WAVES <= at.tile;
            scores(j, more);
            products(j, more);
        }
    }
    if (w == 0 && hh == 0 && q0 + col < n) {
        a.rows_l[h * a.T + at.o + qr] = nl;
        a.rows_d[h * a.T + at.o + qr] = nd;
    }
    write_part<DH>(dq, (float*)sT[w], lane, 32);
    __syncthreads();
    for (int i = tid; i < 32 * (DH / 4); i += 64 * WAVES) {
        const int r = i / (DH / 4), f = i % (DH / 4);
        if (q0 + r >= n) continue;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < WAVES; j++) {
            const float4 v = *(const float4*)&((const float*)sT[j])[4 * part_chunk<DH>(r, f)];
            x.x += v.x;
            x.y += v.y;
            x.z += v.z;
            x.w += v.w;
        }
        *(uint2*)((uint16_t*)a.dq + (long long)(at.o + q0 + r) * a.ld_q + h * DH + 4 * f) =
            make_uint2(pack_bf16x2(x.x * a.scale, x.y * a.scale), pack_bf16x2(x.z * a.scale, x.w * a.scale));
    }
}

template <int DH>
hipError_t dq(const CausalArgs& a, const CausalPlan& p, hipStream_t s) {
    const long long few = (a.T / 32 + a.B) * a.H;
    if (few <= FEW_TILES) causal_dq_few_kernel<DH><<<(int)few + 1, 512, 0, s>>>(a, p);
    else causal_dq_kernel<DH><<<a.slots * a.H + 1, 256, 0, s>>>(a, p);
    return hipGetLastError();
}

}  // namespace

CausalPlan causal_plan(long long T, int B, int H, int Hk, int head_dim) { return make_causal_plan(T, B, H, Hk, head_dim); }

hipError_t launch_causal_dq(const CausalArgs& a, const CausalPlan& p, int head_dim, hipStream_t s) {
    switch (head_dim) {
        case 32: return dq<32>(a, p, s);
        case 64: return dq<64>(a, p, s);
        case 128: return dq<128>(a, p, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace mtgr
