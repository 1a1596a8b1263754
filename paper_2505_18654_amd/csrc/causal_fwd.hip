// Forward of the causal softmax attention.
//
// One workgroup = 4 waves = 128 query rows of one (sequence, head), 32 rows per wave, over the 64-key tiles up to its last
// row.  A wave computes the transposed products: S^T (32 keys x 32 queries) = K Q^T, so that a lane holds 16 scores of one
// query (lane % 32) and the packed probabilities serve directly as the operand of O^T += V^T P^T, whose columns, again a
// query per lane, are rescaled by one multiplication per lane where the running maximum grows.  Rounded to bf16 are the
// probabilities (the matrix instructions take 16 bits; their sum is formed before) and the result.
//
// Bound by the matrix cores at the clock that the power limit leaves: four sequences of up to 16,001 tokens, 16 / 2 heads of
// 128, 1.48 ms = 1.07 PFLOP/s, where a bf16 product of 8,192^3 reaches 1.24 on the same card (matrix cores busy 54 % at 1.7 GHz).
// With the products one after another, before and behind the element arithmetic, it took 1.69 ms; fetching operands two or four
// products ahead, or fences every four products, changes 1 %.  Short sequences are bound by each workgroup's start (the
// search, Q, the first tiles): 64 of 1,024 tokens, 770 TFLOP/s.
#include <type_traits>

#include "causal_device.h"

namespace mtgr {
namespace {

using namespace causal;
constexpr int BN = 64;        // keys of a tile

// 32 rows from row0 on of columns of a matrix into a wave's swizzled tile; rows behind `last` are copies of it.
template <int DH>
__device__ __forceinline__ void copy_rows(uint16_t* tile, const void* src, long long ld, int col0, long long row0, int last,
                                          int lane) {
    constexpr int CPR = DH / 8;
    const uint16_t* base = (const uint16_t*)src + row0 * ld + col0;
#pragma unroll
    for (int i = 0; i < CPR / 2; i++) {
        const int row = i * (64 / CPR) + lane / CPR;
        lds_dma16(lds_address(tile) + i * 1024u, uniform_ptr(base),
                  (uint32_t)(min(row, last) * ld + ((lane % CPR) ^ swz<CPR>(row)) * 8) * 2u);
    }
}

// A wave's 32 queries against halves of 32 keys, first, first + step, .. below end, `diag` the one on the diagonal: maximum,
// sum and outputs of a query in a lane.  issue_k and issue_v copy a half into the wave's tiles; those of the first are under way.
// open(j): whether there is anything left to do behind half j.
template <int DH, class IssueK, class IssueV, class Open>
__device__ __forceinline__ void attend_halves(const CausalArgs& a, const uint16_t* sK, const uint16_t* sV,
                                              const bf16x8 (&qreg)[DH / 16], floatx16 (&oacc)[DH / 32], float& m, float& l,
                                              int first, int step, int end, int diag, IssueK issue_k, IssueV issue_v,
                                              Open open, int lane) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, NI = CPR / 2;
    const int col = lane & 31, hh = lane >> 5;
    for (int j = first; j < end; j += step) {
        const bool more = j + step < end;
        wait_vmcnt<NI>();                                        // K(j)
        floatx16 s{};
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sK, col, 2 * kk + hh), qreg[kk], s, 0, 0, 0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // it is read
        if (more) issue_k(j + step);
        if (j == diag) {
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
        if (more) wait_vmcnt<NI>(); else wait_vmem();            // V(j)
#pragma unroll
        for (int kq = 0; kq < 2; kq++) {
            const bf16x8 pb = as_bf16x8(make_uint4(pk[4 * kq], pk[4 * kq + 1], pk[4 * kq + 2], pk[4 * kq + 3]));
#pragma unroll
            for (int d = 0; d < DBLK; d++)
                oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read_tr<CPR>(sV, 16 * kq, 32 * d, lane), pb, oacc[d], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (!open(j)) break;
        if (more) issue_v(j + step);
    }
}

// Outputs with infinities or NaN among a wave's 32 query rows from q0 on once more.  P = 0 of the keys behind a query, times an
// infinite or NaN value there, is NaN in the products: of the half on the diagonal alone, and only if it holds such a value.  Its
// keys are then taken one by one, each by the queries that see it, behind the others' products formed once more; elements that
// are finite keep what they were.  The rows have been written; sK and sV are tiles of the wave.  8,000 tokens, 8 heads of 128:
// 194 us, with an infinity in the last token 482, in the middle one 271 (the rows behind show it rightly and are left), in
// every token 530.
template <int DH>
__device__ void redo_rows(const CausalArgs& a, const Tile& at, int q0, int h, int hk, uint16_t* sK, uint16_t* sV, int lane) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32;
    // (opaque, so that the compiler does not keep what it has in common with the loop before in registers across that)
    asm volatile("" : "+v"(lane));
    const int col = lane & 31, hh = lane >> 5, n = at.n;
    uint16_t* row = (uint16_t*)a.out + (long long)(at.o + min(q0 + col, n - 1)) * a.ld_o + h * DH + 4 * hh;
    auto issue_k = [&](int j) { copy_rows<DH>(sK, a.k, a.ld_k, hk * DH, at.o + 32 * j, n - 1 - 32 * j, lane); };
    auto issue_v = [&](int j) { copy_rows<DH>(sV, a.v, a.ld_v, hk * DH, at.o + 32 * j, n - 1 - 32 * j, lane); };
    auto special = [](uint32_t bits) { return (bits & 0x7f80u) == 0x7f80u; };
    const int diag = q0 / 32;
    issue_v(diag);
    copy_rows<DH>(sK, a.q, a.ld_q, h * DH, at.o + q0, n - 1 - q0, lane);
    uint32_t bad[DBLK];                                          // a bit for each of the lane's elements, as in the accumulators
#pragma unroll
    for (int d = 0; d < DBLK; d++) {
        bad[d] = 0;
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const uint2 u = *(const uint2*)(row + 32 * d + 8 * g);
            bad[d] |= (uint32_t)(special(u.x) | special(u.x >> 16) << 1 | special(u.y) << 2 | special(u.y >> 16) << 3) << 4 * g;
        }
        if (q0 + col >= n) bad[d] = 0;
    }
    wait_vmem();
    bool any = false;
#pragma unroll
    for (int i = 0; i < CPR / 2; i++) {
        const uint4 u = *(const uint4*)&sV[8 * (lane + 64 * i)];
        const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; e++) any |= special(x[e]) | special(x[e] >> 16);
    }
    if (!__any(any)) return;
    bf16x8 qreg[KSTEPS];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) qreg[kk] = tile_read8<CPR>(sK, col, 2 * kk + hh);
    wait_lgkm_seen();
    floatx16 oacc[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) oacc[d] = floatx16{};
    float m = a.least, l = 0.f;
    // Once all of these are NaN (inputs full of them), they stay so.
    auto open = [&](int j) {
        if (j % 8 != 0) return true;
        bool some = false;
#pragma unroll
        for (int d = 0; d < DBLK; d++)
#pragma unroll
            for (int e = 0; e < 16; e++) some |= (bad[d] >> e & 1) != 0 && oacc[d][e] == oacc[d][e];
        return __any(some) != 0;
    };
    if (diag > 0) {
        issue_k(0);
        issue_v(0);
        attend_halves<DH>(a, sK, sV, qreg, oacc, m, l, 0, 1, diag, -1, issue_k, issue_v, open, lane);
        wait_vmem();
    }
    issue_k(diag);
    issue_v(diag);
    wait_vmem();
    floatx16 s{};
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sK, col, 2 * kk + hh), qreg[kk], s, 0, 0, 0);
    float top = neg_inf();
#pragma unroll
    for (int e = 0; e < 16; e++) {
        if (8 * (e >> 2) + 4 * hh + (e & 3) > col) s[e] = neg_inf();
        top = fmaxf(top, s[e]);
    }
    top = fmaxf(max_halves(top), m);
    const float f = __builtin_amdgcn_exp2f((m - top) * a.c), mc = top * a.c;
    l *= f;
#pragma unroll
    for (int d = 0; d < DBLK; d++) oacc[d] *= f;
    // P [query][key] in place of K
#pragma unroll
    for (int g = 0; g < 4; g++) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; e++) l += p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * g + e], a.c, -mc));
        *(uint2*)&sK[32 * col + 8 * g + 4 * hh] = make_uint2(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]));
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
    for (int key = 0; key <= col; key++) {
        const float p = bf16_to_f32(sK[32 * col + key]);
#pragma unroll
        for (int d = 0; d < DBLK; d++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const uint2 v = *(const uint2*)&sV[8 * tile_chunk<CPR>(key, 4 * d + g) + 4 * hh];
                oacc[d][4 * g] = __builtin_fmaf(p, __uint_as_float(v.x << 16), oacc[d][4 * g]);
                oacc[d][4 * g + 1] = __builtin_fmaf(p, __uint_as_float(v.x & 0xffff0000u), oacc[d][4 * g + 1]);
                oacc[d][4 * g + 2] = __builtin_fmaf(p, __uint_as_float(v.y << 16), oacc[d][4 * g + 2]);
                oacc[d][4 * g + 3] = __builtin_fmaf(p, __uint_as_float(v.y & 0xffff0000u), oacc[d][4 * g + 3]);
            }
    }
    const float inv = 1.0f / sum_halves(l);
#pragma unroll
    for (int d = 0; d < DBLK; d++)
#pragma unroll
        for (int e = 0; e < 16; e++)
            if (bad[d] >> e & 1) row[32 * d + 8 * (e >> 2) + (e & 3)] = (uint16_t)f32_to_bf16_bits(oacc[d][e] * inv);
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
    float m = a.least, mc = m * a.c, l0 = 0.f, l1 = 0.f;
    auto mask = [&](floatx16& s) {                               // on the diagonal: element e is key 8 (e / 4) + 4 hh + e % 4
#pragma unroll
        for (int e = 0; e < 16; e++) s[e] = 8 * (e >> 2) + 4 * hh + (e & 3) > col ? neg_inf() : s[e];
    };
    auto raise = [&](float top) {
        top = max_halves(top);
        // (each query for itself, so that its bits do not depend on the others of the wave, which see later keys)
        const bool up = __builtin_fmaf(top, a.c, -mc) > 8.f;
        if (__any(up)) {
            const float f = up ? __builtin_amdgcn_exp2f((m - top) * a.c) : 1.f;
            l0 *= f;
            l1 *= f;
#pragma unroll
            for (int d = 0; d < DBLK; d++) oacc[d] *= f;
            m = up ? top : m;
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
    const bool bad = __any(zero != 0.f && qi < n);
    uint16_t* sO = sKV[0] + w * 32 * DH;
    store_rows<DH>(oacc, 1.0f / l, sO, (uint16_t*)a.out + (long long)at.o * a.ld_o + h * DH, a.ld_o, qw, n, lane);
    if (bad) {
        wait_vmem();                                             // the rows as they are have been written
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // and their LDS is read
        redo_rows<DH>(a, at, qw, h, hk, sO, sKV[2] + w * 32 * DH, lane);
    }
}

// Few query tiles: a workgroup takes 32 query rows of one (sequence, head), and its 8 waves take their halves of 32 keys in
// turn, each with its own maximum, sum and outputs and its own LDS tiles, joined at the end.  A lone prompt of 700 tokens, 6
// heads, is 36 workgroups of the kernel above, the last of them 11 tiles one after another.  (Heads of 32: registers for three
// workgroups of a CU, which the rare path at the end would make two.)
template <int DH>
__global__ __launch_bounds__(512, DH == 32 ? 6 : 2) void causal_fwd_few_kernel(CausalArgs a) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, TILE = 32 * DH, NI = CPR / 2, WAVES = 8;
    __shared__ __align__(16) uint16_t sT[WAVES][2][TILE];        // K and V of each wave; then its outputs
    __shared__ float sML[WAVES][2][32];
    __shared__ int sBad;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    int id = blockIdx.x;
    const int hk = id % a.Hk;
    id /= a.Hk;
    const int h = hk * a.group + id % a.group;
    const Tile at = tile_of_slot<32>(a.offsets, a.B, a.T, a.slots - 1 - id / a.group);
    if (at.tile < 0) return;
    const int q0 = 32 * at.tile, n = at.n;
    auto issue_k = [&](int j) { copy_rows<DH>(sT[w][0], a.k, a.ld_k, hk * DH, at.o + 32 * j, n - 1 - 32 * j, lane); };
    auto issue_v = [&](int j) { copy_rows<DH>(sT[w][1], a.v, a.ld_v, hk * DH, at.o + 32 * j, n - 1 - 32 * j, lane); };
    const bool any = w <= at.tile;
    if (tid == 0) sBad = 0;
    // (Q through the V tile, as whole lines; a lane's pieces straight from memory, V copied at once: 9.3 -> 10.6 us for 700 tokens,
    // 6 / 2 heads of 128)
    copy_rows<DH>(sT[w][1], a.q, a.ld_q, h * DH, at.o + q0, n - 1 - q0, lane);
    if (any) issue_k(w);
    if (any) wait_vmcnt<NI>(); else wait_vmem();
    bf16x8 qreg[KSTEPS];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) qreg[kk] = tile_read8<CPR>(sT[w][1], col, 2 * kk + hh);
    wait_lgkm_seen();
    if (any) issue_v(w);
    floatx16 oacc[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) oacc[d] = floatx16{};
    float m = a.least, l = 0.f;
    attend_halves<DH>(a, sT[w][0], sT[w][1], qreg, oacc, m, l, w, WAVES, at.tile + 1, at.tile, issue_k, issue_v,
                      [](int) { return true; }, lane);
    l = sum_halves(l);
    if (hh == 0) {
        sML[w][0][col] = m;
        sML[w][1][col] = l;
    }
    write_part<DH>(oacc, (float*)sT[w], lane, 32);
    __syncthreads();
    for (int i = tid; i < 32 * (DH / 4); i += 64 * WAVES) {
        const int r = i / (DH / 4), f = i % (DH / 4), qi = q0 + r;
        if (qi >= n) continue;
        float top, total;
        const float4 o = join_parts<DH, WAVES>(sT, sML, r, f, a.c, top, total);
        const float inv = 1.0f / total;
        *(uint2*)((uint16_t*)a.out + (long long)(at.o + qi) * a.ld_o + h * DH + 4 * f) =
            make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
        if (f == 0 && a.lse) a.lse[h * a.T + at.o + qi] = top * a.scale + logf(total);
        if (o.x * 0.f + o.y * 0.f + o.z * 0.f + o.w * 0.f != 0.f) sBad = 1;
    }
    __syncthreads();
    if (sBad != 0 && w == 0) redo_rows<DH>(a, at, q0, h, hk, sT[0][0], sT[0][1], lane);
}

template <int DH>
hipError_t fwd(CausalArgs a, hipStream_t s) {
    const long long few = (a.T / 32 + a.B) * a.H;
    if (few <= FEW_TILES) {
        a.slots = (int)(a.T / 32 + a.B);
        causal_fwd_few_kernel<DH><<<(int)few, 512, 0, s>>>(a);
    } else {
        causal_fwd_kernel<DH><<<a.slots * a.H, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_causal_fwd(const CausalArgs& a, int head_dim, hipStream_t s) {
    switch (head_dim) {
        case 32: return fwd<32>(a, s);
        case 64: return fwd<64>(a, s);
        case 128: return fwd<128>(a, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace mtgr
