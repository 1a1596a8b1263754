// The products of the feed-forward block and the softmax loss on 128 x 128 tiles, for sizes whose 256 x 256
// tiles (gemm_wide.h: the same layouts, epilogues and arguments) do not fill the chip.
//
// A workgroup of 4 waves computes a tile in k steps of 64, wave w the 64 x 64 part (m half w % 2, n half w / 2)
// as 4 x 4 blocks of 16 x 16, transposed as in gemm_wide.h.  Two LDS stages (64 KB) let two workgroups share a
// CU, so that one's barriers, copies and epilogue run under the other's matrix instructions.  One barrier per
// step: it hands over the stage that has landed and frees the other one for the copies of the next step.
// (A workgroup alone on its CU takes 0.8 us per step, for 0.2 us of matrix work: a chain of the wait, the barrier,
// the copies and the reads.  Without the matrix instructions or the reads it was as long, without the copies
// 0.15 us shorter.  Four stages, operands read a half step ahead, eight waves, and copies spread between the matrix
// instructions, 2 to 15 % slower, gained nothing, so products of few tiles are split over k instead.)  Results pass
// through LDS, so that a lane stores 16 bytes and its neighbours the rest of the line: straight from the accumulators, 8 bytes and
// 32 bytes of a row at a time, dpre of 6,418 tokens, 256 / 704, took 21.6 us, like this 16.3.
#pragma once

#include <stdio.h>

#include <type_traits>

#include "gemm_wide.h"

namespace mtgr {

namespace {

constexpr int MBM = 128, MBN = 128, MBK = 64;
constexpr uint32_t MSLOT = MBM * MBK * 2, MID_LDS = 4 * MSLOT;

// Workgroups per tile grid that fill the chip once: two per CU.
constexpr int MID_WORKGROUPS = 512;

}  // namespace

// The tile of workgroup `block` of a product's own grid; sm: MID_LDS bytes.
template <int LAYOUT, int EPI>
__device__ __forceinline__ void mid_tile(const TileArgs& g, int block, char* sm) {
    constexpr bool A_KR = LAYOUT == GEMM_TN, B_KR = LAYOUT != GEMM_NT;
    constexpr bool ACC = EPI == GEMM_EPI_ACC, SPLIT = LAYOUT == GEMM_TN || ACC || EPI == GEMM_EPI_PART;
    constexpr bool GATED = EPI == GEMM_EPI_GATED || EPI == GEMM_EPI_GATED_SAVE;
    constexpr bool STATS = EPI == GEMM_EPI_SM_STATS, GRAD = EPI == GEMM_EPI_SM_GRAD, B_SHORT = STATS || GRAD;
    constexpr bool DYN = B_SHORT || ACC || EPI == GEMM_EPI_ROWS;
    constexpr int NTILE = GATED ? MBN / 2 : MBN;
    constexpr uint32_t OFF_B = 2 * MSLOT;                    // stages A 0, A 1, B 0, B 1

    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, wm = w & 1, wn = w >> 1;
    const int lr = lane & 15, lg = lane >> 4;
    int M = (int)g.M, K = (int)g.K, mblocks = g.mblocks;
    const int N = (int)g.N;
    if constexpr (DYN) {
        if constexpr (LAYOUT == GEMM_TN) {
            K = min(*g.rows, K);
        } else {
            M = min(*g.rows, M);
            mblocks = (M + MBM - 1) / MBM;
        }
    }
    // items (split, m block, n block), a share of consecutive ones per XCD
    const int tiles = mblocks * g.nblocks, items = tiles * g.splits, share = (items + XCDS - 1) / XCDS;
    const int it = block % XCDS * share + block / XCDS;
    if (block / XCDS >= share || it >= items) return;
    const int split = it / tiles, mb = it % tiles / g.nblocks, nb = it % g.nblocks;
    const int m0 = mb * MBM, n0 = nb * NTILE;
    const int nks = (K + MBK - 1) / MBK, per = (nks + g.splits - 1) / g.splits;
    const int ks0 = split * per, nk = min(nks, ks0 + per) - ks0;      // at most 0: a split without k

    const uint32_t lds0 = lds_address(sm), ldsw = lds0 + __builtin_amdgcn_readfirstlane((uint32_t)w * 1024u);
    // copies: instruction q of wave w fills the 1 KB block 4 q + w of a slot, as in gemm_wide.h
    auto kc_offsets = [&](uint32_t* vo, long long ld, int rvalid, int kvalid) {
        const int r = 8 * w + (lane >> 3), c = min((lane & 7) ^ swz<8>(r), (kvalid >> 3) - 1);
#pragma unroll
        for (int q = 0; q < 4; q++) vo[q] = (uint32_t)(min(32 * q + r, rvalid - 1) * ld + 8 * c) * 2u;
    };
    auto kr_offsets = [&](uint32_t* vo, long long ld, int cvalid, int kvalid) {
        const int r = 4 * w + (lane >> 4), c = min((lane & 15) ^ swz<16>(r), ((cvalid + 7) >> 3) - 1);
#pragma unroll
        for (int q = 0; q < 4; q++) vo[q] = (uint32_t)(min(16 * q + r, kvalid - 1) * ld + 8 * c) * 2u;
    };
    auto gated_offsets = [&](uint32_t* vo, long long ld, int hvalid, int kvalid) {
        const int r = 4 * w + (lane >> 4), c = (lane & 15) ^ swz<16>(r);
        const int col = 8 * min(4 * (c >> 3) + (c & 3), (hvalid >> 3) - 1) + n0 + ((c & 4) ? N : 0);
#pragma unroll
        for (int q = 0; q < 4; q++) vo[q] = (uint32_t)(min(16 * q + r, kvalid - 1) * ld + col) * 2u;
    };
    auto offsets_a = [&](uint32_t* vo, int kvalid) {
        if constexpr (A_KR) kr_offsets(vo, g.lda, M - m0, kvalid);
        else kc_offsets(vo, g.lda, min(MBM, M - m0), kvalid);
    };
    auto offsets_b = [&](uint32_t* vo, int kvalid) {
        if constexpr (GATED) gated_offsets(vo, g.ldb, N - n0, kvalid);
        else if constexpr (B_KR) kr_offsets(vo, g.ldb, N - n0, kvalid);
        else kc_offsets(vo, g.ldb, min(MBN, (B_SHORT ? g.b_rows : N) - n0), kvalid);
    };
    const long long stepA = 2ll * (A_KR ? MBK * g.lda : MBK), stepB = 2ll * (B_KR ? MBK * g.ldb : MBK);
    const char* pa = (const char*)g.A + 2 * (A_KR ? (long long)m0 : (long long)m0 * g.lda) + ks0 * stepA;
    const char* pb = (const char*)g.B + 2 * (GATED ? 0ll : B_KR ? (long long)n0 : (long long)n0 * g.ldb) + ks0 * stepB;
    uint32_t voA[4], voB[4];
    offsets_a(voA, MBK);
    offsets_b(voB, MBK);
    auto copy = [&](int i) {
        const int valid = K - (ks0 + i) * MBK;             // k left; fewer than 64 in the last step of a ragged K
        uint32_t ra[4], rb[4];
#pragma unroll
        for (int q = 0; q < 4; q++) {
            ra[q] = voA[q];
            rb[q] = voB[q];
        }
        if (valid < MBK) {
            offsets_a(ra, valid);
            offsets_b(rb, valid);
        }
        // (the A of these products is padded with zeros in k: only the rows of B end early)
        if constexpr (ACC) {
            if ((ks0 + i + 1) * MBK > g.b_rows) offsets_b(rb, g.b_rows - (ks0 + i) * MBK);
        }
        const uint32_t slot = (uint32_t)(i & 1) * MSLOT;
#pragma unroll
        for (int q = 0; q < 4; q++) lds_dma16(ldsw + slot + 4096u * q, pa, ra[q]);
#pragma unroll
        for (int q = 0; q < 4; q++) lds_dma16(ldsw + OFF_B + slot + 4096u * q, pb, rb[q]);
        pa += stepA;
        pb += stepB;
    };
    // zeros in the k past a ragged K, in both operands
    auto zero_tail = [&](int i) {
        const int valid = K - (ks0 + i) * MBK;
        auto clear = [&](bool kr, char* t) {
            if (kr) {
                for (int c = valid * 16 + tid; c < MBK * 16; c += 256) ((uint4*)t)[c] = make_uint4(0, 0, 0, 0);
            } else {
                for (int c = tid; c < MBM * 8; c += 256)
                    if (((c & 7) ^ swz<8>(c >> 3)) >= (valid >> 3)) ((uint4*)t)[c] = make_uint4(0, 0, 0, 0);
            }
        };
        clear(A_KR, sm + (i & 1) * MSLOT);
        clear(B_KR, sm + OFF_B + (i & 1) * MSLOT);
        lds_barrier();
    };
    // operand reads, as in gemm_wide.h; a k-row slot has 16 chunks per row
    auto kc_base = [&](int r0) { return lds0 + 16u * (uint32_t)((r0 + lr) * 8 + (lg ^ swz<8>(lr))); };
    auto kr_base = [&](int c0, int half) {
        const int row = 8 * lg + 4 * half + (lr >> 2), colx = c0 + 4 * (lr & 3);
        return lds0 + 16u * (uint32_t)tile_chunk<16>(row, colx >> 3) + 2u * (uint32_t)(colx & 7);
    };
    uint32_t rm[2], rn[2];
    rm[0] = A_KR ? kr_base(64 * wm, 0) : kc_base(64 * wm);
    rm[1] = A_KR ? kr_base(64 * wm, 1) : 0;
    rn[0] = OFF_B + (B_KR ? kr_base(64 * wn, 0) : kc_base(64 * wn));
    rn[1] = OFF_B + (B_KR ? kr_base(64 * wn, 1) : 0);
    typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
    auto read_frag = [&](auto kr, const uint32_t (&r)[2], uint32_t slot, int part, int blk) {
        if constexpr (decltype(kr)::value) {
            const uint32_t o0 = ((r[0] + slot) ^ (32u * blk)) + 8192u * part, o1 = ((r[1] + slot) ^ (32u * blk)) + 8192u * part;
            const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)o0);
            const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(uintptr_t)o1);
            const short __attribute__((ext_vector_type(8))) v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            return __builtin_bit_cast(bf16x8, v);
        } else {
            return *(const lds_bf16x8*)(uintptr_t)(((r[0] + slot) ^ (64u * part)) + 2048u * blk);
        }
    };
    using AK = std::integral_constant<bool, A_KR>;
    using BK = std::integral_constant<bool, B_KR>;

    // acc[a][b] will hold row em + 16 b, columns en + 16 a + 0..3; what the epilogue reads there is loaded first
    const int em = m0 + 64 * wm + lr, en = n0 + 64 * wn + 4 * lg;
    // residual of row 8 q + l / 8 of block b, chunk l % 8 of the wave's 64 columns
    uint4 rr[EPI == GEMM_EPI_RESIDUAL ? 4 : 1][2];
    if constexpr (EPI == GEMM_EPI_RESIDUAL) {
        const uint16_t* R = (const uint16_t*)g.R + min(n0 + 64 * wn + 8 * (lane & 7), N - 8);
#pragma unroll
        for (int b = 0; b < 4; b++)
#pragma unroll
            for (int q = 0; q < 2; q++)
                rr[b][q] = *(const uint4*)(R + min(m0 + 64 * wm + 16 * b + 8 * q + (lane >> 3), M - 1) * g.ldr);
    }
    // gate and up values of row 8 q + l / 8 of block b, chunk l % 8 of the wave's 64 columns
    uint4 pg[EPI == GEMM_EPI_GATED_BWD ? 4 : 1][2], pu[EPI == GEMM_EPI_GATED_BWD ? 4 : 1][2];
    if constexpr (EPI == GEMM_EPI_GATED_BWD) {
        const uint16_t* R = (const uint16_t*)g.R + min(n0 + 64 * wn + 8 * (lane & 7), N - 8);
#pragma unroll
        for (int b = 0; b < 4; b++)
#pragma unroll
            for (int q = 0; q < 2; q++) {
                const uint16_t* r = R + min(m0 + 64 * wm + 16 * b + 8 * q + (lane >> 3), M - 1) * g.ldr;
                pg[b][q] = load_nt16(r);
                pu[b][q] = load_nt16(r + N);
            }
    }
    floatx4 acc[4][4];
#pragma unroll
    for (int a = 0; a < 4; a++)
#pragma unroll
        for (int b = 0; b < 4; b++) acc[a][b] = floatx4{};
    if (nk > 0) copy(0);
    for (int i = 0; i < nk; i++) {
        wait_vmem();
        lds_barrier();
        if (i + 1 < nk) copy(i + 1);
        if (K - (ks0 + i) * MBK < MBK) zero_tail(i);
        const uint32_t slot = (uint32_t)(i & 1) * MSLOT;
#pragma unroll
        for (int p = 0; p < 2; p++) {
            bf16x8 fm[4], fn[4];
#pragma unroll
            for (int b = 0; b < 4; b++) fm[b] = read_frag(AK{}, rm, slot, p, b);
#pragma unroll
            for (int a = 0; a < 4; a++) fn[a] = read_frag(BK{}, rn, slot, p, a);
#pragma unroll
            for (int a = 0; a < 4; a++)
#pragma unroll
                for (int b = 0; b < 4; b++)
                    acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fn[a], fm[b], acc[a][b], 0, 0, 0);
        }
    }

    // ---- epilogue
    auto pack = [](floatx4 v) { return make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])); };
    auto unpack = [](uint2 u) {
        return floatx4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u)};
    };
    // The results pass through LDS, 4 KB of its own per wave, so that a lane has 16 bytes of a row and a line is whole.
    char* stg = sm + 4096 * w;
    if constexpr (!STATS) lds_barrier();                       // (the stages are no longer read)
    if constexpr (SPLIT) {
#pragma unroll
        for (int b = 0; b < 4; b++) {
#pragma unroll
            for (int a = 0; a < 4; a++) *(floatx4*)(stg + 256 * lr + 16 * ((4 * a + lg) ^ lr)) = acc[a][b];
            wave_lds_fence();
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const int row = 4 * q + lg, gm = m0 + 64 * wm + 16 * b + row, gn = n0 + 64 * wn + 4 * lr;
                const floatx4 v = *(const floatx4*)(stg + 256 * row + 16 * (lr ^ row));
                if (gm >= M || gn >= N) continue;
                floatx4* dst = (floatx4*)(g.partial + ((long long)split * M + gm) * N + gn);
                *dst = ACC && g.accumulate ? *dst + v : v;
            }
            wave_lds_fence();
        }
    } else if constexpr (STATS) {
        floatx4 bias[4];
#pragma unroll
        for (int a = 0; a < 4; a++) bias[a] = *(const floatx4*)(g.bias + en + 16 * a);
#pragma unroll
        for (int b = 0; b < 4; b++) {
            float top = -3.402823466e38f, sum = 0.f;
#pragma unroll
            for (int a = 0; a < 4; a++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    acc[a][b][e] = fmaf(acc[a][b][e], g.scale, bias[a][e]);
                    top = fmaxf(top, acc[a][b][e]);
                }
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
#pragma unroll
            for (int a = 0; a < 4; a++)
#pragma unroll
                for (int e = 0; e < 4; e++) sum += __builtin_amdgcn_exp2f(acc[a][b][e] - top);
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            const int gm = em + 16 * b;
            if (lg == 0 && gm < M) g.stats[(long long)(2 * nb + wn) * g.M + gm] = make_float2(top, sum);
        }
    } else if constexpr (GRAD) {
        const float top = ((const float*)g.rows)[1];
        floatx4 bias[4], cs[4];
        int4 ri[4];
#pragma unroll
        for (int b = 0; b < 4; b++) ri[b] = g.row_info[em + 16 * b];
#pragma unroll
        for (int a = 0; a < 4; a++) {
            bias[a] = *(const floatx4*)(g.bias + en + 16 * a);
            cs[a] = floatx4{};
        }
#pragma unroll
        for (int b = 0; b < 4; b++) {
            const float lse = __int_as_float(ri[b].x), gr = __int_as_float(ri[b].y) / top;
            const float gp = gr * __int_as_float(ri[b].w);
            const int label = ri[b].z - g.class0 - en;
#pragma unroll
            for (int a = 0; a < 4; a++) {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    acc[a][b][e] = gp * __builtin_amdgcn_exp2f(fmaf(acc[a][b][e], g.scale, bias[a][e]) - lse);
                    if (label == 16 * a + e) acc[a][b][e] -= gr;
                }
                // (dz is rounded as an operand of the next two products; its column sums take it unrounded)
                cs[a] += acc[a][b];
                *(uint2*)(stg + 128 * lr + 16 * ((2 * a + (lg >> 1)) ^ (lr & 7)) + 8 * (lg & 1)) = pack(acc[a][b]);
            }
            wave_lds_fence();
#pragma unroll
            for (int q = 0; q < 2; q++) {
                const int gm = m0 + 64 * wm + 16 * b + 8 * q + (lane >> 3);
                const uint4 v = *(const uint4*)(stg + 128 * (8 * q + (lane >> 3)) + 16 * ((lane & 7) ^ (lane >> 3)));
                if (gm < M) *(uint4*)((uint16_t*)g.C + gm * g.ldc + n0 + 64 * wn + 8 * (lane & 7)) = v;
            }
            wave_lds_fence();
        }
        if (g.col_partial != nullptr) {
#pragma unroll
            for (int a = 0; a < 4; a++) {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    float v = dpp_add<0xB1>(cs[a][e]);
                    v = dpp_add<0x4E>(v);
                    v = dpp_add<0x141>(v);
                    cs[a][e] = dpp_add<0x140>(v);
                }
                if (lr == 0) *(floatx4*)(g.col_partial + (long long)(2 * mb + wm) * g.N + en + 16 * a) = cs[a];
            }
        }
    } else if constexpr (GATED) {
        // h is rounded as an operand of the second product, from unrounded gate and up values.
        // 16 rows at a time, 16-byte chunks: 0..3 the gate columns of a row, 4..7 the up columns (chunk c of row r at
        // c ^ (r & 7)); then h, 32 rows at a time, 4 chunks a row (at c ^ (r / 2 & 3))
        if constexpr (EPI == GEMM_EPI_GATED_SAVE) {
#pragma unroll
            for (int b = 0; b < 4; b++) {
#pragma unroll
                for (int a = 0; a < 4; a++)
                    *(uint2*)(stg + 128 * lr + 16 * ((2 * a + (lg >> 1)) ^ (lr & 7)) + 8 * (lg & 1)) = pack(acc[a][b]);
                wave_lds_fence();
#pragma unroll
                for (int q = 0; q < 2; q++) {
                    const int gm = m0 + 64 * wm + 16 * b + 8 * q + (lane >> 3), gn = n0 + 32 * wn + 8 * (lane & 3);
                    const uint4 v = *(const uint4*)(stg + 128 * (8 * q + (lane >> 3)) + 16 * ((lane & 7) ^ (lane >> 3)));
                    if (gm < M && gn < N) *(uint4*)((uint16_t*)g.C + gm * g.ldc + gn + ((lane & 4) ? N : 0)) = v;
                }
                wave_lds_fence();
            }
        }
#pragma unroll
        for (int b2 = 0; b2 < 2; b2++) {
#pragma unroll
            for (int bb = 0; bb < 2; bb++)
#pragma unroll
                for (int a = 0; a < 2; a++) {
                    const floatx4 z = acc[a][2 * b2 + bb], u = acc[a + 2][2 * b2 + bb];
                    *(uint2*)(stg + 64 * (16 * bb + lr) + 16 * ((2 * a + (lg >> 1)) ^ (lr >> 1 & 3)) + 8 * (lg & 1)) =
                        pack(floatx4{silu(z[0]) * u[0], silu(z[1]) * u[1], silu(z[2]) * u[2], silu(z[3]) * u[3]});
                }
            wave_lds_fence();
#pragma unroll
            for (int q = 0; q < 2; q++) {
                const int row = 16 * q + (lane >> 2), gm = m0 + 64 * wm + 32 * b2 + row, gn = n0 + 32 * wn + 8 * (lane & 3);
                const uint4 v = *(const uint4*)(stg + 64 * row + 16 * ((lane & 3) ^ (row >> 1 & 3)));
                if (gm < M && gn < N) *(uint4*)((uint16_t*)g.C2 + gm * g.ldc2 + gn) = v;
            }
            wave_lds_fence();
        }
    } else {
        // through LDS in fp32, so that dh and the residual are met unrounded
#pragma unroll
        for (int b = 0; b < 4; b++) {
#pragma unroll
            for (int a = 0; a < 4; a++) *(floatx4*)(stg + 256 * lr + 16 * ((4 * a + lg) ^ lr)) = acc[a][b];
            wave_lds_fence();
#pragma unroll
            for (int q = 0; q < 2; q++) {
                const int row = 8 * q + (lane >> 3), ch = lane & 7;
                const int gm = m0 + 64 * wm + 16 * b + row, gn = n0 + 64 * wn + 8 * ch;
                floatx4 x0 = *(const floatx4*)(stg + 256 * row + 16 * ((2 * ch) ^ row));
                floatx4 x1 = *(const floatx4*)(stg + 256 * row + 16 * ((2 * ch + 1) ^ row));
                uint16_t* dst = (uint16_t*)g.C + gm * g.ldc + gn;
                const bool in = gm < M && gn < N;
                if constexpr (EPI == GEMM_EPI_GATED_BWD) {
                    uint4 og, ou;
                    gated_gradient(x0, x1, pg[b][q], pu[b][q], &og, &ou);
                    if (in) {
                        *(uint4*)dst = og;
                        *(uint4*)(dst + N) = ou;
                    }
                } else {
                    if constexpr (EPI == GEMM_EPI_RESIDUAL) {
                        x0 += unpack(make_uint2(rr[b][q].x, rr[b][q].y));
                        x1 += unpack(make_uint2(rr[b][q].z, rr[b][q].w));
                    }
                    const uint2 lo = pack(x0), hi = pack(x1);
                    if (in) *(uint4*)dst = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
            }
            wave_lds_fence();
        }
    }
}

template <int LAYOUT, int EPI>
__global__ __launch_bounds__(256, 2) void gemm_mid_kernel(TileArgs g) {
    __shared__ __align__(1024) char sm[MID_LDS];
    mid_tile<LAYOUT, EPI>(g, blockIdx.x, sm);
}

// Several products in one launch, each from a workgroup of its own on (a multiple of the XCDs).
template <int LAYOUT0, int EPI0, int LAYOUT1, int EPI1>
__global__ __launch_bounds__(256, 2) void gemm_mid_pair_kernel(TileArgs g, TileArgs h, int first) {
    __shared__ __align__(1024) char sm[MID_LDS];
    if ((int)blockIdx.x < first) mid_tile<LAYOUT0, EPI0>(g, blockIdx.x, sm);
    else mid_tile<LAYOUT1, EPI1>(h, blockIdx.x - first, sm);
}

template <int LAYOUT0, int EPI0, int LAYOUT1, int EPI1>
__global__ __launch_bounds__(256, 2) void gemm_mid_trio_kernel(TileArgs g, TileArgs h, TileArgs k, int first, int second) {
    __shared__ __align__(1024) char sm[MID_LDS];
    if ((int)blockIdx.x < first) mid_tile<LAYOUT0, EPI0>(g, blockIdx.x, sm);
    else mid_tile<LAYOUT1, EPI1>((int)blockIdx.x < second ? h : k, blockIdx.x - ((int)blockIdx.x < second ? first : second), sm);
}

static inline int mid_grid(const TileArgs& g) { return XCDS * ((g.mblocks * g.nblocks * g.splits + XCDS - 1) / XCDS); }

template <int LAYOUT, int EPI>
static hipError_t mid_launch(const TileArgs& g, hipStream_t s) {
    gemm_mid_kernel<LAYOUT, EPI><<<mid_grid(g), 256, 0, s>>>(g);
    return hipGetLastError();
}

// ---------------------------------------------------------------- which tiles

// Tiles and K splits of a product, and its kernel: 256 x 256 tiles, one workgroup per CU, or 128 x 128 tiles,
// two per CU.  Whichever is estimated to end first: rounds of workgroups that fill the chip, each of its k steps
// of 64 and a start and an end, and with K splits their fp32 partials, written and read by another kernel.
// The figures are measured ones (T = 312 .. 69,563, d = 256 .. 1024, f = 704 .. 2816).
struct Tiles {
    bool mid;
    int mblocks, nblocks, splits;
    double us;
};

constexpr double MID_START = 4.0, MID_STEP = 1.0, MID_STEP_ALONE = 0.8;     // us; two workgroups on a CU, or one
constexpr double WIDE_START = 7.0, WIDE_STEP = 1.3;

// Writing and reading `elements` of fp32 partials, and the launch that adds them.
static inline double partials_us(double elements) { return 4.0 + elements * 8 / 8e6; }

// n_cols: columns of the result per 256 columns of B (128 for the gated products).
// end: an epilogue's own time per round.
static inline Tiles tiles_of(bool mid, long long M, long long N, long long K, int n_cols, int splits, bool partials, double end = 0.0) {
    Tiles t{};
    t.mid = mid;
    const int side = mid ? MBM : WBM, cols = mid ? n_cols / 2 : n_cols;
    t.mblocks = (int)((unsigned long long)(M + side - 1) / (unsigned)side);
    t.nblocks = (int)((unsigned long long)(N + cols - 1) / (unsigned)cols);
    t.splits = splits;
    const unsigned all = (unsigned)((K + WBK - 1) / WBK), steps = (all + splits - 1) / (unsigned)splits;
    const long long items = (long long)t.mblocks * t.nblocks * splits;
    if (mid) t.us = (double)((items + MID_WORKGROUPS - 1) / MID_WORKGROUPS) *
                    (MID_START + end + (items > WIDE_WORKGROUPS ? MID_STEP : MID_STEP_ALONE) * steps);
    else t.us = (double)((items + WIDE_WORKGROUPS - 1) / WIDE_WORKGROUPS) * (WIDE_START + end + WIDE_STEP * steps);
    if (partials) t.us += partials_us((double)splits * M * N);
    return t;
}

static inline Tiles plan(long long M, long long N, long long K, int n_cols = WBN, double wide_end = 0.0, double mid_end = 0.0) {
    const Tiles wide = tiles_of(false, M, N, K, n_cols, 1, false, wide_end), mid = tiles_of(true, M, N, K, n_cols, 1, false, mid_end);
    return mid.us < wide.us ? mid : wide;
}

constexpr int SPLITS[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64};

// The same with K splits of the 128 x 128 tiles.
static inline Tiles plan_deep(long long M, long long N, long long K) {
    Tiles best = plan(M, N, K);
    if (best.us < 12.0) return best;              // (about what a split's start and end and its sum take)
    for (int s : SPLITS) {
        if (s == 1) continue;
        if (s > 16 || s * 4 * WBK > K) break;
        const Tiles t = tiles_of(true, M, N, K, WBN, s, true);
        if (t.us < best.us) best = t;
    }
    return best;
}

// A product of fp32 partials, or (not `always`) one that 256 x 256 tiles without a split finish in place.
static inline Tiles plan_split(long long M, long long N, long long K, bool always) {
    Tiles best{};
    best.us = 1e30;
    for (int s : SPLITS) {
        if (s > 1 && s * 4ll * WBK > K) break;
        for (int mid = 0; mid < 2; mid++) {
            const Tiles t = tiles_of(mid, M, N, K, WBN, s, always || mid || s > 1);
            if (t.us < best.us) best = t;
        }
    }
    return best;
}

// "128x128/3": the tiles and, beyond one, their K splits.
struct TilesName {
    char text[24];
};
static inline TilesName tiles_name(const char* tiles, int splits) {
    TilesName n;
    snprintf(n.text, sizeof(n.text), splits > 1 ? "%s/%d" : "%s", tiles, splits);
    return n;
}
static inline TilesName tiles_name(const Tiles& t) { return tiles_name(t.mid ? "128x128" : "256x256", t.splits); }

static inline size_t partial_bytes(const Tiles& t, long long M, long long N) {
    return t.splits > 1 ? (size_t)t.splits * M * N * sizeof(float) : 0;
}

static inline void set_tiles(TileArgs* g, const Tiles& t) {
    g->mblocks = t.mblocks;
    g->nblocks = t.nblocks;
    g->splits = t.splits;
    g->ks_per_split = (int)(((g->K + WBK - 1) / WBK + t.splits - 1) / t.splits);
    // (the 256 x 256 kernel wants every split to have k)
    if (!t.mid) g->splits = (int)(((g->K + WBK - 1) / WBK + g->ks_per_split - 1) / g->ks_per_split);
    g->wide = !t.mid;
}

}  // namespace mtgr
