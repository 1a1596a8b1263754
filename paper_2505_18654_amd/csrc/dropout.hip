// Dropout from a counter-based generator: out = [residual +] (keep ? x / (1 - p) : 0).  The mask is
// never stored; the backward pass draws it again.
//
// Generator: Philox4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy
// as 1, 2, 3", SC 2011: 7 rounds is the fewest of Philox4x32 that passes the whole of BigCrush).  The
// key is the 64-bit seed; the counter is (e / 4, low and high word, site, step) for element
// e = row * cols + column, so the mask is a function of the logical element alone: not of strides, of
// the type or of how the work is cut.  Element e takes word e % 4 and is kept when the word is at least
// floor(p 2^32).
//
// Bound by memory: 4 bytes per bf16 element (6 with a residual) against about 30 VALU operations, of
// which 7 products of 32 x 32 -> 64 bits (two per round and four elements, a quarter of the rate).  69,563 x
// 1,024 bf16 with a residual: 69 us for 427 MB, 6.2 TB/s (a large device copy: 5.07), the VALUs busy for half
// of it; small batches are one launch (96 x 32: 2.2 us).
#include "block_internal.h"
#include "mtgr_device.h"

namespace mtgr {

namespace {

struct Philox {
    uint32_t c0, c1, c2, c3;
};

__device__ __forceinline__ Philox philox7(uint32_t k0, uint32_t k1, Philox c) {
#pragma unroll
    for (int i = 0; i < 7; i++) {
        const uint64_t p0 = (uint64_t)c.c0 * 0xD2511F53u, p1 = (uint64_t)c.c2 * 0xCD9E8D57u;
        c = {(uint32_t)(p1 >> 32) ^ c.c1 ^ k0, (uint32_t)p1, (uint32_t)(p0 >> 32) ^ c.c3 ^ k1, (uint32_t)p0};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}

// 16 bytes per thread and step: 8 bf16 (two counters) or 4 fp32 (one).
template <bool BF16, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
    constexpr int N = BF16 ? 8 : 4;
    const unsigned long long seed = a.rng[0];
    const uint32_t step = (uint32_t)a.rng[1], k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
    const int nch = a.cols / N;
    const long long chunks = a.rows * nch, stride = (long long)gridDim.x * 256;
    const long long drow = stride / nch;
    const int dch = (int)(stride % nch);
    long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i / nch;
    int ch = (int)(i % nch);
    for (; i < chunks; i += stride) {
        const long long c = (long long)ch * N;
        const u32x4_nt xv = __builtin_nontemporal_load((const u32x4_nt*)((const char*)a.x + (row * a.ld_x + c) * (16 / N)));
        u32x4_nt rv{};
        if (RES) rv = __builtin_nontemporal_load((const u32x4_nt*)((const char*)a.residual + (row * a.ld_r + c) * (16 / N)));
        uint32_t word[N];
#pragma unroll
        for (int q = 0; q < N / 4; q++) {
            const unsigned long long quad = (unsigned long long)i * (N / 4) + q;
            const Philox o = philox7(k0, k1, {(uint32_t)quad, (uint32_t)(quad >> 32), a.site, step});
            word[4 * q] = o.c0;
            word[4 * q + 1] = o.c1;
            word[4 * q + 2] = o.c2;
            word[4 * q + 3] = o.c3;
        }
        float v[N];
#pragma unroll
        for (int e = 0; e < N; e++) {
            const uint32_t w = xv[BF16 ? e / 2 : e], r = rv[BF16 ? e / 2 : e];
            const float f = __uint_as_float(!BF16 ? w : e & 1 ? w & 0xffff0000u : w << 16);
            // (a dropped element is 0 whatever x holds there)
            v[e] = word[e] >= a.threshold ? f * a.scale : 0.f;
            if (RES) v[e] += __uint_as_float(!BF16 ? r : e & 1 ? r & 0xffff0000u : r << 16);
        }
        u32x4_nt o;
#pragma unroll
        for (int k = 0; k < 4; k++) o[k] = BF16 ? pack_bf16x2(v[2 * k % N], v[(2 * k + 1) % N]) : __float_as_uint(v[k % N]);
        __builtin_nontemporal_store(o, (u32x4_nt*)((char*)a.out + (row * a.ld_out + c) * (16 / N)));
        row += drow;
        ch += dch;
        if (ch >= nch) {
            ch -= nch;
            row++;
        }
    }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, bool bf16, hipStream_t s) {
    const long long chunks = a.rows * (a.cols / (bf16 ? 8 : 4));
    if (chunks <= 0) return hipSuccess;
    const int grid = (int)std::min((chunks + 255) / 256, 8192ll);
    if (bf16) {
        if (a.residual) dropout_kernel<true, true><<<grid, 256, 0, s>>>(a);
        else dropout_kernel<true, false><<<grid, 256, 0, s>>>(a);
    } else {
        if (a.residual) dropout_kernel<false, true><<<grid, 256, 0, s>>>(a);
        else dropout_kernel<false, false><<<grid, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace mtgr
