// One query token of each sequence against its paged cache.
//
// A workgroup takes a chunk of a sequence's keys for one key head and up to 32 of the query heads that share it, a query
// head per column of the 32 x 32 products; its waves take the chunk's tiles of 32 keys in turn, each with its own maximum,
// sum and outputs, and its own LDS tiles, so that no wave waits for another.  A wave copies the next tile's keys while it
// works on this one's probabilities, and the next values once this one's are used, so that half of its 128 DH bytes of LDS at least
// are under way at any time.  The waves are joined through LDS, and the chunks of a sequence, where there are several, by a
// second kernel.  Rounded to bf16 are the probabilities (matrix operands) and the result.
//
// Bound by the read of the cache: 24 sequences of up to 131,072 tokens, 32 / 8 heads of 128, 4.78 GB in 836 us, 5.7 TB/s (a
// device copy: 5.14).  Without the copies ahead 1,227 us.  Less to read is bound by each workgroup's chain of length, pages,
// keys and values, and by the join: one sequence of 100,003 tokens, 6 / 2 heads, 102 MB in 25 us.
#include "causal_device.h"

namespace mtgr {
namespace {

using namespace causal;
constexpr int BN = 32, QT = 32, CHUNKS = 512;

// A wave's copy of 32 rows of a head's pages into a swizzled tile, page0 and page1 those of its halves (16 rows, the
// smallest page).  Rows outside lo .. hi are copies of row lo or hi, so that every row of the tile is one of the sequence's own.
template <int DH>
__device__ __forceinline__ void page_dma(uint16_t* tile, const uint16_t* base, long long page_stride, int in_page, int page0,
                                         int page1, int row0, int lo, int hi, int lane) {
    constexpr int CPR = DH / 8, RPI = 64 / CPR;
    const int rl = lane / CPR;
    const uint32_t dst = lds_address(tile);
#pragma unroll
    for (int i = 0; i < BN / RPI; i++) {
        const int page = min(max(i * RPI, lo), hi) >= 16 ? page1 : page0;
        const int r = min(max(i * RPI + rl, lo), hi);
        const int c = (lane % CPR) ^ swz<CPR>(i * RPI + rl);
        lds_dma16(dst + i * 1024u, uniform_ptr(base + page * page_stride), (uint32_t)(((row0 + r) & in_page) * DH + c * 8) * 2u);
    }
}

template <int DH, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DH == 64 ? 4 : 2) void cache_attn_kernel(CacheAttnArgs a) {
    constexpr int CPR = DH / 8, KSTEPS = DH / 16, DBLK = DH / 32, TILE = BN * DH, NI = CPR / 2;
    __shared__ __align__(16) uint16_t sT[WAVES][2][TILE];        // K and V of each wave; then its outputs
    __shared__ float sML[WAVES][2][QT];
    static_assert(2 * TILE * 2 >= QT * DH * 4, "a wave's outputs fit its tiles");
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    // Chunks slowest: workgroup i runs on XCD i % 8, and with the chunks of a sequence beside each other, where there are 4 or 8
    // of them, some XCDs got the first chunks, which every sequence has, and others the last, which most have not (37 sequences
    // of up to 2,113 tokens, 16 / 8 heads of 128: 30 us, with 4 chunks side by side 41).
    const int qtiles = (a.group + QT - 1) / QT, units = a.cache.kv_heads * qtiles;
    const int unit = blockIdx.x % units, b = blockIdx.x / units % a.B, split = blockIdx.x / units / a.B;
    const int hk = unit / qtiles;
    const int g0 = QT * (unit % qtiles), heads = min(QT, a.group - g0), h0 = hk * a.group + g0;
    const CacheArgs& cache = a.cache;
    const int* table = cache.table + b * cache.ld_table;
    const long long head_ofs = (long long)hk << cache.page_shift, page_stride = ((long long)cache.kv_heads << cache.page_shift) * DH;
    const uint16_t* Kb = (const uint16_t*)cache.keys + head_ofs * DH;
    const uint16_t* Vb = (const uint16_t*)cache.values + head_ofs * DH;
    const int in_page = (1 << cache.page_shift) - 1;
    const int c0 = split * a.chunk;
    // The query rows (columns of the products; those past `heads` are copies) come in through the wave's V tile, the first
    // tile's pages and the sequence's length beside them: one latency for the three.
    {
        const uint16_t* Q = (const uint16_t*)a.q + b * a.ld_q + h0 * DH;
#pragma unroll
        for (int i = 0; i < NI; i++) {
            const int row = i * (64 / CPR) + lane / CPR;
            lds_dma16(lds_address(sT[w][1]) + i * 1024u, uniform_ptr(Q),
                      (uint32_t)(min(row, heads - 1) * DH + ((lane % CPR) ^ swz<CPR>(row)) * 8) * 2u);
        }
    }
    // A tile: its first key, the pages of its halves (the same one where pages are larger) and the rows lo .. hi that have one.
    struct Keys {
        int k0, page0, page1, lo, hi;
    };
    auto entry = [&](int key) { return __builtin_amdgcn_readfirstlane(table[min(key >> cache.page_shift, cache.max_pages - 1)]); };
    const int first = c0 + BN * w;
    const int entry0 = entry(first), entry1 = entry(first + 16);
    const int len = min(max(a.lens[b], 0), a.max_len), c1 = (int)min((long long)c0 + a.chunk, (long long)len);
    if (c0 >= len && split > 0) {
        wait_vmem();
        return;
    }
    // The wave's next tile with a page from k0 on; k0 >= c1: none.
    auto find = [&](int k0, bool known) {
        Keys t{};
        for (; k0 < c1; k0 += BN * WAVES, known = false) {
            const int last = min(c1 - k0, BN) - 1;
            t.page0 = known ? entry0 : entry(k0);
            t.page1 = known ? entry1 : entry(k0 + 16);
            const bool has0 = t.page0 >= 0 && t.page0 < cache.num_pages;
            const bool has1 = last >= 16 && t.page1 >= 0 && t.page1 < cache.num_pages;
            t.lo = has0 ? 0 : 16;
            t.hi = has1 ? last : min(last, 15);
            if (has0 || has1) break;
        }
        t.k0 = k0;
        return t;
    };
    auto issue = [&](const Keys& t, int which) {
        page_dma<DH>(sT[w][which], which ? Vb : Kb, page_stride, in_page, t.page0, t.page1, t.k0 & in_page, t.lo, t.hi, lane);
    };
    Keys t = find(first, true);
    const bool any = t.k0 < c1;
    if (any) issue(t, 0);
    if (any) wait_vmcnt<NI>(); else wait_vmem();
    bf16x8 qreg[KSTEPS];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) qreg[kk] = tile_read8<CPR>(sT[w][1], col, 2 * kk + hh);
    wait_lgkm_seen();
    if (any) issue(t, 1);
    floatx16 oacc[DBLK];
#pragma unroll
    for (int d = 0; d < DBLK; d++) oacc[d] = floatx16{};
    float m = a.least, l = 0.f;
    while (t.k0 < c1) {
        const Keys next = find(t.k0 + BN * WAVES, false);
        const bool more = next.k0 < c1;
        const uint16_t* sK = sT[w][0];
        const uint16_t* sV = sT[w][1];
        wait_vmcnt<NI>();                                        // this tile's keys
        floatx16 s{};
#pragma unroll
        for (int kk = 0; kk < KSTEPS; kk++)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read8<CPR>(sK, col, 2 * kk + hh), qreg[kk], s, 0, 0, 0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // they are read
        if (more) issue(next, 0);
        if (t.lo > 0 || t.hi < BN - 1) {
#pragma unroll
            for (int e = 0; e < 16; e++) {
                const int key = 8 * (e >> 2) + 4 * hh + (e & 3);
                s[e] = key >= t.lo && key <= t.hi ? s[e] : neg_inf();
            }
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
        if (more) wait_vmcnt<NI>(); else wait_vmem();            // this tile's values
        if (t.lo > 0 || t.hi < BN - 1) {
            // The copies' probabilities are 0, which an infinity in the copied row would turn to NaN.
#pragma unroll
            for (int i = 0; i < BN * CPR / 64; i++) {
                const int row = (lane + 64 * i) / CPR;
                if (row < t.lo || row > t.hi) *(uint4*)&sT[w][1][8 * (lane + 64 * i)] = make_uint4(0, 0, 0, 0);
            }
        }
#pragma unroll
        for (int kq = 0; kq < 2; kq++) {
            const bf16x8 pb = as_bf16x8(make_uint4(pk[4 * kq], pk[4 * kq + 1], pk[4 * kq + 2], pk[4 * kq + 3]));
#pragma unroll
            for (int d = 0; d < DBLK; d++)
                oacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_read_tr<CPR>(sV, 16 * kq, 32 * d, lane), pb, oacc[d], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) issue(next, 1);
        t = next;
    }
    l = sum_halves(l);
    if (hh == 0) {
        sML[w][0][col] = m;
        sML[w][1][col] = l;
    }
    write_part<DH>(oacc, (float*)sT[w], lane, heads);
    __syncthreads();
    for (int i = tid; i < heads * (DH / 4); i += 64 * WAVES) {
        const int q = i / (DH / 4), f = 4 * (i % (DH / 4));
        float top, total;
        const float4 o = join_parts<DH, WAVES>(sT, sML, q, f / 4, a.c, top, total);
        const long long row = (long long)b * a.H + h0 + q;
        if (a.splits > 1) {
            *(float4*)&a.part[(row * a.splits + split) * DH + f] = o;
            if (f == 0) a.part_ml[row * a.splits + split] = make_float2(top, total);
        } else {
            const float inv = total != 0.f ? 1.0f / total : 0.f;      // no key: zeros
            *(uint2*)((uint16_t*)a.out + b * a.ld_o + (h0 + q) * DH + f) =
                make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
            if (f == 0 && a.lse) a.lse[row] = total != 0.f ? top * a.scale + logf(total) : neg_inf();
        }
    }
}

// Joins the chunks of a (sequence, head): 32 features of it per workgroup, 8 lanes for them and 32 groups of lanes over the chunks.
template <int DH>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnArgs a) {
    constexpr int L = 8, G = 256 / L;
    __shared__ float sTop[4], sTotal[G];
    __shared__ float4 sO[256];
    const int tid = threadIdx.x, h = blockIdx.x / (DH / 32), f = 32 * (blockIdx.x % (DH / 32)) + 4 * (tid % L), g = tid / L, b = blockIdx.y;
    const long long row = (long long)b * a.H + h;
    const int len = min(max(a.lens[b], 0), a.max_len), n = max(1, (len + a.chunk - 1) / a.chunk);
    const float2* ml = a.part_ml + row * a.splits;
    float top = a.least;
    for (int i = tid; i < n; i += 256) top = fmaxf(top, ml[i].x);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    if ((tid & 63) == 0) sTop[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(sTop[0], sTop[1]), fmaxf(sTop[2], sTop[3]));
    float total = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = g; i < n; i += G) {
        const float2 x = ml[i];
        const float4 v = *(const float4*)&a.part[(row * a.splits + i) * DH + f];
        const float e = __builtin_amdgcn_exp2f((x.x - top) * a.c);
        total = __builtin_fmaf(e, x.y, total);
        o.x = __builtin_fmaf(e, v.x, o.x);
        o.y = __builtin_fmaf(e, v.y, o.y);
        o.z = __builtin_fmaf(e, v.z, o.z);
        o.w = __builtin_fmaf(e, v.w, o.w);
    }
    sO[tid] = o;
    if (tid % L == 0) sTotal[g] = total;
    __syncthreads();
    if (g > 0) return;
    const int groups = min(n, G);
    for (int j = 1; j < groups; j++) {
        const float4 v = sO[j * L + tid];
        total += sTotal[j];
        o.x += v.x;
        o.y += v.y;
        o.z += v.z;
        o.w += v.w;
    }
    const float inv = total != 0.f ? 1.0f / total : 0.f;
    *(uint2*)((uint16_t*)a.out + b * a.ld_o + h * DH + f) =
        make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
    if (f == 0 && a.lse) a.lse[row] = total != 0.f ? top * a.scale + logf(total) : neg_inf();
}

}  // namespace

// Chunks as long as they leave each CU two workgroups of 4 waves.  Of three sequences and more, most are shorter than max_len,
// and half as long chunks balance better (4 sequences of up to 67,056 tokens, 6 / 3 heads of 128: 47 -> 43 us; 13 of up to 27,795,
// 12 / 3: 53 -> 43; one of 100,003, 6 / 2, the other way: 27, with half the length 32).  Up to 1,024 keys, one workgroup per
// (sequence, key head) without a second kernel, of 8 waves where they leave CUs idle.  Against every chunk of 128 to 2,048 keys
// and 4 or 8 waves, 13 sizes back to back: nine within 5 % of the best; 500 of up to 3,000, 8 / 1 heads of 64, 35.2 us where 384
// keys take 33.1; the four of 67,056 37.3 where 2,048 keys and 8 waves take 32.9; 8 of up to 8,000, 8 / 8 of 128, 24.4 where 1,536
// and 8 take 21.4; 64 of up to 4,000, 8 / 2, 28.2 where 768 take 24.0.  (The lengths, by which chunks would be balanced, are not
// known to the host.)
CacheAttnPlan cache_attn_plan(int B, int H, int Hk, int head_dim, long long max_len) {
    CacheAttnPlan p{};
    const int group = H / Hk;
    const int per_seq = Hk * ((group + QT - 1) / QT), fill = B > 2 ? 2 * CHUNKS : CHUNKS;
    const long long units = (long long)B * per_seq;
    const long long want = (fill + units - 1) / units;                               // chunks of a sequence that fill the chip
    long long chunk = (max_len + want - 1) / want;
    chunk = std::min<long long>(std::max<long long>((chunk + 127) / 128 * 128, 128), 2048);
    if (max_len <= 1024) chunk = 1024;
    while (units * ((max_len + chunk - 1) / chunk) >= (1ll << 24)) chunk *= 2;      // (of a launch; units are below 2^23)
    p.chunk = (int)chunk;
    p.splits = (int)std::max<long long>(1, (max_len + chunk - 1) / chunk);
    p.waves = p.splits == 1 && units <= 256 ? 8 : 4;
    // The workspace is sized by a bound of (rows, chunks) that rises with B and max_len, so that one for the longest history and
    // the largest batch serves all others; their number itself falls where chunks grow by a step of 128 keys.  A sequence has at
    // most `want` chunks, or as many as 2,048 keys each make, and no more than of 128 keys.
    auto round = [](long long n) { return ((size_t)n + 255) & ~(size_t)255; };
    const long long rows = (long long)B * H, most = max_len <= 1024 ? 0 : std::min<long long>({
        rows * ((max_len + 127) / 128),
        std::max<long long>(rows + (long long)H * (fill - 1) / per_seq, rows * ((max_len + 2047) / 2048)),
        ((long long)H << 24) / per_seq});                                            // (the launch's bound)
    if (p.splits > 1) {
        p.part_bytes = round(rows * p.splits * head_dim * 4);
        p.need = p.part_bytes + round(rows * p.splits * 8);
    }
    p.bytes = round(most * head_dim * 4) + round(most * 8);
    return p;
}

template <int DH>
static hipError_t cache_attn_dh(const CacheAttnArgs& a, hipStream_t s) {
    const int grid = a.H / a.group * ((a.group + QT - 1) / QT) * a.B * a.splits;
    if (a.waves == 8) cache_attn_kernel<DH, 8><<<grid, 512, 0, s>>>(a);
    else cache_attn_kernel<DH, 4><<<grid, 256, 0, s>>>(a);
    if (a.splits > 1) cache_join_kernel<DH><<<dim3(a.H * (DH / 32), a.B), 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, int head_dim, hipStream_t s) {
    switch (head_dim) {
        case 32: return cache_attn_dh<32>(a, s);
        case 64: return cache_attn_dh<64>(a, s);
        case 128: return cache_attn_dh<128>(a, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace mtgr
