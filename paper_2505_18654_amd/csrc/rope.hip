// Rotary positions, alone and on the way into a paged cache.
//
// A thread takes one item of a token's heads: two 16-byte vectors, features i .. and i + rot / 2 .., which hold whole pairs in
// both layouts, or two of features behind rot, which are copied.  It forms the sines and cosines once and applies them to its
// heads.  Bound by memory: each head is read and written once.  69,563 tokens, 10 heads of 128 (356 MB): 77 us, 4.6 TB/s;
// with one head at a time and a thread's two vectors beside each other 84; with non-temporal loads and stores 86.  The append of
// 21,862 tokens, 8 + 2 heads of 128 and the values: 134 MB in 27.7 us.
#include "causal_device.h"

namespace mtgr {
namespace {

// Sine and cosine of t whole turns: t is brought to an eighth of a turn around the nearest quarter in 64 bits (which
// is exact), then Taylor's series up to x^9 and x^10, whose next terms are below 2e-9 for |x| <= pi / 4.
__device__ __forceinline__ void sincos_turns(double t, float& s, float& c) {
    const double r = t - rint(t), q = rint(4.0 * r);
    const float x = 6.2831853071795865f * (float)(r - 0.25 * q), x2 = x * x;
    float sn = __builtin_fmaf(x2, 2.7557319e-6f, -1.9841270e-4f);          // 1 / 9!, - 1 / 7!
    sn = __builtin_fmaf(x2, sn, 8.3333333e-3f);
    sn = __builtin_fmaf(x2, sn, -1.6666667e-1f);
    sn = __builtin_fmaf(x * x2, sn, x);
    float cs = __builtin_fmaf(x2, -2.7557319e-7f, 2.4801587e-5f);          // - 1 / 10!, 1 / 8!
    cs = __builtin_fmaf(x2, cs, -1.3888889e-3f);
    cs = __builtin_fmaf(x2, cs, 4.1666667e-2f);
    cs = __builtin_fmaf(x2, cs, -0.5f);
    cs = __builtin_fmaf(x2, cs, 1.0f);
    const int k = (int)q & 3;
    const float a = k & 1 ? cs : sn, b = k & 1 ? sn : cs;
    s = k & 2 ? -a : a;
    c = (k == 1 || k == 2) ? -b : b;
}

// 16 bytes of E.
template <class E>
struct Vec {
    static constexpr int N = 16 / (int)sizeof(E);
    E v[N];
};
__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(uint16_t v) { return bf16_to_f32(v); }
template <class E>
__device__ __forceinline__ void unpack(uint4 u, float (&f)[Vec<E>::N]) {
    const Vec<E> x = __builtin_bit_cast(Vec<E>, u);
#pragma unroll
    for (int i = 0; i < Vec<E>::N; i++) f[i] = as_f32(x.v[i]);
}
__device__ __forceinline__ uint4 pack(const float (&f)[4]) { return __builtin_bit_cast(uint4, f); }
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// Features of an item, and its pairs' sines and cosines.  Items beside each other take vectors beside each other.
template <class E>
struct Item {
    static constexpr int N = Vec<E>::N;
    int e0, e1;               // first features of the two vectors; e1 < 0: only one
    bool turns;
    float s[N], c[N];         // half layout: of the pairs (e0 + i, e1 + i); interleaved: of e0's N / 2 pairs, then of e1's
    __device__ __forceinline__ Item(const RopeArgs& a, int item, long long position) {
        const int nrot = a.rot / (2 * N), ncopy = (a.dh - a.rot + 2 * N - 1) / (2 * N);
        turns = item < nrot;
        if (!turns) {
            e0 = a.rot + N * (item - nrot);
            e1 = e0 + N * ncopy < a.dh ? e0 + N * ncopy : -1;
            return;
        }
        e0 = N * item;
        e1 = e0 + a.rot / 2;
        const double p = (double)(a.inverse ? -position : position) * 0.15915494309189533577;   // 1 / 2 pi
#pragma unroll
        for (int i = 0; i < N; i++) {
            const int pair = !a.interleaved ? e0 + i : i < N / 2 ? e0 / 2 + i : e1 / 2 + i - N / 2;
            sincos_turns(p * a.freqs[pair], s[i], c[i]);
            s[i] *= a.amplitude;
            c[i] *= a.amplitude;
        }
    }
    __device__ __forceinline__ void turn(uint4& u0, uint4& u1, bool interleaved) const {
        float x[N], y[N], o[N], p[N];
        unpack<E>(u0, x);
        unpack<E>(u1, y);
        if (interleaved) {
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const int j = i / 2, k = (N + i) / 2;
                o[i] = x[i] * c[j] - x[i + 1] * s[j];
                o[i + 1] = x[i] * s[j] + x[i + 1] * c[j];
                p[i] = y[i] * c[k] - y[i + 1] * s[k];
                p[i + 1] = y[i] * s[k] + y[i + 1] * c[k];
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) {
                o[i] = x[i] * c[i] - y[i] * s[i];
                p[i] = x[i] * s[i] + y[i] * c[i];
            }
        }
        u0 = pack(o);
        u1 = pack(p);
    }
};

// The sequence that row t belongs to; false behind the last one.
__device__ __forceinline__ bool sequence_of(const int* offsets, int B, long long t, int& b) {
    if (B <= 0 || t >= offsets[B]) return false;
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= t) lo = mid;
        else hi = mid;
    }
    b = lo;
    return true;
}

template <class E>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, uint32_t items, uint32_t groups) {
    // (a block's first thread in 64 bits, the threads of a block from it in 32)
    const uint32_t per_token = items * groups;
    const long long first = blockIdx.x * 256ll, t0 = first / per_token;
    const uint32_t i = (uint32_t)(first - t0 * per_token) + threadIdx.x;
    const int item = (int)(i % items), g = (int)(i / items % groups);
    const long long t = t0 + i / per_token;
    if (t >= a.T) return;
    long long position;
    if (a.positions) {
        position = a.positions[t];
    } else {
        int b;
        if (!sequence_of(a.offsets, a.B, t, b)) return;
        position = t - a.offsets[b];
    }
    const Item<E> it(a, item, position);
    const bool same = a.x == a.out && a.ld_x == a.ld_out;
    if (!it.turns && same) return;
    const E* x = (const E*)a.x + t * a.ld_x;
    E* out = (E*)a.out + t * a.ld_out;
    const int h1 = (int)((long long)a.heads * (g + 1) / groups);
    int h = (int)((long long)a.heads * g / groups);
    const int e1 = it.e1 < 0 ? it.e0 : it.e1;                    // (a lone vector is taken twice)
    // Two heads at a time: their loads before either's stores, which out = x keeps apart.
    for (; h + 1 < h1; h += 2) {
        const E* x0 = x + h * a.dh;
        E* o0 = out + h * a.dh;
        uint4 u0 = *(const uint4*)(x0 + it.e0), u1 = *(const uint4*)(x0 + e1);
        uint4 v0 = *(const uint4*)(x0 + a.dh + it.e0), v1 = *(const uint4*)(x0 + a.dh + e1);
        if (it.turns) {
            it.turn(u0, u1, a.interleaved);
            it.turn(v0, v1, a.interleaved);
        }
        *(uint4*)(o0 + it.e0) = u0;
        *(uint4*)(o0 + e1) = u1;
        *(uint4*)(o0 + a.dh + it.e0) = v0;
        *(uint4*)(o0 + a.dh + e1) = v1;
    }
    if (h < h1) {
        uint4 u0 = *(const uint4*)(x + h * a.dh + it.e0), u1 = *(const uint4*)(x + h * a.dh + e1);
        if (it.turns) it.turn(u0, u1, a.interleaved);
        *(uint4*)(out + h * a.dh + it.e0) = u0;
        *(uint4*)(out + h * a.dh + e1) = u1;
    }
}

__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a, uint32_t items, uint32_t groups) {
    typedef uint16_t E;
    const RopeArgs& r = a.rope;
    const CacheArgs& cache = a.cache;
    const uint32_t per_token = items * groups;
    const long long block0 = blockIdx.x * 256ll, t0 = block0 / per_token;
    const uint32_t i = (uint32_t)(block0 - t0 * per_token) + threadIdx.x;
    const int item = (int)(i % items), g = (int)(i / items % groups);
    const long long t = t0 + i / per_token;
    if (t >= r.T) return;
    int b = (int)t;
    long long at = 0;
    if (r.offsets) {
        if (!sequence_of(r.offsets, r.B, t, b)) return;
        at = t - r.offsets[b];
    }
    const int past = a.past[b];
    if (past < 0) return;
    at += past;
    const long long column = at >> cache.page_shift;
    if (column >= cache.max_pages) return;
    const int page = cache.table[b * cache.ld_table + column];
    const bool is_page = page >= 0 && page < cache.num_pages;
    const int row = (int)(at & ((1 << cache.page_shift) - 1));
    const Item<E> it(r, item, at);
    const int Hk = cache.kv_heads, all = r.heads + 2 * Hk, h1 = (int)((long long)all * (g + 1) / groups);
    for (int h = (int)((long long)all * g / groups); h < h1; h++) {
        const E* src;
        E* dst;
        if (h < r.heads) {
            src = (const E*)r.x + t * r.ld_x + h * r.dh;
            dst = (E*)r.out + t * r.ld_out + h * r.dh;
        } else {
            if (!is_page) continue;
            const int j = (h - r.heads) % Hk;
            const bool key = h < r.heads + Hk;
            src = (key ? (const E*)a.k + t * a.ld_k : (const E*)a.v + t * a.ld_v) + j * r.dh;
            dst = (E*)(key ? cache.keys : cache.values) + ((((long long)page * Hk + j) << cache.page_shift) + row) * r.dh;
        }
        uint4 u0 = *(const uint4*)(src + it.e0), u1{};
        if (it.e1 >= 0) u1 = *(const uint4*)(src + it.e1);
        if (it.turns && h < r.heads + Hk) it.turn(u0, u1, r.interleaved);
        *(uint4*)(dst + it.e0) = u0;
        if (it.e1 >= 0) *(uint4*)(dst + it.e1) = u1;
    }
}

// Heads go to so many threads each that a launch has about `most` threads; a thread's sines serve its heads.  For positions four
// waves for each SIMD (40,000 tokens, 8 heads of 64: 17.7 us, with two 20.8, with eight 18.1; 10,000 of 128: 8.9, 8.9, 12.4), for
// the append, whose threads also find their page, two (21,862 tokens, 8 + 2 heads of 128: 27.8, with four 29.5).
constexpr long long ROPE_THREADS = 262144, APPEND_THREADS = 131072;
int head_groups(long long threads, int heads, long long most) {
    return (int)std::min<long long>(heads, std::max<long long>(1, (most + threads - 1) / threads));
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, bool bf16, hipStream_t s) {
    const int n = bf16 ? 8 : 4, items = a.rot / (2 * n) + (a.dh - a.rot + 2 * n - 1) / (2 * n);
    const int groups = head_groups(a.T * items, a.heads, ROPE_THREADS);
    const long long blocks = (a.T * items * groups + 255) / 256;
    if (bf16) rope_kernel<uint16_t><<<(unsigned)blocks, 256, 0, s>>>(a, items, groups);
    else rope_kernel<float><<<(unsigned)blocks, 256, 0, s>>>(a, items, groups);
    return hipGetLastError();
}

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t s) {
    const RopeArgs& r = a.rope;
    const int items = r.rot / 16 + (r.dh - r.rot + 15) / 16;
    const int groups = head_groups(r.T * items, r.heads + 2 * a.cache.kv_heads, APPEND_THREADS);
    const long long blocks = (r.T * items * groups + 255) / 256;
    kv_append_kernel<<<(unsigned)blocks, 256, 0, s>>>(a, items, groups);
    return hipGetLastError();
}

}  // namespace mtgr
