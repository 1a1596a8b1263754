// The gated feed-forward block for few tokens (serving): both products as streams of the weights.
//
// With few rows each weight is used for a few operations, so what counts is how fast the weights arrive: a
// workgroup takes 16 CPL columns of a weight matrix (for the gated product half of them gate, half up columns
// of the same numbers) and up to 16 MB rows, and its waves share the k range, each reading its own rows of
// the weights straight into registers.  Nothing is handed over between waves until their partial products
// are added through LDS, in a fixed order, where the activation, the product and the residual are applied.
//
// The weights are row-major [K, N], the matrix instruction wants eight k of one column in a lane.  Lane l
// reads columns CPL (l % 16) .. + CPL - 1 of the rows 8 (l / 16) .. + 7 of a k block of 32, and v_perm
// pairs the rows' 16-bit halves: fragment j then holds the columns CPL (l % 16) + j, a row order of the
// (transposed) result that only the epilogue sees.
//
// Bound by latency (start, one chain of weight loads, the additions through LDS) and, the larger the weights, by what
// the few workgroups can load: one token, 512 / 1408, 44 and 16 workgroups: 4.3 and 3.9 us for 2.9 and 1.4 MB; 1024 /
// 2816, 88 and 32 workgroups: 8.2 us for 11.5 MB, 1.4 TB/s, and 7.9 for 5.8 MB, 0.7 TB/s.
#include "block_internal.h"
#include "mtgr_device.h"

namespace mtgr {

namespace {

constexpr int FR_GATED = 0, FR_SAVE = 1, FR_OUT = 2;

struct RowsArgs {
    int T, K, N;              // N: hidden columns (gated), or columns of y
    const uint16_t *x, *w;
    long long ld_x, ld_w;
    uint16_t *out, *pre;      // h, or y; pre
    const uint16_t* residual;
    long long ld_out, ld_pre, ld_r;
};

template <int CPL>
struct WordsOf;
template <>
struct WordsOf<4> {
    typedef uint2 type;
    __device__ static uint32_t word(uint2 v, int j) { return j ? v.y : v.x; }
};
template <>
struct WordsOf<2> {
    typedef uint32_t type;
    __device__ static uint32_t word(uint32_t v, int) { return v; }
};

template <int KIND, int MB, int CPL, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void ffn_rows_kernel(RowsArgs a) {
    typedef typename WordsOf<CPL>::type Words;
    constexpr int NC = 16 * CPL, LD = NC + 4, ROWS = 16 * MB, HALF = WAVES / 2;
    __shared__ __align__(16) float red[HALF][ROWS][LD];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, cl = lane & 15, kg = lane >> 4;
    const int c0 = blockIdx.x * (KIND == FR_OUT ? NC : NC / 2), m0 = blockIdx.y * ROWS;
    int col;
    if (KIND == FR_OUT) col = min(c0 + CPL * cl, a.N - CPL);
    else col = c0 + CPL * (cl & 7) + (cl >= 8 ? a.N : 0);
    uint32_t wo[8];
#pragma unroll
    for (int i = 0; i < 8; i++) wo[i] = (uint32_t)((8 * kg + i) * a.ld_w + col) * 2u;
    const uint16_t* xr[MB];
#pragma unroll
    for (int m = 0; m < MB; m++) xr[m] = a.x + min(m0 + 16 * m + cl, a.T - 1) * a.ld_x + 8 * kg;
    floatx4 acc[MB][CPL];
#pragma unroll
    for (int m = 0; m < MB; m++)
#pragma unroll
        for (int j = 0; j < CPL; j++) acc[m][j] = floatx4{};
    const int nkb = a.K / 32;
    const char* wp = (const char*)(a.w + (long long)w * 32 * a.ld_w);
    const long long wstep = (long long)WAVES * 32 * a.ld_w * 2;
#pragma unroll (MB == 4 ? 2 : 4)
    for (int kb = w; kb < nkb; kb += WAVES, wp += wstep) {
        Words r[8];
#pragma unroll
        for (int i = 0; i < 8; i++) r[i] = *(const Words*)(wp + wo[i]);
        bf16x8 xf[MB];
#pragma unroll
        for (int m = 0; m < MB; m++) xf[m] = *(const bf16x8*)(xr[m] + 32 * kb);
#pragma unroll
        for (int j = 0; j < CPL; j++) {
            uint4 f;
            const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
            f.x = __builtin_amdgcn_perm(WordsOf<CPL>::word(r[1], j >> 1), WordsOf<CPL>::word(r[0], j >> 1), sel);
            f.y = __builtin_amdgcn_perm(WordsOf<CPL>::word(r[3], j >> 1), WordsOf<CPL>::word(r[2], j >> 1), sel);
            f.z = __builtin_amdgcn_perm(WordsOf<CPL>::word(r[5], j >> 1), WordsOf<CPL>::word(r[4], j >> 1), sel);
            f.w = __builtin_amdgcn_perm(WordsOf<CPL>::word(r[7], j >> 1), WordsOf<CPL>::word(r[6], j >> 1), sel);
#pragma unroll
            for (int m = 0; m < MB; m++)
                acc[m][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(f), xf[m], acc[m][j], 0, 0, 0);
        }
    }
    // acc[m][j][r]: row 16 m + cl, column CPL (4 kg + r) + j of the workgroup's.  The upper half of the waves
    // hands its part to the lower half, lane for lane, so that LDS holds half as many (two workgroups per CU).
    typedef float Part __attribute__((ext_vector_type(CPL)));
    auto pass = [&](bool add) {
#pragma unroll
        for (int m = 0; m < MB; m++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                Part v, *p = (Part*)&red[w % HALF][16 * m + cl][CPL * (4 * kg + r)];
#pragma unroll
                for (int j = 0; j < CPL; j++) v[j] = acc[m][j][r];
                *p = add ? *p + v : v;
            }
    };
    if (w >= HALF) pass(false);
    __syncthreads();
    if (w < HALF) pass(true);
    __syncthreads();
    constexpr int OC = KIND == FR_OUT ? NC : NC / 2;         // output columns, four per thread
    for (int i = tid; i < ROWS * (OC / 4); i += 64 * WAVES) {
        const int row = i / (OC / 4), c = i % (OC / 4) * 4;
        const long long gm = m0 + row;
        const int gn = c0 + c;
        if (gm >= a.T || gn >= a.N) continue;
        floatx4 s = *(const floatx4*)&red[0][row][c];
#pragma unroll
        for (int k = 1; k < HALF; k++) s += *(const floatx4*)&red[k][row][c];
        if (KIND == FR_OUT) {
            if (a.residual) {
                const uint2 r = *(const uint2*)(a.residual + gm * a.ld_r + gn);
                s[0] += __uint_as_float(r.x << 16);
                s[1] += __uint_as_float(r.x & 0xffff0000u);
                s[2] += __uint_as_float(r.y << 16);
                s[3] += __uint_as_float(r.y & 0xffff0000u);
            }
        } else {
            floatx4 u = *(const floatx4*)&red[0][row][c + OC];
#pragma unroll
            for (int k = 1; k < HALF; k++) u += *(const floatx4*)&red[k][row][c + OC];
            if (KIND == FR_SAVE) {
                uint16_t* p = a.pre + gm * a.ld_pre + gn;
                *(uint2*)p = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
                *(uint2*)(p + a.N) = make_uint2(pack_bf16x2(u[0], u[1]), pack_bf16x2(u[2], u[3]));
            }
#pragma unroll
            for (int e = 0; e < 4; e++)       // (rounded below: an operand of the second product)
                s[e] = s[e] * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * s[e])) * u[e];
        }
        *(uint2*)(a.out + gm * a.ld_out + gn) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
    }
}

template <int KIND, int CPL>
hipError_t rows_launch(const RowsArgs& a, hipStream_t s) {
    const int per = KIND == FR_OUT ? 16 * CPL : 8 * CPL, gx = (a.N + per - 1) / per;
    if (a.T <= 16) ffn_rows_kernel<KIND, 1, CPL, 16><<<dim3(gx, 1), 1024, 0, s>>>(a);
    else if (a.T <= 32) ffn_rows_kernel<KIND, 2, CPL, 8><<<dim3(gx, 1), 512, 0, s>>>(a);
    else ffn_rows_kernel<KIND, 4, CPL, 8><<<dim3(gx, (a.T + 63) / 64), 512, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

// Up to one workgroup of 64 rows per CU: beyond that the tiles of gemm_mid.h read the weights less often (gated
// product of 64 tokens, d = 1024, f = 2816, 176 workgroups: 10.9 us here and 13.0 there; 600 tokens, d = 256,
// f = 704, 220: 6.3 and 6.3; 312 tokens, d = 768, f = 2048, 320: 15.2 and 12.2; 1,024 tokens, d = 512, f = 1408,
// 704: 18 and 9.4).
bool ffn_rows_fit(long long T, int N, int columns) {
    return T <= 16384 && (T + 63) / 64 * ((N + columns - 1) / columns) <= 256;
}

hipError_t launch_ffn_rows_hidden(const FfnArgs& f, hipStream_t s) {
    RowsArgs a{};
    a.T = (int)f.T;
    a.K = f.d;
    a.N = f.f;
    a.x = (const uint16_t*)f.x;
    a.w = (const uint16_t*)f.w_in;
    a.ld_x = f.ld_x;
    a.ld_w = f.ld_win;
    a.out = (uint16_t*)f.h;
    a.ld_out = f.ld_h;
    a.pre = (uint16_t*)f.pre;
    a.ld_pre = f.ld_pre;
    return f.pre ? rows_launch<FR_SAVE, 4>(a, s) : rows_launch<FR_GATED, 4>(a, s);
}

hipError_t launch_ffn_rows_out(const FfnArgs& f, hipStream_t s) {
    RowsArgs a{};
    a.T = (int)f.T;
    a.K = f.f;
    a.N = f.d;
    a.x = (const uint16_t*)f.h;
    a.w = (const uint16_t*)f.w_out;
    a.ld_x = f.ld_h;
    a.ld_w = f.ld_wout;
    a.out = (uint16_t*)f.y;
    a.ld_out = f.ld_y;
    a.residual = (const uint16_t*)f.residual;
    a.ld_r = f.ld_r;
    return rows_launch<FR_OUT, 2>(a, s);
}

}  // namespace mtgr
