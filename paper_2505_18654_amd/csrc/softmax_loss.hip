// Softmax cross entropy of token rows against a set of class rows, in pieces of the classes, without
// keeping the logits:
//   z_nc = scale x_n . w_c + b_c,  lse_n = log sum_c exp z_nc,  loss_n = lse_n - z_n,t(n)
// and its gradients
//   dz_nc = g_n (exp(z_nc - lse_n) - [c = t(n)]),  dx = scale dz W,  dW = scale dz^T x,  db = sum_n dz.
//
// Only rows with a label (0 <= t < V) take part.  They are gathered once into consecutive rows, so that
// the products' cost follows their number, which stays on the device (no synchronisation): the grids are
// laid out for N rows and the kernels stop at the count.
//
// Forward: x W^T on the matrix cores (gemm_wide.h; up to 256 columns mostly softmax_tiles.h, small batches
// gemm_mid.h).  A workgroup walks class tiles of its rows, and every lane
// keeps a reference and a sum of exponentials for the columns that it saw of a row; a second kernel joins
// them.  2 n V d operations; written are at most 8 bytes per row and 64 classes, a sixteenth of the logits in
// bf16.
// Backward, per piece of classes: x W^T again, its epilogue turning the products into dz (rounded to bf16
// as operand of the next two products' matrix instructions; the bias gradient is summed from dz before that rounding),
// then dx += dz W (fp32, over the pieces) and the piece's dW = dz^T x.  6 n V d operations.  dz is kept divided by
// the largest |g| of the rows, which multiplies the finished sums: under a mean the g are one number, whose
// rounding error would be common to all labels' terms (-g), and a label's own term -1 is exact.
//
// Bound by the matrix cores (power) and by the epilogues' vector work, which does not run beside them
// in gemm_wide.h.  Kernel traces of ten calls in a row: 24,000 rows of 69,563, 50,021 classes, d = 512: statistics 1.23 ms
// (1.00 PFLOP/s); backward, of 2 pieces, dz 1.48 ms (0.83; 2.4 GB written), dx 1.14 (1.08), dW 1.14 (1.08), sums 0.15.
// 1,900 rows, 400,003 classes, d = 256: 0.38 (1.04); dz 0.57 (0.68; 1.5 GB written), dx 0.40 (0.98), dW 0.46 (0.84).
// (The rules' and the tiles' figures are of short bursts, in which the clock is up to a fifth higher.)
#include <stdio.h>

#include "gemm_mid.h"
#include "softmax_tiles.h"

namespace mtgr {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LOG2E_LOW = (float)(1.4426950408889634 - (double)LOG2E);
constexpr int ROWS_PER_BLOCK = 256;               // of the gather
constexpr int GROUP_M = 4;                        // see gemm_wide.h (tile_of)

struct SmPlan {
    int piece;                // classes per piece, a multiple of 256
    int pieces;
    int vpad;                 // V rounded up to whole tiles
    bool regs;                // x W^T on the tiles of softmax_tiles.h, otherwise on those of `logits`
    Tiles logits;             // of x W^T (forward and backward), dx and dW; which kernel
    Tiles dx, dw;
    bool direct;              // dW without partials
    int items;                // most of the wide dx kernel
    size_t rows /* their count, the largest |g|, class tiles of an item */, counts, tops, index, xc, bias, info, stats, running, dz, dxp, dwp, colp, total;
};

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Most items of a product with accumulated partials, over all numbers of labels (acc_splits in gemm_wide.h).
long long acc_items(long long N, int d) {
    const long long tiles = (N + WBM - 1) / WBM * ((d + WBN - 1) / WBN);
    return std::max(tiles, std::min(256ll * ACC_ROUNDS, tiles * ACC_SPLITS));
}

// Pieces of the classes: the statistics (forward, 8 bytes per row and 64 classes) or dz (backward, 2 bytes
// per row and class) of one piece take about half or four gigabytes (backward of 24,000 of 69,563 rows, 50,021
// classes, d = 512: 3.82 ms; with one gigabyte, 7 pieces instead of 2, 3.94; 1,900 of 2,048 rows, 400,003 classes,
// d = 256, one piece instead of two: 1.50, 1.57).  At most 2^22 classes: 32-bit copy offsets over 256 rows of dz.
SmPlan sm_plan(long long N, int V, int d, bool backward) {
    SmPlan p{};
    const long long mblocks = (N + WBM - 1) / WBM, npad = mblocks * WBM;
    const long long blocks = (V + WBN - 1ll) / WBN;
    const long long budget = backward ? std::min((4ll << 30) / (npad * 2 * WBN), (1ll << 22) / WBN) : (512ll << 20) / (npad * 32);
    long long per = std::max(1ll, std::min(budget, blocks));
    p.pieces = (int)((blocks + per - 1) / per);
    per = (blocks + p.pieces - 1) / p.pieces;     // pieces of equal size
    p.piece = (int)(per * WBN);
    p.vpad = (int)(blocks * WBN);
    // The number of labels is not known here: x W^T is planned for all rows, dx and dW for half of them.
    const long long half = (N + 1) / 2;
    const Tiles lw = tiles_of(false, N, p.piece, d, WBN, 1, false), lm = tiles_of(true, N, p.piece, d, WBN, 1, false);
    p.logits = lm.us < lw.us ? lm : lw;
    // (where both were measured: 2,900 rows, 20,011 classes, d = 256: 35 us, 48 on `logits`; 1,900, 400,003: 312, 513;
    // 300, 100,003: 32, 36; 64, 100,003: 14, 11; 600, 20,011, d = 192: 14, 14; 2,007 of 6,418, 5,003, d = 128: 11, 10.
    // The margin is for rows without a label, whose tiles of 256 rows are the coarser ones.)
    p.regs = d <= CT_MAX_D && sm_tiles_us(N, p.piece, d) < 0.86 * p.logits.us;
    p.dx = plan_split(half, d, p.piece, true);
    p.dw = plan_split(p.piece, d, half, false);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align256(bytes);
        return here;
    };
    p.rows = take(256);
    p.counts = take(sizeof(int) * mblocks);
    p.tops = take(sizeof(float) * mblocks);
    p.index = take(sizeof(int) * npad);
    p.bias = take(sizeof(float) * p.vpad);
    p.xc = take((size_t)npad * d * 2);
    if (!backward) {
        p.stats = take((size_t)(p.piece / 64) * N * sizeof(float2));
        p.running = take((size_t)N * sizeof(float2));
    } else {
        p.info = take(sizeof(int4) * npad);
        p.dz = take((size_t)N * p.piece * 2);
        // fp32 partials (of the wide dx kernel: as many tiles as it may have items; none of a dW that the wide kernel
        // finishes in place)
        p.items = (int)acc_items(N, d);
        p.dxp = take((p.dx.mid ? (size_t)p.dx.splits * N * d : (size_t)p.items * WBM * WBN) * sizeof(float));
        p.direct = p.dw.splits == 1 && !p.dw.mid;
        p.dwp = take(p.direct ? 0 : (size_t)p.dw.splits * p.piece * d * sizeof(float));
        p.colp = take((size_t)(p.regs || p.logits.mid ? 4 : 2) * mblocks * p.piece * sizeof(float));
    }
    p.total = at;
    return p;
}

template <class T>
__device__ __forceinline__ int label_of(const void* targets, long long i, int V) {
    const T t = ((const T*)targets)[i];
    return t >= 0 && t < V ? (int)t : -1;
}

// |g| for the largest of a batch: an infinite or NaN gradient stays that of its own row.
__device__ __forceinline__ float size_of(float g) { return fabsf(g) < __builtin_inff() ? fabsf(g) : 0.f; }

// The class bias in units of log 2, padded to whole tiles with classes that do not count.
__device__ __forceinline__ void padded_bias(const SoftmaxLossArgs& a, float* bias2, int vpad, int c) {
    if (c < vpad) bias2[c] = c >= a.V ? -__builtin_inff() : a.bias ? a.bias[c] * LOG2E : 0.f;
}

// Labels of every 256 rows, their largest |g| (backward), and the class bias (the last workgroups).
template <class T, bool BWD>
__global__ __launch_bounds__(256) void sm_count_kernel(SoftmaxLossArgs a, int* counts, float* tops, float* bias2, int vpad,
                                                       int row_blocks) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if ((int)blockIdx.x >= row_blocks) return padded_bias(a, bias2, vpad, ((int)blockIdx.x - row_blocks) * 256 + tid);
    __shared__ int n[4];
    __shared__ float top[4];
    const long long r = (long long)blockIdx.x * ROWS_PER_BLOCK + tid;
    const bool on = r < a.N && label_of<T>(a.targets, r, a.V) >= 0;
    float g = BWD && on ? size_of(a.dloss[r]) : 0.f;
    if (BWD) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) g = fmaxf(g, __shfl_xor(g, o, 64));
    }
    const int k = __popcll(__ballot(on));
    if (lane == 0) {
        n[w] = k;
        top[w] = g;
    }
    __syncthreads();
    if (tid == 0) {
        counts[blockIdx.x] = n[0] + n[1] + n[2] + n[3];
        if (BWD) tops[blockIdx.x] = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    }
}

// Gathers the rows with a label (index[k] = row, xc[k] = x[row]) in order, counts them, and finishes the
// rows without one: loss = lse = 0 (forward), dx = 0 (backward).  A workgroup has 256 rows.  SCAN: the labels
// before them, and the last workgroup's largest |g|, are counted here instead of by sm_count_kernel, and the
// last workgroups write the class bias (up to SCAN_ROWS rows: at 6,418 rows the two kernels take 7 us, this
// one 5; at 69,563 20 and 23, and 28 and 85 in the backward).
constexpr int SCAN_ROWS = 8192;
template <class T, bool BWD, bool SCAN>
__global__ __launch_bounds__(1024) void sm_rows_kernel(SoftmaxLossArgs a, int* rows, const int* block_counts,
                                                       const float* block_tops, int* index, uint16_t* xc, int4* info,
                                                       float* bias2, int vpad, int row_blocks, int class_tiles) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    if (SCAN && (int)blockIdx.x >= row_blocks)
        return padded_bias(a, bias2, vpad, ((int)blockIdx.x - row_blocks) * 1024 + tid);
    __shared__ int counts[16], own[4], list[ROWS_PER_BLOCK], off[ROWS_PER_BLOCK];
    __shared__ float tops[16];
    const long long r0 = (long long)blockIdx.x * ROWS_PER_BLOCK;
    const bool last = (int)blockIdx.x == row_blocks - 1;
    float top = 0.f;                                     // the largest |g| of all rows (backward, last workgroup)
    if (BWD && last) {
        if (SCAN) {
#pragma unroll 8
            for (int i = tid; i < (int)a.N; i += 1024) {
                const float g = size_of(a.dloss[i]);
                top = fmaxf(top, label_of<T>(a.targets, i, a.V) >= 0 ? g : 0.f);
            }
        } else {
            for (int i = tid; i < row_blocks; i += 1024) top = fmaxf(top, block_tops[i]);
        }
    }
    int before = 0;
    if (SCAN) {
#pragma unroll 8
        for (int i = tid; i < (int)r0; i += 1024) before += label_of<T>(a.targets, i, a.V) >= 0;
    } else {
        for (int i = tid; i < (int)blockIdx.x; i += 1024) before += block_counts[i];
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) before += __shfl_xor(before, o, 64);
    if (lane == 0) counts[w] = before;
    const long long r = r0 + tid;
    const int t = tid < ROWS_PER_BLOCK && r < a.N ? label_of<T>(a.targets, r, a.V) : -1;
    const unsigned long long on = __ballot(t >= 0);
    if (lane == 0 && w < 4) own[w] = __popcll(on);
    __syncthreads();
    before = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) before += counts[i];
    int at = 0, n = 0;                                   // labelled rows of the waves before, of the workgroup
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if (i < w) at += own[i];
        n += own[i];
    }
    // (one thread, while the others gather)
    if (last && class_tiles > 0 && tid == 1023) {
        int cost;
        rows[2] = tile_run((before + n + CT_ROWS - 1) / CT_ROWS, class_tiles, &cost);
    }
    const int in_block = (int)min((long long)ROWS_PER_BLOCK, a.N - r0);
    if (tid < in_block) {
        const int lower = __popcll(on & ((1ull << lane) - 1ull));
        if (t >= 0) {
            const int k = at + lower;
            list[k] = tid;
            index[before + k] = (int)r;
            if (BWD) {
                // an empty row (no class that counts: lse = -inf) has no gradient
                // lse in units of log 2: what its rounding (an error common to the row's terms) leaves out goes
                // into the factor 2^-low
                const float lse = a.lse[r], g = a.dloss[r], high = lse * LOG2E;
                const bool empty = lse == -__builtin_inff();
                const float low = fmaf(lse, LOG2E_LOW, fmaf(lse, LOG2E, -high));
                info[before + k] = make_int4(__float_as_int(empty ? __builtin_inff() : high), __float_as_int(empty ? 0.f : g),
                                             t, __float_as_int(empty ? 0.f : __builtin_amdgcn_exp2f(-low)));
            }
        } else {
            off[tid - at - lower] = tid;                 // (64 w + lane rows before, at + lower of them labelled)
            if (!BWD) {
                a.loss[r] = 0.f;
                a.lse[r] = 0.f;
            }
        }
    }
    __syncthreads();
    const int ch = a.d / 8;
    for (int i = tid; i < n * ch; i += 1024) {
        const int k = i / ch, c = i % ch;
        *(uint4*)(xc + (long long)(before + k) * a.d + 8 * c) =
            *(const uint4*)((const uint16_t*)a.x + (r0 + list[k]) * a.ld_x + 8 * c);
    }
    if (BWD)
        for (int i = tid; i < (in_block - n) * ch; i += 1024)
            *(uint4*)((uint16_t*)a.dx + (r0 + off[i / ch]) * a.ld_x + 8 * (i % ch)) = make_uint4(0, 0, 0, 0);
    if (last) {
        const int total = before + n;
        if (BWD) {
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
            if (lane == 0) tops[w] = top;
            __syncthreads();
            if (tid == 0) {
#pragma unroll
                for (int i = 1; i < 16; i++) top = fmaxf(top, tops[i]);
                ((float*)rows)[1] = top > 0.f ? top : 1.f;
            }
        }
        if (tid == 0) *rows = total;
        // rows up to the end of the last tile: no gradient
        if (BWD && total + tid < (total + WBM - 1) / WBM * WBM)
            info[total + tid] = make_int4(__float_as_int(__builtin_inff()), 0, -1, 0);
    }
}

__device__ __forceinline__ float2 join(float2 p, float2 q) {
    const float top = fmaxf(p.x, q.x);
    return make_float2(top, p.y * __builtin_amdgcn_exp2f(p.x - top) + q.y * __builtin_amdgcn_exp2f(q.x - top));
}

// Joins a piece's statistics, [parts][N], of 16 rows per workgroup (64 threads a row, so that a large class
// set is not one thread's chain of loads), with those of the pieces before.  After the last piece: loss and
// lse, the label's logit from its own product.
template <class T>
__global__ __launch_bounds__(1024) void sm_join_kernel(SoftmaxLossArgs a, const int* rows, const int* index,
                                                       const uint16_t* xc, const float* bias2, const float2* stats,
                                                       bool regs, bool mid, int nblocks, float2* running, bool first, bool last) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, count = *rows;
    const int parts = regs ? (nblocks + rows[2] - 1) / rows[2] : mid ? 2 * nblocks : 4 * stat_chunks((count + WBM - 1) / WBM, nblocks);
    const int r0 = (int)blockIdx.x * 16;
    if (r0 >= count) return;
    __shared__ float2 part[16][16];
    __shared__ float zt[16];
    const int r = r0 + (tid & 15);
    float2 s = make_float2(-3.402823466e38f, 0.f);
    if (r < count) {
#pragma unroll 4
        for (int p = tid >> 4; p < parts; p += 64) s = join(s, stats[(long long)p * a.N + r]);
    }
#pragma unroll
    for (int o = 16; o <= 32; o <<= 1) s = join(s, make_float2(__shfl_xor(s.x, o, 64), __shfl_xor(s.y, o, 64)));
    if (lane < 16) part[w][lane] = s;
    if (last && r0 + w < count) {
        const long long row = index[r0 + w];
        const int t = label_of<T>(a.targets, row, a.V);
        const uint16_t *x = xc + (long long)(r0 + w) * a.d, *c = (const uint16_t*)a.w + (long long)t * a.ld_w;
        float dot = 0.f;
        for (int i = lane; i < a.d; i += 64) dot = fmaf(bf16_to_f32(x[i]), bf16_to_f32(c[i]), dot);
        dot = wave_sum(dot);
        if (lane == 0) zt[w] = fmaf(dot, a.scale * LOG2E, bias2[t]);
    }
    __syncthreads();
    if (tid < 16 && r < count) {
        s = part[0][tid];
#pragma unroll
        for (int i = 1; i < 16; i++) s = join(s, part[i][tid]);
        if (!first) s = join(s, running[r]);
        if (!last) {
            running[r] = s;
        } else {
            const long long row = index[r];
            const float lse = s.x + __builtin_amdgcn_logf(s.y);
            const bool empty = s.y == 0.f;               // no class counts
            a.lse[row] = empty ? -__builtin_inff() : lse * LN2;
            a.loss[row] = empty ? 0.f : (lse - zt[tid]) * LN2;
        }
    }
}

// What ends a piece: its dW (the K splits' sums, unless finished in place), its bias gradient and, with the last
// piece, dx of the rows with a label; each scaled and rounded once.  Each has workgroups of its own.
struct FinishArgs {
    const int* rows;
    const int* index;
    const float *dw_partial, *col_partial, *dx_partial;
    int dw_splits, dx_splits; // dx_splits 0: those of the wide kernel, of dx_steps k steps
    int dx_steps;
    int v0, nv, ld_col;
    bool mid;                 // col_partial has two parts per 128 rows, not per 256
    int dw_blocks, col_blocks;
};

__global__ __launch_bounds__(256) void sm_finish_kernel(SoftmaxLossArgs a, FinishArgs f) {
    // (scale and the largest |g| one after the other: their product alone may leave the float range)
    const float top = ((const float*)f.rows)[1], scale = a.scale;
    int block = blockIdx.x;
    if (block < f.dw_blocks) {
        const int ch = a.d / 4;
        const long long per = (long long)f.nv * a.d;
        for (long long i = (long long)block * 256 + threadIdx.x; i < (long long)f.nv * ch; i += (long long)f.dw_blocks * 256) {
            const long long r = i / ch;
            const int c = (int)(i % ch) * 4;
            const float* p = f.dw_partial + r * a.d + c;
            floatx4 s = *(const floatx4*)p;
            for (int k = 1; k < f.dw_splits; k++) s += *(const floatx4*)(p + k * per);
            s = s * scale * top;
            *(uint2*)((uint16_t*)a.dw + (f.v0 + r) * a.ld_w + c) = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
        }
        return;
    }
    block -= f.dw_blocks;
    const int count = *f.rows;
    if (block < f.col_blocks) {
        const int c = block * 256 + threadIdx.x;
        if (c >= f.nv) return;
        const int side = f.mid ? MBM : WBM, parts = 2 * ((count + side - 1) / side);
        // (in 64 bits: softmax sums and label counts cancel, and the parts are hundreds)
        double s = 0.;
#pragma unroll 8
        for (int p = 0; p < parts; p++) s += f.col_partial[(long long)p * f.ld_col + c];
        a.dbias[f.v0 + c] = (float)(s * top);
        return;
    }
    block -= f.col_blocks;
    const int blocks = gridDim.x - f.dw_blocks - f.col_blocks, ch = a.d / 8;
    const int splits = f.dx_splits > 0 ? f.dx_splits : acc_splits((count + WBM - 1) / WBM * ((a.d + WBN - 1) / WBN), f.dx_steps);
    const long long per = (long long)count * a.d;
    for (long long i = (long long)block * 256 + threadIdx.x; i < (long long)count * ch; i += (long long)blocks * 256) {
        const long long r = i / ch;
        const int c = (int)(i % ch) * 8;
        const float* p = f.dx_partial + r * a.d + c;
        floatx4 lo = *(const floatx4*)p, hi = *(const floatx4*)(p + 4);
#pragma unroll 4
        for (int k = 1; k < splits; k++) {
            lo += *(const floatx4*)(p + k * per);
            hi += *(const floatx4*)(p + k * per + 4);
        }
        lo = lo * scale * top;
        hi = hi * scale * top;
        *(uint4*)((uint16_t*)a.dx + f.index[r] * a.ld_x + c) =
            make_uint4(pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3]));
    }
}

// Class tiles of the first piece on the tiles of softmax_tiles.h.
int register_tiles(const SmPlan& p, int V) { return std::min(p.piece / CT_CLASSES, (V + CT_CLASSES - 1) / CT_CLASSES); }

template <bool BWD>
hipError_t launch_rows(const SoftmaxLossArgs& a, const SmPlan& p, char* ws, hipStream_t s) {
    const int rb = (int)((a.N + ROWS_PER_BLOCK - 1) / ROWS_PER_BLOCK);
    int* counts = (int*)(ws + p.counts);
    float* tops = (float*)(ws + p.tops);
    int *rows = (int*)(ws + p.rows), *index = (int*)(ws + p.index);
    uint16_t* xc = (uint16_t*)(ws + p.xc);
    float* bias2 = (float*)(ws + p.bias);
    int4* info = (int4*)(ws + p.info);
    const int class_tiles = p.regs ? register_tiles(p, a.V) : 0;
    auto launch = [&](auto type) {
        typedef decltype(type) T;
        if (a.N <= SCAN_ROWS) {
            sm_rows_kernel<T, BWD, true><<<rb + (p.vpad + 1023) / 1024, 1024, 0, s>>>(a, rows, counts, tops, index, xc, info,
                                                                                   bias2, p.vpad, rb, class_tiles);
            return hipGetLastError();
        }
        sm_count_kernel<T, BWD><<<rb + p.vpad / 256, 256, 0, s>>>(a, counts, tops, bias2, p.vpad, rb);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        sm_rows_kernel<T, BWD, false><<<rb, 1024, 0, s>>>(a, rows, counts, tops, index, xc, info, bias2, p.vpad, rb,
                                                                class_tiles);
        return hipGetLastError();
    };
    return a.targets64 ? launch(int64_t{}) : launch(int{});
}

// x W^T of the piece at class v0.
TileArgs logits_product(const SoftmaxLossArgs& a, const SmPlan& p, char* ws, int v0) {
    TileArgs g{};
    g.layout = GEMM_NT;
    g.M = a.N;
    g.N = std::min(p.piece, p.vpad - v0);
    g.K = a.d;
    g.A = ws + p.xc;
    g.lda = a.d;
    g.B = (const uint16_t*)a.w + v0 * a.ld_w;
    g.ldb = a.ld_w;
    g.bias = (const float*)(ws + p.bias) + v0;
    g.scale = a.scale * LOG2E;
    g.rows = (const int*)(ws + p.rows);
    g.b_rows = std::min(p.piece, a.V - v0);
    g.class0 = v0;
    g.group_m = GROUP_M;
    const int side = p.logits.mid ? MBM : WBM, cols = p.regs ? CT_CLASSES : side;
    g.mblocks = (int)((a.N + side - 1) / side);
    g.nblocks = (g.b_rows + cols - 1) / cols;
    g.splits = 1;
    g.ks_per_split = (a.d + WBK - 1) / WBK;
    return g;
}

}  // namespace

size_t softmax_loss_workspace_bytes(long long N, int V, int d, bool backward) {
    return N > 0 && V > 0 ? sm_plan(N, V, d, backward).total : 0;
}

// run: class tiles that an item (256 rows, or a tile's) goes through, of the first piece.
int softmax_loss_kernels(long long N, int V, int d, bool backward, long long labels, char* text, size_t n) {
    const SmPlan p = sm_plan(N, V, d, backward);
    const int mblocks = (int)((labels + WBM - 1) / WBM), nblocks = (std::min(p.piece, V) + WBN - 1) / WBN;
    int cost, run = 1;
    if (p.regs) run = tile_run(mblocks, register_tiles(p, V), &cost);
    else if (!p.logits.mid && !backward) run = (nblocks + stat_chunks(mblocks, nblocks) - 1) / stat_chunks(mblocks, nblocks);
    const char* logits = p.regs ? "registers" : p.logits.mid ? "128x128" : "256x256";
    if (!backward) return snprintf(text, n, "logits=%s run=%d pieces=%d piece=%d", logits, run, p.pieces, p.piece);
    Tiles dx = p.dx;
    if (!dx.mid) dx.splits = acc_splits(mblocks * ((d + WBN - 1) / WBN), p.piece / WBK);
    return snprintf(text, n, "logits=%s run=%d pieces=%d piece=%d dz=%s dx=%s dw=%s%s", logits, run, p.pieces, p.piece,
                    (!p.regs && p.logits.mid) || dz_stays(labels, p.piece) ? "cached" : "streamed", tiles_name(dx).text,
                    tiles_name(p.dw).text, p.direct ? "/direct" : "");
}

hipError_t launch_softmax_loss_fwd(const SoftmaxLossArgs& a, void* workspace, hipStream_t s) {
    const SmPlan p = sm_plan(a.N, a.V, a.d, false);
    char* ws = (char*)workspace;
    hipError_t e = launch_rows<false>(a, p, ws, s);
    for (int i = 0; i < p.pieces && e == hipSuccess; i++) {
        TileArgs g = logits_product(a, p, ws, i * p.piece);
        g.stats = (float2*)(ws + p.stats);
        e = p.regs ? sm_tile_launch<false>(g, s)
            : p.logits.mid ? mid_launch<GEMM_NT, GEMM_EPI_SM_STATS>(g, s) : wide_launch<GEMM_NT, GEMM_EPI_SM_STATS, false>(g, s);
        if (e != hipSuccess) break;
        const int blocks = (int)((a.N + 15) / 16);
        const bool first = i == 0, last = i == p.pieces - 1;
        const int *rows = (const int*)(ws + p.rows), *index = (const int*)(ws + p.index);
        const uint16_t* xc = (const uint16_t*)(ws + p.xc);
        const float* bias2 = (const float*)(ws + p.bias);
        float2* running = (float2*)(ws + p.running);
        if (a.targets64) sm_join_kernel<int64_t><<<blocks, 1024, 0, s>>>(a, rows, index, xc, bias2, g.stats, p.regs, p.logits.mid, g.nblocks, running, first, last);
        else sm_join_kernel<int><<<blocks, 1024, 0, s>>>(a, rows, index, xc, bias2, g.stats, p.regs, p.logits.mid, g.nblocks, running, first, last);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_softmax_loss_bwd(const SoftmaxLossArgs& a, void* workspace, hipStream_t s) {
    if (a.N == 0) {
        const hipError_t z = launch_zero_rows(a.V, a.d / 8, a.dw, a.ld_w / 8, s);
        return z != hipSuccess || !a.dbias ? z : launch_fill_f32(a.dbias, a.V, 0.f, s);
    }
    const SmPlan p = sm_plan(a.N, a.V, a.d, true);
    char* ws = (char*)workspace;
    const int* rows = (const int*)(ws + p.rows);
    hipError_t e = launch_rows<true>(a, p, ws, s);
    for (int i = 0; i < p.pieces && e == hipSuccess; i++) {
        const int v0 = i * p.piece;
        TileArgs g = logits_product(a, p, ws, v0);
        const int nv = g.b_rows;
        g.C = ws + p.dz;
        g.ldc = p.piece;
        g.row_info = (const int4*)(ws + p.info);
        g.col_partial = a.dbias ? (float*)(ws + p.colp) : nullptr;
        e = p.regs ? sm_tile_launch<true>(g, s)
            : p.logits.mid ? mid_launch<GEMM_NT, GEMM_EPI_SM_GRAD>(g, s) : wide_launch<GEMM_NT, GEMM_EPI_SM_GRAD, false>(g, s);
        if (e != hipSuccess) break;

        TileArgs x{};                                    // dx += dz W
        x.layout = GEMM_NN;
        x.M = a.N;
        x.N = a.d;
        x.K = (nv + WBK - 1) / WBK * WBK;                // (dz is zero behind the last class)
        x.A = ws + p.dz;
        x.lda = p.piece;
        x.B = g.B;
        x.ldb = a.ld_w;
        x.rows = rows;
        x.b_rows = nv;
        x.accumulate = i > 0;
        x.partial = (float*)(ws + p.dxp);
        TileArgs w{};                                    // the piece's dW = dz^T x
        w.layout = GEMM_TN;
        w.M = nv;
        w.N = a.d;
        w.K = a.N;
        w.A = ws + p.dz;
        w.lda = p.piece;
        w.B = ws + p.xc;
        w.ldb = a.d;
        w.rows = rows;
        w.partial = (float*)(ws + p.dwp);
        w.splits = p.dw.splits;
        w.scale = a.scale;
        w.C = (uint16_t*)a.dw + v0 * a.ld_w;
        w.ldc = a.ld_w;
        const int side = p.dw.mid ? MBM : WBM;
        w.mblocks = (nv + side - 1) / side;
        w.nblocks = (a.d + side - 1) / side;
        // (without a split the 256 x 256 tiles finish dW in place)
        const bool last = i == p.pieces - 1;
        if (p.dx.mid) {
            x.mblocks = (int)((a.N + MBM - 1) / MBM);
            x.nblocks = (a.d + MBN - 1) / MBN;
            x.splits = p.dx.splits;
        } else {
            x.mblocks = (int)((a.N + WBM - 1) / WBM);
            x.nblocks = (a.d + WBN - 1) / WBN;
            x.splits = 1;                                // (chosen on the device, from the rows with a label)
        }
        if (p.dx.mid && p.dw.mid) {
            gemm_mid_pair_kernel<GEMM_NN, GEMM_EPI_ACC, GEMM_TN, GEMM_EPI_ROWS><<<mid_grid(x) + mid_grid(w), 256, 0, s>>>(x, w, mid_grid(x));
            e = hipGetLastError();
        } else {
            if (p.dx.mid) {
                e = mid_launch<GEMM_NN, GEMM_EPI_ACC>(x, s);
            } else {
                x.ks_per_split = p.piece / WBK;
                gemm_wide_kernel<GEMM_NN, GEMM_EPI_ACC, false><<<XCDS * ((p.items + XCDS - 1) / XCDS), 512, 0, s>>>(x);
                e = hipGetLastError();
            }
            if (e != hipSuccess) break;
            e = p.dw.mid ? mid_launch<GEMM_TN, GEMM_EPI_ROWS>(w, s)
                : p.direct ? wide_launch<GEMM_TN, GEMM_EPI_ROWS_DIRECT, false>(w, s) : wide_launch<GEMM_TN, GEMM_EPI_ROWS, false>(w, s);
        }
        if (e != hipSuccess) break;
        FinishArgs f{};
        f.rows = rows;
        f.index = (const int*)(ws + p.index);
        f.dw_partial = w.partial;
        f.col_partial = g.col_partial;
        f.dx_partial = x.partial;
        f.dw_splits = w.splits;
        f.dx_splits = p.dx.mid ? p.dx.splits : 0;
        f.dx_steps = p.piece / WBK;
        f.v0 = v0;
        f.nv = nv;
        f.ld_col = (int)g.N;
        f.mid = p.regs || p.logits.mid;
        f.dw_blocks = p.direct ? 0 : (int)std::min(((long long)nv * a.d / 4 + 255) / 256, 8192ll);
        f.col_blocks = a.dbias ? (nv + 255) / 256 : 0;
        const int dx_blocks = last ? (int)std::min((a.N * (a.d / 8) + 255) / 256, 8192ll) : 0;
        if (f.dw_blocks + f.col_blocks + dx_blocks == 0) continue;
        sm_finish_kernel<<<f.dw_blocks + f.col_blocks + dx_blocks, 256, 0, s>>>(a, f);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace mtgr
