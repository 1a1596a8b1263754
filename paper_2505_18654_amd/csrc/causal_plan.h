// The dK / dV kernel's work: items of at most about a thousandth of all units, costliest first.
//
// A tile of keys is read by all queries from it to its sequence's end, of every query head that shares its key head, so the
// first tiles of a long sequence are most of the work of a few workgroups.  Cut into items of at most U units and started
// costliest first (a counting sort), the workgroups end together: 64 sequences with 68,000 tokens, 8 query heads on 2 of 128, in
// the batch's order 997 us, costliest first 745, cut as well 538 and 31 for the joins.  U is a 1,024th of all units; of little
// work a 256th, an item for each CU, of at most 16 units (smaller ones cost more in the joins than they end sooner) and at least
// 8: the whole backward of 700 tokens, 6 / 2 heads of 128, 33 us, with at least 16 37.5, 4 35, 2 41.5; of 1,000, 8 / 1 heads,
// 42, 45, 49, 49; of two of 2,000 and less, 8 / 2 heads, 70, with 512 items of at most 16 units 83.  One workgroup of the dQ
// kernel, which runs before, makes the plan.  Which of two items of equal size comes first may differ from run to run; results
// do not depend on it.
#pragma once

#include "causal_device.h"

namespace mtgr {
namespace causal {

constexpr int PLAN_CLASSES = 1024, MOST_ITEMS = 1024, LEAST_UNITS = 8, FEW_ITEMS = 256, PLAN_STARTS = 2048;
constexpr long long FEW_UNITS = 16;

// The workgroup's THREADS threads; lds: PLAN_LDS ints, 8-byte aligned.
constexpr int PLAN_LDS = PLAN_CLASSES + PLAN_STARTS + 32;
template <int THREADS>
__device__ __forceinline__ void make_plan(const CausalArgs& a, const CausalPlan& p, int* lds) {
    int* count = lds;                                            // of a class, then its next position
    int* start = lds + PLAN_CLASSES;                             // first slots of every step-th sequence
    constexpr int WAVES = THREADS / 64, OWN = PLAN_CLASSES / THREADS;
    int* wave_sum = start + PLAN_STARTS;                         // 8
    int* joined = wave_sum + 8;
    int* parted = wave_sum + 9;
    unsigned long long* sum64 = (unsigned long long*)(wave_sum + 16);        // 8
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int step = (a.B + PLAN_STARTS - 1) / PLAN_STARTS, starts = (a.B + step - 1) / step;
    for (int i = tid; i < starts; i += THREADS) start[i] = a.offsets[i * step] / BM + i * step;
    for (int i = tid; i < PLAN_CLASSES; i += THREADS) count[i] = 0;
    if (tid == 0) *joined = *parted = 0;
    __syncthreads();
    struct Work {
        Tile t;
        int units, n, size;                                      // its units, items and their size
    };
    auto tile = [&](int slot) {
        int lo = 0, hi = starts;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (start[mid] <= slot) lo = mid;
            else hi = mid;
        }
        lo *= step;
        hi = min(lo + step, a.B);
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.offsets[mid] / BM + mid <= slot) lo = mid;
            else hi = mid;
        }
        return tile_at(a.offsets[lo], a.offsets[lo + 1], a.T, lo, slot);
    };
    auto units_of = [&](const Tile& t) { return t.tile < 0 ? 0 : (t.n - t.tile * BM + 31) / 32 * a.group; };
    unsigned long long units = 0;
    for (int slot = tid; slot < a.slots; slot += THREADS) units += units_of(tile(slot));
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) units += __shfl_xor(units, off, 64);
    if (lane == 0) sum64[w] = units;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; i++) all += (long long)sum64[i];
    all *= a.Hk;
    const int U = (int)max(max((all + MOST_ITEMS - 1) / MOST_ITEMS, min(all / FEW_ITEMS, FEW_UNITS)), (long long)LEAST_UNITS);
    auto work = [&](int slot) {
        Work x;
        x.t = tile(slot);
        x.units = units_of(x.t);
        x.n = (x.units + U - 1) / U;
        x.size = x.n > 0 ? (x.units + x.n - 1) / x.n : 0;
        return x;
    };
    auto class_of = [&](const Work& x) { return PLAN_CLASSES - 1 - (int)((long long)(x.size - 1) * PLAN_CLASSES / U); };
    for (int slot = tid; slot < a.slots; slot += THREADS) {
        const Work x = work(slot);
        if (x.n > 0) atomicAdd(&count[class_of(x)], x.n);
    }
    __syncthreads();
    // first positions: a thread's classes, sums over a wave, then over the waves before it
    int own[OWN], sum = 0;
#pragma unroll
    for (int i = 0; i < OWN; i++) sum += own[i] = count[OWN * tid + i];
    const int mine = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int v = __shfl_up(sum, off, 64);
        if (lane >= off) sum += v;
    }
    if (lane == 63) wave_sum[w] = sum;
    __syncthreads();
    int at = sum - mine, total = 0;
#pragma unroll
    for (int i = 0; i < WAVES; i++) {
        if (i < w) at += wave_sum[i];
        total += wave_sum[i];
    }
#pragma unroll
    for (int i = 0; i < OWN; i++) {
        count[OWN * tid + i] = at;
        at += own[i];
    }
    __syncthreads();
    for (int slot = tid; slot < a.slots; slot += THREADS) {
        const Work x = work(slot);
        if (x.n == 0) continue;
        const int first = atomicAdd(&count[class_of(x)], x.n), part = x.n > 1 ? atomicAdd(parted, x.n) : -1;
        CausalItem item;
        item.o = x.t.o;
        item.n = x.t.n;
        item.tile = part + x.n <= p.parts ? x.t.tile : -1;       // (within p.parts, as below, for offsets that ascend)
        item.parts = x.n;
        item.pad = 0;
        for (int i = 0; i < x.n; i++) {
            item.first = i * x.size;
            item.last = min(x.units, item.first + x.size);
            item.part = part < 0 ? -1 : part + i;
            if (first + i < p.items) a.items[first + i] = item;  // (always, by the bounds of causal_plan)
        }
        if (x.n > 1) {
            item.part = part;
            const int j = atomicAdd(joined, 1);
            if (j < p.joins) a.joins[j] = item;
        }
    }
    __syncthreads();
    CausalItem none{};
    none.tile = -1;
    for (int i = total + tid; i < p.items; i += THREADS) a.items[i] = none;
    if (tid == 0) {
        none.parts = *joined;
        a.joins[p.joins] = none;                                 // how many there are
    }
}

}  // namespace causal

// With u units of a key head in all and U >= max(8, u Hk / 1024): tiles of more than U units are at most u / U, their items at
// most 2 u / U, all items at most slots + u / U.  A sequence of n tokens has at most (n / 32 + 1) (n / 128 + 1) units per
// query head.
inline CausalPlan make_causal_plan(long long T, int B, int H, int Hk, int head_dim) {
    const long long slots = T / causal::BM + B, G = H / Hk, most = (T / 64 + 1) * (T * G / 64 + 1) + (T * 5 / 128 + 1 + B) * G;
    const long long cuts = std::min<long long>(causal::MOST_ITEMS / Hk, most / causal::LEAST_UNITS) + 1;
    CausalPlan p{};
    p.items = (int)(slots + cuts);
    p.joins = (int)std::min<long long>(slots, cuts);
    p.parts = (int)(2 * cuts);
    auto round = [](size_t n) { return (n + 255) & ~(size_t)255; };
    p.joins_ofs = round((size_t)p.items * sizeof(CausalItem));
    p.parts_ofs = p.joins_ofs + round((size_t)(p.joins + 1) * sizeof(CausalItem));
    p.bytes = p.parts_ofs + round((size_t)p.parts * Hk * 2 * causal::BM * head_dim * 4);
    return p;
}

}  // namespace mtgr
