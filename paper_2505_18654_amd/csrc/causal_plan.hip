// The dK / dV kernel's work: items of at most about a thousandth of all units, costliest first.
//
// A tile of keys is read by all queries from it to its sequence's end, of every query head that shares its key head, so the
// first tiles of a long sequence are most of the work of a few workgroups.  Cut into items of at most U = max(64, all units
// / 1024) units, and started costliest first (a counting sort), the workgroups end together: 64 sequences with 68,000 tokens,
// 8 query heads on 2 of 128: PLAN_FIGURES.
#include "causal_device.h"

namespace mtgr {
namespace {

using namespace causal;
constexpr int CLASSES = 1024, MOST_ITEMS = 1024, LEAST_UNITS = 64;

__global__ __launch_bounds__(1024) void causal_plan_kernel(CausalArgs a, CausalPlan p, CausalItem* items, CausalItem* joins) {
    __shared__ int sCount[CLASSES], sFirst[CLASSES], sWave[16], sJoins, sParts;
    __shared__ long long sUnits[16];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    sCount[tid] = 0;
    if (tid == 0) sJoins = sParts = 0;
    struct Work {
        Tile t;
        int units, n, size;   // its units, items and their size
    };
    auto tile = [&](int slot) {
        int lo = 0, hi = a.B;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((a.offsets[mid] >> 7) + mid <= slot) lo = mid;
            else hi = mid;
        }
        return tile_at(a.offsets, a.T, lo, slot);
    };
    auto units_of = [&](const Tile& t) { return t.tile < 0 ? 0 : (t.n - t.tile * BM + 31) / 32 * a.group; };
    long long units = 0;
    for (int slot = tid; slot < a.slots; slot += 1024) units += units_of(tile(slot));
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) units += __shfl_xor(units, off, 64);
    if (lane == 0) sUnits[w] = units;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) all += sUnits[i];
    const int U = (int)max((all * a.Hk + MOST_ITEMS - 1) / MOST_ITEMS, (long long)LEAST_UNITS);
    auto work = [&](int slot) {
        Work x;
        x.t = tile(slot);
        x.units = units_of(x.t);
        x.n = (x.units + U - 1) / U;
        x.size = x.n > 0 ? (x.units + x.n - 1) / x.n : 0;
        return x;
    };
    auto class_of = [&](const Work& x) { return CLASSES - 1 - (int)((long long)(x.size - 1) * CLASSES / U); };
    for (int slot = tid; slot < a.slots; slot += 1024) {
        const Work x = work(slot);
        if (x.n > 0) atomicAdd(&sCount[class_of(x)], x.n);
    }
    __syncthreads();
    // first positions: sums over a wave, then over the waves before it
    const int own = sCount[tid];
    int sum = own;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int v = __shfl_up(sum, off, 64);
        if (lane >= off) sum += v;
    }
    if (lane == 63) sWave[w] = sum;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        if (i < w) before += sWave[i];
        total += sWave[i];
    }
    sFirst[tid] = before + sum - own;
    __syncthreads();
    for (int slot = tid; slot < a.slots; slot += 1024) {
        const Work x = work(slot);
        if (x.n == 0) continue;
        const int at = atomicAdd(&sFirst[class_of(x)], x.n), part = x.n > 1 ? atomicAdd(&sParts, x.n) : -1;
        CausalItem item;
        item.o = x.t.o;
        item.n = x.t.n;
        item.tile = x.t.tile;
        item.parts = x.n;
        item.pad = 0;
        for (int i = 0; i < x.n; i++) {
            item.first = i * x.size;
            item.last = min(x.units, item.first + x.size);
            item.part = part < 0 ? -1 : part + i;
            if (at + i < p.items) items[at + i] = item;          // (always, by the bounds of causal_plan)
        }
        if (x.n > 1) {
            item.part = part;
            const int j = atomicAdd(&sJoins, 1);
            if (j < p.joins) joins[j] = item;
        }
    }
    __syncthreads();
    CausalItem none{};
    none.tile = -1;
    for (int i = total + tid; i < p.items; i += 1024) items[i] = none;
    for (int i = sJoins + tid; i < p.joins; i += 1024) joins[i] = none;
}

}  // namespace

// With u units of a key head in all and U = max(64, u Hk / 1024): tiles of more than U units are at most u / U, their items at
// most 2 u / U, all items at most slots + u / U.  A sequence of n tokens has at most (n / 32 + 1) (n / 128 + 1) units per
// query head.
CausalPlan causal_plan(long long T, int B, int H, int Hk, int head_dim) {
    const long long slots = T / BM + B, G = H / Hk, most = (T / 64 + 1) * (T * G / 64 + 1) + (T * 5 / 128 + 1 + B) * G;
    const long long cuts = std::min<long long>(MOST_ITEMS / Hk, most / LEAST_UNITS) + 1;
    CausalPlan p{};
    p.items = (int)(slots + cuts);
    p.joins = (int)std::min<long long>(slots, cuts);
    p.parts = (int)(2 * cuts);
    auto round = [](size_t n) { return (n + 255) & ~(size_t)255; };
    p.joins_ofs = round((size_t)p.items * sizeof(CausalItem));
    p.parts_ofs = p.joins_ofs + round((size_t)p.joins * sizeof(CausalItem));
    p.bytes = p.parts_ofs + round((size_t)p.parts * Hk * 2 * BM * head_dim * 4);
    return p;
}

hipError_t launch_causal_plan(const CausalArgs& a, const CausalPlan& p, CausalItem* items, CausalItem* joins, hipStream_t s) {
    causal_plan_kernel<<<1, 1024, 0, s>>>(a, p, items, joins);
    return hipGetLastError();
}

}  // namespace mtgr
