// Which tiles a CTA of the attention kernels works on, from the lengths that the device holds.
#pragma once
#include "mxq_attend_items.cuh"

namespace mxq {
namespace {

// The run of a CTA: the next tile and one past its last, the sequence that the next one lies in, that sequence's first tile and tiles per
// head; and the item: its first tile and tiles, its head and first row.
struct Plan {
    uint32_t total, from, to, base, per_head;
    int b;
    Sequence s;
    uint32_t item, tiles;
    int head, r0;
};

// The item of tile `from`, in its sequence.
__device__ __forceinline__ void find_item(const AttendArgs& p, Plan& plan)
{
    plan.head = (int)((plan.from - plan.base) / plan.per_head);
    plan.item = plan.base + plan.per_head * (uint32_t)plan.head;
    plan.tiles = plan.per_head;
    plan.r0 = 0;
    if (plan.s.n * p.group <= p.rows) return;
    ItemWalk w(p);
    uint32_t item = plan.item, tiles = w.tiles(p, plan.s);
    while (plan.from - item >= tiles) {
        item += tiles;
        w.next(p);
        tiles = w.tiles(p, plan.s);
    }
    plan.item = item;
    plan.tiles = tiles;
    plan.r0 = w.r0;
}

// On to the item behind the one that the plan is at, where the run has one.  One thread's; the items of a run are followed, not searched for
// again, since a sequence may have thousands of them.  (Searched for each time, 32768 FP32 queries of 16 heads over one with a window of 64
// took 803 ms, and take 3.8.)
__device__ __noinline__ void next_item(const AttendArgs& p, Plan& plan)
{
    plan.from = min(plan.item + plan.tiles, plan.to);
    if (plan.from == plan.to) return;
    if (plan.from - plan.base < plan.per_head * p.cache.heads) {
        plan.item += plan.tiles;
        plan.r0 += p.rows;
        if (plan.r0 >= plan.s.n * p.group) {
            plan.r0 = 0;
            ++plan.head;
        }
        if (plan.s.n * p.group > p.rows) plan.tiles = item_tiles(p, plan.s, plan.r0);
        return;
    }
    do {
        if (plan.b + 1 >= p.batch.batch) {                   // (only where sums of tiles passed 32 bits: rows that several sequences claim)
            plan.from = plan.to;
            return;
        }
        plan.base += plan.per_head * p.cache.heads;
        ++plan.b;
        plan.s = sequence(p.batch, plan.b, p.cache.page_shift);
        plan.per_head = sequence_tiles(p, plan.s);
    } while (plan.from - plan.base >= plan.per_head * p.cache.heads);
    find_item(p, plan);
}

__device__ __forceinline__ void make_plan(const AttendArgs& p, int warps, Plan& plan, uint32_t (&warp_sum)[32])
{
    const int threads = warps * 32, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // a sequence per thread, or a few in a row
    const int per = p.batch.batch <= threads ? 1 : (p.batch.batch + threads - 1) / threads;
    const int first = min((int)threadIdx.x * per, p.batch.batch), last = min(first + per, p.batch.batch);
    Sequence s = {0, 0, 0};
    uint32_t mine = 0, per_head = 0;
    for (int b = first; b < last; ++b) {
        s = sequence(p.batch, b, p.cache.page_shift);
        per_head = sequence_tiles(p, s);
        mine += per_head * p.cache.heads;
    }
    uint32_t before = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, before, o);
        if (lane >= o) before += up;
    }
    if (lane == 31) warp_sum[warp] = before;
    if (threadIdx.x == 0) plan.total = plan.from = plan.to = 0;        // (a run that lies in no sequence, likewise)
    __syncthreads();
    uint32_t sum = lane < warps ? warp_sum[lane] : 0u;
    const uint32_t total = __reduce_add_sync(0xFFFFFFFFu, sum);
    if (lane >= warp) sum = 0;
    before += __reduce_add_sync(0xFFFFFFFFu, sum) - mine;
    const uint32_t ctas = working_ctas(total, gridDim.x);
    const Runs runs(total, ctas);
    const uint32_t from = blockIdx.x < ctas ? runs.start(blockIdx.x) : total, to = blockIdx.x < ctas ? runs.start(blockIdx.x + 1) : total;
    if (from < to ? from >= before && from < before + mine : threadIdx.x == 0) {            // one thread's
        int b = first;
        if (per > 1) {
            for (; from < to && b < last; ++b) {
                s = sequence(p.batch, b, p.cache.page_shift);
                per_head = sequence_tiles(p, s);
                if (from < before + per_head * p.cache.heads) break;
                before += per_head * p.cache.heads;
            }
        }
        plan = Plan{total, from, to, before, per_head, b, s, 0, 0, 0, 0};
        if (from < to) find_item(p, plan);
    }
    __syncthreads();
}

}  // namespace
}  // namespace mxq
