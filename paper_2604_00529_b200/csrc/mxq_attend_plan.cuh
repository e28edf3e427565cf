// Which tiles a CTA of the attention kernels works on, from the lengths that the device holds.
#pragma once
#include "mxq_attend_items.cuh"

namespace mxq {
namespace {

// The run of a CTA: its first and one past its last tile, the sequence that the first lies in and the tiles in front of that.
struct Plan {
    uint32_t total, from, to, base, per_head;
    int b;
    Sequence s;
};

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
        plan = Plan{total, from, to, before, per_head, b, s};
    }
    __syncthreads();
}

}  // namespace
}  // namespace mxq
