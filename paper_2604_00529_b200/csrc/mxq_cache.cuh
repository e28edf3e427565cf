// What the kernels over a paged cache of keys and values share: the cache's and a batch's description as kernels take them,
// and the way from a token's row to its sequence, its position and its page.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "../../include/mxq.h"
#include "mxq_access.cuh"

namespace mxq {

constexpr int kCachePageMin = 16, kCachePageMax = 256;      // 16: the keys of one matrix step lie in one page

// A page holds `page` tokens of every head: codes [pages, heads, page, row], scales [pages, heads, page, srow], row and srow in bytes.
struct CacheArgs {
    const uint8_t *kc, *ks, *vc, *vs;
    int pages, page_shift, heads, block_shift;
};

// Sequence b: tokens table[b * width ...], lengths[b] of them, the last starts[b + 1] - starts[b] (1 without starts) new.
struct BatchArgs {
    const int *table, *lengths, *starts;
    int batch, width, tokens;                               // tokens: rows of the new tokens' tensors
};

__device__ __forceinline__ int ld_int(const int* p)
{
    MXQ_CHECKED(p, 4, return 0)
    return *p;
}

// What the device says of a sequence, kept inside what the host said: rows first ... first + n - 1 of `tokens`, 0 <= length <= width pages.
struct Sequence {
    int first, n, length;
};

__device__ __forceinline__ Sequence sequence(const BatchArgs& p, int b, int page_shift)
{
    Sequence s;
    if (p.starts) {
        s.first = min(max(ld_int(p.starts + b), 0), p.tokens);
        s.n = max(min(ld_int(p.starts + b + 1), p.tokens) - s.first, 0);
    } else {
        s.first = b;
        s.n = 1;
    }
    const long long most = (long long)p.width << page_shift;
    s.length = (int)min((long long)max(ld_int(p.lengths + b), 0), min(most, (long long)0x7FFFFFFF));
    return s;
}

// The last b with starts[b] <= row, among 0 ... batch - 1 (starts[0] <= row).
__device__ __forceinline__ int find_sequence(const int* starts, int batch, int row)
{
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (ld_int(starts + mid) <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Row number of a token's head in the cache (codes and scales alike), or -1 if the table gives no page for it.
__device__ __forceinline__ long long cache_row(const CacheArgs& c, const BatchArgs& p, int b, int pos, int head)
{
    const int page = ld_int(p.table + (size_t)b * p.width + (pos >> c.page_shift));
    if ((unsigned)page >= (unsigned)c.pages) return -1;
    return ((((long long)page * c.heads + head) << c.page_shift) | (pos & ((1 << c.page_shift) - 1)));
}

// What the kernels of mxq_cache_attention take.
struct AttendArgs {
    CacheArgs cache;
    BatchArgs batch;
    const uint8_t* q;
    size_t q_token, q_head;                                 // in bytes
    uint8_t* out;
    float* lse;
    uint8_t* ws;
    int group, rows;                                        // rows of a cache head per token; rows of an item
    int causal, window;
    float scale;                                            // times log2 e
    int ctas, warps, tile_shift;                            // of the first kernel; keys of a tile: what is shared out among CTAs
    int share;                                              // CTAs of a cluster, which has one item; 0: all tiles in runs
};

template <int FMT>
int launch_attend(int dim, int nt, int dtype, const AttendArgs& p, cudaStream_t stream);
int launch_attend_many(int fmt, int dim, const AttendArgs& p, cudaStream_t stream);      // BF16, dim 64 or 128, 256 rows to an item
int many_status(int reset);                                  // as tc_status, of that kernel's waits

// Checks of a cache's and a batch's description, and of their addresses, as the entry points make them (an mxq_status).
int check_cache(const mxq_cache* c);
int check_batch(const mxq_batch* b, size_t tokens);
int check_places(const mxq_cache* c, const mxq_batch* b, bool lengths);
CacheArgs cache_args(const mxq_cache* c);
BatchArgs batch_args(const mxq_batch* b, size_t tokens);
void debug_expect_cache(const mxq_cache* c, const mxq_batch* b);

}  // namespace mxq
