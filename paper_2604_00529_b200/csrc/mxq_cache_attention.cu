// mxq_cache_attention: checks, the choice of a kernel's width, and the kernel that adds up what the first one did in parts.
#include "mxq_attend_items.cuh"
#include "mxq_launch.h"

namespace mxq {
namespace {

// Items that the first kernel worked on in several parts: CTA c (and a row of its grid's second dimension) takes the item that run c begins
// inside, if no earlier run begins inside it too.
template <int PIECES>
__global__ void __launch_bounds__(256)
join_kernel(const __grid_constant__ AttendArgs p, int dim)
{
    pdl_release();
    pdl_acquire();
    __shared__ float sums[256 * 4];
    __shared__ float weight[256];
    const PartMeta* metas = reinterpret_cast<const PartMeta*>(p.ws);
    const PartMeta meta0 = metas[0];
    const int ctas = (int)min((long long)p.ctas, max(meta0.total, 1ll)), c = blockIdx.x + 1, r = blockIdx.y;
    if (c >= ctas) return;
    const PartMeta meta = metas[c];
    if (meta.from <= meta.item_from || r >= meta.rows) return;
    if (run_start(meta.total, ctas, c - 1) > meta.item_from) return;
    int last = c;                                            // the runs c - 1 ... last have parts of it
    {
        long long lo = c, hi = ctas;                         // the last run that begins in front of the item's end
        while (hi - lo > 1) {
            const long long mid = (lo + hi) >> 1;
            if (run_start(meta.total, ctas, (int)mid) < meta.item_to) lo = mid;
            else hi = mid;
        }
        last = (int)lo;
    }
    const uint8_t* const parts = p.ws + (size_t)p.ctas * sizeof(PartMeta);
    const size_t part = part_bytes(p.rows, dim);
    const bool own = run_start(meta.total, ctas, c - 1) == meta.item_from;      // the item is the first of run c - 1
    const int n = last - c + 2;
    auto at = [&](int i) { return reinterpret_cast<const float*>(parts + ((size_t)(c - 1 + i) * 2 + (i == 0 && !own ? 1 : 0)) * part); };
    // the largest maximum, then every part's weight
    float top = kNone;
    for (int i = threadIdx.x; i < n; i += 256) top = fmaxf(top, at(i)[p.rows * dim + 2 * r]);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if ((threadIdx.x & 31) == 0) weight[threadIdx.x >> 5] = top;
    __syncthreads();
    top = weight[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) top = fmaxf(top, weight[w]);
    __syncthreads();
    const int quads = dim / 4, lanes = 256 / quads;          // parts in turn among `lanes` threads of the same elements
    const int d = threadIdx.x % quads * 4, mine = threadIdx.x / quads;
    float v[4] = {}, sum = 0.f;
    for (int i0 = 0; i0 < n; i0 += 256) {
        if (i0 + (int)threadIdx.x < n) {
            const float* x = at(i0 + threadIdx.x) + p.rows * dim + 2 * r;
            weight[threadIdx.x] = x[1] * exp2_approx(x[0] - top);
        }
        __syncthreads();
        const int some = min(256, n - i0);
#pragma unroll 4
        for (int i = mine; i < some; i += lanes) {
            const float4 x = *reinterpret_cast<const float4*>(at(i0 + i) + r * dim + d);
            const float w = weight[i];
            sum += w;
            v[0] += w * x.x;
            v[1] += w * x.y;
            v[2] += w * x.z;
            v[3] += w * x.w;
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[threadIdx.x * 4 + j] = v[j];
    weight[threadIdx.x] = sum;
    __syncthreads();
    if (mine != 0) return;
    for (int k = 1; k < lanes; ++k) {
        sum += weight[threadIdx.x + k * quads];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += sums[(threadIdx.x + k * quads) * 4 + j];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= inv;
    const Sequence s = sequence(p.batch, meta.b, p.cache.page_shift);
    const int row = meta.r0 + r;
    write_row<PIECES>(p, (size_t)(s.first + row / p.group) * (p.cache.heads * p.group) + meta.head * p.group + row % p.group, dim, d, v, top, sum);
}

// ---- launches -------------------------------------------------------------------------------------------------

// Column groups of a kernel for `tokens` new tokens of `batch` sequences: as many as their rows fill, as registers allow.
inline int column_groups(size_t tokens, size_t batch, int group, int pieces, int dim)
{
    const size_t per = (tokens + batch - 1) / (batch ? batch : 1), columns = per * (size_t)group * (size_t)pieces;
    const int most = dim == 256 ? 2 : 4;
    int nt = 1;
    while (nt < most && columns > (size_t)8 * nt) nt *= 2;
    return nt;
}

inline int ctas_per_sm(int nt, int dim) { return nt == 4 ? 2 : nt * dim <= 128 ? 4 : nt * dim <= 256 ? 3 : 2; }

// CTAs of the first kernel: as many as the GPU holds, or tiles there can be.
inline size_t grid_size(size_t batch, size_t tokens, int heads, int group, int rows, size_t width, int page, int nt, int dim)
{
    const size_t room = (size_t)148 * ctas_per_sm(nt, dim);
    const size_t items = (tokens * group / rows + batch) * heads, tiles = (width * page + kTile - 1) / kTile + 1;
    return items >= room || tiles >= room ? room : (items * tiles < room ? items * tiles : room);
}

struct Sizes {
    int nt, rows;
    size_t ctas, bytes;
};

Sizes sizes(const mxq_cache* c, const mxq_batch* b, int q_heads, int dtype, size_t tokens)
{
    Sizes z;
    const int pieces = dtype == MXQ_F32 ? 2 : 1, group = q_heads / c->heads;
    z.nt = column_groups(tokens, b->batch, group, pieces, c->head_dim);
    z.rows = 8 * z.nt / pieces;
    z.ctas = grid_size(b->batch, tokens, c->heads, group, z.rows, b->width, c->page, z.nt, c->head_dim);
    z.bytes = z.ctas * (sizeof(PartMeta) + 2 * part_bytes(z.rows, c->head_dim));
    return z;
}

int check(const mxq_cache* c, const mxq_batch* b, int q_heads, int dtype, size_t tokens)
{
    if (int rc = check_cache(c)) return rc;
    if (int rc = check_batch(b, tokens)) return rc;
    if (dtype != MXQ_F32 && dtype != MXQ_BF16) return MXQ_ERR_FORMAT;
    if (q_heads < 1 || q_heads > (1 << 16) || q_heads % c->heads) return MXQ_ERR_SIZE;
    if (tokens * (size_t)(q_heads / c->heads) >= ((size_t)1 << 31)) return MXQ_ERR_SIZE;
    return MXQ_OK;
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace
}  // namespace mxq

using namespace mxq;

#pragma GCC visibility push(default)
extern "C" {

size_t mxq_cache_attention_workspace_bytes(const mxq_cache* cache, const mxq_batch* batch, int q_heads, int dtype, size_t tokens)
{
    if (check(cache, batch, q_heads, dtype, tokens) != MXQ_OK || tokens == 0 || batch->batch == 0) return 0;
    return sizes(cache, batch, q_heads, dtype, tokens).bytes;
}

int mxq_cache_attention(const mxq_cache* cache, const mxq_batch* batch, const mxq_rows* q, int q_heads, int dtype, size_t tokens, float scale,
                        int causal, size_t window, void* out, float* lse, void* workspace, size_t workspace_bytes, mxq_stream stream)
{
    if (int rc = check(cache, batch, q_heads, dtype, tokens)) return rc;
    if (window && !causal) return MXQ_ERR_SIZE;
    if (!q) return MXQ_ERR_NULL;
    if (tokens == 0 || batch->batch == 0) return MXQ_OK;
    if (!q->data || !out || !workspace) return MXQ_ERR_NULL;
    if (int rc = check_places(cache, batch, true)) return rc;
    const size_t size = dtype == MXQ_F32 ? 4 : 2;
    AttendArgs a;
    a.cache = cache_args(cache);
    a.batch = batch_args(batch, tokens);
    a.q = static_cast<const uint8_t*>(q->data);
    a.q_token = q->token_stride * size;
    a.q_head = q->head_stride * size;
    if (!aligned(a.q, 32) || a.q_token % 32 || a.q_head % 32 || !aligned(out, 32) || !aligned(workspace, 32) || !aligned(lse, 4)) return MXQ_ERR_ALIGN;
    const Sizes z = sizes(cache, batch, q_heads, dtype, tokens);
    if (workspace_bytes < z.bytes) return MXQ_ERR_SIZE;
    MXQ_DEBUG_SCOPE();
    debug_expect_cache(cache, batch);
    MXQ_DEBUG_EXPECT(a.q, (tokens - 1) * a.q_token + (q_heads - 1) * a.q_head + cache->head_dim * size);
    MXQ_DEBUG_EXPECT(out, tokens * q_heads * cache->head_dim * size);
    MXQ_DEBUG_EXPECT(lse, lse ? tokens * q_heads * 4 : 0);
    MXQ_DEBUG_EXPECT(workspace, z.bytes);
    a.out = static_cast<uint8_t*>(out);
    a.lse = lse;
    a.ws = static_cast<uint8_t*>(workspace);
    a.group = q_heads / cache->heads;
    a.rows = z.rows;
    a.causal = causal != 0;
    a.window = window > (size_t)0x7FFFFFFF ? 0 : (int)window;
    a.scale = scale * 1.4426950408889634f;
    a.ctas = (int)z.ctas;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int rc = MXQ_ERR_FORMAT;
    switch (cache->fmt) {
    case MXQ_FP8_E4M3: rc = launch_attend<MXQ_FP8_E4M3>(cache->head_dim, z.nt, dtype, a, s); break;
    case MXQ_FP4_E2M1: rc = launch_attend<MXQ_FP4_E2M1>(cache->head_dim, z.nt, dtype, a, s); break;
    case MXQ_INT8: rc = launch_attend<MXQ_INT8>(cache->head_dim, z.nt, dtype, a, s); break;
    case MXQ_INT4: rc = launch_attend<MXQ_INT4>(cache->head_dim, z.nt, dtype, a, s); break;
    default: break;
    }
    if (rc != MXQ_OK || a.ctas == 1) return rc;
    auto join = dtype == MXQ_F32 ? join_kernel<2> : join_kernel<1>;
    return launch_grid(join, dim3((unsigned)a.ctas - 1, (unsigned)a.rows), 256, 0, 1, s, a, cache->head_dim);
}

}  // extern "C"
#pragma GCC visibility pop
