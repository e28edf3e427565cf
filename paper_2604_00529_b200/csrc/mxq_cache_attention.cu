// mxq_cache_attention: checks, the choice of a kernel's width, and the kernel that adds up what the first one did in parts.
#include "mxq_attend_items.cuh"
#include "mxq_launch.h"

namespace mxq {
namespace {

// Items that the first kernel worked on in several parts: CTA c takes the item that run c + 1 begins inside, if no earlier run begins
// inside it too.  Its threads are shared out among the item's elements, four to a thread, and what is left of them among its parts.
constexpr int kJoinThreads = 512;

template <int PIECES>
__global__ void __launch_bounds__(kJoinThreads)
join_kernel(const __grid_constant__ AttendArgs p, int dim)
{
    pdl_release();
    pdl_acquire();
    __shared__ float4 sums[kJoinThreads];
    __shared__ float2 weights[kJoinThreads];
    const PartMeta* metas = reinterpret_cast<const PartMeta*>(p.ws);
    const uint32_t c = blockIdx.x + 1;
    const PartMeta meta = ld_part<PartMeta>(metas + c);    // (every CTA has written its own)
    const uint32_t total = ld_part<uint32_t>(&metas->total);
    if (c >= working_ctas(total, p.ctas)) return;
    const Runs runs(total, working_ctas(total, p.ctas));
    const uint32_t before = runs.start(c - 1);
    if (meta.from <= meta.item_from || before > meta.item_from) return;
    const int n = (int)(runs.of(min(meta.item_to, total) - 1) - (c - 1) + 1);      // runs c - 1 ... have parts of it
    const size_t part = part_bytes(p.rows, dim) / 4;        // in floats
    const float* const parts = reinterpret_cast<const float*>(p.ws + (size_t)p.ctas * sizeof(PartMeta));
    // the first part is its run's last piece (slot 1), unless the item is that run's first; the others are their runs' first pieces (slot 0)
    const float* const part0 = parts + ((size_t)(c - 1) * 2 + (before == meta.item_from ? 0 : 1)) * part;
    const float* const part1 = parts + (size_t)c * 2 * part;
    const int quads = dim / 4, slots = meta.rows * quads, lanes = slots < kJoinThreads ? kJoinThreads / slots : 1;
    for (int slot0 = (int)blockIdx.y * kJoinThreads; slot0 < slots; slot0 += (int)gridDim.y * kJoinThreads) {
        const int slot = lanes > 1 ? (int)threadIdx.x % slots : slot0 + (int)threadIdx.x, mine = lanes > 1 ? (int)threadIdx.x / slots : 0;
        const bool on = mine < lanes && slot < slots;
        const int r = on ? slot / quads : 0, d = on ? slot % quads * 4 : 0;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float top = kNone, sum = 0.f;                       // carried along, like the softmax that they are parts of
        auto add = [&](float2 w, float4 e) {                // w: a part's maximum and its weight there
            const float up = fmaxf(top, w.x), keep = exp2_approx(top - up), by = w.y * exp2_approx(w.x - up);
            top = up;
            sum = sum * keep + by;
            v.x = v.x * keep + by * e.x;
            v.y = v.y * keep + by * e.y;
            v.z = v.z * keep + by * e.z;
            v.w = v.w * keep + by * e.w;
        };
        if (on) {
#pragma unroll 4
            for (int i = mine; i < n; i += lanes) {
                const float* x = i ? part1 + (size_t)(i - 1) * 2 * part : part0;
                add(ld_part<float2>(x + p.rows * dim + 2 * r), ld_part<float4>(x + r * dim + d));
            }
        }
        if (lanes > 1) {
            sums[threadIdx.x] = v;
            weights[threadIdx.x] = make_float2(top, sum);
            __syncthreads();
            if (mine != 0) return;
            // (v is not divided yet: a weight of 1 at its maximum)
            for (int k = 1; k < lanes; ++k) {
                const float4 e = sums[threadIdx.x + k * slots];
                const float2 w = weights[threadIdx.x + k * slots];
                const float up = fmaxf(top, w.x), keep = exp2_approx(top - up), by = exp2_approx(w.x - up);
                top = up;
                sum = sum * keep + by * w.y;
                v.x = v.x * keep + by * e.x;
                v.y = v.y * keep + by * e.y;
                v.z = v.z * keep + by * e.z;
                v.w = v.w * keep + by * e.w;
            }
        }
        if (!on) continue;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const float out[4] = {v.x * inv, v.y * inv, v.z * inv, v.w * inv};
        const int i = meta.r0 + r < p.group ? 0 : (meta.r0 + r) / p.group;      // the row's token
        write_row<PIECES>(p, (size_t)(meta.first + i) * (p.cache.heads * p.group) + meta.head * p.group + meta.r0 + r - i * p.group, dim, d, out, top, sum);
    }
}

// ---- launches -------------------------------------------------------------------------------------------------

// How a call is cut up: column groups of its kernel, rows of an item, CTAs and their warps, a tile's keys, bytes of workspace.
// Rows of a cache head in a mean sequence, above which they are many: items of 256 of them in tiles instead of 16 in two column groups.  Both, us, 32 heads
// over 8 of 128:
//   rows                                     16        20        32        40        48        64        96
//   12 sequences of 4096 INT8 tokens      49 / 93   67 / 93   70 / 93   92 / 95   93 / 95   114 / 95  165 / 97
//   8 of 8192 E2M1                        48 / 95   71 / 95   73 / 93   97 / 96   99 / 96   123 / 95  172 / 98
//   32 of 2048 E4M3                       55 / 128  86 / 129  90 / 128 117 / 130 119 / 131  153 / 131 216 / 133
//   1 of 16384 INT8                       48 / 54   43 / 53   46 / 53   49 / 53   50 / 55   55 / 54   68 / 56
// Where one sequence of 64 brings a piece of a prompt and the others one query each, 4096 E2M1 tokens: 256 queries (20 rows in the mean) 236 / 412, 512
// (36) 338 / 432, 1024 (68) 528 / 482.
constexpr size_t kManyColumns = 48;
// Keys per CTA of a cluster, at most.  Clusters and runs with the second kernel, us: one sequence of 1000 E2M1 tokens, 8 heads of 128, 7.3 and 10.8, of
// 16000 15.7 and 20.0; 8 of 2000 11.8 and 19.7; 32 of 2048 to 4096 E4M3 tokens, one head of 256, 22.6 and 33.2.  Lengths are known on the device
// alone, and a cluster has its sequence to itself: beyond this a long one among short ones would keep the call waiting (8 of 8000, all alike, would
// still take 25 and 33).
constexpr size_t kClusterKeys = 2048;

struct Sizes {
    bool many;
    int nt, rows, warps, tile_shift, share;
    size_t ctas, bytes;
};

// `window`: 0 for none, or what the call says; the workspace does not depend on it.
Sizes sizes(const mxq_cache* c, const mxq_batch* b, int q_heads, int dtype, size_t tokens, size_t window)
{
    constexpr size_t kSms = 148;
    Sizes z;
    const int pieces = dtype == MXQ_F32 ? 2 : 1, group = q_heads / c->heads, dim = c->head_dim;
    // as many column groups as the rows of a mean sequence fill, as registers allow
    const size_t columns = (tokens + b->batch - 1) / b->batch * (size_t)group * (size_t)pieces;
    z.nt = 1;
    while (z.nt < (dim == 256 || pieces == 1 ? 2 : 4) && columns > (size_t)8 * z.nt) z.nt *= 2;
    // Many rows: items of 256 of them on the tensor cores that take whole tiles.
    z.many = dtype == MXQ_BF16 && dim <= 128 && columns > kManyColumns;
    z.rows = z.many ? 256 : 8 * z.nt / pieces;
    const size_t items = (b->starts ? tokens * group / z.rows + b->batch : b->batch * ((size_t)(group + z.rows - 1) / z.rows)) * c->heads, keys = b->width * (size_t)c->page < (size_t)1 << 31 ? b->width * (size_t)c->page : (size_t)1 << 31;     // at most
    const int ctas = z.nt == 4 ? 2 : z.nt * dim <= 128 ? 4 : z.nt * dim <= 256 ? 3 : 2;      // per SM, of four warps
    // Few items: one CTA per SM with all the warps that it holds, so that an item has a quarter of the parts.
    const bool wide = z.many || (z.nt == 1 && items <= kSms);
    z.warps = wide ? 4 * ctas : 4;
    const size_t room = wide ? kSms : kSms * ctas;
    // tiles of 64 (128) keys, longer ones where there could be more of them than 32 bits count
    z.tile_shift = z.many ? 7 : 6;
    while ((keys >> z.tile_shift) + 1 > (((size_t)1 << 31) - 1) / items) ++z.tile_shift;
    const size_t tiles = items * ((keys >> z.tile_shift) + 1);
    z.ctas = tiles < room ? tiles : room;
    z.bytes = z.ctas * (sizeof(PartMeta) + 2 * part_bytes(z.rows, dim));
    // Few items that cannot be long: a cluster of CTAs each, which joins its sums itself, without a plan and a second kernel.
    z.share = 0;
    if (wide && !z.many && !b->starts && group <= z.rows) {
        const size_t most = window && window < keys ? window + 64 : keys, own = (size_t)b->batch * c->heads;
        size_t share = 1;
        while (share < 8 && own * share * 2 <= kSms) share *= 2;
        if (most <= share * kClusterKeys) {
            z.share = (int)share;
            z.ctas = own * share;
        }
    }
    return z;
}

int check(const mxq_cache* c, const mxq_batch* b, int q_heads, int dtype, size_t tokens)
{
    if (int rc = check_cache(c)) return rc;
    if (int rc = check_batch(b, tokens)) return rc;
    if (dtype != MXQ_F32 && dtype != MXQ_BF16) return MXQ_ERR_FORMAT;
    if (q_heads < 1 || q_heads > (1 << 16) || q_heads % c->heads) return MXQ_ERR_SIZE;
    if (tokens * (size_t)q_heads + b->batch * (size_t)c->heads > MXQ_CACHE_ROWS_MAX) return MXQ_ERR_SIZE;
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
    return sizes(cache, batch, q_heads, dtype, tokens, 0).bytes;
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
    const Sizes z = sizes(cache, batch, q_heads, dtype, tokens, window);
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
    a.warps = z.warps;
    a.tile_shift = z.tile_shift;
    a.share = z.share;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int rc = MXQ_ERR_FORMAT;
    if (z.many) rc = launch_attend_many(cache->fmt, cache->head_dim, a, s);
    else switch (cache->fmt) {
    case MXQ_FP8_E4M3: rc = launch_attend<MXQ_FP8_E4M3>(cache->head_dim, z.nt, dtype, a, s); break;
    case MXQ_FP4_E2M1: rc = launch_attend<MXQ_FP4_E2M1>(cache->head_dim, z.nt, dtype, a, s); break;
    case MXQ_INT8: rc = launch_attend<MXQ_INT8>(cache->head_dim, z.nt, dtype, a, s); break;
    case MXQ_INT4: rc = launch_attend<MXQ_INT4>(cache->head_dim, z.nt, dtype, a, s); break;
    default: break;
    }
    if (rc != MXQ_OK || a.share || a.ctas == 1) return rc;
    auto join = dtype == MXQ_F32 ? join_kernel<2> : join_kernel<1>;
    return launch_grid(join, dim3((unsigned)a.ctas - 1, z.many ? 8 : 1), kJoinThreads, 0, 1, s, a, cache->head_dim);
}

}  // extern "C"
#pragma GCC visibility pop
