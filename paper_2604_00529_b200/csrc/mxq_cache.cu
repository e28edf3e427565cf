// Keys and values on their way into and out of a paged cache of MX codes.
//   mxq_cache_write  codes and scales of the new tokens' rows [tokens, heads, dim], Q_f along the head (Eq. 1-3)
//   mxq_cache_read   V^ = X P of the cached tokens of sequences, as rows [total, heads, dim]
// Both move each byte once and are bound by that, or by latency where there are few tokens: a lane takes 32 bytes of the plain
// tensors, the keys' and the values' halves of a launch lie side by side in the grid's second dimension.
#include "mxq_cache.cuh"
#include "mxq_kernels.cuh"
#include "mxq_launch.h"

namespace mxq {
namespace {

constexpr int kThreads = 128, kUnits = 2;                   // lane units per thread

// The token of row r of [tokens, heads].  (A division of 64 bits costs more than the rest of a unit: 390 MB of BF16 out of a 4-bit
// cache READ_FIGURE.)
__device__ __forceinline__ int token_of(size_t r, uint32_t heads)
{
    return r >> 32 ? (int)(r / heads) : (int)((uint32_t)r / heads);
}

struct WriteArgs {
    CacheArgs cache;
    BatchArgs batch;
    const uint8_t* src[2];                                  // keys, values
    size_t token_stride[2], head_stride[2];                 // in bytes
    uint32_t row_shift;                                     // lane units of a row, as a power of two
};

// Lane unit u of [tokens, heads, row units]; a unit never straddles a block, the lanes of a block are neighbours.
template <class T, class F>
__global__ void __launch_bounds__(kThreads)
cache_write_kernel(const __grid_constant__ WriteArgs p)
{
    pdl_release();
    pdl_acquire();
    constexpr int OB = T::epl * F::bits / 8, NW = code_words(T::epl, F::bits);
    const int kind = blockIdx.y;
    const uint8_t* src = kind ? p.src[1] : p.src[0];
    const size_t ts = kind ? p.token_stride[1] : p.token_stride[0], hs = kind ? p.head_stride[1] : p.head_stride[0];
    uint8_t* codes = const_cast<uint8_t*>(kind ? p.cache.vc : p.cache.kc);
    uint8_t* scales = const_cast<uint8_t*>(kind ? p.cache.vs : p.cache.ks);
    const uint32_t heads = (uint32_t)p.cache.heads, lpb = (1u << p.cache.block_shift) / T::epl;
    const size_t total = ((size_t)p.batch.tokens * heads) << p.row_shift;
    uint32_t w[kUnits][8];
    long long row[kUnits];
    const size_t u0 = (size_t)blockIdx.x * (kThreads * kUnits) + threadIdx.x;
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
        const size_t u = u0 + j * kThreads;
        row[j] = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[j][i] = 0;
        if (u >= total) continue;
        const size_t r = u >> p.row_shift;
        const int token = token_of(r, heads), head = (int)(r - (size_t)token * heads);
        ld256(w[j], src + token * ts + head * hs + (u & ((1u << p.row_shift) - 1u)) * 32);
        int b = token, pos;
        if (p.batch.starts) {
            if (token < ld_int(p.batch.starts)) continue;   // (rows in front of the first and behind the last sequence)
            b = find_sequence(p.batch.starts, p.batch.batch, token);
        }
        const Sequence s = sequence(p.batch, b, p.cache.page_shift);
        pos = s.length - s.n + (token - s.first);
        if (pos < 0 || token - s.first >= s.n) continue;
        row[j] = cache_row(p.cache, p.batch, b, pos, head);
    }
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
        uint32_t amax = unit_amax_bits<T>(w[j]);
        for (uint32_t o = 1; o < lpb; o <<= 1) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
        const BlockScale s = block_scale<F>(amax);
        uint32_t out[NW];
        if constexpr (T::size == 2 && F::kind == KIND_INT) quantize_unit_bf16_int<F>(w[j], s.inv, out);
        else quantize_unit<T, F>(w[j], s.inv, out);
        if (s.byte == 0xFFu) {
#pragma unroll
            for (int i = 0; i < NW; ++i) out[i] = 0;
        }
        if (row[j] < 0) continue;
        const uint32_t at = (uint32_t)(u0 + j * kThreads) & ((1u << p.row_shift) - 1u);
        store_bytes<OB>(codes + ((size_t)row[j] << p.row_shift) * OB + at * OB, out);
        if ((at & (lpb - 1)) == 0) st_u8(scales + (((size_t)row[j] << p.row_shift) + at) / lpb, s.byte);
    }
}

struct ReadArgs {
    CacheArgs cache;
    BatchArgs batch;                                        // starts: of the rows; lengths unused
    uint8_t* dst[2];
    uint32_t row_shift;
};

template <class F, class T>
__global__ void __launch_bounds__(kThreads)
cache_read_kernel(const __grid_constant__ ReadArgs p)
{
    pdl_release();
    pdl_acquire();
    constexpr int IB = T::epl * F::bits / 8, NWI = (IB + 3) / 4;
    const int kind = blockIdx.y;
    const uint8_t *codes = kind ? p.cache.vc : p.cache.kc, *scales = kind ? p.cache.vs : p.cache.ks;
    uint8_t* dst = kind ? p.dst[1] : p.dst[0];
    const uint32_t heads = (uint32_t)p.cache.heads, spb = (1u << p.cache.block_shift) / T::epl;
    const size_t total = ((size_t)p.batch.tokens * heads) << p.row_shift;
    const size_t u0 = (size_t)blockIdx.x * (kThreads * kUnits) + threadIdx.x;
    uint32_t w[kUnits][NWI], sb[kUnits];
    bool in[kUnits];
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
        const size_t u = u0 + j * kThreads;
        in[j] = false;
        sb[j] = 0;
#pragma unroll
        for (int i = 0; i < NWI; ++i) w[j][i] = 0;
        if (u >= total) continue;
        const size_t r = u >> p.row_shift;
        const int token = token_of(r, heads), head = (int)(r - (size_t)token * heads);
        if (token < ld_int(p.batch.starts)) continue;
        const int b = find_sequence(p.batch.starts, p.batch.batch, token);
        const int first = max(ld_int(p.batch.starts + b), 0), pos = token - first;
        if (token >= ld_int(p.batch.starts + b + 1)) continue;      // behind the last sequence: left as it is
        in[j] = true;
        if ((pos >> p.cache.page_shift) >= p.batch.width) continue;
        const long long row = cache_row(p.cache, p.batch, b, pos, head);
        if (row < 0) continue;                              // no page: zeros
        const uint32_t at = (uint32_t)u & ((1u << p.row_shift) - 1u);
        load_bytes<IB>(w[j], codes + ((size_t)row << p.row_shift) * IB + at * IB);
        sb[j] = ld_u8(scales + (((size_t)row << p.row_shift) + at) / spb);
    }
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
        uint32_t out[8];
        widen_unit<F, T>(w[j], sb[j], out);
        if (in[j]) st256(dst + (u0 + j * kThreads) * 32, out);
    }
}

inline int shift_of(int v)
{
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

template <class FN>
int by_cache_format(int fmt, FN&& fn)
{
    switch (fmt) {
    case MXQ_FP8_E4M3: return fn(Fmt<MXQ_FP8_E4M3>{});
    case MXQ_FP4_E2M1: return fn(Fmt<MXQ_FP4_E2M1>{});
    case MXQ_INT8: return fn(Fmt<MXQ_INT8>{});
    case MXQ_INT4: return fn(Fmt<MXQ_INT4>{});
    default: return MXQ_ERR_FORMAT;
    }
}

template <class T, class F>
int run_write(const WriteArgs& a, size_t units, cudaStream_t stream)
{
    const size_t ctas = (units + kThreads * kUnits - 1) / (kThreads * kUnits);
    if (ctas > 0x7FFFFFFFu) return MXQ_ERR_SIZE;
    return launch_grid(cache_write_kernel<T, F>, dim3((unsigned)ctas, 2), kThreads, 0, 1, stream, a);
}

template <class F, class T>
int run_read(const ReadArgs& a, size_t units, cudaStream_t stream)
{
    const size_t ctas = (units + kThreads * kUnits - 1) / (kThreads * kUnits);
    if (ctas > 0x7FFFFFFFu) return MXQ_ERR_SIZE;
    return launch_grid(cache_read_kernel<F, T>, dim3((unsigned)ctas, 2), kThreads, 0, 1, stream, a);
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace

// Checks of a cache's description: format, block, sizes.
int check_cache(const mxq_cache* c)
{
    if (!c) return MXQ_ERR_NULL;
    if (c->fmt != MXQ_FP8_E4M3 && c->fmt != MXQ_FP4_E2M1 && c->fmt != MXQ_INT8 && c->fmt != MXQ_INT4) return MXQ_ERR_FORMAT;
    if (c->block != 32 && c->block != 64 && c->block != 128) return MXQ_ERR_BLOCK;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return MXQ_ERR_SIZE;
    if (c->head_dim % c->block) return MXQ_ERR_SIZE;
    if (c->page < kCachePageMin || c->page > kCachePageMax || (c->page & (c->page - 1))) return MXQ_ERR_SIZE;
    if (c->heads < 1 || c->heads > MXQ_CACHE_HEADS_MAX || c->pages >= ((size_t)1 << 31)) return MXQ_ERR_SIZE;
    return MXQ_OK;
}

int check_batch(const mxq_batch* b, size_t tokens)
{
    if (!b) return MXQ_ERR_NULL;
    if (b->batch >= ((size_t)1 << 31) || b->width >= ((size_t)1 << 31) || tokens >= ((size_t)1 << 31)) return MXQ_ERR_SIZE;
    if (!b->starts && tokens != b->batch) return MXQ_ERR_SIZE;
    return MXQ_OK;
}

// Addresses of both, for calls that have something to do.
int check_places(const mxq_cache* c, const mxq_batch* b, bool lengths)
{
    if (c->pages && (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales)) return MXQ_ERR_NULL;
    if ((b->width && !b->table) || (lengths && !b->lengths)) return MXQ_ERR_NULL;
    if (!aligned(c->k_codes, 32) || !aligned(c->v_codes, 32) || !aligned(c->k_scales, 16) || !aligned(c->v_scales, 16) || !aligned(b->table, 4) ||
        !aligned(b->lengths, 4) || !aligned(b->starts, 4))
        return MXQ_ERR_ALIGN;
    return MXQ_OK;
}

CacheArgs cache_args(const mxq_cache* c)
{
    CacheArgs a;
    a.kc = static_cast<const uint8_t*>(c->k_codes);
    a.ks = c->k_scales;
    a.vc = static_cast<const uint8_t*>(c->v_codes);
    a.vs = c->v_scales;
    a.pages = (int)c->pages;
    a.page_shift = shift_of(c->page);
    a.heads = c->heads;
    a.block_shift = shift_of(c->block);
    return a;
}

BatchArgs batch_args(const mxq_batch* b, size_t tokens)
{
    return BatchArgs{b->table, b->lengths, b->starts, (int)b->batch, (int)b->width, (int)tokens};
}

void debug_expect_cache(const mxq_cache* c, const mxq_batch* b)
{
    const size_t elements = c->pages * (size_t)c->heads * (size_t)c->page * (size_t)c->head_dim;
    (void)elements;
    MXQ_DEBUG_EXPECT(c->k_codes, mxq_codes_bytes(elements, c->fmt));
    MXQ_DEBUG_EXPECT(c->v_codes, mxq_codes_bytes(elements, c->fmt));
    MXQ_DEBUG_EXPECT(c->k_scales, elements / (size_t)c->block);
    MXQ_DEBUG_EXPECT(c->v_scales, elements / (size_t)c->block);
    MXQ_DEBUG_EXPECT(b->table, b->batch * b->width * 4);
    MXQ_DEBUG_EXPECT(b->lengths, b->lengths ? b->batch * 4 : 0);
    MXQ_DEBUG_EXPECT(b->starts, b->starts ? (b->batch + 1) * 4 : 0);
}

}  // namespace mxq

using namespace mxq;

#pragma GCC visibility push(default)
extern "C" {

int mxq_cache_write(const mxq_cache* cache, const mxq_batch* batch, const mxq_rows* k, const mxq_rows* v, int dtype, size_t tokens, mxq_stream stream)
{
    if (int rc = check_cache(cache)) return rc;
    if (int rc = check_batch(batch, tokens)) return rc;
    if (!k || !v) return MXQ_ERR_NULL;
    if (dtype != MXQ_F32 && dtype != MXQ_BF16) return MXQ_ERR_FORMAT;
    if (tokens == 0 || batch->batch == 0 || batch->width == 0 || cache->pages == 0) return MXQ_OK;
    if (!k->data || !v->data) return MXQ_ERR_NULL;
    if (int rc = check_places(cache, batch, true)) return rc;
    const size_t size = dtype == MXQ_F32 ? 4 : 2;
    WriteArgs a;
    a.cache = cache_args(cache);
    a.batch = batch_args(batch, tokens);
    const mxq_rows* rows[2] = {k, v};
    MXQ_DEBUG_SCOPE();
    for (int i = 0; i < 2; ++i) {
        a.src[i] = static_cast<const uint8_t*>(rows[i]->data);
        a.token_stride[i] = rows[i]->token_stride * size;
        a.head_stride[i] = rows[i]->head_stride * size;
        if (!aligned(a.src[i], 32) || a.token_stride[i] % 32 || a.head_stride[i] % 32) return MXQ_ERR_ALIGN;
        MXQ_DEBUG_EXPECT(a.src[i], (tokens - 1) * a.token_stride[i] + (cache->heads - 1) * a.head_stride[i] + cache->head_dim * size);
    }
    debug_expect_cache(cache, batch);
    const size_t per_row = cache->head_dim * size / 32;
    a.row_shift = (uint32_t)shift_of((int)per_row);
    const size_t units = tokens * cache->heads * per_row;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return by_cache_format(cache->fmt, [&](auto f) {
        using F = decltype(f);
        return dtype == MXQ_F32 ? run_write<F32, F>(a, units, s) : run_write<BF16, F>(a, units, s);
    });
}

int mxq_cache_read(const mxq_cache* cache, const mxq_batch* batch, size_t total, void* k, void* v, int dtype, mxq_stream stream)
{
    if (int rc = check_cache(cache)) return rc;
    if (!batch) return MXQ_ERR_NULL;
    if (dtype != MXQ_F32 && dtype != MXQ_BF16) return MXQ_ERR_FORMAT;
    if (total == 0 || batch->batch == 0) return MXQ_OK;
    if (!batch->starts) return MXQ_ERR_NULL;
    if (int rc = check_batch(batch, total)) return rc;
    if (!k || !v) return MXQ_ERR_NULL;
    if (int rc = check_places(cache, batch, false)) return rc;
    if (!aligned(k, 32) || !aligned(v, 32)) return MXQ_ERR_ALIGN;
    const size_t size = dtype == MXQ_F32 ? 4 : 2, per_row = cache->head_dim * size / 32, units = total * cache->heads * per_row;
    MXQ_DEBUG_SCOPE();
    debug_expect_cache(cache, batch);
    MXQ_DEBUG_EXPECT(k, units * 32);
    MXQ_DEBUG_EXPECT(v, units * 32);
    ReadArgs a;
    a.cache = cache_args(cache);
    a.batch = batch_args(batch, total);
    a.dst[0] = static_cast<uint8_t*>(k);
    a.dst[1] = static_cast<uint8_t*>(v);
    a.row_shift = (uint32_t)shift_of((int)per_row);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return by_cache_format(cache->fmt, [&](auto f) {
        using F = decltype(f);
        return dtype == MXQ_F32 ? run_read<F, F32>(a, units, s) : run_read<F, BF16>(a, units, s);
    });
}

}  // extern "C"
#pragma GCC visibility pop
