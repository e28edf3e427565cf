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

constexpr int kThreads = 128;

// A thread has one lane unit of a token, the same one of kTokens tokens in a row: what places it (a division, the search for the sequence,
// mostly the page) is worked out once for all of them.  (For every unit by itself it was two thirds of the instructions: 98504 tokens of
// 8 heads of 128 from E2M1 to BF16 took 113 us, and take 87 this way.)
struct Place {
    int token, head;                                        // the first token
    uint32_t unit;                                          // of the row
};

template <int kTokens>
__device__ __forceinline__ bool place_of(const BatchArgs& p, uint32_t heads, uint32_t row_shift, Place& at)
{
    const uint32_t per = heads << row_shift;
    const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x, group = i >> 32 ? i / per : (uint32_t)i / per;
    const uint32_t u = (uint32_t)(i - group * per);
    at.head = (int)(u >> row_shift);
    at.unit = u & ((1u << row_shift) - 1u);
    at.token = (int)min(group * kTokens, (size_t)0x7FFFFFFF);
    return at.token < p.tokens;
}

// The sequence of a token and its rows [first, next), followed from token to token.
struct Cursor {
    int b, first, next;
    __device__ __forceinline__ void start(const BatchArgs& p, int token)
    {
        if (!p.starts) {
            b = first = token;
            next = token + 1;
            return;
        }
        b = find_sequence(p.starts, p.batch, token);
        first = ld_int(p.starts + b);
        next = ld_int(p.starts + b + 1);
    }
    // Whether the token is some sequence's.
    __device__ __forceinline__ bool at(const BatchArgs& p, int token)
    {
        while (token >= next && b + 1 < p.batch) {
            ++b;
            first = next;
            next = p.starts ? ld_int(p.starts + b + 1) : next + 1;
        }
        return token >= first && token < next && first >= 0;
    }
};

struct WriteArgs {
    CacheArgs cache;
    BatchArgs batch;
    const uint8_t* src[2];                                  // keys, values
    size_t token_stride[2], head_stride[2];                 // in bytes
    uint32_t row_shift;                                     // lane units of a row, as a power of two
};

// A unit never straddles a block, the lanes of a block are neighbours.
template <class T, class F, int kTokens>
__global__ void __launch_bounds__(kThreads)
cache_write_kernel(const __grid_constant__ WriteArgs p)
{
    pdl_release();
    pdl_acquire();
    constexpr int OB = T::epl * F::bits / 8, NW = code_words(T::epl, F::bits);
    const int kind = blockIdx.y;
    const size_t ts = kind ? p.token_stride[1] : p.token_stride[0], hs = kind ? p.head_stride[1] : p.head_stride[0];
    uint8_t* codes = const_cast<uint8_t*>(kind ? p.cache.vc : p.cache.kc);
    uint8_t* scales = const_cast<uint8_t*>(kind ? p.cache.vs : p.cache.ks);
    const uint32_t lpb = (1u << p.cache.block_shift) / T::epl;
    Place at = {0, 0, 0};
    const bool in = place_of<kTokens>(p.batch, (uint32_t)p.cache.heads, p.row_shift, at);
    const uint8_t* src = (kind ? p.src[1] : p.src[0]) + at.head * hs + at.unit * 32;
    uint32_t w[kTokens][8];
    long long row[kTokens];
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
        row[j] = -1;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[j][i] = 0;
        if (in && at.token + j < p.batch.tokens) ld256(w[j], src + (size_t)(at.token + j) * ts);
    }
    if (in) {
        Cursor c;
        c.start(p.batch, at.token);
        int b = -1, length = 0;
#pragma unroll
        for (int j = 0; j < kTokens; ++j) {
            const int token = at.token + j;
            if (token >= p.batch.tokens || !c.at(p.batch, token)) continue;
            if (c.b != b) {
                b = c.b;
                length = sequence(p.batch, b, p.cache.page_shift).length;
            }
            const int pos = length - (min(c.next, p.batch.tokens) - token);
            if (pos >= 0) row[j] = cache_row(p.cache, p.batch, b, pos, at.head);
        }
    }
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
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
        store_bytes<OB>(codes + ((size_t)row[j] << p.row_shift) * OB + at.unit * OB, out);
        if ((at.unit & (lpb - 1)) == 0) st_u8(scales + (((size_t)row[j] << p.row_shift) + at.unit) / lpb, s.byte);
    }
}

struct ReadArgs {
    CacheArgs cache;
    BatchArgs batch;                                        // starts: of the rows; lengths unused
    uint8_t* dst[2];
    uint32_t row_shift;
};

template <class F, class T, int kTokens>
__global__ void __launch_bounds__(kThreads)
cache_read_kernel(const __grid_constant__ ReadArgs p)
{
    pdl_release();
    pdl_acquire();
    constexpr int IB = T::epl * F::bits / 8, NWI = (IB + 3) / 4;
    const int kind = blockIdx.y;
    const uint8_t *codes = kind ? p.cache.vc : p.cache.kc, *scales = kind ? p.cache.vs : p.cache.ks;
    const uint32_t block_units_shift = p.cache.block_shift - (T::size == 4 ? 3 : 4);
    Place at;
    if (!place_of<kTokens>(p.batch, (uint32_t)p.cache.heads, p.row_shift, at)) return;
    uint32_t w[kTokens][NWI], sb[kTokens];
    bool in[kTokens];
    Cursor c;
    c.start(p.batch, at.token);
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
        const int token = at.token + j;
        sb[j] = 0;
#pragma unroll
        for (int i = 0; i < NWI; ++i) w[j][i] = 0;
        in[j] = token < p.batch.tokens && c.at(p.batch, token);       // (rows of no sequence: left as they are)
        const int pos = token - c.first;
        if (!in[j] || (pos >> p.cache.page_shift) >= p.batch.width) continue;
        const long long row = cache_row(p.cache, p.batch, c.b, pos, at.head);
        if (row < 0) continue;                              // no page: zeros
        const size_t unit = ((size_t)row << p.row_shift) + at.unit;
        load_bytes<IB>(w[j], codes + unit * IB);
        sb[j] = ld_u8(scales + (unit >> block_units_shift));
    }
    uint8_t* dst = (kind ? p.dst[1] : p.dst[0]) + ((((size_t)at.token * p.cache.heads + at.head) << p.row_shift) + at.unit) * 32;
    const size_t next = ((size_t)p.cache.heads << p.row_shift) * 32;
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
        uint32_t out[8];
        widen_unit<F, T>(w[j], sb[j], out);
        if (in[j]) st256(dst + j * next, out);
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

// Tokens per thread: one in short calls, where time is what one thread takes; four, placed together, from 20 CTAs of single ones per SM on.  One and four,
// us, 8 heads of 128, INT8 and BF16: writing 1024 tokens 2.9 and 4.3, 4096 6.0 and 5.8, 8192 12.3 and 13.3, 32768 39.9 and 36.4; reading 1024 3.2 and
// 3.3, 5900 7.9 and 6.7, 32768 38.2 and 33.5.
template <class FN>
int by_tokens(size_t tokens, size_t units_per_token, FN&& fn)
{
    const bool few = tokens * units_per_token < (size_t)148 * 20 * kThreads;
    const size_t groups = few ? tokens : (tokens + 3) / 4, ctas = (groups * units_per_token + kThreads - 1) / kThreads;
    if (ctas > 0x7FFFFFFFu) return MXQ_ERR_SIZE;
    return few ? fn(std::integral_constant<int, 1>{}, (unsigned)ctas) : fn(std::integral_constant<int, 4>{}, (unsigned)ctas);
}

template <class T, class F>
int run_write(const WriteArgs& a, size_t units, cudaStream_t stream)
{
    return by_tokens((size_t)a.batch.tokens, units, [&](auto u, unsigned ctas) { return launch_grid(cache_write_kernel<T, F, decltype(u)::value>, dim3(ctas, 2), kThreads, 0, 1, stream, a); });
}

template <class F, class T>
int run_read(const ReadArgs& a, size_t units, cudaStream_t stream)
{
    return by_tokens((size_t)a.batch.tokens, units, [&](auto u, unsigned ctas) { return launch_grid(cache_read_kernel<F, T, decltype(u)::value>, dim3(ctas, 2), kThreads, 0, 1, stream, a); });
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
    const size_t units = cache->heads * per_row;            // of a token
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
    const size_t size = dtype == MXQ_F32 ? 4 : 2, per_row = cache->head_dim * size / 32, units = cache->heads * per_row;
    MXQ_DEBUG_SCOPE();
    debug_expect_cache(cache, batch);
    MXQ_DEBUG_EXPECT(k, total * units * 32);
    MXQ_DEBUG_EXPECT(v, total * units * 32);
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
