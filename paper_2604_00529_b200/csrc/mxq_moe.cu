// A mixture-of-experts layer for a few tokens over experts held as MX codes (the products that the converted weights are for,
// Sec. 3.5), in two kernels:
//   choice     p = softmax(logits[t]); the top_k largest logits (ties: the lowest expert; -inf is never chosen);
//              w = p / (sum of the chosen p), or p
//   kernel 1   h[t, e] = silu(G_e x_t) * (U_e x_t), G_e and U_e the two halves of expert e's up matrix [2 inner, hidden]
//   kernel 2   out[t] = sum over the chosen e of w[t, e] D_e h[t, e], D_e = [hidden, inner]
// Bound by reading the chosen experts' codes once.  Both kernels work the choice out for themselves from the logits (a few
// hundred cycles), so that no third launch stands in front, and kernel 2 does so before it waits for kernel 1.
//
// Products: a warp takes 16 rows of a matrix and a chunk of 16 bytes of codes per lane, widens the codes to BF16 with their
// block's scale multiplied in (exact, see Widen) and multiplies them with up to eight tokens by the warp's matrix instruction,
// sums in FP32.  FP32 operands go in as BF16 parts that add up to them: FP32 tokens as three (all 24 bits), h as two for
// BF16 tokens (16 bits: its error, 2^-17 of a value, is far below the output's rounding) and as three for FP32 ones.
// Warps meet in shared memory in a fixed order: results do not depend on timing.
#include "mxq_kernels.cuh"
#include "mxq_launch.h"
#include "mxq_product.cuh"

namespace mxq {
namespace {

constexpr int kMaxTokens = MXQ_MOE_TOKENS_MAX, kMaxExperts = MXQ_MOE_EXPERTS_MAX, kMaxTopK = MXQ_MOE_TOP_K_MAX;
constexpr int kUpWarps = 4;             // warps per CTA of kernel 1
constexpr int kUpTiles = 2;             // m16 tiles per CTA of kernel 1: eight rows of the gate and eight of the up half each
constexpr int kDownWarps = 16;

struct MoeArgs {
    const uint8_t *x, *up, *up_s, *down, *down_s;
    const float* logits;
    uint8_t *h, *out;
    size_t hidden, inner;
    int tokens, experts, top_k, renormalize, block_shift;
};

// ---- the choice -------------------------------------------------------------------------------------------

// What a CTA knows of the choice: the experts that have tokens, in order, and each one's tokens, in order.
struct Choice {
    unsigned long long mask[kMaxExperts];          // tokens of an expert
    unsigned short first[kMaxExperts + 1];         // its first pair, by position among the active experts
    unsigned short expert[kMaxExperts];            // the active experts
    unsigned short place[kMaxExperts];             // expert -> position
    unsigned char token[kMaxTokens * kMaxTopK];    // pair -> token
    float weight[kMaxTokens * kMaxTopK];           // pair -> weight
    float picked_w[kMaxTokens][kMaxTopK];
    short picked[kMaxTokens][kMaxTopK];
    int active;
};

// A logit's place in the order: NaN above everything, -0 equal to +0.  0 is below -inf.
__device__ __forceinline__ uint32_t order_key(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

__device__ __forceinline__ void choose(const MoeArgs& p, Choice& ch)
{
    constexpr int PER = kMaxExperts / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) ch.mask[e] = 0;
    __syncthreads();
    const uint32_t none = order_key(-INFINITY);
    for (int t = warp; t < p.tokens; t += warps) {
        uint32_t key[PER];
        float own[PER];
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = j * 32 + lane;
            key[j] = 0;
            own[j] = -INFINITY;
            if (j * 32 < p.experts && e < p.experts) {
                const float* at = p.logits + (size_t)t * p.experts + e;
                bool ok = true;
                MXQ_CHECKED(at, 4, ok = false)
                own[j] = ok ? *at : 0.f;
                key[j] = order_key(own[j]);
            }
        }
        float total = 0.f, mine = 0.f;
        int chosen = -1;
        for (int r = 0; r < p.top_k; ++r) {
            uint32_t best = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (j * 32 < p.experts) best = max(best, key[j]);
            best = __reduce_max_sync(0xFFFFFFFFu, best);
            if (best <= none) break;                         // nothing but -inf is left
            uint32_t who = 0xFFFFFFFFu;
#pragma unroll
            for (int j = PER - 1; j >= 0; --j)
                if (j * 32 < p.experts && key[j] == best) who = (uint32_t)(j * 32 + lane);
            who = __reduce_min_sync(0xFFFFFFFFu, who);
            float v = 0.f;
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (j * 32 < p.experts && (uint32_t)(j * 32 + lane) == who) {
                    v = own[j];
                    key[j] = 0;
                }
            v = __shfl_sync(0xFFFFFFFFu, v, (int)(who & 31u));
            if (r == 0) top = v;
            const float e = expf(v - top);
            total += e;
            if (lane == r) {
                chosen = (int)who;
                mine = e;
            }
        }
        if (!p.renormalize) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (j * 32 < p.experts) s += expf(own[j] - top);
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            total = s;
        }
        if (lane < p.top_k) {
            ch.picked[t][lane] = (short)chosen;
            ch.picked_w[t][lane] = mine / total;
            if (chosen >= 0) atomicOr(&ch.mask[chosen], 1ull << t);
        }
    }
    __syncthreads();
    if (warp == 0) {
        int active = 0, pairs = 0;
        for (int e0 = 0; e0 < p.experts; e0 += 32) {
            const int e = e0 + lane;
            const int cnt = e < p.experts ? __popcll(ch.mask[e]) : 0;
            const uint32_t has = __ballot_sync(0xFFFFFFFFu, cnt > 0);
            int before = cnt;                                // inclusive scan of the counts
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xFFFFFFFFu, before, o);
                if (lane >= o) before += up;
            }
            if (cnt > 0) {
                const int a = active + __popc(has & ((1u << lane) - 1u));
                ch.expert[a] = (unsigned short)e;
                ch.place[e] = (unsigned short)a;
                ch.first[a] = (unsigned short)(pairs + before - cnt);
            }
            active += __popc(has);
            pairs += __shfl_sync(0xFFFFFFFFu, before, 31);
        }
        if (lane == 0) {
            ch.first[active] = (unsigned short)pairs;
            ch.active = active;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.tokens * p.top_k; i += blockDim.x) {
        const int t = i / p.top_k, e = ch.picked[t][i % p.top_k];
        if (e < 0) continue;
        const int pair = ch.first[ch.place[e]] + __popcll(ch.mask[e] & ((1ull << t) - 1ull));
        ch.token[pair] = (unsigned char)t;
        ch.weight[pair] = ch.picked_w[t][i % p.top_k];
    }
    __syncthreads();
}

// ---- operands ---------------------------------------------------------------------------------------------

// v as BF16 parts that add up to it: each takes the upper 16 bits of what is left, the last of two rounds.  An infinity or a
// NaN is the first part alone.
template <int PARTS>
__device__ __forceinline__ void bf16_parts(float v, uint32_t (&o)[PARTS])
{
    const bool fine = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
    float left = v;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        uint32_t h = __float_as_uint(left) >> 16;
        if (i == 0 && v != v) h = 0x7FC0u;
        if (PARTS == 2 && i == 1) h = pack_bf16x2(left, 0.f) & 0xFFFFu;
        o[i] = h;
        left = fine ? left - __uint_as_float(h << 16) : 0.f;
    }
}

// One row's consecutive elements for a lane's piece of codes, as BF16 pairs per part.
template <class T, int N>
struct TokenPiece;
template <int N>
struct TokenPiece<BF16, N> {
    static constexpr int PARTS = 1;
    uint32_t v[1][N / 2];
    __device__ __forceinline__ void load(const uint8_t* row, size_t at, bool in)
    {
#pragma unroll
        for (int i = 0; i < N / 16; ++i) {
            uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (in) ld256(w, row + (at + i * 16) * 2);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[0][i * 8 + j] = w[j];
        }
    }
};
template <int N>
struct TokenPiece<F32, N> {
    static constexpr int PARTS = 3;
    uint32_t v[3][N / 2];
    __device__ __forceinline__ void load(const uint8_t* row, size_t at, bool in)
    {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (in) ld256(w, row + (at + i * 8) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t lo[3], hi[3];
                bf16_parts<3>(__uint_as_float(w[2 * j]), lo);
                bf16_parts<3>(__uint_as_float(w[2 * j + 1]), hi);
#pragma unroll
                for (int q = 0; q < 3; ++q) v[q][i * 4 + j] = lo[q] | hi[q] << 16;
            }
        }
    }
};
// h as kernel 1 left it: PARTS planes of BF16 values, `plane` bytes apart
template <int P, int N>
struct StoredPiece {
    static constexpr int PARTS = P;
    uint32_t v[P][N / 2];
    __device__ __forceinline__ void load(const uint8_t* row, size_t at, bool in, size_t plane)
    {
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int i = 0; i < N / 16; ++i) {
                uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (in) ld256(w, row + q * plane + (at + i * 16) * 2);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[q][i * 8 + j] = w[j];
            }
    }
};

// Codes of rows g and g + 8 of a 16-row tile, one piece each, and their scale bytes.
template <int FMT>
struct CodePiece {
    using W = Widen<FMT>;
    static constexpr int N = 128 / W::bits;                  // elements of a piece
    uint4 c[2];
    uint32_t byte[2];

    __device__ __forceinline__ void load(const uint8_t* r0, const uint8_t* r1, const uint8_t* s0, const uint8_t* s1, size_t at, size_t k,
                                         int block_shift)
    {
        c[0] = c[1] = make_uint4(0, 0, 0, 0);
        byte[0] = byte[1] = 127;
        if (at >= k) return;
        c[0] = ld_once(r0 + at * W::bits / 8);
        c[1] = ld_once(r1 + at * W::bits / 8);
        byte[0] = ld_u8(s0 + (at >> block_shift));
        byte[1] = ld_u8(s1 + (at >> block_shift));
    }

    // acc += the tile times the token pieces
    template <class X>
    __device__ __forceinline__ void multiply(float (&acc)[4], const X& x) const
    {
        constexpr int NP = W::NP;
        const uint32_t f0 = W::factor(byte[0]), f1 = W::factor(byte[1]);
        uint32_t g0 = 0, g1 = 0;
        bool wide = false;                                   // a scale beyond what one BF16 factor holds
        if constexpr (W::fp) {
            wide = __any_sync(0xFFFFFFFFu, max(byte[0], byte[1]) > W::limit);
            if (wide) {
                g0 = W::factor2(byte[0]);
                g1 = W::factor2(byte[1]);
            }
        }
        const uint32_t w0[4] = {c[0].x, c[0].y, c[0].z, c[0].w}, w1[4] = {c[1].x, c[1].y, c[1].z, c[1].w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t a0[NP], a1[NP];
            W::pairs(w0[w], f0, a0);
            W::pairs(w1[w], f1, a1);
            if (W::fp && wide) {
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    a0[i] = W::mul(a0[i], g0);
                    a1[i] = W::mul(a1[i], g1);
                }
            }
#pragma unroll
            for (int q = 0; q < X::PARTS; ++q) {
                uint32_t raw[NP], b[NP];
#pragma unroll
                for (int i = 0; i < NP; ++i) raw[i] = x.v[q][w * NP + i];
                order_pairs<NP>(raw, b);
#pragma unroll
                for (int i = 0; i < NP; i += 2) Bf16Mma::mma(acc, a0[i], a1[i], a0[i + 1], a1[i + 1], b[i], b[i + 1]);
            }
        }
    }
};

// ---- kernel 1 ---------------------------------------------------------------------------------------------
// A CTA of four warps works on units of 32 rows, 16 of the gate and the 16 of the up half that go with them, of one expert; the
// warps share k out and meet in shared memory.  In a 16-row tile the first eight rows are the gate's and the last eight
// the up half's.

template <class T, int FMT, int HPARTS>
__global__ void __launch_bounds__(kUpWarps * 32, 4)
moe_up_kernel(const MoeArgs p)
{
    constexpr int TILES = kUpTiles, N = CodePiece<FMT>::N, CHUNK = 4 * N;
    __shared__ Choice ch;
    __shared__ float s_sum[kUpWarps][TILES][4][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    pdl_acquire();
    pdl_release();                                           // after the wait: kernel 2 may read the logits at once
    choose(p, ch);

    const size_t H = p.hidden, I = p.inner, hrow = H * CodePiece<FMT>::W::bits / 8, srow = H >> p.block_shift;
    const size_t plane = (size_t)p.tokens * p.top_k * I * 2;
    const int per_expert = (int)(I / (8 * TILES)), units = ch.active * per_expert;
    for (int u = blockIdx.x; u < units; u += gridDim.x) {
        const int pos = u / per_expert, e = ch.expert[pos], first = ch.first[pos], cnt = ch.first[pos + 1] - first;
        const size_t i0 = (size_t)(u % per_expert) * (8 * TILES);
        const uint8_t* codes = p.up + (size_t)e * 2 * I * hrow;
        const uint8_t* scales = p.up_s + (size_t)e * 2 * I * srow;
        for (int c0 = 0; c0 < cnt; c0 += 8) {                // eight tokens at a time
            const bool live = c0 + g < cnt;
            const uint8_t* xrow = p.x + (size_t)(live ? ch.token[first + c0 + g] : 0) * H * T::size;
            float acc[TILES][4] = {}, sum[TILES][4] = {};
#pragma unroll 2
            for (size_t k0 = (size_t)warp * CHUNK; k0 < H; k0 += kUpWarps * CHUNK) {
                const size_t at = k0 + (size_t)t * N;
                CodePiece<FMT> cp[TILES];
                TokenPiece<T, N> x;
#pragma unroll
                for (int m = 0; m < TILES; ++m) {
                    const size_t r0 = i0 + m * 8 + g, r1 = I + r0;
                    cp[m].load(codes + r0 * hrow, codes + r1 * hrow, scales + r0 * srow, scales + r1 * srow, at, H, p.block_shift);
                }
                x.load(xrow, at, live && at < H);
#pragma unroll
                for (int m = 0; m < TILES; ++m) {
                    if constexpr (T::size == 4) {            // sums kept outside the matrix instruction, which truncates
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[m][j] = 0.f;
                    }
                    cp[m].multiply(T::size == 4 ? acc[m] : sum[m], x);
                    if constexpr (T::size == 4) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) sum[m][j] += acc[m][j];
                    }
                }
            }
            __syncthreads();                                 // the last unit's sums have been read
#pragma unroll
            for (int m = 0; m < TILES; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) s_sum[warp][m][j][lane] = sum[m][j];
            __syncthreads();
            // row r of the gate and of the up half, token c: elements (c & 1) and 2 + (c & 1) of lane r * 4 + c / 2
            for (int o = threadIdx.x; o < TILES * 64; o += kUpWarps * 32) {
                const int m = o >> 6, c = (o >> 3) & 7, r = o & 7, ln = r * 4 + (c >> 1);
                if (c0 + c >= cnt) continue;
                float gate = 0.f, lift = 0.f;
#pragma unroll
                for (int w = 0; w < kUpWarps; ++w) {
                    gate += s_sum[w][m][c & 1][ln];
                    lift += s_sum[w][m][2 + (c & 1)][ln];
                }
                const float h = gate / (1.f + expf(-gate)) * lift;
                uint32_t part[HPARTS];
                bf16_parts<HPARTS>(h, part);
                uint8_t* at = p.h + ((size_t)(first + c0 + c) * I + i0 + m * 8 + r) * 2;
#pragma unroll
                for (int q = 0; q < HPARTS; ++q) st_u16(at + q * plane, part[q]);
            }
        }
    }
}

// ---- kernel 2 ---------------------------------------------------------------------------------------------
// A CTA of 16 warps covers 16 rows of the output for all tokens.  The chunks of all active experts, laid end to end, are shared
// out between the warps; a warp adds its weighted sums to its own copy of the tile, and the copies are added in order.

template <class T, int FMT, int HPARTS>
__global__ void __launch_bounds__(kDownWarps * 32, 1)
moe_down_kernel(const MoeArgs p)
{
    constexpr int N = CodePiece<FMT>::N, CHUNK = 4 * N;
    __shared__ Choice ch;
    extern __shared__ float s_tile[];                        // [warp][token][16]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    pdl_release();
    choose(p, ch);                                           // (the logits were complete when kernel 1 let this one start)
    const size_t H = p.hidden, I = p.inner, irow = I * CodePiece<FMT>::W::bits / 8, srow = I >> p.block_shift;
    const size_t plane = (size_t)p.tokens * p.top_k * I * 2, j0 = (size_t)blockIdx.x * 16;
    float* mine = s_tile + (size_t)warp * p.tokens * 16;
    for (int i = lane; i < p.tokens * 16; i += 32) mine[i] = 0.f;
    __syncwarp();
    pdl_acquire();

    const int per_expert = (int)((I + CHUNK - 1) / CHUNK), total = ch.active * per_expert;
    int q = (int)((long long)total * warp / kDownWarps);
    const int end = (int)((long long)total * (warp + 1) / kDownWarps);
    while (q < end) {
        const int pos = q / per_expert, e = ch.expert[pos], first = ch.first[pos], cnt = ch.first[pos + 1] - first;
        const int lo = q - pos * per_expert, hi = min(per_expert, lo + end - q);
        const size_t r0 = (size_t)e * H + j0 + g, r1 = r0 + 8;
        for (int c0 = 0; c0 < cnt; c0 += 8) {
            const bool live = c0 + g < cnt;
            const uint8_t* hrow = p.h + (size_t)(first + c0 + (live ? g : 0)) * I * 2;
            float acc[4] = {0.f, 0.f, 0.f, 0.f}, sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
            for (int c = lo; c < hi; ++c) {
                const size_t at = (size_t)c * CHUNK + (size_t)t * N;
                CodePiece<FMT> cp;
                StoredPiece<HPARTS, N> x;
                cp.load(p.down + r0 * irow, p.down + r1 * irow, p.down_s + r0 * srow, p.down_s + r1 * srow, at, I, p.block_shift);
                x.load(hrow, at, live && at < I, plane);
                if constexpr (T::size == 4) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = 0.f;
                }
                cp.multiply(T::size == 4 ? acc : sum, x);
                if constexpr (T::size == 4) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[j] += acc[j];
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {                    // row g + 8 (j >> 1), token 2 t + (j & 1) of the eight
                const int c = c0 + 2 * t + (j & 1);
                if (c < cnt) mine[ch.token[first + c] * 16 + g + 8 * (j >> 1)] += ch.weight[first + c] * sum[j];
            }
            __syncwarp();
        }
        q += hi - lo;
    }
    __syncthreads();
    for (int o = threadIdx.x; o < p.tokens * 16; o += kDownWarps * 32) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kDownWarps; ++w) v += s_tile[(size_t)w * p.tokens * 16 + o];
        const size_t i = (size_t)(o >> 4) * H + j0 + (o & 15);
        if constexpr (T::size == 4) {
            MXQ_CHECKED(p.out + i * 4, 4, continue)
            reinterpret_cast<float*>(p.out)[i] = v;
        } else {
            st_u16(p.out + i * 2, pack_bf16x2(v, 0.f) & 0xFFFFu);
        }
    }
}

constexpr int h_parts(int dtype) { return dtype == MXQ_F32 ? 3 : 2; }

template <class T, int FMT>
int run(const MoeArgs& p, cudaStream_t stream)
{
    constexpr int P = h_parts(T::id);
    const size_t most = (size_t)p.tokens * p.top_k < (size_t)p.experts ? (size_t)p.tokens * p.top_k : (size_t)p.experts;
    const size_t units = most * (p.inner / (8 * kUpTiles));
    const unsigned grid = (unsigned)(units < 148 * 4 ? units : 148 * 4);
    if (int rc = launch_grid(moe_up_kernel<T, FMT, P>, dim3(grid), kUpWarps * 32, 0, 1, stream, p)) return rc;
    static std::atomic<uint64_t> done{0};
    auto down = moe_down_kernel<T, FMT, P>;
    if (int rc = allow_smem(reinterpret_cast<const void*>(down), (size_t)kDownWarps * kMaxTokens * 64, done)) return rc;
    return launch_grid(down, dim3((unsigned)(p.hidden / 16)), kDownWarps * 32, (size_t)kDownWarps * p.tokens * 64, 1, stream, p);
}

template <class T>
int by_format(int fmt, const MoeArgs& p, cudaStream_t stream)
{
    switch (fmt) {
    case MXQ_FP8_E4M3: return run<T, MXQ_FP8_E4M3>(p, stream);
    case MXQ_FP4_E2M1: return run<T, MXQ_FP4_E2M1>(p, stream);
    case MXQ_INT8: return run<T, MXQ_INT8>(p, stream);
    case MXQ_INT4: return run<T, MXQ_INT4>(p, stream);
    default: return MXQ_ERR_FORMAT;
    }
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline size_t workspace_bytes(size_t tokens, int top_k, size_t inner, int dtype)
{
    return (tokens * (size_t)top_k * inner * 2 * h_parts(dtype) + 255) / 256 * 256;
}

}  // namespace

}  // namespace mxq

using namespace mxq;

#pragma GCC visibility push(default)
extern "C" {

size_t mxq_moe_workspace_bytes(size_t tokens, int top_k, size_t inner, int dtype)
{
    if (tokens > (size_t)kMaxTokens || top_k < 1 || top_k > kMaxTopK || inner >= ((size_t)1 << 31) || (dtype != MXQ_F32 && dtype != MXQ_BF16)) return 0;
    return workspace_bytes(tokens, top_k, inner, dtype);
}

int mxq_moe(const mxq_moe_layer* layer, const void* x, int dtype, const float* logits, size_t tokens, int top_k, int renormalize,
            void* out, void* workspace, size_t workspace_size, mxq_stream stream)
{
    if (!layer) return MXQ_ERR_NULL;
    const mxq_moe_layer& l = *layer;
    if (dtype != MXQ_F32 && dtype != MXQ_BF16) return MXQ_ERR_FORMAT;
    if (l.fmt != MXQ_FP8_E4M3 && l.fmt != MXQ_FP4_E2M1 && l.fmt != MXQ_INT8 && l.fmt != MXQ_INT4) return MXQ_ERR_FORMAT;
    if (l.block != 32 && l.block != 64 && l.block != 128) return MXQ_ERR_BLOCK;
    const size_t most = (size_t)1 << 20;
    if (tokens > (size_t)kMaxTokens || l.experts < 1 || l.experts > kMaxExperts || top_k < 1 || top_k > kMaxTopK || top_k > l.experts) return MXQ_ERR_SIZE;
    if (l.hidden == 0 || l.inner == 0 || l.hidden > most || l.inner > most || l.hidden % (size_t)l.block || l.inner % (size_t)l.block)
        return MXQ_ERR_SIZE;
    if (tokens == 0) return MXQ_OK;
    const size_t need = workspace_bytes(tokens, top_k, l.inner, dtype);
    if (!x || !logits || !out || !workspace || !l.up_codes || !l.up_scales || !l.down_codes || !l.down_scales) return MXQ_ERR_NULL;
    if (workspace_size < need) return MXQ_ERR_SIZE;
    if (!aligned(x, 32) || !aligned(out, 32) || !aligned(workspace, 32) || !aligned(logits, 16) || !aligned(l.up_codes, 32) || !aligned(l.down_codes, 32) ||
        !aligned(l.up_scales, 16) || !aligned(l.down_scales, 16))
        return MXQ_ERR_ALIGN;
    const size_t size = dtype == MXQ_F32 ? 4u : 2u, weights = (size_t)l.experts * l.hidden * l.inner;
    MXQ_DEBUG_SCOPE();
    MXQ_DEBUG_EXPECT(x, tokens * l.hidden * size);
    MXQ_DEBUG_EXPECT(logits, tokens * (size_t)l.experts * 4);
    MXQ_DEBUG_EXPECT(l.up_codes, mxq_codes_bytes(2 * weights, l.fmt));
    MXQ_DEBUG_EXPECT(l.up_scales, 2 * weights / (size_t)l.block);
    MXQ_DEBUG_EXPECT(l.down_codes, mxq_codes_bytes(weights, l.fmt));
    MXQ_DEBUG_EXPECT(l.down_scales, weights / (size_t)l.block);
    MXQ_DEBUG_EXPECT(workspace, need);
    MXQ_DEBUG_EXPECT(out, tokens * l.hidden * size);
    MoeArgs p;
    p.x = static_cast<const uint8_t*>(x);
    p.up = static_cast<const uint8_t*>(l.up_codes);
    p.up_s = l.up_scales;
    p.down = static_cast<const uint8_t*>(l.down_codes);
    p.down_s = l.down_scales;
    p.logits = logits;
    p.h = static_cast<uint8_t*>(workspace);
    p.out = static_cast<uint8_t*>(out);
    p.hidden = l.hidden;
    p.inner = l.inner;
    p.tokens = (int)tokens;
    p.experts = l.experts;
    p.top_k = top_k;
    p.renormalize = renormalize;
    p.block_shift = l.block == 32 ? 5 : l.block == 64 ? 6 : 7;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == MXQ_F32 ? by_format<F32>(l.fmt, p, s) : by_format<BF16>(l.fmt, p, s);
}

}  // extern "C"
#pragma GCC visibility pop
