// A mixture-of-experts layer for a few tokens over experts held as MX codes, anchors or converted to 4 bits (Sec. 3.5), in two
// kernels:
//   choice     p = softmax(logits[t]); the top_k largest logits (ties: the lowest expert; -inf is never chosen);
//              w = p / (sum of the chosen p), or p
//   kernel 1   h[t, e] = silu(G_e x_t) * (U_e x_t), G_e and U_e the two halves of expert e's up matrix [2 inner, hidden]
//   kernel 2   out[t] = sum over the chosen e of w[t, e] D_e h[t, e], D_e = [hidden, inner]
// Bound by reading the chosen experts' codes once.  Both kernels work the choice out for themselves from the logits (2 us for one
// token and 64 experts, 4.4 for 32 tokens), so that no third launch stands in front, and kernel 2 does so before it waits for
// kernel 1 (leaving the choice in the workspace for it instead was 2 to 4 % slower: it then starts only when kernel 1 is done).  A CTA of
// either kernel fills an SM, so that kernel 2's begin where CTAs of kernel 1 have left.
//
// Products: a warp takes 16 rows of a matrix and a chunk of 16 bytes of codes per lane, widens the codes to BF16 with their
// block's scale multiplied in (exact, see Widen) and multiplies them with up to eight tokens by the warp's matrix instruction,
// sums in FP32.  FP32 operands go in as BF16 parts that add up to them: FP32 tokens as three (all 24 bits), h as two for
// BF16 tokens (16 bits: its error, 2^-17 of a value, is far below the output's rounding) and as three for FP32 ones.  The instruction cuts
// its sums, by less than 2^-23 of them per step of 16 values: with BF16 tokens a warp's share of k stays in it (64 steps for
// hidden = 4096, 2^-17.6 in norm at worst), with FP32 ones its sums leave it chunk by chunk.  With BF16 tokens these two move outputs
// next to a halfway point, 1e-4 of them in norm, and leave their distance to 64 bits at 1.7e-3; three parts of h cost 3 to 9 %
// (one token, two of eight 4096 x 14336 E4M3 experts 115 us where two parts took 111; eight small experts 24.9 and 22.9), with sums
// outside as well 5 to 11 % (117 and 25.4).
// Warps meet in shared memory in a fixed order: results do not depend on timing.
#include "mxq_kernels.cuh"
#include "mxq_launch.h"
#include "mxq_product.cuh"
#include "mxq_tensor.cuh"

namespace mxq {
namespace {

constexpr int kMaxTokens = MXQ_MOE_TOKENS_MAX, kMaxExperts = MXQ_MOE_EXPERTS_MAX, kMaxTopK = MXQ_MOE_TOP_K_MAX;
constexpr int kTeam = 4, kUpTeams = 4;  // kernel 1: warps of a team, teams of a CTA
constexpr int kUpWarps = kTeam * kUpTeams;
constexpr int kUpTiles = 2;             // 16-row tiles of a team's unit: eight rows of the gate and eight of the up half each
constexpr int kDownWarps = 16;          // kernel 2: warps of a CTA
constexpr int kDownTiles = 2;           // 16-row tiles of its rows of the output

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

template <int PER>                                           // logits per lane: experts <= 32 PER
__device__ __forceinline__ void choose_tokens(const MoeArgs& p, Choice& ch)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
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
            if (e < p.experts) {
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
            for (int j = 0; j < PER; ++j) best = max(best, key[j]);
            best = __reduce_max_sync(0xFFFFFFFFu, best);
            if (best <= none) break;                         // nothing but -inf is left
            uint32_t who = 0xFFFFFFFFu;
#pragma unroll
            for (int j = PER - 1; j >= 0; --j)
                if (key[j] == best) who = (uint32_t)(j * 32 + lane);
            who = __reduce_min_sync(0xFFFFFFFFu, who);
            float v = 0.f;
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if ((uint32_t)(j * 32 + lane) == who) {
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
            for (int j = 0; j < PER; ++j) s += expf(own[j] - top);
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
}

__device__ __forceinline__ void choose(const MoeArgs& p, Choice& ch)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int e = threadIdx.x; e < p.experts; e += blockDim.x) ch.mask[e] = 0;
    __syncthreads();
    if (p.experts <= 64) choose_tokens<2>(p, ch);
    else if (p.experts <= 128) choose_tokens<4>(p, ch);
    else choose_tokens<kMaxExperts / 32>(p, ch);
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

// ---- the pipeline of a warp -------------------------------------------------------------------------------
// A warp's codes of a few chunks are always under way to shared memory (asynchronous copies, each lane's own 16 bytes in a
// place of its own: no lane reads what another one copied, so waiting for the own copies is enough).
// A chunk is 16 bytes of codes per lane and row: four lanes cover 64 (128) elements of k of an 8-bit (4-bit) row.

__device__ __forceinline__ void copy16(uint32_t to, const uint8_t* from, bool in)      // zeros where `in` is false
{
    uint32_t size = in ? 16u : 0u;
    MXQ_CHECKED(from, size, size = 0)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(size) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }

__device__ __forceinline__ uint4 lds16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// 16-row tiles of codes times eight tokens.  What a lane holds of a row lies at byte 16 t of the chunk's 64 bytes.
template <int FMT, int TILES>
struct Chunk {
    using W = Widen<FMT>;
    static constexpr int N = 128 / W::bits;                  // elements of k per lane
    static constexpr int K = 4 * N;                          // and per chunk
    static constexpr int bytes = TILES * 2 * 512;            // of a warp's slot

    // The codes of rows g and g + 8 of each tile: `lo` and `hi` point to the first tile's rows 0 and 8, `next` bytes apart from the next
    // tile's; `off` is the lane's byte from there (row g, byte 16 t of the chunk), `left` the row's bytes from the chunk on.
    static __device__ __forceinline__ void fetch_codes(uint32_t slot, int lane, const uint8_t* lo, const uint8_t* hi, uint32_t next, uint32_t off,
                                                       uint32_t left)
    {
        const uint32_t to = slot + lane * 16;
        const bool in = (uint32_t)(lane & 3) * 16 < left;
        if (!in) off = next = 0;
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
            copy16(to + m * 1024, lo + (m * next + off), in);
            copy16(to + m * 1024 + 512, hi + (m * next + off), in);
        }
    }

    // acc += the tiles times the token pieces.  ORDERED: the tokens' values lie in the order of the widened pairs already.
    template <bool ORDERED, class X>
    static __device__ __forceinline__ void multiply(float (&acc)[TILES][4], uint32_t slot, int lane, const X& x, const uint32_t (&byte)[TILES][2])
    {
        uint32_t f[TILES][2], top = 0;
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f[m][h] = W::factor(byte[m][h]);
                top = max(top, byte[m][h]);
            }
        if (W::fp && __any_sync(0xFFFFFFFFu, top > W::limit)) products<ORDERED, true>(acc, slot, lane, x, byte, f);
        else products<ORDERED, false>(acc, slot, lane, x, byte, f);
    }
    // WIDE: some scale is beyond what one BF16 factor holds
    template <bool ORDERED, bool WIDE, class X>
    static __device__ __forceinline__ void products(float (&acc)[TILES][4], uint32_t slot, int lane, const X& x, const uint32_t (&byte)[TILES][2],
                                                    const uint32_t (&f)[TILES][2])
    {
        constexpr int NP = W::NP;
        uint4 c[TILES][2];
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) c[m][h] = lds16(slot + (m * 2 + h) * 512 + lane * 16);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            uint32_t b[X::PARTS][NP];
#pragma unroll
            for (int q = 0; q < X::PARTS; ++q) {
                uint32_t raw[NP];
#pragma unroll
                for (int i = 0; i < NP; ++i) raw[i] = x.v[q][w * NP + i];
                if constexpr (ORDERED) {
#pragma unroll
                    for (int i = 0; i < NP; ++i) b[q][i] = raw[i];
                } else {
                    order_pairs<NP>(raw, b[q]);
                }
            }
#pragma unroll
            for (int m = 0; m < TILES; ++m) {
                uint32_t a[2][NP];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    W::pairs(w == 0 ? c[m][h].x : w == 1 ? c[m][h].y : w == 2 ? c[m][h].z : c[m][h].w, f[m][h], a[h]);
                    if constexpr (WIDE) {
                        const uint32_t g = W::factor2(byte[m][h]);
#pragma unroll
                        for (int i = 0; i < NP; ++i) a[h][i] = W::mul(a[h][i], g);
                    }
                }
#pragma unroll
                for (int q = 0; q < X::PARTS; ++q)
#pragma unroll
                    for (int i = 0; i < NP; i += 2) Bf16Mma::mma(acc[m], a[0][i], a[1][i], a[0][i + 1], a[1][i + 1], b[q][i], b[q][i + 1]);
            }
        }
        if constexpr (W::has_nan) nan_rows(acc, c);
    }
    // The sums of rows with a NaN code become NaN: a matrix step of NaN by zeros for those rows, of zeros by zeros for the others.  One
    // question for all of the warp's codes, behind the products: one token, two of eight 4096 x 14336 E4M3 experts 109.2 us, 103.7
    // without it; 8 tokens over eight experts 316 and 302.  (NaN as the multiplier of a lane's codes that hold one 112.3 and 336; NaN
    // into the sums without asking first 112.2 and 330; kept over a unit's chunks 112.0 and 329; the codes through an 8-bit
    // matrix step by zeros slower still.)
    static __device__ __forceinline__ void nan_rows(float (&acc)[TILES][4], const uint4 (&c)[TILES][2])
    {
        uint32_t any = 0;
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) W::note_nan(c[m][h], any);
        if (!__any_sync(0xFFFFFFFFu, W::saw_nan(any))) return;
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
            uint32_t lo = 0, hi = 0;
            W::note_nan(c[m][0], lo);
            W::note_nan(c[m][1], hi);
            lo = W::saw_nan(lo) ? 0x7FC07FC0u : 0u;
            hi = W::saw_nan(hi) ? 0x7FC07FC0u : 0u;
            Bf16Mma::mma(acc[m], lo, hi, lo, hi, 0u, 0u);
        }
    }
};

// Where element i of h is stored: in the order of Widen's pairs, within its code word's elements.
template <int FMT>
__device__ __forceinline__ uint32_t ordered_index(uint32_t i)
{
    if constexpr (Widen<FMT>::NP == 2) return (i & ~3u) | (i & 1u) << 1 | (i >> 1 & 1u);
    else return (i & ~7u) | (i & 3u) << 1 | (i >> 2 & 1u);
}

// A lane's BF16 pairs of a token's elements, per part.
template <int P, int N>
struct TokenPiece {
    static constexpr int PARTS = P;
    uint32_t v[P][N / 2];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int i = 0; i < N / 2; ++i) v[q][i] = 0;
    }
    // BF16 elements.  Lanes without a token keep what they have: finite values or not, their sums are not looked at.  Beyond k: zeros.
    __device__ __forceinline__ void load(const uint8_t* at, bool live, bool in, size_t plane = 0)
    {
        if (!live) return;
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int i = 0; i < N / 16; ++i) {
                uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                if (in) ld256(w, at + q * plane + i * 32);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[q][i * 8 + j] = w[j];
            }
    }
    // FP32 elements from global memory, split into parts
    __device__ __forceinline__ void load_f32(const uint8_t* at, bool in)
    {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            uint32_t w[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (in) ld256(w, at + i * 32);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t lo[P], hi[P];
                bf16_parts<P>(__uint_as_float(w[2 * j]), lo);
                bf16_parts<P>(__uint_as_float(w[2 * j + 1]), hi);
#pragma unroll
                for (int q = 0; q < P; ++q) v[q][i * 4 + j] = lo[q] | hi[q] << 16;
            }
        }
    }
};

constexpr int kSlots = 4;                                    // chunks under way per warp: two to four, as shared memory allows
inline int slots_for(size_t shared, int warps, int bytes) { return (int)(shared / ((size_t)warps * bytes) < kSlots ? shared / ((size_t)warps * bytes) : kSlots); }

__device__ __forceinline__ void wait_slot(int slots)         // all copies but those of the last slots - 1 groups
{
    if (slots == 4) wait_copies<3>();
    else if (slots == 3) wait_copies<2>();
    else wait_copies<1>();
}

// ---- kernel 1 ---------------------------------------------------------------------------------------------
// One CTA per SM, of four teams of four warps.  A team works on units of 32 rows, 16 of the gate and the 16 of the up half that go
// with them, of one expert, for eight of its tokens at a time; its warps share k out and meet in shared memory, once per unit (in
// two sets of sums in turn).  In a 16-row tile the first eight rows are the gate's and the last eight the up half's.  Units go
// to the CTAs' first teams before their second ones, so that few of them are on many SMs (256 units of 4096: both kernels 25 us;
// four at a time 31).  A warp's copies run on into its next unit.
// Bound by instructions: one token, two of eight 4096 x 14336 E4M3 experts 65 us for 235 MB, about 5 more since NaN codes are looked
// for (67 us when tried: 57 without the widening, 46 with the copies alone; about 6 of them for the last 16 of 1792 units, which 592
// teams share.  The whole CTA on each of those saved 3 us there and cost other shapes 0.3 to 0.6; teams of 8 or 16 for all units
// cost 5 and 16 us).  Tokens go through L1, not through the copies (82 us: every SM asking L2 for the same few lines).  Asking for a
// unit's scales as early as for its codes, 20 or 24 warps of fewer registers: nothing gained.

template <class T, int FMT, int HPARTS>
__global__ void __launch_bounds__(kUpWarps * 32, 1)
moe_up_kernel(const MoeArgs p, const int slots)
{
    using C = Chunk<FMT, kUpTiles>;
    constexpr int TILES = kUpTiles;
    constexpr int bytes = C::bytes;
    extern __shared__ __align__(16) uint8_t s_ring[];        // the warps' slots, then two sets of the warps' sums
    __shared__ Choice ch;
    using Sums = float[TILES][4][32];
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int team = warp / kTeam, part = warp % kTeam;
    Sums* sums = reinterpret_cast<Sums*>(s_ring + kUpWarps * slots * bytes) + team * kTeam;      // this unit's, of the team
    int other = kUpWarps;                                    // the other set lies there
    pdl_acquire();
    pdl_release();                                           // after the wait: kernel 2 may read the logits at once
    choose(p, ch);

    const uint32_t H = (uint32_t)p.hidden, I = (uint32_t)p.inner, hrow = H * C::W::bits / 8, srow = H >> p.block_shift;
    const size_t plane = (size_t)p.tokens * p.top_k * I * 2, half = (size_t)I * hrow, half_s = (size_t)I * srow;
    const int per_expert = (int)(I / (8 * TILES)), units = ch.active * per_expert, stride = gridDim.x * kUpTeams;
    const int turns = (int)((H + kTeam * C::K - 1) / (kTeam * C::K));    // chunks of a warp per unit and group of tokens
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + warp * slots * bytes;

    // A warp's sequence of chunks: units, groups of eight of the unit's tokens, turns.  It is followed three times: where the copies
    // are; one turn ahead, where the loads of scale bytes and BF16 tokens are; and where the products are.
    struct At {
        int unit, group, turn;
    };
    auto step = [&](At& a) {                                 // true: a new unit or group
        if (++a.turn < turns) return false;
        a.turn = 0;
        a.group += 8;
        const int pos = a.unit / per_expert;
        if (a.group >= ch.first[pos + 1] - ch.first[pos]) {
            a.group = 0;
            a.unit += stride;
        }
        return true;
    };
    auto row_of = [&](int unit) { return ((size_t)ch.expert[unit / per_expert] * 2) * I + (size_t)(unit % per_expert) * (8 * TILES); };

    At ahead{team * (int)gridDim.x + (int)blockIdx.x, 0, 0};
    const uint8_t* a_lo = nullptr;
    auto enter_copies = [&] {
        if (ahead.unit < units) a_lo = p.up + row_of(ahead.unit) * hrow;
    };
    auto fetch = [&](int slot) {
        if (ahead.unit < units) {
            const uint32_t kb = (uint32_t)(ahead.turn * kTeam + part) * 64, at = kb + t * 16;      // bytes of codes of a row
            C::fetch_codes(ring + slot * bytes, lane, a_lo, a_lo + half, 8 * hrow, g * hrow + at, kb < hrow ? hrow - kb : 0);
            if (step(ahead)) enter_copies();
        }
        copies_done();
    };
    At soon = ahead;
    const uint8_t *s_lo = nullptr, *s_x = nullptr;
    bool s_live = false;
    auto enter_operands = [&] {
        if (soon.unit >= units) return;
        s_lo = p.up_s + row_of(soon.unit) * srow + (size_t)g * srow;
        const int pos = soon.unit / per_expert, first = ch.first[pos], cnt = ch.first[pos + 1] - first;
        s_live = soon.group + g < cnt;
        s_x = p.x + (size_t)(s_live ? ch.token[first + soon.group + g] : 0) * H * T::size;
    };
    uint32_t byte[TILES][2];
    TokenPiece<1, C::N> x_next;                              // (BF16 tokens)
    x_next.zero();
    auto fetch_operands = [&] {
        if (soon.unit >= units) return;
        const uint32_t at = ((uint32_t)(soon.turn * kTeam + part) * 64 + t * 16) * (8 / C::W::bits);
        const uint8_t* s = s_lo + (at < H ? at >> p.block_shift : 0);
#pragma unroll
        for (int m = 0; m < TILES; ++m) {
            byte[m][0] = ld_u8(s + m * 8 * srow);
            byte[m][1] = ld_u8(s + half_s + m * 8 * srow);
        }
        if constexpr (T::size == 2) x_next.load(s_x + (at < H ? (size_t)at * 2 : 0), s_live, at < H);
        if (step(soon)) enter_operands();
    };
    At now = ahead;
    enter_copies();
    enter_operands();
    for (int i = 0; i < slots - 1; ++i) fetch(i);
    fetch_operands();
    int slot = 0;
    while (now.unit < units) {
        const int pos = now.unit / per_expert, first = ch.first[pos], cnt = ch.first[pos + 1] - first, unit = now.unit, group = now.group;
        const bool live = group + g < cnt;
        const uint8_t* xrow = p.x + (size_t)(T::size == 4 && live ? ch.token[first + group + g] : 0) * H * T::size;
        float sum[TILES][4] = {};
#pragma unroll 2
        for (int turn = 0; turn < turns; ++turn) {
            fetch(slot == 0 ? slots - 1 : slot - 1);         // (that slot was read in the turn before)
            wait_slot(slots);
            const uint32_t at = ring + slot * bytes;
            uint32_t scale[TILES][2];
#pragma unroll
            for (int m = 0; m < TILES; ++m) {
                scale[m][0] = byte[m][0];
                scale[m][1] = byte[m][1];
            }
            const TokenPiece<1, C::N> x_now = x_next;
            fetch_operands();
            if constexpr (T::size == 2) {
                C::template multiply<false>(sum, at, lane, x_now, scale);
            } else {                                         // sums kept outside the matrix instruction, which truncates
                const uint32_t k = ((uint32_t)(turn * kTeam + part) * 64 + t * 16) * (8 / C::W::bits);
                TokenPiece<3, C::N> x;
                x.load_f32(xrow + (size_t)(k < H ? k : 0) * 4, live && k < H);
                float acc[TILES][4] = {};
                C::template multiply<false>(acc, at, lane, x, scale);
#pragma unroll
                for (int m = 0; m < TILES; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[m][j] += acc[m][j];
            }
            slot = slot + 1 == slots ? 0 : slot + 1;
        }
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[part][m][j][lane] = sum[m][j];
        asm volatile("bar.sync %0, %1;" :: "r"(1 + team), "n"(kTeam * 32) : "memory");
        // row r of the gate and of the up half, token c: elements (c & 1) and 2 + (c & 1) of lane r * 4 + c / 2
        for (int o = part * 32 + lane; o < TILES * 64; o += kTeam * 32) {
            const int m = o >> 6, c = (o >> 3) & 7, r = o & 7, ln = r * 4 + (c >> 1);
            if (group + c >= cnt) continue;
            float gate = 0.f, lift = 0.f;
#pragma unroll
            for (int w = 0; w < kTeam; ++w) {
                gate += sums[w][m][c & 1][ln];
                lift += sums[w][m][2 + (c & 1)][ln];
            }
            const float h = gate / (1.f + expf(-gate)) * lift;
            uint32_t hp[HPARTS];
            bf16_parts<HPARTS>(h, hp);
            uint8_t* to = p.h + ((size_t)(first + group + c) * I + ordered_index<FMT>((uint32_t)(unit % per_expert) * (8 * TILES) + m * 8 + r)) * 2;
#pragma unroll
            for (int q = 0; q < HPARTS; ++q) st_u16(to + q * plane, hp[q]);
        }
        sums += other;                                       // (what the team reads now is written again after its next meeting)
        other = -other;
        now.turn = turns - 1;
        step(now);
    }
    wait_copies<0>();
}

// ---- kernel 2 ---------------------------------------------------------------------------------------------
// A CTA covers 32 rows of the output for all tokens; where that makes few CTAs, a cluster of them covers the same rows.  The
// chunks of all active experts, laid end to end, are shared out between the warps; a warp adds its weighted sums to its own
// copy of the tile, and the copies are added in order, then the cluster's.  The first chunks' codes are fetched before the
// wait for kernel 1.  (The same experts: 37 us for 117 MB; with 16 rows per CTA 46.)  Spills, FP32 tokens: 192 bytes per thread over
// MXINT4 experts, 240 over E2M1 ones (kernel 1: 4 and 20).

template <class T, int FMT, int HPARTS>
__global__ void __launch_bounds__(kDownWarps * 32, 1)
moe_down_kernel(const MoeArgs p, const int slots, const int share)
{
    constexpr int TILES = kDownTiles, WARPS = kDownWarps, ROWS = 16 * TILES;
    using C = Chunk<FMT, TILES>;
    constexpr int bytes = C::bytes;
    __shared__ Choice ch;
    extern __shared__ __align__(16) uint8_t s_ring[];        // the warps' slots, then [warp][token][16] sums
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    pdl_release();
    choose(p, ch);                                           // (the logits were complete when kernel 1 let this one start)
    const uint32_t H = (uint32_t)p.hidden, I = (uint32_t)p.inner, irow = I * C::W::bits / 8, srow = I >> p.block_shift;
    const size_t plane = (size_t)p.tokens * p.top_k * I * 2, j0 = (size_t)(blockIdx.x / share) * ROWS;
    const int rank = blockIdx.x % share;                     // of the cluster's CTAs, which share the chunks of one group of rows
    float* const tile = reinterpret_cast<float*>(s_ring + WARPS * slots * bytes);
    float* const mine = tile + (size_t)warp * p.tokens * ROWS;
    for (int i = lane; i < p.tokens * ROWS; i += 32) mine[i] = 0.f;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + warp * slots * bytes;

    // A warp's sequence of chunks: its part of each expert's, for eight of the expert's tokens at a time; followed three times as
    // in kernel 1 (one turn ahead, h in the tokens' place).
    const int per_expert = (int)((irow + 63) / 64), total = ch.active * per_expert;
    const int begin = (int)((long long)total * (rank * WARPS + warp) / (share * WARPS)), end = (int)((long long)total * (rank * WARPS + warp + 1) / (share * WARPS));
    struct At {
        int pos, lo, hi, group, c;                           // the expert, the warp's chunks [lo, hi) of it, ...; pos < 0: the end
    };
    auto start = [&](int q) {
        if (q >= end) return At{-1, 0, 0, 0, 0};
        const int pos = q / per_expert, lo = q - pos * per_expert;
        return At{pos, lo, min(per_expert, lo + end - q), 0, lo};
    };
    auto step = [&](At& a) {                                 // true: another expert or group
        if (++a.c < a.hi) return false;
        a.group += 8;
        a.c = a.lo;
        if (a.group >= ch.first[a.pos + 1] - ch.first[a.pos]) a = start(a.pos * per_expert + a.hi);
        return true;
    };
    At ahead = start(begin), soon = ahead, now = ahead;
    const uint8_t *a_lo = nullptr, *s_lo = nullptr, *s_h = nullptr;
    bool s_live = false;
    auto enter_copies = [&] {
        if (ahead.pos >= 0) a_lo = p.down + ((size_t)ch.expert[ahead.pos] * H + j0) * irow;
    };
    auto fetch = [&](int slot) {
        if (ahead.pos >= 0) {
            const uint32_t kb = (uint32_t)ahead.c * 64;
            C::fetch_codes(ring + slot * bytes, lane, a_lo, a_lo + 8 * (size_t)irow, 16 * irow, g * irow + kb + t * 16, irow - kb);
            if (step(ahead)) enter_copies();
        }
        copies_done();
    };
    auto enter_operands = [&] {
        if (soon.pos < 0) return;
        s_lo = p.down_s + ((size_t)ch.expert[soon.pos] * H + j0 + g) * srow;
        const int first = ch.first[soon.pos], cnt = ch.first[soon.pos + 1] - first;
        s_live = soon.group + g < cnt;
        s_h = p.h + (size_t)(first + soon.group + (s_live ? g : 0)) * I * 2;
    };
    uint32_t byte[TILES][2] = {};
    TokenPiece<HPARTS, C::N> x_next;
    x_next.zero();
    auto fetch_operands = [&] {
        if (soon.pos < 0) return;
        const uint32_t at = ((uint32_t)soon.c * 64 + t * 16) * (8 / C::W::bits);
        const uint8_t* s = s_lo + (at < I ? at >> p.block_shift : 0);
#pragma unroll
        for (int m = 0; m < TILES; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) byte[m][h] = ld_u8(s + (uint32_t)(m * 16 + h * 8) * srow);
        x_next.load(s_h + (at < I ? (size_t)at * 2 : 0), s_live, at < I, plane);
        if (step(soon)) enter_operands();
    };
    // the first slots' codes before the wait for kernel 1
    enter_copies();
    for (int i = 0; i < slots - 1; ++i) fetch(i);
    pdl_acquire();
    enter_operands();
    fetch_operands();
    int slot = 0;
    while (now.pos >= 0) {
        const int first = ch.first[now.pos], cnt = ch.first[now.pos + 1] - first, chunks = now.hi - now.lo, group = now.group;
        float sum[TILES][4] = {};
        for (int i = 0; i < chunks; ++i) {
            fetch(slot == 0 ? slots - 1 : slot - 1);
            wait_slot(slots);
            const uint32_t at = ring + slot * bytes;
            uint32_t scale[TILES][2];
#pragma unroll
            for (int m = 0; m < TILES; ++m) {
                scale[m][0] = byte[m][0];
                scale[m][1] = byte[m][1];
            }
            const TokenPiece<HPARTS, C::N> x = x_next;
            fetch_operands();
            if constexpr (T::size == 2) {
                C::template multiply<true>(sum, at, lane, x, scale);
            } else {
                float acc[TILES][4] = {};
                C::template multiply<true>(acc, at, lane, x, scale);
#pragma unroll
                for (int m = 0; m < TILES; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[m][j] += acc[m][j];
            }
            slot = slot + 1 == slots ? 0 : slot + 1;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {                        // row g + 8 (j >> 1) of a tile, token 2 t + (j & 1) of the eight
            const int c = group + 2 * t + (j & 1);
            if (c >= cnt) continue;
            float* const to = mine + ch.token[first + c] * ROWS + g + 8 * (j >> 1);
            const float w = ch.weight[first + c];
#pragma unroll
            for (int m = 0; m < TILES; ++m) to[16 * m] += w * sum[m][j];
        }
        __syncwarp();
        now.c = now.hi - 1;
        step(now);
    }
    wait_copies<0>();
    __syncthreads();
    const int outs = p.tokens * ROWS;
    if (share > 1) {                                         // the CTA's own sum into its first copy, then the cluster's in order of rank
        for (int o = threadIdx.x; o < outs; o += WARPS * 32) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) v += tile[(size_t)w * outs + o];
            tile[o] = v;
        }
        cluster_sync();
    }
    const uint32_t tile_at = smem_addr(tile);
    for (int o = threadIdx.x + rank * WARPS * 32; o < outs; o += share * WARPS * 32) {
        float v = 0.f;
        if (share > 1) {
            for (int r = 0; r < share; ++r) v += ld_peer(peer_addr(tile_at + o * 4, r));
        } else {
#pragma unroll
            for (int w = 0; w < WARPS; ++w) v += tile[(size_t)w * outs + o];
        }
        const size_t i = (size_t)(o / ROWS) * H + j0 + o % ROWS;
        if constexpr (T::size == 4) {
            MXQ_CHECKED(p.out + i * 4, 4, continue)
            reinterpret_cast<float*>(p.out)[i] = v;
        } else {
            st_u16(p.out + i * 2, pack_bf16x2(v, 0.f) & 0xFFFFu);
        }
    }
    if (share > 1) cluster_sync();                           // no CTA leaves while another one reads its sums
}

constexpr int h_parts(int dtype) { return dtype == MXQ_F32 ? 3 : 2; }

constexpr size_t kShared = 226 * 1024;                       // what a CTA may use of an SM, less a little

template <class T, int FMT>
int run(const MoeArgs& p, cudaStream_t stream)
{
    static std::atomic<uint64_t> done{0};
    auto up = moe_up_kernel<T, FMT, h_parts(T::id)>;
    constexpr size_t kUpStatic = sizeof(Choice) + 64, kUpSums = (size_t)2 * kUpWarps * kUpTiles * 512;
    constexpr int up_bytes = Chunk<FMT, kUpTiles>::bytes;
    if (int rc = allow_smem(reinterpret_cast<const void*>(up), kShared - kUpStatic, done)) return rc;
    const size_t most = (size_t)p.tokens * p.top_k < (size_t)p.experts ? (size_t)p.tokens * p.top_k : (size_t)p.experts;
    const size_t units = most * (p.inner / (8 * kUpTiles));    // as many CTAs as may have one
    const int up_slots = slots_for(kShared - kUpStatic - kUpSums, kUpWarps, up_bytes);
    if (int rc = launch_grid(up, dim3((unsigned)(units < 148 ? units : 148)), kUpWarps * 32, (size_t)kUpWarps * up_slots * up_bytes + kUpSums, 1, stream, p, up_slots))
        return rc;
    static std::atomic<uint64_t> down_done{0};
    auto down = moe_down_kernel<T, FMT, h_parts(T::id)>;
    const size_t free = kShared - sizeof(Choice) - 64, sums = (size_t)kDownWarps * p.tokens * 64 * kDownTiles;
    if (int rc = allow_smem(reinterpret_cast<const void*>(down), free, down_done)) return rc;
    static_assert(kShared - sizeof(Choice) - 64 - (size_t)kDownWarps * kMaxTokens * 64 * kDownTiles >= 2 * kDownWarps * Chunk<FMT, kDownTiles>::bytes, "two slots at least");
    const int slots = slots_for(free - sums, kDownWarps, Chunk<FMT, kDownTiles>::bytes);
    const size_t groups = p.hidden / (16 * kDownTiles);
    int share = 1;                                           // CTAs of a cluster: so many that there is about one CTA per SM
    while (share < 8 && groups * share * 2 <= 148) share *= 2;
    return launch_grid(down, dim3((unsigned)(groups * share)), kDownWarps * 32, (size_t)kDownWarps * slots * Chunk<FMT, kDownTiles>::bytes + sums, share, stream, p,
                       slots, share);
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
    if (!aligned(x, 32) || !aligned(out, 32) || !aligned(workspace, 32) || !aligned(logits, 4) || !aligned(l.up_codes, 32) || !aligned(l.down_codes, 32) ||
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
