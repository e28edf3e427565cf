// What the two kernels of mxq_cache_attention share: how rows and keys are cut into items and tiles, how runs of tiles are
// shared out among CTAs, and how a row of the output is written.
#pragma once
#include "mxq_cache.cuh"
#include "mxq_kernels.cuh"

namespace mxq {
namespace {

constexpr float kNone = -3.402823466e38f;                   // m of a row that has seen nothing: no score is less (finite: -inf - kNone is no NaN)
// Beyond it a maximum differs from the exact product that it was rounded from by one and more: scores are rounded before it is taken from them.
constexpr float kSteep = 16777216.f;

// ---- items ----------------------------------------------------------------------------------------------------

// The new token that a row belongs to.  (A division costs some thirty instructions that depend on one another; one token is the common case.)
__device__ __forceinline__ int row_token(const AttendArgs& p, const Sequence& s, int row) { return s.n == 1 ? 0 : row / p.group; }

// The keys [lo, hi) that a new token of a sequence sees.
__device__ __forceinline__ int token_hi(const AttendArgs& p, const Sequence& s, int i) { return p.causal ? max(s.length - s.n + i + 1, 0) : s.length; }
// (A token in front of position 0 is taken to be there, so that no window passes 32 bits.)
__device__ __forceinline__ int token_lo(const AttendArgs& p, const Sequence& s, int i) { return p.window ? max(max(s.length - s.n + i + 1, 0) - p.window, 0) : 0; }

__device__ __forceinline__ uint32_t span_tiles(const AttendArgs& p, int lo, int hi)
{
    const int tiles = (int)(((uint32_t)hi + ((1u << p.tile_shift) - 1u)) >> p.tile_shift) - (lo >> p.tile_shift);
    return (uint32_t)max(tiles, 1);                         // (an item that sees nothing still writes its zeros)
}

// Tiles of the item that begins with row r0.
__device__ __forceinline__ uint32_t item_tiles(const AttendArgs& p, const Sequence& s, int r0)
{
    const int last = min(r0 + p.rows, s.n * p.group) - 1;
    return span_tiles(p, token_lo(p, s, row_token(p, s, r0)), token_hi(p, s, row_token(p, s, last)));
}

// The items of one head of a sequence in order, without a division for each: first and last token of an item follow from the item before.
struct ItemWalk {
    int r0, first, over, tokens, rest, last_tokens, last_rest;     // over: rows of token `first` that lie in front of r0
    __device__ __forceinline__ explicit ItemWalk(const AttendArgs& p)
        : r0(0), first(0), over(0), tokens(p.rows / p.group), rest(p.rows % p.group), last_tokens((p.rows - 1) / p.group), last_rest((p.rows - 1) % p.group) {}
    __device__ __forceinline__ uint32_t tiles(const AttendArgs& p, const Sequence& s) const
    {
        const int last = min(first + last_tokens + (over + last_rest >= p.group), s.n - 1);
        return span_tiles(p, token_lo(p, s, first), token_hi(p, s, last));
    }
    __device__ __forceinline__ void next(const AttendArgs& p)
    {
        r0 += p.rows;
        first += tokens;
        over += rest;
        if (over >= p.group) {
            over -= p.group;
            ++first;
        }
    }
};

// Tiles of one head of a sequence.
__device__ __forceinline__ uint32_t sequence_tiles(const AttendArgs& p, const Sequence& s)
{
    const int rows = s.n * p.group;                         // far below 2^31: the host has seen to that, and to the sum of all tiles
    if (rows == 0) return 0;
    if (rows <= p.rows) return span_tiles(p, token_lo(p, s, 0), token_hi(p, s, s.n - 1));
    uint32_t sum = 0;
    for (ItemWalk w(p); w.r0 < rows; w.next(p)) sum += w.tiles(p, s);
    return sum;
}

// Run c of `ctas` nearly equal runs of tiles 0 ... total - 1: each has `each` of them, the first `more` one besides.
struct Runs {
    uint32_t each, more;
    __device__ __forceinline__ Runs(uint32_t total, uint32_t ctas) : each(total / ctas), more(total % ctas) {}
    __device__ __forceinline__ uint32_t start(uint32_t c) const { return each * c + min(c, more); }
    __device__ __forceinline__ uint32_t of(uint32_t tile) const         // the run that a tile lies in
    {
        const uint32_t big = (each + 1) * more;
        return tile < big ? tile / (each + 1) : more + (tile - big) / each;
    }
};

// What the second kernel needs of a CTA of the first: its run's first tile, the tiles of the item that it lies in, all tiles; and that
// item's rows.
struct PartMeta {
    uint32_t from, item_from, item_to, total;
    int first, head, r0, rows;                              // first: the row of the tokens' tensors that its sequence begins with
};

// CTAs that work, of `ctas`: those that there is a tile for.
__device__ __forceinline__ uint32_t working_ctas(uint32_t total, uint32_t ctas) { return min(ctas, max(total, 1u)); }

// Words of the workspace: what the first kernel leaves of an item's row beside its sums, and what the second one reads.
__device__ __forceinline__ void write_weight(float* to, float m, float l)
{
    MXQ_CHECKED(to, 8, return)
    to[0] = m;
    to[1] = l;
}
template <class T>
__device__ __forceinline__ T ld_part(const void* from)
{
    MXQ_CHECKED(from, sizeof(T), return T{})
    return *reinterpret_cast<const T*>(from);
}

__host__ __device__ inline size_t part_bytes(int rows, int dim) { return ((size_t)rows * (dim + 2) * 4 + 31) / 32 * 32; }

__device__ __forceinline__ float exp2_approx(float v)
{
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(v));
    return d;
}

__device__ __forceinline__ void write_lse(const AttendArgs& p, size_t row, float m, float l)
{
    if (!p.lse) return;
    float* to = p.lse + row;
    MXQ_CHECKED(to, 4, return)
    *to = l == 0.f ? __uint_as_float(0xFF800000u) : (m + log2f(l)) * 0.6931471805599453f;
}

// Four elements of an output row, and the row's logarithm with the first of them.
template <int PIECES>
__device__ __forceinline__ void write_row(const AttendArgs& p, size_t row, int dim, int d, const float (&v)[4], float m, float l)
{
    if constexpr (PIECES == 2) {
        float* to = reinterpret_cast<float*>(p.out) + row * dim + d;
        MXQ_CHECKED(to, 16, return)
        *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
        uint8_t* to = p.out + (row * dim + d) * 2;
        MXQ_CHECKED(to, 8, return)
        *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
    if (d == 0) write_lse(p, row, m, l);
}

}  // namespace
}  // namespace mxq
