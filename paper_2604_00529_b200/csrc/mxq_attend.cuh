// Attention over a paged cache of MX codes: out = sum over t of softmax_t(scale q . K^[t]) V^[t], the codes read once.
//
// A row is a query head of a token; the rows that use one cache head read the same keys and values and are worked on together, up
// to 8 NT of them at a time.  An item is one such group of rows, one cache head and the range of keys that its rows see, cut into tiles of
// 64 keys.  All items' tiles, laid end to end, are shared out evenly among the CTAs, whatever the lengths are: a CTA works on a run of
// tiles that may begin and end inside an item, and the parts of such an item are added up, in order, by a second kernel.
//
// A warp takes 16 keys at a time, with the maximum and the sum of a softmax carried along:
//   S^T = K Q^T     keys are the 16 rows of the matrix step, the group's rows its 8 columns; codes become FP16, exactly, and
//                   the sum over a block of 32 is multiplied by its scale in FP32
//   P = 2^(S - m)   m is moved only when a score exceeds it by 2^12; FP16 holds what lies below
//   O^T += V^T P^T  V^T by the transposing load of shared memory; the scales, which belong to (key, block) here, are multiplied
//                   into P, relative to a reference of the block of dimensions.  A step with a scale that lies too far from it (the products
//                   would not be FP16 numbers) takes products relative to each row's largest
//                   instead (far_step), whatever other rows see or what a key weighs
// FP32 rows enter as two FP16 parts, neighbouring columns of the same step, and so do their P.
//
// Bound by HBM for 8-bit codes (64 sequences of 16384 to 32768 tokens, 32 heads over 8 of 128: 6.1 TB/s E4M3, 5.9 INT8), by instructions for 4-bit ones
// (E2M1 4.5 TB/s; issue slots 56 %, ALU pipe 55 %): widening takes 4 instructions per 8 codes of K and 7 of V, which is transposed on the way, of
// some 320 per 16 keys of a warp.  Sequences of up to 8192 tokens, E2M1: 147 us as first written (16 keys at a time, every row of a copy asked for by
// itself, scales worked out by every lane), 126 with two groups of keys per round and offsets in the instructions, 115 with the parts joined by
// one block per item, 110 with one question per fetched step, 112 with a way for scales that are far apart.
#pragma once
#include "mxq_attend_items.cuh"
#include "mxq_attend_plan.cuh"
#include "mxq_kernels.cuh"
#include "mxq_launch.h"
#include "mxq_product.cuh"
#include "mxq_tensor.cuh"

namespace mxq {
namespace {

constexpr int kWarps = 4;                                   // of a CTA, where that is not the launch's choice
constexpr int kGroup = 16;                                  // keys of a matrix step
constexpr int kStagesMax = 6;
constexpr float kBias = 8.f;                                // P is held as 2^kBias times itself: more of FP16's range below 1
constexpr float kSlack = 12.f;                              // m moves when 2^kSlack would be exceeded
// Scales from 2^-below to 2^kAbove of a block's reference are multiplied into P as they are: what FP16 cuts off is then 2^-21 of a row's largest
// product of weight and scale for BF16 rows, where a small first token should not cost time, 2^-24 for FP32 ones.
constexpr int kAbove = 3;
constexpr int below_of(int pieces) { return pieces == 1 ? 8 : 5; }

// ---- codes to FP16 pairs --------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t add_f16(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t mul_f16(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float f16_lo(uint32_t v)
{
    float f;
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, l; }" : "=f"(f) : "r"(v));
    return f;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ void e2m1_word(uint32_t w, uint32_t& b0, uint32_t& b1, uint32_t& b2, uint32_t& b3)
{
    asm("{ .reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, a; cvt.rn.f16x2.e2m1x2 %1, b; cvt.rn.f16x2.e2m1x2 %2, c; cvt.rn.f16x2.e2m1x2 %3, d; }"
        : "=r"(b0), "=r"(b1), "=r"(b2), "=r"(b3) : "r"(w));
}
__device__ __forceinline__ void e4m3_word(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }" : "=r"(lo), "=r"(hi) : "r"(w));
}
// Nibbles i and i + 4 of a word (MXINT4): under the exponent of 1024 a nibble, its sign bit flipped, is 1024 + 8 + its value.
__device__ __forceinline__ void int4_word(uint32_t w, uint32_t (&o)[4])
{
    const uint32_t h = w >> 8;
    o[0] = add_f16((w & 0x000F000Fu) ^ 0x64086408u, 0xE408E408u);                       // - 1032
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(o[1]) : "r"((w & 0x00F000F0u) ^ 0x64806480u), "r"(0x2C002C00u), "r"(0xD480D480u));   // / 16 - 72
    o[2] = add_f16((h & 0x000F000Fu) ^ 0x64086408u, 0xE408E408u);
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(o[3]) : "r"((h & 0x00F000F0u) ^ 0x64806480u), "r"(0x2C002C00u), "r"(0xD480D480u));
}
// Two bytes of a word (MXINT8), the word's sign bits flipped: under the exponent of 1024 a byte is 1024 + 128 + its value.
template <uint32_t SEL>
__device__ __forceinline__ uint32_t int8_pair(uint32_t flipped) { return add_f16(__byte_perm(flipped, 0x64646464u, SEL), 0xE480E480u); }

// K: the word that a lane holds of a row, as pairs of neighbouring elements (MXINT4: elements i and i + 4).
template <int FMT, int NP>
__device__ __forceinline__ void key_pairs(uint32_t w, uint32_t (&o)[NP])
{
    if constexpr (FMT == MXQ_FP4_E2M1) e2m1_word(w, o[0], o[1], o[2], o[3]);
    else if constexpr (FMT == MXQ_INT4) int4_word(w, o);
    else if constexpr (FMT == MXQ_FP8_E4M3) e4m3_word(w, o[0], o[1]);
    else {
        const uint32_t x = w ^ 0x80808080u;
        o[0] = int8_pair<0x4140>(x);
        o[1] = int8_pair<0x4342>(x);
    }
}

// V: x holds 16 bits of key 2t in its lower half and of key 2t + 1 in its upper one, y of keys 2t + 8 and 2t + 9: pairs of two keys'
// codes of the same dimension, X of x and Y of y, dimensions in order.
template <int FMT, int NP>
__device__ __forceinline__ void value_pairs(uint32_t x, uint32_t y, uint32_t (&X)[NP], uint32_t (&Y)[NP])
{
    if constexpr (FMT == MXQ_FP4_E2M1) {
        const uint32_t u = __byte_perm(x, y, 0x5410), w = __byte_perm(x, y, 0x7632);
        e2m1_word((u & 0x0F0F0F0Fu) | ((w << 4) & 0xF0F0F0F0u), X[0], X[2], Y[0], Y[2]);
        e2m1_word(((u >> 4) & 0x0F0F0F0Fu) | (w & 0xF0F0F0F0u), X[1], X[3], Y[1], Y[3]);
    } else if constexpr (FMT == MXQ_INT4) {
        int4_word(x, X);
        int4_word(y, Y);
    } else if constexpr (FMT == MXQ_FP8_E4M3) {
        e4m3_word(__byte_perm(x, x, 0x3120), X[0], X[1]);
        e4m3_word(__byte_perm(y, y, 0x3120), Y[0], Y[1]);
    } else {
        const uint32_t a = x ^ 0x80808080u, b = y ^ 0x80808080u;
        X[0] = int8_pair<0x4240>(a);
        X[1] = int8_pair<0x4341>(a);
        Y[0] = int8_pair<0x4240>(b);
        Y[1] = int8_pair<0x4341>(b);
    }
}

// The top bit of each byte that is an E4M3 NaN code.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) { return ((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

template <int AT>
__device__ __forceinline__ void ldmatrix4(uint32_t at, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4 + %5];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(at), "n"(AT) : "memory");
}
template <int AT>
__device__ __forceinline__ void ldmatrix4_trans(uint32_t at, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4 + %5];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(at), "n"(AT) : "memory");
}

// 16 bytes to shared memory, asynchronously; copy16_some: only the first `size` of them, zeros behind.  (Offsets that are known here go
// into the instructions.)
template <int TO, int FROM>
__device__ __forceinline__ void copy16(uint32_t to, const uint8_t* from)
{
    MXQ_CHECKED(from + FROM, 16, return)
    asm volatile("cp.async.cg.shared.global [%0 + %2], [%1 + %3], 16;" :: "r"(to), "l"(from), "n"(TO), "n"(FROM) : "memory");
}
template <int TO, int FROM>
__device__ __forceinline__ void copy16_some(uint32_t to, const uint8_t* from, uint32_t size)
{
    MXQ_CHECKED(from + FROM, size, size = 0)
    asm volatile("cp.async.cg.shared.global [%0 + %2], [%1 + %3], 16, %4;" :: "r"(to), "l"(from), "n"(TO), "n"(FROM), "r"(size) : "memory");
}

template <int AT = 0>
__device__ __forceinline__ float lds_f32(uint32_t at)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1 + %2];" : "=f"(v) : "r"(at), "n"(AT) : "memory");
    return v;
}
template <int AT = 0>
__device__ __forceinline__ uint32_t lds_u32(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1 + %2];" : "=r"(v) : "r"(at), "n"(AT) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
template <int N, int AT = 0>
__device__ __forceinline__ void lds_words(uint32_t at, uint32_t (&v)[N])      // N = 1, 2, 4, 8
{
    if constexpr (N == 1) {
        asm volatile("ld.shared.u32 %0, [%1 + %2];" : "=r"(v[0]) : "r"(at), "n"(AT) : "memory");
    } else if constexpr (N == 2) {
        asm volatile("ld.shared.v2.u32 {%0,%1}, [%2 + %3];" : "=r"(v[0]), "=r"(v[1]) : "r"(at), "n"(AT) : "memory");
    } else {
        static_for<N / 4>([&](auto k) {
            constexpr int I = 4 * decltype(k)::value;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4 + %5];" : "=r"(v[I]), "=r"(v[I + 1]), "=r"(v[I + 2]), "=r"(v[I + 3]) : "r"(at), "n"(AT + I * 4) : "memory");
        });
    }
}
template <int AT>
__device__ __forceinline__ void sts_u16(uint32_t at, uint32_t v)
{
    asm volatile("st.shared.u16 [%0 + %2], %1;" :: "r"(at), "h"((unsigned short)v), "n"(AT) : "memory");
}

// The first of a chain of matrix steps: sums from zero.
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// ---- layout of shared memory ----------------------------------------------------------------------------------

template <int FMT, int D, int NT>
struct Shape {
    static constexpr int bits = fmt_info(FMT).bits;
    static constexpr int RB = D * bits / 8;                 // bytes of a row of codes
    static constexpr int CPR = RB / 16;                     // its 16-byte chunks
    static constexpr int NB = D / 32;                       // blocks of 32 elements
    static constexpr int MT = D / 16;                       // 16-row tiles of V^T
    static constexpr int NP = bits == 8 ? 2 : 4;            // pairs in a word of codes
    // Keys that a warp takes at a time: two matrix steps where their codes are few, for one round of waiting, page lookup and votes.
    static constexpr int groups = RB <= 64 && NT == 1 ? 2 : 1, step = groups * kGroup;
    // a warp's slot: a step's keys, values and scale bytes
    static constexpr int k_at = 0, v_at = step * RB, ks_at = 2 * step * RB, vs_at = ks_at + step * NB, slot = vs_at + step * NB;
    // tables of a warp's step: the keys' scales (FP32), the values' multipliers (FP16, pairs of keys)
    static constexpr int kf_at = 0, vm_at = step * NB * 4, far_at = vm_at + step * NB * 2;
    static constexpr int tables = far_at + NT * NB * 16;    // far_at: units of the sums, 16 bits each (far_step)
    static constexpr int q_row = D * 2 + (bits == 4 ? 16 : 32);       // padded: lanes of a read lie in different banks
    static constexpr int q_bytes = 8 * NT * q_row;
    static constexpr int columns_at = q_bytes;                        // of each column: its factor, the keys that its row sees
    static constexpr int rows_bytes = q_bytes + 8 * NT * 12;
    static constexpr int ctas = NT == 4 ? 2 : NT * D <= 128 ? 4 : NT * D <= 256 ? 3 : 2;     // of kWarps warps per SM, by registers
    // Warps of a CTA: kWarps, or with one column group as many as an SM holds.
    static constexpr int most = NT > 1 ? kWarps : kWarps * ctas;
    // steps of a warp under way to shared memory, and the one worked on: as many as the CTA's share of an SM holds
    static constexpr int fit = (227 * 1024 / ctas - 1536 - rows_bytes - kWarps * tables) / (kWarps * slot);
    static constexpr int stages = fit < kStagesMax ? fit : kStagesMax;
    static constexpr int ring = stages * slot;
    static constexpr int merge = 8 * NT * (D + 2) * 4;                // a warp's results, in the rings' place
    static constexpr int work = ring > merge ? ring : merge;
    static constexpr size_t total(int warps) { return (size_t)warps * (work + tables) + rows_bytes; }
    // (Heads of 256 leave no registers for their queries: 32 sequences of up to 4096 E4M3 tokens, 8 heads over one, 27.8 us with them there, 25.8 without.)
    static constexpr bool q_in_registers = NT * MT * 2 <= 32 && D < 256;
    static_assert(stages >= 2 && (total(kWarps) + 1536) * ctas <= 227 * 1024, "shared memory");

    // Chunk c of row r lies at r * RB + (c ^ twist(r)) * 16: the eight rows that a matrix load reads at once are in different banks.
    static __host__ __device__ constexpr int twist(int r) { return CPR >= 8 ? r & 7 : CPR == 4 ? (r >> 1) & 3 : (r >> 2) & 1; }
};

template <int FMT, int D, int NT, int PIECES>
struct Attend {
    using S = Shape<FMT, D, NT>;
    static constexpr int NB = S::NB, MT = S::MT, NP = S::NP, GROUPS = S::groups;
    static constexpr bool has_nan = FMT == MXQ_FP8_E4M3;
    static constexpr int kBelow = below_of(PIECES);

    const AttendArgs& p;
    const int warps, warp, lane, g, t;
    uint32_t ring, tables, qs;                              // shared addresses: the warp's ring and tables, the CTA's rows
    uint32_t twisted;                                       // a lane's part of its matrix loads' addresses
    float acc[MT][NT][4], l[NT][2], m[NT][2], f[NT][2];
    // Of the lane's blocks (make_tables), the smallest scale byte that is multiplied into P as it is: kBelow under the reference, which is the
    // unit of the block's sums.  kUnset before a key was seen.
    static constexpr int kUnset = -1000;
    int low[NB * S::step / 32];
    bool apart;                                             // the sums have units of their own, by row and block, in shared memory
    bool steep;                                             // some row's maximum is beyond kSteep
    uint32_t q[S::q_in_registers ? NT * MT : 1][2];
    // the item
    int b, head, row0, rows;                                // rows: how many of the item are there
    Sequence s;
    int some_lo, some_hi, all_lo, all_hi;                   // keys that some row sees, that all rows see

    __device__ __forceinline__ void item(int sequence, int h, int r0, const Sequence& of)
    {
        b = sequence;
        head = h;
        row0 = r0;
        s = of;
        rows = min(p.rows, s.n * p.group - r0);
        const int first = row_token(p, s, r0), last = row_token(p, s, r0 + rows - 1);
        some_lo = token_lo(p, s, first);
        some_hi = token_hi(p, s, last);
        all_lo = token_lo(p, s, last);
        all_hi = token_hi(p, s, first);
    }

    // The first key of a tile of the item, none behind its last key.  (Keys are below 2^31, tiles behind the last one reach no further than
    // one tile beyond it.)
    __device__ __forceinline__ uint32_t tile_key(uint32_t tile) const
    {
        return min((uint32_t)(some_lo >> p.tile_shift << p.tile_shift) + (tile << p.tile_shift), (uint32_t)some_hi);
    }
    // Warps that have keys of these; one where there are none.
    __device__ __forceinline__ int with_keys(uint32_t from, uint32_t to) const { return min(warps, max((int)((to - from + S::step - 1) / S::step), 1)); }

    // -- a step's codes and scales on their way to shared memory

    // Where the lane's chunks of keys and values and its chunk of scales would lie in page 0, and the bytes from page to page.
    const uint8_t *k_lane, *v_lane, *s_lane;
    uint32_t page_bytes, page_scales;
    uint32_t to_codes, to_scales;                           // the same in a slot (chunks of j > 0: see fetch)
    const int* pages_of;                                    // the sequence's page table
    int page_next[GROUPS];                                  // the entries for the next fetch, on their way
    uint32_t there;                                         // bit GROUPS i + h: group h of the step fetched i fetches ago has a page

    __device__ __forceinline__ void place(int h)
    {
        const uint32_t nb = (uint32_t)D >> p.cache.block_shift;
        const size_t rows_before = (size_t)h << p.cache.page_shift;
        page_bytes = ((uint32_t)p.cache.heads << p.cache.page_shift) * S::RB;
        page_scales = ((uint32_t)p.cache.heads << p.cache.page_shift) * nb;
        k_lane = p.cache.kc + rows_before * S::RB + lane * 16;
        v_lane = p.cache.vc + rows_before * S::RB + lane * 16;
        const bool v = lane >= (int)nb;                     // 16 rows' scales are nb chunks
        s_lane = (v ? p.cache.vs : p.cache.ks) + rows_before * nb + (v ? lane - nb : lane) * 16;
        to_scales = (v ? S::vs_at + (lane - nb) * 16 : S::ks_at + lane * 16);
    }
    // (Keys are unsigned on the way: those that a warp looks ahead to may lie beyond 2^31, the most that a sequence has.)
    __device__ __forceinline__ void ask_page(uint32_t key, uint32_t to)
    {
        page_next[0] = ld_int(pages_of + (key >> p.cache.page_shift));
        if constexpr (GROUPS == 2) {
            page_next[1] = page_next[0];
            if (p.cache.page_shift == 4 && key + kGroup < to) page_next[1] = ld_int(pages_of + (key >> 4) + 1);
        }
    }

    // The step of `key`; the next one to be fetched is that of `after`.
    __device__ __forceinline__ void fetch(uint32_t slot, uint32_t key, uint32_t after, uint32_t to)
    {
        there <<= GROUPS;
        if (key < to) {
            uint32_t page[GROUPS];
#pragma unroll
            for (int h = 0; h < GROUPS; ++h) page[h] = (uint32_t)page_next[h];
            if (after < to) ask_page(after, to);
            if constexpr (GROUPS == 2) {
                // Mostly the step lies in one page and every row of it exists: one place, the rest is in the instructions.
                if (p.cache.page_shift > 4 && key + S::step <= (uint32_t)some_hi && page[0] < (uint32_t)p.cache.pages) {
                    there |= 3u;
                    const uint32_t in_page = key & ((1u << p.cache.page_shift) - 1u);
                    const uint32_t nb = (uint32_t)D >> p.cache.block_shift;
                    const size_t off = (size_t)page[0] * page_bytes + in_page * S::RB;
                    const uint8_t *k = k_lane + off, *v = v_lane + off;
                    static_for<S::CPR>([&](auto jc) {
                        constexpr int J = decltype(jc)::value;
                        const uint32_t at = slot + (to_codes ^ (S::twist(J * (32 / S::CPR)) << 4));
                        copy16<S::k_at + J * 512, J * 512>(at, k);
                        copy16<S::v_at + J * 512, J * 512>(at, v);
                    });
                    if (lane < 2 * (int)nb) {
                        const uint8_t* from = s_lane + ((size_t)page[0] * page_scales + in_page * nb);
                        copy16<0, 0>(slot + to_scales, from);
                        copy16<0, 0>(slot + to_scales + kGroup * nb, from + kGroup * nb);
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                    return;
                }
            }
            static_for<GROUPS>([&](auto hc) {
                constexpr int H = decltype(hc)::value;
                const int left = (int)((uint32_t)some_hi - key) - H * kGroup;      // rows from here on that exist
                if (page[H] >= (uint32_t)p.cache.pages || (H > 0 && left <= 0)) return;
                there |= 1u << H;
                const uint32_t in_page = (key + H * kGroup) & ((1u << p.cache.page_shift) - 1u);
                const uint32_t nb = (uint32_t)D >> p.cache.block_shift;
                const size_t off = (size_t)page[H] * page_bytes + in_page * S::RB;
                const uint8_t *k = k_lane + off, *v = v_lane + off;
                constexpr int per = S::CPR / 2;              // chunks of 16 rows per lane: 16 CPR / 32
                constexpr int rows_apart = 32 / S::CPR;
                if (left >= kGroup) {
                    static_for<per>([&](auto jc) {
                        constexpr int J = decltype(jc)::value;
                        const uint32_t at = slot + (to_codes ^ (S::twist(J * rows_apart) << 4));
                        copy16<S::k_at + H * kGroup * S::RB + J * 512, J * 512>(at, k);
                        copy16<S::v_at + H * kGroup * S::RB + J * 512, J * 512>(at, v);
                    });
                } else {
                    static_for<per>([&](auto jc) {
                        constexpr int J = decltype(jc)::value;
                        const uint32_t at = slot + (to_codes ^ (S::twist(J * rows_apart) << 4)), size = lane / S::CPR + J * rows_apart < left ? 16u : 0u;
                        copy16_some<S::k_at + H * kGroup * S::RB + J * 512, J * 512>(at, k, size);
                        copy16_some<S::v_at + H * kGroup * S::RB + J * 512, J * 512>(at, v, size);
                    });
                }
                if (lane < 2 * (int)nb) copy16<0, 0>(slot + to_scales + H * kGroup * nb, s_lane + ((size_t)page[H] * page_scales + in_page * nb));
            });
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }

    // -- the scales of a step, shared out among the lanes: with two groups a lane has a key, with one half of a key's blocks

    static constexpr int LPK = 32 / S::step, HB = NB / LPK; // lanes per key, blocks of a lane

    // Bytes of the lane's blocks (up to eight), from the scale bytes at `at`.
    __device__ __forceinline__ void scale_bytes(uint32_t at, uint32_t (&w)[(HB + 3) / 4]) const
    {
        const int bs = p.cache.block_shift - 5;
        if (bs == 0) {
            const uint32_t from = at + lane * HB;
            if constexpr (HB == 1) w[0] = lds_u8(from);
            else if constexpr (HB == 2) asm volatile("ld.shared.u16 %0, [%1];" : "=r"(w[0]) : "r"(from) : "memory");
            else lds_words(from, w);
            return;
        }
        const uint32_t from = at + (lane / LPK) * (NB >> bs);
#pragma unroll
        for (int j = 0; j < HB; ++j) {
            const uint32_t byte = lds_u8(from + (((lane % LPK) * HB + j) >> bs));
            w[j / 4] = j % 4 ? w[j / 4] | byte << (8 * (j % 4)) : byte;
        }
    }

    // The tables of a step; whether a scale of a value that some row sees lies too far from its block's reference.
    template <bool CAREFUL>
    __device__ __forceinline__ bool make_tables(uint32_t slot, uint32_t key, uint32_t has)
    {
        uint32_t kw[(HB + 3) / 4], vw[(HB + 3) / 4];
        scale_bytes(slot + S::ks_at, kw);
        scale_bytes(slot + S::vs_at, vw);
        const uint32_t mine = key + lane / LPK;
        // seen by no row, or not there
        const bool hidden = CAREFUL && (mine < (uint32_t)some_lo || mine >= (uint32_t)some_hi || !((has >> (lane / LPK / kGroup)) & 1u));
        uint32_t kb[HB], vb[HB];
        bool rare = false;
#pragma unroll
        for (int j = 0; j < HB; ++j) {
            kb[j] = __byte_perm(kw[j / 4], 0, 0x4440 + j % 4);
            vb[j] = __byte_perm(vw[j / 4], 0, 0x4440 + j % 4);
            rare |= kb[j] == 255u || (vb[j] - (uint32_t)low[j] > (uint32_t)(kBelow + kAbove) && !hidden);
        }
        const bool any_rare = __any_sync(0xFFFFFFFFu, rare);
        bool far = false;
        if (any_rare) far = settle(vb, hidden);
        float kf[HB], mult[HB];
#pragma unroll
        for (int j = 0; j < HB; ++j) {
            kf[j] = __uint_as_float(max(kb[j] << 23, 0x00400000u));
            mult[j] = __uint_as_float((vb[j] - (uint32_t)low[j] + (uint32_t)(127 - kBelow)) << 23);
            if (hidden) mult[j] = 0.f;
        }
        uint32_t h[(HB + 1) / 2];
#pragma unroll
        for (int j = 0; j < HB; j += 2) h[j / 2] = pack_f16(mult[j], j + 1 < HB ? mult[j + 1] : 0.f);
        if (any_rare) {                         // poisoned blocks, scales too far away (or just a reference settled)
#pragma unroll
            for (int j = 0; j < HB; ++j) {
                if (kb[j] == 255u) kf[j] = __uint_as_float(0x7FC00000u);
                if (vb[j] - (uint32_t)low[j] > (uint32_t)(kBelow + kAbove)) h[j / 2] &= j & 1 ? 0xFFFFu : 0xFFFF0000u;
                if (vb[j] == 255u && !hidden) h[j / 2] = j & 1 ? (h[j / 2] & 0xFFFFu) | 0x7E000000u : (h[j / 2] & 0xFFFF0000u) | 0x7E00u;
            }
        }
        const uint32_t kt = tables + lane * HB * 4;
        if constexpr (HB == 1) {
            asm volatile("st.shared.f32 [%0], %1;" :: "r"(kt), "f"(kf[0]) : "memory");
        } else if constexpr (HB == 2) {
            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" :: "r"(kt), "f"(kf[0]), "f"(kf[1]) : "memory");
        } else {
            static_for<HB / 4>([&](auto jc) {
                constexpr int J = 4 * decltype(jc)::value;
                asm volatile("st.shared.v4.f32 [%0 + %5], {%1, %2, %3, %4};" :: "r"(kt), "f"(kf[J]), "f"(kf[J + 1]), "f"(kf[J + 2]), "f"(kf[J + 3]), "n"(J * 4) : "memory");
            });
        }
        // the values' multipliers as pairs of keys: [pair][block]
        const int kk = lane / LPK;
        const uint32_t vt = tables + ((kk >> 1) * NB + (lane % LPK) * HB) * 4 + (kk & 1) * 2;
        static_for<HB>([&](auto jc) {
            constexpr int J = decltype(jc)::value;
            sts_u16<S::vm_at + J * 4>(vt, J & 1 ? h[J / 2] >> 16 : h[J / 2]);
        });
        return far;
    }

    // References of blocks that have none yet: the largest scale of the step that some row sees (vb: the bytes of the lane's key and blocks;
    // 251 at most, so that a poisoned block is never near).  Whether a scale lies too far from its block's reference then.
    __device__ __forceinline__ bool settle(const uint32_t (&vb)[HB], bool hidden)
    {
        bool far = false;
#pragma unroll
        for (int j = 0; j < HB; ++j) {
            const bool counts = !hidden && vb[j] != 255u;
            int top = counts ? (int)min(vb[j], 251u) : kUnset;
#pragma unroll
            for (int o = LPK; o < 32; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            if (low[j] == kUnset && top != kUnset) low[j] = top - kBelow;
            far |= counts && vb[j] - (uint32_t)low[j] > (uint32_t)(kBelow + kAbove);
        }
        return __any_sync(0xFFFFFFFFu, far);
    }

    // -- one step

    // Scores of group H, 16 keys x 8 NT columns, without their rows' factors.
    template <int H>
    __device__ __forceinline__ void scores(uint32_t slot, float (&sc)[NT][4]) const
    {
        uint32_t kf_lo[NB], kf_hi[NB];
        lds_words<NB, S::kf_at + H * kGroup * NB * 4>(tables + g * NB * 4, kf_lo);
        lds_words<NB, S::kf_at + H * kGroup * NB * 4 + 32 * NB>(tables + g * NB * 4, kf_hi);
        constexpr int per_load = S::bits == 4 ? 2 : 1;       // blocks of 32 in two chunks
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[n][j] = 0.f;
#pragma unroll
        for (int c = 0; c < S::CPR; c += 2) {
            uint32_t w[2][2];                                // [chunk][row g, row g + 8]
            ldmatrix4<S::k_at + H * kGroup * S::RB>(slot + (twisted ^ (c << 4)), w[0][0], w[0][1], w[1][0], w[1][1]);
#pragma unroll
            for (int h = 0; h < per_load; ++h) {
                const int blk = S::bits == 4 ? c + h : c / 2;
                uint32_t a[2][4];                            // [row g, row g + 8][pairs of the block]
                if constexpr (S::bits == 4) {
                    key_pairs<FMT>(w[h][0], a[0]);
                    key_pairs<FMT>(w[h][1], a[1]);
                } else {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        uint32_t x[2], y[2];
                        key_pairs<FMT>(w[0][r], x);
                        key_pairs<FMT>(w[1][r], y);
                        a[r][0] = x[0];
                        a[r][1] = x[1];
                        a[r][2] = y[0];
                        a[r][3] = y[1];
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint32_t qb[4];
                    q_block(n, blk, qb);
                    float d[4];
                    mma_first(d, a[0][0], a[1][0], a[0][1], a[1][1], qb[0], qb[1]);
                    F16Mma::mma(d, a[0][2], a[1][2], a[0][3], a[1][3], qb[2], qb[3]);
                    const float lo = __uint_as_float(kf_lo[blk]), hi = __uint_as_float(kf_hi[blk]);
                    sc[n][0] = fmaf(d[0], lo, sc[n][0]);
                    sc[n][1] = fmaf(d[1], lo, sc[n][1]);
                    sc[n][2] = fmaf(d[2], hi, sc[n][2]);
                    sc[n][3] = fmaf(d[3], hi, sc[n][3]);
                }
            }
        }
        if constexpr (PIECES == 2) {                         // the two parts' columns are one row's
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                sc[n][0] = sc[n][1] = sc[n][0] + sc[n][1];
                sc[n][2] = sc[n][3] = sc[n][2] + sc[n][3];
            }
        }
    }

    // Hidden scores of a group become -inf; `seen` gets a one (FP16) for each of the others.
    __device__ __forceinline__ void hide(uint32_t key, float (&sc)[NT][4], uint32_t (&seen)[NT][2]) const
    {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            seen[n][0] = seen[n][1] = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t at_column = qs + S::columns_at + (8 * n + 2 * t + j) * 12;
                const uint32_t lo = lds_u32<4>(at_column), hi = lds_u32<8>(at_column);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t at = key + g + 8 * h;
                    const bool on = at >= lo && at < hi;
                    if (!on) sc[n][2 * h + j] = __uint_as_float(0xFF800000u);
                    seen[n][h] |= (on ? 0x3C00u : 0u) << (16 * j);
                }
            }
        }
    }

    // O^T += V^T P^T of group H, P as matrix operands; or (FAR) as the weights of each block, from the scores.
    template <int H, bool CAREFUL, bool FAR = false>
    __device__ __forceinline__ void add_values(uint32_t slot, uint32_t (&pb)[NT][2], const uint32_t (&seen)[NT][2], const float (*sc)[4] = nullptr)
    {
        uint32_t vm_lo[NB], vm_hi[NB];                       // keys 2t, 2t + 1 and 2t + 8, 2t + 9
        lds_words<NB, S::vm_at + H * 8 * NB * 4>(tables + t * NB * 4, vm_lo);
        lds_words<NB, S::vm_at + H * 8 * NB * 4 + 16 * NB>(tables + t * NB * 4, vm_hi);
        uint32_t nan_lo[CAREFUL ? NB : 1], nan_hi[CAREFUL ? NB : 1], any_nan = 0;
        if constexpr (CAREFUL) {                             // poisoned blocks: flags in the place of NaN
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                nan_lo[i] = take_nan(vm_lo[i]);
                nan_hi[i] = take_nan(vm_hi[i]);
                any_nan |= nan_lo[i] | nan_hi[i];
            }
        }
#pragma unroll
        for (int c = 0; c < S::CPR; c += 2) {
            uint32_t w[2][2];                                // [chunk][keys 0 - 7, keys 8 - 15]
            ldmatrix4_trans<S::v_at + H * kGroup * S::RB>(slot + (twisted ^ (c << 4)), w[0][0], w[0][1], w[1][0], w[1][1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int blk = S::bits == 4 ? c + h : c / 2;
                if constexpr (CAREFUL && has_nan) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t bad = nan_bytes(w[h][k]);
                        any_nan |= bad;
                        w[h][k] &= ~((bad >> 7) * 255u);
                    }
                }
                uint32_t X[NP], Y[NP];
                value_pairs<FMT>(w[h][0], w[h][1], X, Y);
                if constexpr (FAR) {
                    if (S::bits == 4 || h == 0) far_weights<H>(slot, blk, sc, pb);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint32_t b0 = FAR ? pb[n][0] : mul_f16(pb[n][0], vm_lo[blk]), b1 = FAR ? pb[n][1] : mul_f16(pb[n][1], vm_hi[blk]);
#pragma unroll
                    for (int j = 0; j < NP / 2; ++j)
                        F16Mma::mma(acc[(c + h) * (NP / 2) + j][n], X[2 * j], X[2 * j + 1], Y[2 * j], Y[2 * j + 1], b0, b1);
                }
            }
        }
        if constexpr (CAREFUL) {
            if (__any_sync(0xFFFFFFFFu, any_nan != 0)) spread_nan<H>(slot, seen, nan_lo, nan_hi);
        }
    }

    // Groups FIRST ... FIRST + N - 1 of a step.
    template <int FIRST, int N, bool CAREFUL>
    __device__ __forceinline__ void step(uint32_t slot, uint32_t key)
    {
        float sc[N][NT][4], x[N][NT][4];                     // scores; times their rows' factors, less m
        uint32_t seen[N][NT][2];
        static_for<N>([&](auto hc) {
            constexpr int H = decltype(hc)::value;
            scores<FIRST + H>(slot, sc[H]);
            if constexpr (CAREFUL) hide(key + (FIRST + H) * kGroup, sc[H], seen[H]);
        });
        float over = 0.f;
#pragma unroll
        for (int h = 0; h < N; ++h)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[h][n][j] = CAREFUL ? less(sc[h][n][j], f[n][j & 1], m[n][j & 1]) : fmaf(sc[h][n][j], f[n][j & 1], -m[n][j & 1]);
                    over = fmaxf(over, x[h][n][j]);
                }
        if (__any_sync(0xFFFFFFFFu, over > kSlack)) raise_maximum<N>(sc, x);
        uint32_t pb[N][NT][2];
#pragma unroll
        for (int h = 0; h < N; ++h)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float e[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) e[j] = exp2_approx(x[h][n][j]);
                l[n][0] += e[0] + e[2];
                if constexpr (PIECES == 1) {
                    l[n][1] += e[1] + e[3];
                    pb[h][n][0] = transpose8x8(pack_f16(e[0], e[1]));
                    pb[h][n][1] = transpose8x8(pack_f16(e[2], e[3]));
                } else {
                    const uint32_t a = pack_f16(e[0], 0.f), c = pack_f16(e[2], 0.f);
                    pb[h][n][0] = transpose8x8(a | pack_f16(0.f, e[0] - f16_lo(a)));
                    pb[h][n][1] = transpose8x8(c | pack_f16(0.f, e[2] - f16_lo(c)));
                }
            }
        static_for<N>([&](auto hc) {
            constexpr int H = decltype(hc)::value;
            add_values<FIRST + H, CAREFUL>(slot, pb[H], seen[H]);
        });
    }

    // A fetched step: all of it at once where every row sees all of it, else group by group.  Without FAR a step with scales that lie too far
    // from their references, or with scores beyond kSteep in front of it, is not taken (false).
    template <bool FAR>
    __device__ __forceinline__ bool take(uint32_t slot, uint32_t key)
    {
        constexpr uint32_t every = (1u << GROUPS) - 1u;
        const uint32_t has = (there >> (GROUPS * (S::stages - 1))) & every;
        const uint32_t lo = (uint32_t)some_lo, hi = (uint32_t)some_hi;
        if (!has || key + S::step <= lo || key >= hi) return true;
        const bool all = has == every && key >= (uint32_t)all_lo && key + S::step <= (uint32_t)all_hi;
        const bool far = (all ? make_tables<false>(slot, key, has) : make_tables<true>(slot, key, has)) || steep;
        __syncwarp();
        if constexpr (FAR) {
            if (far || apart) {                              // (steep is among what makes `far`)
                far_step(slot, key, has);
                return true;
            }
        } else if (far) {
            return false;
        }
        if (all) {
            step<0, GROUPS, false>(slot, key);
        } else {
            static_for<GROUPS>([&](auto hc) {
                constexpr int H = decltype(hc)::value;
                const uint32_t at = key + H * kGroup;
                if (((has >> H) & 1u) && at + kGroup > lo && at < hi) step<H, 1, true>(slot, key);
            });
        }
        return true;
    }

    // FP16 NaN halves of v become zeros and are flagged as ones (0x3C00) in the result.
    static __device__ __forceinline__ uint32_t take_nan(uint32_t& v)
    {
        const uint32_t bit = (v >> 13) & (v >> 14) & 0x00010001u;      // multipliers stay below 2^9: bits 13 and 14 are NaN's
        v &= ~(bit * 0xFFFFu);
        return bit * 0x3C00u;
    }

    // Accumulators of dimensions in which a key that their row sees holds a NaN become NaN: counts such keys by matrix steps.
    template <int H>
    __device__ __forceinline__ void spread_nan(uint32_t slot, const uint32_t (&seen)[NT][2], const uint32_t (&nan_lo)[NB], const uint32_t (&nan_hi)[NB])
    {
        uint32_t vis[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            vis[n][0] = transpose8x8(seen[n][0]);
            vis[n][1] = transpose8x8(seen[n][1]);
        }
#pragma unroll
        for (int c = 0; c < S::CPR; c += 2) {
            uint32_t w[2][2];
            ldmatrix4_trans<S::v_at + H * kGroup * S::RB>(slot + (twisted ^ (c << 4)), w[0][0], w[0][1], w[1][0], w[1][1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int blk = S::bits == 4 ? c + h : c / 2;
#pragma unroll
                for (int j = 0; j < NP / 2; ++j) {
                    uint32_t a[4] = {nan_lo[blk], nan_lo[blk], nan_hi[blk], nan_hi[blk]};
                    if constexpr (has_nan) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const uint32_t bad = nan_bytes(w[h][k]);
                            a[2 * k] |= ((bad >> 7) & 0x00010001u) * 0x3C00u;
                            a[2 * k + 1] |= ((bad >> 15) & 0x00010001u) * 0x3C00u;
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float d[4] = {};
                        F16Mma::mma(d, a[0], a[1], a[2], a[3], vis[n][0], vis[n][1]);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (d[i] > 0.f) acc[(c + h) * (NP / 2) + j][n][i] = __uint_as_float(0x7FC00000u);
                    }
                }
            }
        }
    }

    // A score less m; hidden ones are -inf, which a factor that is NaN must not make NaN of.
    __device__ __forceinline__ float less(float sc, float f, float m) const { return sc == __uint_as_float(0xFF800000u) ? sc : fmaf(sc, f, -m); }
    // The same of the rounded score, for maxima of every size.
    __device__ __forceinline__ float rounded_less(float sc, float f, float m) const { return sc == __uint_as_float(0xFF800000u) ? sc : __fmul_rn(sc, f) - m; }

    // The columns' maxima moved up to the step's scores.
    template <int N>
    __device__ __forceinline__ void raise_maximum(const float (&sc)[N][NT][4], float (&x)[N][NT][4])
    {
        bool high = false;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float top = kNone;
#pragma unroll
                for (int h = 0; h < N; ++h) top = fmaxf(top, fmaxf(less(sc[h][n][j], f[n][j], 0.f), less(sc[h][n][2 + j], f[n][j], 0.f)));
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                const float lower = top - kBias, to = fmaxf(m[n][j], top - lower > kSlack ? top : lower), by = exp2_approx(m[n][j] - to);
                m[n][j] = to;
                high |= fabsf(to) > kSteep && to != kNone;
                l[n][j] *= by;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    acc[i][n][j] *= by;
                    acc[i][n][2 + j] *= by;
                }
#pragma unroll
                for (int h = 0; h < N; ++h) {
                    x[h][n][j] = rounded_less(sc[h][n][j], f[n][j], to);
                    x[h][n][2 + j] = rounded_less(sc[h][n][2 + j], f[n][j], to);
                }
            }
        steep = __any_sync(0xFFFFFFFFu, high);
    }

    // -- a step whose values' scales lie too far apart for weights times multipliers: each row and block has a unit of its own for its sums, 2^(m +
    // unit - 127), which follows the largest product of weight and scale so far, and the weights of a block are worked out from the scores and the
    // scales, in FP32, before they become FP16.  The row's m and l are what they are elsewhere.  Behind the step the sums go back to the blocks' references,
    // to the step's largest scales, where FP32 has room for that; else the units stay (apart), and the next step takes this way too.

    // Two units of a block, of the lane's columns 2t and 2t + 1 of group n.
    __device__ __forceinline__ uint32_t unit_at(int n, int blk) const { return tables + S::far_at + ((blk * NT + n) * 4 + t) * 4; }
    static __device__ __forceinline__ int unit_of(uint32_t units, int j) { return (int)(units << (16 - 16 * j)) >> 16; }
    static __device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23); }
    // The largest sum of a column's block, of all lanes that have some of it.
    __device__ __forceinline__ float largest_sum(int n, int j, int blk) const
    {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a = fmaxf(a, fmaxf(fabsf(acc[2 * blk + i][n][j]), fabsf(acc[2 * blk + i][n][2 + j])));
            if constexpr (PIECES == 2) a = fmaxf(a, fmaxf(fabsf(acc[2 * blk + i][n][1]), fabsf(acc[2 * blk + i][n][3])));
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
        return a;
    }
    // A column's block (of both of its parts) times 2^e.
    __device__ __forceinline__ void scale_sums(int n, int j, int blk, int e)
    {
        const int half = min(max(e, -252), 252) / 2;
        const float by0 = two_to(half), by1 = two_to(min(max(e, -252), 252) - half);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float* const v = acc[2 * blk + i][n];
            v[j] = v[j] * by0 * by1;
            v[2 + j] = v[2 + j] * by0 * by1;
            if constexpr (PIECES == 2) {
                v[1] = v[1] * by0 * by1;
                v[3] = v[3] * by0 * by1;
            }
        }
    }
    static __device__ __forceinline__ int exponent_of(float v) { return (int)(__float_as_uint(v) >> 23) - 127; }

    // Weights times scales of block blk and the 16 keys of group H, as matrix operands, the sums of the block in their units.
    template <int H>
    __device__ __forceinline__ void far_weights(uint32_t slot, int blk, const float (*sc)[4], uint32_t (&pb)[NT][2])
    {
        const int bs = p.cache.block_shift - 5;
        int byte[2];                                         // of keys g and g + 8; a poisoned block's values are taken out elsewhere
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            byte[h] = (int)lds_u8(slot + S::vs_at + (H * kGroup + g + 8 * h) * (NB >> bs) + (blk >> bs));
            if (byte[h] == 255) byte[h] = 0;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t was = lds_u32(unit_at(n, blk));
            int unit[2];
            float w[4];
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 3 - PIECES; ++j) {
                float x[2] = {rounded_less(sc[n][j], f[n][j], m[n][j]), rounded_less(sc[n][2 + j], f[n][j], m[n][j])};
                float top = fmaxf(x[0] + (float)byte[0], x[1] + (float)byte[1]);
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                const float a = largest_sum(n, j, blk);
                const int old = unit_of(was, j);
                // (sums so far at 2^10 or less, products at 2^kBias or less)
                unit[j] = max(a > 0.f ? old + exponent_of(a) - 10 : kUnset, (int)fminf(fmaxf(ceilf(top) - kBias, (float)kUnset), 1000.f));
                scale_sums(n, j, blk, old - unit[j]);
#pragma unroll
                for (int h = 0; h < 2; ++h) w[2 * h + j] = exp2_approx(x[h] + (float)(byte[h] - unit[j]));
            }
            if constexpr (PIECES == 1) {
                pb[n][0] = transpose8x8(pack_f16(w[0], w[1]));
                pb[n][1] = transpose8x8(pack_f16(w[2], w[3]));
            } else {
                unit[1] = unit[0];
                const uint32_t a = pack_f16(w[0], 0.f), c = pack_f16(w[2], 0.f);
                pb[n][0] = transpose8x8(a | pack_f16(0.f, w[0] - f16_lo(a)));
                pb[n][1] = transpose8x8(c | pack_f16(0.f, w[2] - f16_lo(c)));
            }
            if (g == 0) asm volatile("st.shared.u32 [%0], %1;" :: "r"(unit_at(n, blk)), "r"(((uint32_t)unit[0] & 0xFFFFu) | (uint32_t)unit[1] << 16) : "memory");
        }
    }

    template <int H>
    __device__ __forceinline__ void far_group(uint32_t slot, uint32_t key)
    {
        float sc[NT][4];
        uint32_t seen[NT][2], pb[NT][2];
        scores<H>(slot, sc);
        hide(key + H * kGroup, sc, seen);
        bool high = false;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            int down[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float top = fmaxf(less(sc[n][j], f[n][j], 0.f), less(sc[n][2 + j], f[n][j], 0.f));
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                // m moves by a whole number: the sums stay, their units relative to m sink
                const float up = top - m[n][j] > kSlack ? ceilf(top - m[n][j]) - kBias : 0.f, to = m[n][j] == kNone ? fmaxf(top - kBias, kNone) : fminf(m[n][j] + up, fmaxf(top, m[n][j]));
                l[n][j] *= exp2_approx(m[n][j] - to);
                down[j] = (int)fminf(rintf(to - m[n][j]), 4000.f);
                m[n][j] = to;
                high |= fabsf(to) > kSteep && to != kNone;
                l[n][j] += exp2_approx(rounded_less(sc[n][j], f[n][j], to)) + exp2_approx(rounded_less(sc[n][2 + j], f[n][j], to));
            }
#pragma unroll 1
            for (int blk = 0; blk < NB; ++blk) {
                const uint32_t at = unit_at(n, blk), was = lds_u32(at);
                __syncwarp();
                const int u0 = max(unit_of(was, 0) - down[0], kUnset), u1 = max(unit_of(was, 1) - down[1], kUnset);
                if (g == 0) asm volatile("st.shared.u32 [%0], %1;" :: "r"(at), "r"(((uint32_t)u0 & 0xFFFFu) | (uint32_t)u1 << 16) : "memory");
            }
        }
        steep = __any_sync(0xFFFFFFFFu, high);
        __syncwarp();
        add_values<H, true, true>(slot, pb, seen, sc);
        __syncwarp();
    }

    __device__ __forceinline__ void far_step(uint32_t slot, uint32_t key, uint32_t has)
    {
        if (!apart) {
#pragma unroll
            for (int blk = 0; blk < NB; ++blk) {
                const uint32_t unit = (uint32_t)max(__shfl_sync(0xFFFFFFFFu, low[blk % HB], blk / HB) + kBelow, kUnset) & 0xFFFFu;
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    if (g == 0) asm volatile("st.shared.u32 [%0], %1;" :: "r"(unit_at(n, blk)), "r"(unit | unit << 16) : "memory");
            }
            __syncwarp();
        }
        static_for<GROUPS>([&](auto hc) {
            constexpr int H = decltype(hc)::value;
            const uint32_t at = key + H * kGroup;
            if (((has >> H) & 1u) && at + kGroup > (uint32_t)some_lo && at < (uint32_t)some_hi) far_group<H>(slot, key);
        });
        // back to references: the step's largest scales, but for blocks of zeros
        int to[HB];
        uint32_t vw[(HB + 3) / 4];
        scale_bytes(slot + S::vs_at, vw);
        const uint32_t mine = key + lane / LPK;
        const bool hidden = mine < (uint32_t)some_lo || mine >= (uint32_t)some_hi || !((has >> (lane / LPK / kGroup)) & 1u);
#pragma unroll
        for (int j = 0; j < HB; ++j) {
            const uint32_t byte = __byte_perm(vw[j / 4], 0, 0x4440 + j % 4);
            int top = hidden || byte == 255u ? 0 : (int)min(byte, 251u);
#pragma unroll
            for (int o = LPK; o < 32; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            to[j] = top > 0 ? top : max(low[j] + kBelow, 0);
        }
        bool fits = true;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) {
            const int unit = __shfl_sync(0xFFFFFFFFu, to[blk % HB], blk / HB);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 3 - PIECES; ++j) {
                    const float a = largest_sum(n, j, blk);
                    const int e = exponent_of(a) + unit_of(lds_u32(unit_at(n, blk)), j) - unit;
                    fits &= !(a > 0.f && a < __uint_as_float(0x7F800000u)) || (e >= -60 && e <= 90);
                }
        }
        apart = !__all_sync(0xFFFFFFFFu, fits);
        if (apart) return;
#pragma unroll
        for (int blk = 0; blk < NB; ++blk) {
            const int unit = __shfl_sync(0xFFFFFFFFu, to[blk % HB], blk / HB);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 3 - PIECES; ++j) scale_sums(n, j, blk, unit_of(lds_u32(unit_at(n, blk)), j) - unit);
        }
#pragma unroll
        for (int j = 0; j < HB; ++j) low[j] = to[j] - kBelow;
        __syncwarp();
    }

    // Sums in units of their own become the warp's results: divided by the weights' sum, then times their units.
    __device__ __forceinline__ void give_back_units()
    {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 3 - PIECES; ++j) {
                float sum = l[n][j];
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    acc[i][n][j] *= inv;
                    acc[i][n][2 + j] *= inv;
                    if constexpr (PIECES == 2) {
                        acc[i][n][1] *= inv;
                        acc[i][n][3] *= inv;
                    }
                }
#pragma unroll
                for (int blk = 0; blk < NB; ++blk) scale_sums(n, j, blk, unit_of(lds_u32(unit_at(n, blk)), j) - 127);
            }
    }

    // -- rows

    // The step operands of block blk and column group n: four pairs of column g.
    __device__ __forceinline__ void q_block(int n, int blk, uint32_t (&o)[4]) const
    {
        if constexpr (S::q_in_registers) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                o[2 * i] = q[n * MT + 2 * blk + i][0];
                o[2 * i + 1] = q[n * MT + 2 * blk + i][1];
            }
        } else {
            load_q_block(n, blk, o);
        }
    }
    __device__ __forceinline__ void load_q_block(int n, int blk, uint32_t (&o)[4]) const
    {
        const uint32_t at = qs + (8 * n + g) * S::q_row + blk * 64;
        if constexpr (S::bits == 4) {
            lds_words<4>(at + t * 16, o);
        } else {
            uint32_t x[2], y[2];
            lds_words<2>(at + t * 8, x);
            lds_words<2>(at + 32 + t * 8, y);
            o[0] = x[0];
            o[1] = x[1];
            o[2] = y[0];
            o[3] = y[1];
        }
    }

    // The item's rows to shared memory as FP16 parts, each row times the power of two that brings its largest element to
    // [2^14, 2^15): BF16's eight bits fit FP16's eleven, down to 2^-31 of the largest.  The columns get the factor that
    // takes that back and the keys that their rows see.
    __device__ __forceinline__ void load_rows() const
    {
        constexpr int per = D / 32, columns = 8 * NT / kWarps;         // of a lane; of a warp, at most
        float all[columns][per];
#pragma unroll
        for (int k = 0; k < columns; ++k) {                  // (all of them under way before the first is looked at)
            const int c = warp + k * warps, r = c / PIECES, row = row0 + min(r, rows - 1);
#pragma unroll
            for (int i = 0; i < per; ++i) all[k][i] = 0.f;
            if (c < 8 * NT && r < rows) {
                const int i = row_token(p, s, row);
                const uint8_t* at = p.q + (size_t)(s.first + i) * p.q_token + (size_t)(head * p.group + row - i * p.group) * p.q_head;
                if constexpr (PIECES == 2) {
#pragma unroll
                    for (int j = 0; j < per; ++j) all[k][j] = __uint_as_float(ld_u32(at + (lane * per + j) * 4));
                } else {
#pragma unroll
                    for (int j = 0; j < per; j += 2) {
                        const uint32_t x = ld_u32(at + (lane * per + j) * 2);
                        all[k][j] = __uint_as_float(x << 16);
                        all[k][j + 1] = __uint_as_float(x & 0xFFFF0000u);
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < columns; ++k) {
            const int c = warp + k * warps, row = row0 + min(c / PIECES, rows - 1);
            if (c >= 8 * NT) break;
            const float(&v)[per] = all[k];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < per; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
            top = __reduce_max_sync(0xFFFFFFFFu, top) >> 23;
            const int up = 127 + 14 - (int)max(top, 1u), half = up / 2;
            const float by0 = __uint_as_float((uint32_t)(127 + half) << 23), by1 = __uint_as_float((uint32_t)(127 + up - half) << 23);
            const float back0 = __uint_as_float((uint32_t)(127 - half) << 23), back1 = __uint_as_float((uint32_t)(127 - up + half) << 23);
#pragma unroll
            for (int i = 0; i < per; ++i) {
                const float x = v[i] * by0 * by1;
                uint32_t h = pack_f16(x, 0.f);
                if (PIECES == 2 && c % 2 == 1) h = pack_f16(x - f16_lo(h), 0.f);
                int e = lane * per + i;                      // MXINT4's pairs are elements i and i + 4 of eight
                if constexpr (FMT == MXQ_INT4) e = (e & ~7) | (e & 3) << 1 | ((e >> 2) & 1);
                asm volatile("st.shared.u16 [%0], %1;" :: "r"(qs + c * S::q_row + e * 2), "h"((unsigned short)h) : "memory");
            }
            if (lane == 0) {
                float back = p.scale * back0 * back1;
                if (top == 255u) back = __uint_as_float(0x7FC00000u);
                const uint32_t at = qs + S::columns_at + c * 12;
                asm volatile("st.shared.f32 [%0], %1;" :: "r"(at), "f"(back) : "memory");
                asm volatile("st.shared.u32 [%0 + 4], %1;" :: "r"(at), "r"(token_lo(p, s, row_token(p, s, row))) : "memory");
                asm volatile("st.shared.u32 [%0 + 8], %1;" :: "r"(at), "r"(token_hi(p, s, row_token(p, s, row))) : "memory");
            }
        }
    }

    // -- a run of keys [from, to) of the item, from a multiple of a tile on

    __device__ __forceinline__ void run(uint32_t from, uint32_t to)
    {
        place(head);
        pages_of = p.batch.table + (size_t)b * p.batch.width;
        there = 0;
        uint32_t key = from + warp * S::step;
        const uint32_t stride = warps * S::step;
        if (key < to) ask_page(key, to);
#pragma unroll
        for (int i = 0; i < S::stages - 1; ++i) fetch(ring + i * S::slot, key + i * stride, key + (i + 1) * stride, to);
        load_rows();
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f[n][j] = lds_f32(qs + S::columns_at + (8 * n + 2 * t + j) * 12);
                m[n][j] = kNone;
                l[n][j] = 0.f;
            }
        if constexpr (S::q_in_registers) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int blk = 0; blk < NB; ++blk) {
                    uint32_t o[4];
                    load_q_block(n, blk, o);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        q[n * MT + 2 * blk + i][0] = o[2 * i];
                        q[n * MT + 2 * blk + i][1] = o[2 * i + 1];
                    }
                }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][n][j] = 0.f;
#pragma unroll
        for (int j = 0; j < HB; ++j) low[j] = kUnset;
        apart = steep = false;
        int slot = 0, next = S::stages - 1;
        auto next_step = [&] {
            const uint32_t ahead = key + (S::stages - 1) * stride;
            fetch(ring + next * S::slot, ahead, ahead + stride, to);
            asm volatile("cp.async.wait_group %0;" :: "n"(S::stages - 1) : "memory");
            __syncwarp();
        };
        auto step_done = [&] {
            __syncwarp();
            slot = slot + 1 == S::stages ? 0 : slot + 1;
            next = next + 1 == S::stages ? 0 : next + 1;
            key += stride;
        };
        bool near = true;
        while (key < to) {
            next_step();
            near = take<false>(ring + slot * S::slot, key);
            if (!near) break;
            step_done();
        }
        // The first step with scales far apart and all behind it: a loop of its own, whose registers are not the common one's.  (64 sequences of up
        // to 8192 tokens, E2M1, none of it far: 112 us; 115 with everything in one loop; 110 without a way for scales that are far apart.)
        while (!near) {
            take<true>(ring + slot * S::slot, key);
            step_done();
            if (key >= to) break;
            next_step();
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
    }

    // -- the warps' results together: normalized sums and their weights in shared memory, then to the output or to a part

    // (some: warps that had keys, one at least; share: CTAs of the cluster that has the item, 0 without one)
    __device__ __forceinline__ void finish(float* area, bool whole, uint8_t* part, int some, int share)
    {
        constexpr int R = 8 * NT / PIECES;                   // rows of the tile
        float* const o_at = area + warp * R * D;
        float* const ml = area + warps * R * D;             // [warp][row][m, l]
        float* const shared_ml = area + (size_t)warps * S::work / 4;          // [row][m, l] for the cluster, where the first warp's tables were
        if (warp < some) {
            float scales[NB];
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const int byte = __shfl_sync(0xFFFFFFFFu, low[i % HB], i / HB) + kBelow;
                scales[i] = apart ? 1.f : scale_value((uint32_t)max(byte, 0));
            }
            if (apart) give_back_units();
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 3 - PIECES; ++j) {
                    float sum = l[n][j];
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                    const float inv = apart ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
                    const int r = PIECES == 1 ? 8 * n + 2 * t + j : 4 * n + t;
                    if (g == 0) {
                        ml[(warp * R + r) * 2] = m[n][j];
                        ml[(warp * R + r) * 2 + 1] = sum;
                    }
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        float x = acc[i][n][j], y = acc[i][n][2 + j];
                        if constexpr (PIECES == 2) {
                            x += acc[i][n][1];
                            y += acc[i][n][3];
                        }
                        const int d = S::bits == 4 ? (i >> 1) * 32 + 4 * g + (i & 1) * 2 : i * 16 + 2 * g;
                        *reinterpret_cast<float2*>(o_at + r * D + d) = make_float2(x * inv * scales[i >> 1], y * inv * scales[i >> 1]);
                    }
                }
        }
        __syncthreads();
        for (int at = threadIdx.x; at < rows * (D / 4); at += warps * 32) {
            const int r = at / (D / 4), d = at % (D / 4) * 4;
            float top = kNone;
#pragma unroll 4
            for (int w = 0; w < some; ++w) top = fmaxf(top, ml[(w * R + r) * 2]);
            float sum = 0.f, v[4] = {};
#pragma unroll 4
            for (int w = 0; w < some; ++w) {
                const float wt = ml[(w * R + r) * 2 + 1] * exp2_approx(ml[(w * R + r) * 2] - top);
                const float4 x = *reinterpret_cast<const float4*>(area + (w * R + r) * D + d);
                sum += wt;
                v[0] += wt * x.x;
                v[1] += wt * x.y;
                v[2] += wt * x.z;
                v[3] += wt * x.w;
            }
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= inv;
            if (share > 1) {                                 // (this thread alone has read what lies here)
                *reinterpret_cast<float4*>(area + r * D + d) = make_float4(v[0], v[1], v[2], v[3]);
                if (d == 0) reinterpret_cast<float2*>(shared_ml)[r] = make_float2(top, sum);
            } else if (whole) {
                put(r, d, v, top, sum);
            } else {
                float* const to = reinterpret_cast<float*>(part);
                MXQ_CHECKED(to + r * D + d, 16, continue)
                *reinterpret_cast<float4*>(to + r * D + d) = make_float4(v[0], v[1], v[2], v[3]);
                if (d == 0) write_weight(to + p.rows * D + 2 * r, top, sum);
            }
        }
        if (share > 1) {
            cluster_sync();
            const uint32_t at = smem_addr(area), at_ml = smem_addr(shared_ml);
            for (int slot = threadIdx.x * share + cluster_rank(); slot < rows * (D / 4); slot += warps * 32 * share) {
                const int r = slot / (D / 4), d = slot % (D / 4) * 4;
                float top = kNone, sum = 0.f, v[4] = {};
#pragma unroll 8
                for (int c = 0; c < share; ++c) top = fmaxf(top, ld_peer(peer_addr(at_ml + r * 8, c)));
#pragma unroll 8
                for (int c = 0; c < share; ++c) {
                    const float wt = ld_peer(peer_addr(at_ml + r * 8 + 4, c)) * exp2_approx(ld_peer(peer_addr(at_ml + r * 8, c)) - top);
                    const float4 x = ld_peer4(peer_addr(at + (r * D + d) * 4, c));
                    sum += wt;
                    v[0] += wt * x.x;
                    v[1] += wt * x.y;
                    v[2] += wt * x.z;
                    v[3] += wt * x.w;
                }
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] *= inv;
                put(r, d, v, top, sum);
            }
            cluster_sync();                                  // no CTA leaves while another one reads its sums
        } else {
            __syncthreads();
        }
    }
    __device__ __forceinline__ void put(int r, int d, const float (&v)[4], float top, float sum) const
    {
        const int row = row0 + r, i = row_token(p, s, row);
        write_row<PIECES>(p, (size_t)(s.first + i) * (p.cache.heads * p.group) + head * p.group + row - i * p.group, D, d, v, top, sum);
    }
};

template <int FMT, int D, int NT, int PIECES>
__global__ void __launch_bounds__(Shape<FMT, D, NT>::most * 32, NT == 1 ? 1 : Shape<FMT, D, NT>::ctas)
attend_kernel(const __grid_constant__ AttendArgs p)
{
    using S = Shape<FMT, D, NT>;
    extern __shared__ __align__(1024) uint8_t shared[];
    __shared__ Plan plan;
    __shared__ uint32_t warp_sum[32];
    pdl_acquire();
    pdl_release();                                           // (the second kernel reads nothing before its own wait)
    const int warps = NT == 1 ? p.warps : kWarps;
    const uint32_t base = smem_addr(shared);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Attend<FMT, D, NT, PIECES> a{p, warps, warp, lane, lane >> 2, lane & 3};
    a.ring = base + warp * S::ring;
    a.tables = base + warps * S::work + warp * S::tables;
    a.qs = base + warps * (S::work + S::tables);
    a.to_codes = (lane / S::CPR) * S::RB + ((lane % S::CPR ^ S::twist(lane / S::CPR)) << 4);
    // matrix i of a load: keys 8 (i & 1) ..., chunk i >> 1; the lane gives the address of row lane % 8 of matrix lane / 8
    a.twisted = (((lane >> 3) & 1) * 8 + (lane & 7)) * S::RB + (((lane >> 4) ^ S::twist(lane & 7)) << 4);
    uint8_t* const parts = p.ws + (size_t)p.ctas * sizeof(PartMeta);
    PartMeta* const meta = reinterpret_cast<PartMeta*>(p.ws) + blockIdx.x;
    const size_t part = part_bytes(p.rows, D);
    // A cluster's item, its tiles by rank, one token per sequence; or a run of tiles.
    const int share = NT == 1 ? p.share : 0;
    bool first = true, whole = true;
    uint32_t from_key = 0, to_key = 0;
    if (share) {
        const int item = blockIdx.x / share, rank = share > 1 ? (int)cluster_rank() : 0, b = item / p.cache.heads;
        const Sequence s = sequence(p.batch, b, p.cache.page_shift);
        const uint32_t tiles = sequence_tiles(p, s);
        a.item(b, item - b * p.cache.heads, 0, s);
        from_key = a.tile_key(tiles * rank / share);
        to_key = a.tile_key(tiles * (rank + 1) / share);
    } else {
        make_plan(p, warps, plan, warp_sum);
        if (plan.from >= plan.to && threadIdx.x == 0) {
            bool ok = true;
            MXQ_CHECKED(meta, sizeof(PartMeta), ok = false)
            if (ok) *meta = PartMeta{0, 0, 0, plan.total, 0, 0, 0, 0};
        }
    }
    while (share || plan.from < plan.to) {
        if (!share) {
            a.item(plan.b, plan.head, plan.r0, plan.s);
            const uint32_t end = min(plan.item + plan.tiles, plan.to);
            from_key = a.tile_key(plan.from - plan.item);
            to_key = a.tile_key(end - plan.item);
            whole = plan.from == plan.item && end == plan.item + plan.tiles;
        }
        a.run(from_key, to_key);
        if (first && !share && threadIdx.x == 0) {
            bool ok = true;
            MXQ_CHECKED(meta, sizeof(PartMeta), ok = false)
            if (ok) *meta = PartMeta{plan.from, plan.item, plan.item + plan.tiles, plan.total, a.s.first, a.head, a.row0, a.rows};
        }
        a.finish(reinterpret_cast<float*>(shared), whole, parts + ((size_t)blockIdx.x * 2 + (first ? 0 : 1)) * part, a.with_keys(from_key, to_key), share);
        if (share) break;
        first = false;
        if (threadIdx.x == 0) next_item(p, plan);
        __syncthreads();
    }
}

// ---- launches -------------------------------------------------------------------------------------------------

template <int FMT, int D, int NT, int PIECES>
int run(const AttendArgs& p, cudaStream_t stream)
{
    using S = Shape<FMT, D, NT>;
    static std::atomic<uint64_t> done{0};
    auto kern = attend_kernel<FMT, D, NT, PIECES>;
    if (int rc = allow_smem(reinterpret_cast<const void*>(kern), S::total(S::most), done)) return rc;
    return launch_grid(kern, dim3((unsigned)p.ctas), p.warps * 32, S::total(p.warps), p.share > 1 ? p.share : 1, stream, p);
}

// (Four column groups: FP32 rows alone, since BF16 ones are many before that, and heads of 256 leave no registers.)
template <int FMT, int D, int PIECES>
int by_columns(int nt, const AttendArgs& p, cudaStream_t stream)
{
    if (nt == 1) return run<FMT, D, 1, PIECES>(p, stream);
    if constexpr (PIECES == 2 && D < 256) {
        if (nt == 4) return run<FMT, D, 4, PIECES>(p, stream);
    }
    return nt == 2 ? run<FMT, D, 2, PIECES>(p, stream) : MXQ_ERR_SIZE;
}

template <int FMT, int PIECES>
int by_dim(int dim, int nt, const AttendArgs& p, cudaStream_t stream)
{
    if (dim == 64) return by_columns<FMT, 64, PIECES>(nt, p, stream);
    if (dim == 128) return by_columns<FMT, 128, PIECES>(nt, p, stream);
    return by_columns<FMT, 256, PIECES>(nt, p, stream);
}

}  // namespace

// The first kernel for a cache of format FMT: its `nt` column groups, 16- or 32-bit rows.
template <int FMT>
int launch_attend(int dim, int nt, int dtype, const AttendArgs& p, cudaStream_t stream)
{
    return dtype == MXQ_F32 ? by_dim<FMT, 2>(dim, nt, p, stream) : by_dim<FMT, 1>(dim, nt, p, stream);
}

}  // namespace mxq
