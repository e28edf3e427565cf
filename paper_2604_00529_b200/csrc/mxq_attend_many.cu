// Attention over a paged cache of MX codes where sequences bring many queries (a piece of a prompt): bound by the tensor cores, so
// both products are on the fifth-generation ones.  A CTA works on two tiles of 128 rows (rows and runs of tiles as in mxq_attend.cuh)
// against tiles of 128 keys:
//   warps 0 - 3, 4 - 7   a tile of rows each, a row per thread: S from tensor memory, the softmax with its maximum and sum
//                        carried along, P as BF16 back into tensor memory over S; the sums O are rescaled there in the rare case that m moves
//   warps 8 - 15         codes of keys and values from global memory, a tile ahead in registers, widened to BF16 with their scales
//                        multiplied in (exact: eight significant bits, a power of two), into swizzled shared memory
//   warp 16              issues S_i = Q_i K^T and O_i += P_i V for the two row tiles in turn, so that one's softmax overlaps the other's products
// Queries are BF16 as they are.  P is rounded to BF16, by 2^-8 of a weight or less, because V^ is BF16 and both operands of a product have one
// type (FP16 would hold P to 11 bits, but not every V^): results are 2.3e-3 in norm from 64 bits, where the output's own rounding is 1.7e-3.  The
// sum is that of the rounded weights, so that they add up to one: a row that sees one key gives that key's value.  Sums are FP32.
//
// 2048 queries over 8192 tokens, 32 heads over 8 of 128, E2M1: 348 us, 690 TFLOP/s.  A pair of row tiles takes 5300 cycles per tile of keys (at 360 us): 3300 for
// a row tile's softmax (its exponentials alone 1024, two warps of each scheduler at it), 1400 until its scores are there, 500 of waiting; the
// products themselves take 2900.  With the maximum found in a pass of its own the softmax took 5900 cycles (495 us); 16 scores at a time with the next
// ones on their way 3900 (384 us).
#include "mxq_attend_items.cuh"
#include "mxq_attend_plan.cuh"
#include "mxq_launch.h"
#include "mxq_product.cuh"
#include "mxq_tensor.cuh"

namespace mxq {
namespace {

__device__ unsigned int g_many_status;                       // a bounded wait gave up

constexpr int kRowWarps = 8, kWideners = 8, kIssuer = kRowWarps + kWideners, kManyWarps = kIssuer + 1, kManyThreads = kManyWarps * 32;
constexpr int kRowTile = 128, kKeys = 128;
constexpr float kManySlack = 8.f;                            // m moves when 2^8 would be exceeded
constexpr uint32_t kLoudByte = 247;                          // the smallest scale under which an element (448, E4M3) passes BF16's range

template <int FMT, int D>
struct ManyShape {
    using W = Widen<FMT>;
    static constexpr int bits = W::bits, RB = D * bits / 8, CPR = RB / 16, NB = D / 32, panels = D / 64, NP = W::NP;
    static constexpr int panel = kKeys * 128;                // bytes: 128 rows of 64 elements
    static constexpr int q_bytes = 2 * panels * kRowTile * 128, stage = panels * panel;
    static constexpr int k_at = q_bytes, v_at = k_at + 2 * stage, nan_at = v_at + 2 * stage, absent_at = nan_at + 2 * kKeys * NB * 4;
    static constexpr int total = absent_at + 2 * kKeys + 1024;
    static constexpr int chunks = kKeys * CPR / (kWideners * 32);      // of 16 bytes of codes per widening thread
    // tensor memory: S (P over it) and O of both row tiles
    static constexpr uint32_t s_cols = kKeys, o_at = 2 * s_cols, cols = 512;
};

// Instruction descriptor of kind::f16: BF16 x BF16, FP32 sums of 128 x n; A K-major, B K-major or (transposed) N-major.
__host__ __device__ constexpr uint32_t bf16_desc(int n, bool b_by_n)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)b_by_n << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
}
// Shared-memory descriptor of an operand whose rows of 128 bytes (64 elements of n, 128-byte swizzle) follow k: groups of eight k are
// 1024 bytes apart, the next 64 elements of n a panel.
__device__ __forceinline__ uint64_t by_n_desc(uint32_t addr, uint32_t panel)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(panel >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// The first operand from tensor memory, two elements of k in a column.
__device__ __forceinline__ void mma_bf16_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc)
{
    asm volatile("{ .reg .pred p; setp.eq.u32 p, 0, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc) : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                    "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
                 :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                    "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
                    "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void st_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" :: "r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Two FP32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{ .reg .b64 x, y, z, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 w, x, y, z; mov.b64 {%0, %1}, w; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{ .reg .b64 x, y, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 w, x, y; mov.b64 {%0, %1}, w; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// A row's sums in tensor memory times `by`.
template <int D>
__device__ __forceinline__ void rescale_sums(uint32_t oc, float by)
{
#pragma unroll 1
    for (int c = 0; c < D; c += 32) {
        uint32_t v[32];
        tmem_ld32(v, oc + c);
        tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * by);
        tmem_st32(oc + c, v);
    }
    tmem_st_wait();
}
__device__ __forceinline__ void tmem_ld16(uint32_t (&r)[16], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr));
}

// The top bit of each byte that is an E4M3 NaN code.
__device__ __forceinline__ uint32_t nan_codes(uint32_t x) { return ((x & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// Where element e of a row lies among the widened ones: codes widen in the order of order_pairs.
template <int NP>
__host__ __device__ constexpr int widened_place(int e)
{
    return NP == 4 ? (e & ~7) | (e & 3) << 1 | ((e >> 2) & 1) : (e & ~3) | (e & 1) << 1 | ((e >> 1) & 1);
}

// What all warps know of the item.
struct ManyItem {
    int b, head, row0, rows, some_lo, some_hi, all_lo, all_hi, from, to;
};

struct ManyBars {
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_ready[2], o_full;
};

template <int FMT, int D>
__global__ void __launch_bounds__(kManyThreads, 1)
attend_many_kernel(const __grid_constant__ AttendArgs p)
{
    using M = ManyShape<FMT, D>;
    using W = Widen<FMT>;
    constexpr int NB = M::NB, NP = M::NP;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) ManyBars bars;
    __shared__ Plan plan;
    __shared__ uint32_t warp_sum[32], s_tmem, s_gave_up;
    __shared__ uint32_t s_info[2][kWideners];                // of a tile of values: 1: some key has no page, 2: something that is no finite number was taken out
    __shared__ uint8_t s_bad[2 * kRowTile];                  // rows whose query holds a NaN or an infinity
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    uint8_t* const base_p = raw + (base - smem_addr(raw));
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&bars.k_full[i]), kWideners);
            mbar_init(smem_addr(&bars.k_empty[i]), 1);
            mbar_init(smem_addr(&bars.v_full[i]), kWideners);
            mbar_init(smem_addr(&bars.v_empty[i]), 1);
            mbar_init(smem_addr(&bars.s_full[i]), 1);
            mbar_init(smem_addr(&bars.p_ready[i]), 4);
        }
        mbar_init(smem_addr(&bars.o_full), 1);
        s_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssuer) tmem_alloc<1>(smem_addr(&s_tmem), M::cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_acquire();
    pdl_release();                                           // (the second kernel reads nothing before its own wait)
    make_plan(p, kManyWarps, plan, warp_sum);
    auto wait = [&](uint64_t& bar, uint32_t parity) { return mbar_wait(smem_addr(&bar), parity, &s_gave_up, &g_many_status); };

    PartMeta* const meta = reinterpret_cast<PartMeta*>(p.ws) + blockIdx.x;
    uint8_t* const parts = p.ws + (size_t)p.ctas * sizeof(PartMeta);
    const size_t part = part_bytes(p.rows, D);
    bool first = true, ok = true;
    uint32_t n0 = 0, n1 = 0, pieces = 0;                     // tiles that the first and the second row tile have seen, pieces done
    if (plan.from >= plan.to && threadIdx.x == 0) {
        bool good = true;
        MXQ_CHECKED(meta, sizeof(PartMeta), good = false)
        if (good) *meta = PartMeta{0, 0, 0, plan.total, 0, 0, 0, 0};
    }
    while (plan.from < plan.to) {
        ManyItem it;
        const Sequence s = plan.s;
        const uint32_t item = plan.item, tiles = plan.tiles, at = plan.from, end = min(item + tiles, plan.to);
        {
            const int r0 = plan.r0;
            it.b = plan.b;
            it.head = plan.head;
            it.row0 = r0;
            it.rows = min(p.rows, s.n * p.group - r0);
            const int t0 = row_token(p, s, r0), t1 = row_token(p, s, r0 + it.rows - 1);
            it.some_lo = token_lo(p, s, t0);
            it.some_hi = token_hi(p, s, t1);
            it.all_lo = token_lo(p, s, t1);
            it.all_hi = token_hi(p, s, t0);
            const uint32_t key0 = (uint32_t)(it.some_lo >> p.tile_shift << p.tile_shift);
            it.from = (int)min(key0 + ((at - item) << p.tile_shift), (uint32_t)it.some_hi);
            it.to = (int)min(key0 + ((end - item) << p.tile_shift), (uint32_t)it.some_hi);
        }
        const bool two = it.rows > kRowTile, whole = at == item && end == item + tiles;
        const int count = (int)(((uint32_t)it.to - (uint32_t)it.from + kKeys - 1) / kKeys);       // key tiles, maybe none

        // rows to shared memory, in the order that the keys' elements are widened in; O from zero
        for (int i = threadIdx.x; i < 2 * kRowTile; i += kManyThreads) s_bad[i] = 0;
        __syncthreads();
        if (ok) {
            constexpr int batch = 4;                         // loads under way per thread
            const int pieces16 = (two ? 2 : 1) * kRowTile * (D / 8);
            for (int c0 = threadIdx.x; c0 < pieces16; c0 += kManyThreads * batch) {
                uint4 v[batch];
#pragma unroll
                for (int k = 0; k < batch; ++k) {
                    const int c = c0 + k * kManyThreads, r = c / (D / 8), e = c % (D / 8);       // eight elements
                    v[k] = make_uint4(0, 0, 0, 0);
                    if (r < it.rows) {
                        const int row = it.row0 + r, i = row_token(p, s, row);
                        v[k] = ld_once(p.q + (size_t)(s.first + i) * p.q_token + (size_t)(it.head * p.group + row - i * p.group) * p.q_head + e * 16);
                    }
                }
#pragma unroll
                for (int k = 0; k < batch; ++k) {
                    const int c = c0 + k * kManyThreads, r = c / (D / 8), e = c % (D / 8);
                    if (c >= pieces16) continue;
                    const uint32_t x[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
                    uint32_t o[4];
                    bool bad = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j) bad |= (x[j] & 0x7F80u) == 0x7F80u || (x[j] & 0x7F800000u) == 0x7F800000u;
                    if (bad) s_bad[r] = 1;
                    if constexpr (NP == 4) {
                        order_pairs<4>(x, o);
                    } else {
                        const uint32_t lo[2] = {x[0], x[1]}, hi[2] = {x[2], x[3]};
                        uint32_t l[2], h[2];
                        order_pairs<2>(lo, l);
                        order_pairs<2>(hi, h);
                        o[0] = l[0];
                        o[1] = l[1];
                        o[2] = h[0];
                        o[3] = h[1];
                    }
                    const uint32_t tile = base + ((r >> 7) * M::panels + (e >> 3)) * (kRowTile * 128);
                    st_shared16(tile + (r & 127) * 128 + (((e & 7) ^ (r & 7)) << 4), o[0], o[1], o[2], o[3]);
                }
            }
            fence_async();
        }
        if (ok && warp < kRowWarps && (two || warp < 4)) {
            uint32_t z[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) z[i] = 0;
#pragma unroll
            for (int c = 0; c < D; c += 32) tmem_st32(tmem + M::o_at + (warp >> 2) * D + c + ((uint32_t)(warp & 3) * 32 << 16), z);
            tmem_st_wait();
            tc_fence_before();
        }
        __syncthreads();
        tc_fence_after();

        if (ok && warp == kIssuer) {
            bool fine = true;
            const uint32_t sdesc = bf16_desc(kKeys, false), odesc = bf16_desc(D, true);
            auto scores = [&](int i, int j) {                // S_i of key tile j
                if (!elect_one()) return;
                const uint32_t k = base + M::k_at + ((n0 + j) & 1) * M::stage, q = base + i * M::panels * (kRowTile * 128);
#pragma unroll
                for (int e = 0; e < D / 16; ++e)
                    mma_bf16(tmem + i * M::s_cols, operand_desc(q + (e >> 2) * (kRowTile * 128) + (e & 3) * 32),
                             operand_desc(k + (e >> 2) * M::panel + (e & 3) * 32), sdesc, e > 0);
                mma_commit<1>(smem_addr(&bars.s_full[i]), 0);
            };
            auto sums = [&](int i, int j) {                  // O_i += P_i V of key tile j
                if (!elect_one()) return;
                const uint32_t v = base + M::v_at + ((n0 + j) & 1) * M::stage;
#pragma unroll
                for (int e = 0; e < kKeys / 16; ++e)
                    mma_bf16_tmem(tmem + M::o_at + i * D, tmem + i * M::s_cols + e * 8, by_n_desc(v + e * 2048, M::panel), odesc);
            };
            auto freed = [&](uint64_t& bar) {
                if (elect_one()) mma_commit<1>(smem_addr(&bar), 0);
            };
            auto tile_wait = [&](uint64_t (&bar)[2], int j) { return warp_agrees(wait(bar[(n0 + j) & 1], ((n0 + j) >> 1) & 1)); };
            if (count > 0) {
                fine = tile_wait(bars.k_full, 0);
                if (fine) {
                    tc_fence_after();
                    scores(0, 0);
                    if (two) scores(1, 0);
                    freed(bars.k_empty[n0 & 1]);
                }
            }
            for (int j = 0; fine && j < count; ++j) {
                const bool more = j + 1 < count;
                if (!(fine = tile_wait(bars.v_full, j))) break;
                if (!(fine = warp_agrees(wait(bars.p_ready[0], (n0 + j) & 1)))) break;
                tc_fence_after();
                sums(0, j);
                if (more) {
                    if (!(fine = tile_wait(bars.k_full, j + 1))) break;
                    tc_fence_after();
                    scores(0, j + 1);
                }
                if (two) {
                    if (!(fine = warp_agrees(wait(bars.p_ready[1], (n1 + j) & 1)))) break;
                    tc_fence_after();
                    sums(1, j);
                }
                freed(bars.v_empty[(n0 + j) & 1]);
                if (more) {
                    if (two) scores(1, j + 1);
                    freed(bars.k_empty[(n0 + j + 1) & 1]);
                }
            }
            freed(bars.o_full);
            ok = fine;
        } else if (ok && warp >= kRowWarps && warp < kIssuer) {
            const int me = threadIdx.x - kRowWarps * 32;
            const int* const pages_of = p.batch.table + (size_t)it.b * p.batch.width;
            uint4 code[2][M::chunks];                        // keys and values of the tile to come
            uint32_t byte[2][M::chunks];
            uint32_t absent = 0, outside = 0;                // bit per chunk: its key has no page, is seen by no row
            uint32_t row_at[M::chunks], row_page[M::chunks]; // where the tile to come lies
            auto locate = [&](uint32_t k0) {                 // (keys of a last tile may lie beyond 2^31: unsigned, here and below)
                absent = outside = 0;
#pragma unroll
                for (int i = 0; i < M::chunks; ++i) {
                    const uint32_t key = k0 + (me + i * kWideners * 32) / M::CPR;
                    const bool in = key >= (uint32_t)it.some_lo && key < (uint32_t)it.some_hi;
                    if (!in) outside |= 1u << i;
                    row_page[i] = (uint32_t)ld_int(pages_of + ((in ? key : (uint32_t)it.some_lo) >> p.cache.page_shift));
                    row_at[i] = key & ((1u << p.cache.page_shift) - 1u);
                }
#pragma unroll
                for (int i = 0; i < M::chunks; ++i)
                    if (row_page[i] >= (uint32_t)p.cache.pages) absent |= 1u << i;
                absent &= ~outside;
            };
            auto load = [&](int kind) {
#pragma unroll
                for (int i = 0; i < M::chunks; ++i) {
                    const int c = (me + i * kWideners * 32) % M::CPR;
                    code[kind][i] = make_uint4(0, 0, 0, 0);
                    byte[kind][i] = 127;
                    if (((absent | outside) >> i) & 1u) continue;
                    const size_t row = (((size_t)row_page[i] * p.cache.heads + it.head) << p.cache.page_shift) | row_at[i];
                    code[kind][i] = ld_once((kind ? p.cache.vc : p.cache.kc) + row * M::RB + c * 16);
                    byte[kind][i] = ld_u8((kind ? p.cache.vs : p.cache.ks) + row * (D >> p.cache.block_shift) + (c * (128 / M::bits) >> p.cache.block_shift));
                }
            };
            // Widens a chunk to `at` (row of its key, first panel).  With `some` (a key that not all rows see) elements that are NaN or beyond BF16's
            // range become zeros, which a weight of zero takes away, and are returned, a bit each.
            auto widen = [&](uint32_t at, int key, int c, uint4 v, uint32_t sb, bool some) {
                uint32_t out_of = 0;
                const uint32_t f = W::factor(sb);
                const uint32_t words[4] = {v.x, v.y, v.z, v.w};
                uint32_t o[4 * NP];
                bool odd = sb > W::limit || (some && sb >= kLoudByte);
                if constexpr (W::has_nan) {
                    uint32_t seen = 0;
                    W::note_nan(v, seen);
                    odd |= W::saw_nan(seen);
                }
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t x[NP];
                    W::pairs(words[w], f, x);
#pragma unroll
                    for (int j = 0; j < NP; ++j) o[w * NP + j] = x[j];
                }
                if (odd) {
                    const uint32_t f2 = W::factor2(sb);
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
#pragma unroll
                        for (int j = 0; j < NP; ++j) {
                            o[w * NP + j] = W::mul(o[w * NP + j], f2);
                            if constexpr (W::has_nan) {      // bytes j and j + 2 of the word
                                const uint32_t bad = nan_codes(words[w]) >> (7 + 8 * j) & 0x00010001u;
                                o[w * NP + j] = (o[w * NP + j] & ~(bad * 0xFFFFu)) | bad * 0x7FC0u;
                            }
                        }
                    }
                    if (some) {
#pragma unroll
                        for (int e = 0; e < 4 * NP * 2; ++e) {
                            const int place = widened_place<NP>(e);
                            if (((o[place / 2] >> (16 * (place & 1))) & 0x7F80u) != 0x7F80u) continue;
                            out_of |= 1u << e;
                            o[place / 2] &= place & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                        }
                    }
                }
                constexpr int per = 128 / M::bits / 8;       // 16-byte pieces of a chunk
#pragma unroll
                for (int q = 0; q < per; ++q) {
                    const int piece = c * per + q;
                    st_shared16(at + (piece >> 3) * M::panel + (((piece & 7) ^ (key & 7)) << 4), o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
                }
                return out_of;
            };
            bool fine = true;
            if (count > 0) {
                locate(it.from);
                load(0);
                load(1);
            }
            for (int j = 0; fine && j < count; ++j) {
                const uint32_t n = n0 + j, st = n & 1, again = ((n >> 1) & 1) ^ 1;
                const uint32_t k0 = (uint32_t)it.from + j * kKeys, all_lo = (uint32_t)it.all_lo, all_hi = (uint32_t)it.all_hi;
                if (!(fine = warp_agrees(wait(bars.k_empty[st], again)))) break;
#pragma unroll
                for (int i = 0; i < M::chunks; ++i) {
                    const int id = me + i * kWideners * 32, key = id / M::CPR;
                    widen(base + M::k_at + st * M::stage + key * 128, key, id % M::CPR, code[0][i], byte[0][i], false);
                }
                fence_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&bars.k_full[st]));
                const uint32_t gone = absent;
                if (j + 1 < count) {
                    locate(k0 + kKeys);
                    load(0);
                }
                if (!(fine = warp_agrees(wait(bars.v_empty[st], again)))) break;
                const bool edge = k0 < all_lo || k0 + kKeys > all_hi;
                uint32_t info = gone ? 1u : 0u;
#pragma unroll
                for (int i = 0; i < M::chunks; ++i) {
                    const int id = me + i * kWideners * 32, key = id / M::CPR, c = id % M::CPR;
                    const bool some = edge && (k0 + key < all_lo || k0 + key >= all_hi);
                    const uint32_t out_of = widen(base + M::v_at + st * M::stage + key * 128, key, c, code[1][i], byte[1][i], some);
                    if (edge) {
                        if (out_of) info |= 2u;
                        uint8_t* const to = base_p + M::nan_at + (st * kKeys + key) * NB * 4;
                        if constexpr (M::bits == 4) reinterpret_cast<uint32_t*>(to)[c] = out_of;
                        else reinterpret_cast<uint16_t*>(to)[c] = (uint16_t)out_of;
                    }
                    if (c == 0) base_p[M::absent_at + st * kKeys + key] = (uint8_t)((gone >> i) & 1u);
                }
                fence_async();
                info = __reduce_or_sync(0xFFFFFFFFu, info);
                if (lane == 0) s_info[st][warp - kRowWarps] = info;
                __syncwarp();                                // (the reduction orders no stores: the lanes' values and masks stand in front of the arrival)
                if (lane == 0) mbar_arrive(smem_addr(&bars.v_full[st]));
                if (j + 1 < count) load(1);
            }
            ok = fine;
        } else if (ok && (two || warp < 4)) {
            const int i = warp >> 2, r = threadIdx.x & 127, row = i * kRowTile + r;
            const uint32_t quarter = (uint32_t)(warp & 3) * 32 << 16, sc = tmem + i * M::s_cols + quarter, oc = tmem + M::o_at + i * D + quarter;
            const uint32_t nth = i ? n1 : n0;
            const bool mine = row < it.rows;
            const int token = mine ? row_token(p, s, it.row0 + row) : 0;
            const int lo = mine ? token_lo(p, s, token) : 0, hi = mine ? token_hi(p, s, token) : 0;
            const float f = s_bad[row] ? __uint_as_float(0x7FC00000u) : p.scale;
            float m = kNone, l = 0.f;
            bool fine = true, steep = false;                 // steep: some row's m is beyond kSteep
            for (int j = 0; fine && j < count; ++j) {
                const uint32_t st = (n0 + j) & 1;
                if (!(fine = warp_agrees(wait(bars.v_full[st], ((n0 + j) >> 1) & 1) && wait(bars.s_full[i], (nth + j) & 1)))) break;
                tc_fence_after();
                uint32_t info = 0;
#pragma unroll
                for (int w = 0; w < kWideners; ++w) info |= s_info[st][w];
                const int k0 = it.from + j * kKeys, from = lo - k0, to_key = hi - k0;
                const bool edge = k0 < it.all_lo || (uint32_t)k0 + kKeys > (uint32_t)it.all_hi || (info & 1u);
                const uint8_t* const absent = base_p + M::absent_at + st * kKeys;
                if (info & 2u) {                             // what was taken out of values that not every row sees: NaN in the sums of those that do
                    uint32_t bad[NB] = {};
                    for (int k = 0; k < kKeys; ++k) {
                        if (k < from || k >= to_key || ((info & 1u) && absent[k])) continue;
                        const uint32_t* words = reinterpret_cast<const uint32_t*>(base_p + M::nan_at + (st * kKeys + k) * NB * 4);
#pragma unroll
                        for (int w = 0; w < NB; ++w) bad[w] |= words[w];
                    }
#pragma unroll
                    for (int w = 0; w < NB; ++w) {
                        if (!__any_sync(0xFFFFFFFFu, bad[w] != 0)) continue;
                        uint32_t v[32];
                        tmem_ld32(v, oc + w * 32);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if ((bad[w] >> e) & 1u) v[widened_place<NP>(e)] = 0x7FC00000u;
                        tmem_st32(oc + w * 32, v);
                        tmem_st_wait();
                    }
                }
                // 32 keys at a time from key c on: scores less m, P over scores that are read already.  Returns where it stopped: in front of keys that
                // moved some row's m beyond kSteep (STEEP: none).
                auto weigh = [&](auto edge_t, auto steep_t, int c) {
                    constexpr bool EDGE = decltype(edge_t)::value, STEEP = decltype(steep_t)::value;
#pragma unroll 1
                    for (; c < kKeys; c += 32) {
                        float2 x[16];
                        auto scores = [&] {                  // less m (or 0, before any key was seen); hidden ones -inf
                            uint32_t v[32];
                            tmem_ld32(v, sc + c);
                            tmem_ld_wait();
                            const float less = m == kNone ? 0.f : -m;
#pragma unroll
                            for (int k = 0; k < 16; ++k) {
                                if constexpr (STEEP)
                                    x[k] = make_float2(__fmul_rn(__uint_as_float(v[2 * k]), f) + less, __fmul_rn(__uint_as_float(v[2 * k + 1]), f) + less);
                                else
                                    x[k] = fma2(make_float2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), make_float2(f, f), make_float2(less, less));
                                if constexpr (EDGE) {
                                    const int at = c + 2 * k;
                                    if (at < from || at >= to_key || ((info & 1u) && absent[at])) x[k].x = __uint_as_float(0xFF800000u);
                                    if (at + 1 < from || at + 1 >= to_key || ((info & 1u) && absent[at + 1])) x[k].y = __uint_as_float(0xFF800000u);
                                }
                            }
                        };
                        scores();
                        float top = x[0].x;
#pragma unroll
                        for (int k = 0; k < 16; ++k) top = max3(top, x[k].x, x[k].y);
                        if (__any_sync(0xFFFFFFFFu, m == kNone ? top > kNone : top > kManySlack)) {
                            // m moved, by a whole number, so that nothing is rounded again: the sums so far and P so far in this tile
                            const float up = fmaxf(m, ceilf(top + (m == kNone ? 0.f : m))), by = exp2_approx(m - up);
                            m = up;
                            l *= by;
                            rescale_sums<D>(oc, by);
                            const uint32_t by2 = pack_bf16x2(by, by);
#pragma unroll 1
                            for (int done = 0; done < c / 2; done += 16) {
                                uint32_t w[16];
                                tmem_ld16(w, sc + done);
                                tmem_ld_wait();
#pragma unroll
                                for (int k = 0; k < 16; ++k) w[k] = W::mul(w[k], by2);
                                tmem_st16(sc + done, w);
                            }
                            tmem_st_wait();
                            if (!STEEP && __any_sync(0xFFFFFFFFu, fabsf(m) > kSteep && m != kNone)) return c;
                            scores();
                        }
                        uint32_t o[16];
                        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            // (the sum is that of the rounded weights: a row of few keys keeps what they are together)
                            o[k] = pack_bf16x2(exp2_approx(x[k].x), exp2_approx(x[k].y));
                            sum = add2(sum, make_float2(__uint_as_float(o[k] << 16), __uint_as_float(o[k] & 0xFFFF0000u)));
                        }
                        l += sum.x + sum.y;
                        tmem_st16(sc + c / 2, o);
                    }
                    return (int)kKeys;
                };
                const int c = steep ? 0 : edge ? weigh(std::true_type{}, std::false_type{}, 0) : weigh(std::false_type{}, std::false_type{}, 0);
                if (c < kKeys) {
                    steep = true;
                    weigh(std::true_type{}, std::true_type{}, c);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&bars.p_ready[i]));
            }
            if (fine) fine = warp_agrees(wait(bars.o_full, pieces & 1));
            if (fine) {
                tc_fence_after();
                const float inv = l == 0.f ? 0.f : 1.f / l;
                const size_t out_row = (size_t)(s.first + token) * (p.cache.heads * p.group) + it.head * p.group + (it.row0 + row - token * p.group);
                float* const to_part = reinterpret_cast<float*>(parts + ((size_t)blockIdx.x * 2 + (first ? 0 : 1)) * part);
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t v[32];
                    tmem_ld32(v, oc + c);
                    tmem_ld_wait();
                    if (!mine) continue;
                    float o[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(v[widened_place<NP>(e)]) * inv;
                    if (whole) {
#pragma unroll
                        for (int e = 0; e < 32; e += 16) {
                            uint32_t w[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) w[k] = pack_bf16x2(o[e + 2 * k], o[e + 2 * k + 1]);
                            st256(p.out + (out_row * D + c + e) * 2, w);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t w[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(o[e + k]);
                            st256(to_part + row * D + c + e, w);
                        }
                    }
                }
                if (mine && whole) write_lse(p, out_row, m, l);
                if (mine && !whole) write_weight(to_part + p.rows * D + 2 * row, m, l);
                tc_fence_before();
            }
            ok = fine;
        }
        if (first && threadIdx.x == 0) {
            bool good = true;
            MXQ_CHECKED(meta, sizeof(PartMeta), good = false)
            if (good) *meta = PartMeta{at, item, item + tiles, plan.total, s.first, it.head, it.row0, it.rows};
        }
        __syncwarp();
        __syncthreads();
        if (s_gave_up) ok = false;
        n0 += count;
        if (two) n1 += count;
        ++pieces;
        first = false;
        if (threadIdx.x == 0) next_item(p, plan);
        __syncthreads();
    }
    // A wait that gave up, in whichever warp, may have left products under way: let them end before their memory goes.
    if (s_gave_up) {
        const uint64_t began = global_ns();
        while (global_ns() - began < 1000ull * 1000) {}
    }
    __syncthreads();
    if (warp == kIssuer) tmem_free<1>(tmem, M::cols);
}

template <int FMT, int D>
int run_many(const AttendArgs& p, cudaStream_t stream)
{
    static std::atomic<uint64_t> done{0};
    auto kern = attend_many_kernel<FMT, D>;
    constexpr size_t smem = ManyShape<FMT, D>::total;
    if (int rc = allow_smem(reinterpret_cast<const void*>(kern), smem, done)) return rc;
    return launch_grid(kern, dim3((unsigned)p.ctas), kManyThreads, smem, 1, stream, p);
}

template <int FMT>
int many_by_dim(int dim, const AttendArgs& p, cudaStream_t stream)
{
    return dim == 64 ? run_many<FMT, 64>(p, stream) : run_many<FMT, 128>(p, stream);
}

}  // namespace

int launch_attend_many(int fmt, int dim, const AttendArgs& p, cudaStream_t stream)
{
    switch (fmt) {
    case MXQ_FP8_E4M3: return many_by_dim<MXQ_FP8_E4M3>(dim, p, stream);
    case MXQ_FP4_E2M1: return many_by_dim<MXQ_FP4_E2M1>(dim, p, stream);
    case MXQ_INT8: return many_by_dim<MXQ_INT8>(dim, p, stream);
    case MXQ_INT4: return many_by_dim<MXQ_INT4>(dim, p, stream);
    default: return MXQ_ERR_FORMAT;
    }
}

int many_status(int reset)
{
    unsigned int v = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, g_many_status, sizeof v) != cudaSuccess) {
        (void)cudaGetLastError();
        return MXQ_ERR_CUDA;
    }
    if (v && reset) {
        const unsigned int zero = 0;
        if (cudaMemcpyToSymbol(g_many_status, &zero, sizeof zero) != cudaSuccess) {
            (void)cudaGetLastError();
            return MXQ_ERR_CUDA;
        }
    }
    return v ? MXQ_ERR_TIMEOUT : MXQ_OK;
}

}  // namespace mxq
