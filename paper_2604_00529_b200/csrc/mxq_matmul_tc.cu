// D = L^ R^T on the fifth-generation tensor cores (block-scaled E4M3 matrix instructions): the product of mxq_matmul for more
// rows than a few.  L's rows go to the accumulator's lanes, R's rows to its columns: A and B, or, where parts are added (SPLIT), B and A,
// so that a lane's neighbours are consecutive elements of a row of D.
//
// The instruction takes one scale byte per row and 32 values of k, multiplied in by the hardware; a block of 64 or 128
// repeats its byte.  Scales therefore come in as plain bytes and are spread by the warps that bring them to shared memory
// (four bytes per row and k tile of 128), from where they are copied to tensor memory in front of the tile's four instructions.
// They are brought for eight k tiles at a time: a hand-over (a fence between the two memory proxies, an arrival across the pair)
// takes longer than the tensor cores take for one.
//
// Warps of a CTA: 0 loads operand tiles (TMA), 1 issues the matrix instructions (of the pair: the first CTA's), 2 - 7 bring the
// scales, 8 - 11 write results.  Tiles are worked on one after another by a CTA (pair) per SM (pair of SMs); or,
// where there are too few of them for that (SPLIT), a cluster shares one tile's k out and adds its parts through distributed
// shared memory, in a fixed order.  A CTA pair (CG = 2) works on 256 rows of L, 128 per CTA, and shares the tile of R half and half.
//
// Measured (blocks of 128, BF16 results): 8192 x 14336 x 4096 352 us in short runs, 2.7 PFLOP/s; in a loop of seconds 411 us, at the
// card's power limit and a clock of 1.28 GHz.  13 x 14336 x 4096 14.8 us, 4.0 TB/s of codes.  What the loops of the issuing warp
// cost decides: with one lane in a branch of its own, addresses went through vector registers and a k tile took 570 ns
// instead of 430; copying the next tile's scales ahead of this one's products, or writing them to tensor memory from registers,
// was slower (13 x 14336 x 4096 15.9 and 18.5 us).  The two issuing warps agree on what a wait answered (warp_agrees) behind what they
// issue: 200 x 4096 x 14336 takes 24.4 us, 24.5 with that in front, 24.1 where each lane goes by itself.
//
// The accumulator is FP32 and the instruction cuts: it loses less than 2^-23 of the sum at each step of 32 values, always toward zero
// (k = 14336 in one run 8.4e-6 of D in norm; in four parts, whose sum rounds, 2.1e-6).
#include <cuda.h>

#include "mxq_kernels.cuh"
#include "mxq_launch.h"
#include "mxq_tensor.cuh"

namespace mxq {
namespace {

__device__ unsigned int g_status;                            // a bounded wait gave up

constexpr int kRowsL = 128;                                  // rows of L per CTA
constexpr int kTileK = 128;                                  // bytes = elements of k per stage
constexpr int kThreads = 384;

template <int CG, int BN>
struct Shape {
    static constexpr int ahead = 8;                          // k tiles whose scales are brought together
    static constexpr int budget = 205 * 1024;
    static constexpr int rows_r = BN / CG;                   // rows of R that a CTA loads
    static constexpr int sf_r = (BN + 127) / 128;            // 512-byte scale tiles of R
    static constexpr int bytes_l = kRowsL * kTileK, bytes_r = rows_r * kTileK;
    static constexpr int sets = 1 + sf_r;                    // groups of 128 rows that have scales
    static constexpr int slot = ahead * sets * 512;          // the scale words of `ahead` k tiles
    static constexpr int stage = bytes_l + bytes_r;
    static constexpr int stages = (budget - 2 * slot) / stage < 8 ? (budget - 2 * slot) / stage : 8;
    static constexpr int sf_cols = 4 * sets;                 // columns of tensor memory per stage
    // Two accumulators, so that one tile's results leave while the next is computed.  Where tensor memory does not hold both
    // (BN = 256), the second begins inside the first; the columns that they share are read first.
    static constexpr int over = 2 * BN + stages * sf_cols <= 512 ? 0 : (2 * BN + stages * sf_cols - 512 + 31) / 32 * 32;
    static constexpr int second = BN - over;                 // where the second one begins
    static constexpr int sf_at = 2 * BN - over;
    static constexpr int tmem_used = sf_at + stages * sf_cols;
    static constexpr int tmem_cols = tmem_used <= 64 ? 64 : tmem_used <= 128 ? 128 : tmem_used <= 256 ? 256 : 512;
    static constexpr int smem = stages * stage + 2 * slot + 1024;       // (the base is aligned up to 1024)
    static_assert(tmem_used <= 512, "tensor memory");
};

struct TcArgs {
    const uint8_t *ls, *rs;                                  // scale bytes
    uint8_t* dst;
    size_t rows_l, rows_r;
    uint32_t kblocks, tiles_l, tiles_r, ktiles, split;
    size_t ld;                                               // elements between rows of dst
};

// Where tile number t lies: groups of eight tile rows of L, so that the tiles in flight share operands in L2.
__device__ __forceinline__ void tile_at(uint32_t t, uint32_t tiles_l, uint32_t tiles_r, uint32_t& tl, uint32_t& tr)
{
    constexpr uint32_t G = 8;
    const uint32_t group = t / (G * tiles_r), first = group * G, height = min(G, tiles_l - first), in = t - group * G * tiles_r;
    tl = first + in % height;
    tr = in / height;
}

// The scale bytes of a row for AHEAD k tiles, as they lie in memory.  Bytes beyond k, or of a row beyond the matrix, are 1.0:
// what they scale is 0.
template <int BLOCK, int AHEAD>
struct RowScales {
    static constexpr int PER = kTileK / BLOCK;               // bytes per k tile
    static constexpr int NW = AHEAD * PER / 4;
    uint32_t w[NW];

    __device__ __forceinline__ void load(const uint8_t* s, size_t row, size_t rows, uint32_t kt, uint32_t kblocks)
    {
#pragma unroll
        for (int j = 0; j < NW; ++j) w[j] = 0x7F7F7F7Fu;
        if (row >= rows) return;
        const uint8_t* at = s + row * kblocks;
        const uint32_t first = kt * PER;
        const uint32_t skip = (uint32_t)reinterpret_cast<uintptr_t>(at + first) & 3u, have = kblocks > first ? kblocks - first : 0;
        const uint8_t* const from = at + first - skip;
        if (skip == 0 && (kblocks & 3u) == 0) {
#pragma unroll
            for (int j = 0; j < NW; ++j)
                if (4u * j < have) w[j] = ld_u32(at + first + 4 * j);
        } else if (from + 4 * (NW + 1) <= s + rows * kblocks) {      // any alignment: the words that hold the bytes, shifted together
            uint32_t v[NW + 1];
#pragma unroll
            for (int j = 0; j <= NW; ++j) v[j] = ld_u32(from + 4 * j);
#pragma unroll
            for (int j = 0; j < NW; ++j) {
                const uint32_t left = have > 4u * j ? have - 4u * j : 0u, x = __funnelshift_r(v[j], v[j + 1], 8 * skip);
                w[j] = left >= 4 ? x : left ? (x & ((1u << 8 * left) - 1u)) | (0x7F7F7F7Fu << 8 * left) : 0x7F7F7F7Fu;
            }
        } else {                                             // the last rows
#pragma unroll
            for (int j = 0; j < 4 * NW; ++j)
                if (j < have) w[j / 4] = __byte_perm(w[j / 4], ld_u8(at + first + j), (0x3210u & ~(0xFu << 4 * (j % 4))) | 4u << 4 * (j % 4));
        }
    }
    // the four bytes of k tile i, one per 32 values of k
    __device__ __forceinline__ uint32_t word(int i) const
    {
        if constexpr (BLOCK == 32) return w[i];
        else if constexpr (BLOCK == 64) return __byte_perm(w[i / 2], 0, i % 2 ? 0x3322 : 0x1100);
        else return __byte_perm(w[i / 4], 0, 0x1111u * (i % 4));
    }
};

template <class OUT>
__device__ __forceinline__ void put(uint8_t* dst, size_t i, float v)
{
    if constexpr (OUT::size == 4) {
        MXQ_CHECKED(dst + i * 4, 4, return)
        reinterpret_cast<float*>(dst)[i] = v;
    } else {
        st_u16(dst + i * 2, pack_bf16x2(v, 0.f) & 0xFFFFu);
    }
}

// 32 columns of one row per lane to memory.
template <class OUT>
__device__ __forceinline__ void store_block(const TcArgs& p, const uint32_t (&v)[32], size_t row, size_t col, float* stage, int lane)
{
    if (p.ld % (32 / OUT::size) == 0) {               // whole 32-byte sectors
        constexpr int PER = 32 / OUT::size;
        if (row >= p.rows_l) return;
#pragma unroll
        for (int s = 0; s < 32 / PER; ++s) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (OUT::size == 4) w[j] = v[s * 8 + j];
                else w[j] = pack_bf16x2(__uint_as_float(v[s * 16 + 2 * j]), __uint_as_float(v[s * 16 + 2 * j + 1]));
            }
            if (col + s * PER < p.rows_r) st256(p.dst + (row * p.ld + col + s * PER) * OUT::size, w);
        }
    } else {                                                 // any alignment: through shared memory, lanes along the row
        const size_t row0 = row - lane;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 32; ++j) stage[lane * 33 + j] = __uint_as_float(v[j]);
        __syncwarp();
        for (int r = 0; r < 32; ++r)
            if (row0 + r < p.rows_l && col + lane < p.rows_r) put<OUT>(p.dst, (row0 + r) * p.ld + col + lane, stage[r * 33 + lane]);
    }
}

template <class OUT, int CG, int BN, int BLOCK, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1)
matmul_tc_kernel(const __grid_constant__ CUtensorMap map_l, const __grid_constant__ CUtensorMap map_r, const TcArgs p)
{
    using S = Shape<CG, BN>;
    extern __shared__ uint8_t s_raw[];
    __shared__ __align__(8) uint64_t s_full[S::stages], s_empty[S::stages], s_sf_full[2], s_sf_empty[2], s_acc_full[2], s_acc_free;
    __shared__ uint32_t s_tmem, s_gave_up;
    __shared__ float s_out[SPLIT ? 1 : 4 * 32 * 33];
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t in_cluster = CG == 2 || SPLIT ? cluster_rank() : 0u, rank = in_cluster % CG, leader = in_cluster - rank;
    const uint32_t base = (smem_addr(s_raw) + 1023u) & ~1023u;
    uint8_t* const base_p = s_raw + (base - smem_addr(s_raw));
    pdl_release();
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::stages; ++i) {
            mbar_init(smem_addr(&s_full[i]), 1);
            mbar_init(smem_addr(&s_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&s_sf_full[i]), S::sets * CG);
            mbar_init(smem_addr(&s_sf_empty[i]), 1);
            mbar_init(smem_addr(&s_acc_full[i]), 1);
        }
        mbar_init(smem_addr(&s_acc_free), 4 * CG);
        s_gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        tmem_alloc<CG>(smem_addr(&s_tmem), S::tmem_cols);
        if (lane == 0) {
            tma_prefetch_map(&map_l);
            tma_prefetch_map(&map_r);
        }
    }
    tc_fence_before();
    if constexpr (CG == 2 || SPLIT) cluster_sync();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_acquire();

    // the tiles of this CTA (pair) and its k tiles of each: all of them, or a part that begins at a whole word of scale bytes
    const uint32_t tiles = p.tiles_l * p.tiles_r, step = SPLIT ? tiles : gridDim.x / CG, first = blockIdx.x / (SPLIT ? CG * p.split : CG);
    uint32_t k_lo = 0, k_hi = p.ktiles;
    if constexpr (SPLIT) {
        const uint32_t unit = p.ktiles >= 8 * p.split ? 4 : 1, units = (p.ktiles + unit - 1) / unit, part = in_cluster / CG;
        k_lo = min(units * part / p.split * unit, p.ktiles);
        k_hi = min(units * (part + 1) / p.split * unit, p.ktiles);
    }
    auto wait = [&](uint64_t& bar, uint32_t parity) { return mbar_wait(smem_addr(&bar), parity, &s_gave_up, &g_status); };
    uint32_t stage = 0, phase = 0, slot = 0;                 // slots are numbered through: slot & 1, parity (slot >> 1) & 1
    const uint32_t slots = base + S::stages * S::stage;
    auto advance = [&] {
        if (++stage == (uint32_t)S::stages) {
            stage = 0;
            phase ^= 1;
        }
    };

    if (warp == 0) {                                         // operand tiles
        bool ok = true;
        for (uint32_t t = first; ok && t < tiles; t += step) {
            uint32_t tl, tr;
            tile_at(t, p.tiles_l, p.tiles_r, tl, tr);
            const int yl = (int)(tl * (kRowsL * CG) + rank * kRowsL), yr = (int)(tr * BN + rank * S::rows_r);
            for (uint32_t kt = k_lo; ok && kt < k_hi; ++kt, advance()) {
                ok = wait(s_empty[stage], phase ^ 1);
                if (elect_one() && ok) {
                    uint32_t bar = smem_addr(&s_full[stage]);
                    const uint32_t at = base + stage * S::stage;
                    if (rank == 0) mbar_expect(bar, CG * (S::bytes_l + S::bytes_r));
                    if constexpr (CG == 2) bar = peer_addr(bar, leader);
                    tma_tile<CG>(at, &map_l, (int)(kt * kTileK), yl, bar);
                    tma_tile<CG>(at + S::bytes_l, &map_r, (int)(kt * kTileK), yr, bar);
                }
                ok = warp_agrees(ok);
            }
        }
    } else if (warp == 1 && rank == 0) {                     // matrix instructions
        bool ok = true;
        uint32_t n = 0;
        for (uint32_t t = first; ok && t < tiles; t += step, ++n) {
            // The last tile's shared columns have been read; and since whoever read them had done with the tile before, so has
            // the accumulator that this tile goes to.
            if (n > 0 && !(ok = warp_agrees(wait(s_acc_free, (n - 1) & 1)))) break;
            tc_fence_after();
            const uint32_t buf = n & 1, d = tmem + buf * S::second;
            for (uint32_t kt = 0; ok && kt < k_hi - k_lo; ++kt, advance()) {
                ok = wait(s_full[stage], phase);
                if (kt % S::ahead == 0) ok = wait(s_sf_full[slot & 1], (slot >> 1) & 1) && ok;
                tc_fence_after();
                const uint32_t at = base + stage * S::stage, sf = slots + (slot & 1) * S::slot + kt % S::ahead * (S::sets * 512);
                const uint32_t tsf = tmem + S::sf_at + stage * S::sf_cols;
                const uint64_t a = operand_desc(at), b = operand_desc(at + S::bytes_l);
                const bool end = kt + 1 == k_hi - k_lo, last = kt % S::ahead == S::ahead - 1 || end;
                if (elect_one() && ok) {
#pragma unroll
                    for (int i = 0; i < S::sets; ++i) scales_to_tmem<CG>(tsf + 4 * i, scales_desc(sf + 512 * i));
#pragma unroll
                    for (int j = 0; j < 4; ++j)              // 32 bytes of k further inside the swizzled rows
                        mma_scaled<CG>(d, a + 2 * j, b + 2 * j, instr_desc(kRowsL * CG, BN, j), tsf, tsf + 4, kt > 0 || j > 0);
                    mma_commit<CG>(smem_addr(&s_empty[stage]), leader);
                    if (last) mma_commit<CG>(smem_addr(&s_sf_empty[slot & 1]), leader);
                    if (end) mma_commit<CG>(smem_addr(&s_acc_full[buf]), leader);
                }
                ok = warp_agrees(ok);
                slot += last;
            }
        }
    } else if (warp >= 2 && warp < 8 && (warp - 2) % 3 < S::sets) {
        // Scales: rows lane, lane + 32, + 64 and + 96 of a group of 128, for every other slot: two warps take turns, since filling one
        // (loads, a fence that waits for them, an arrival) takes longer than the tensor cores take for its k tiles.
        const int set = (warp - 2) % 3;
        const uint32_t turn = (warp - 2) / 3, chunks = (k_hi - k_lo + S::ahead - 1) / S::ahead;
        const uint8_t* s = set == 0 ? p.ls : p.rs;
        uint32_t t = first, c = turn;
        RowScales<BLOCK, S::ahead> w[4];
        auto load = [&] {                                    // the warp's next chunk, which may lie in a later tile
            for (; t < tiles && c >= chunks; t += step) c -= chunks;
            if (t >= tiles) return;
            uint32_t tl, tr;
            tile_at(t, p.tiles_l, p.tiles_r, tl, tr);
            const size_t row0 = set == 0 ? (size_t)tl * (kRowsL * CG) + rank * kRowsL : (size_t)tr * BN + 128 * (set - 1);
            const size_t rows = set == 0 ? p.rows_l : min(p.rows_r, (size_t)(tr + 1) * BN);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i].load(s, row0 + lane + 32 * i, rows, k_lo + c * S::ahead, p.kblocks);
        };
        load();
        for (slot = turn; t < tiles; slot += 2) {
            if (!warp_agrees(wait(s_sf_empty[turn], ((slot >> 1) & 1) ^ 1))) break;
            uint4* to = reinterpret_cast<uint4*>(base_p + S::stages * S::stage + turn * S::slot + set * 512) + lane;
#pragma unroll
            for (int j = 0; j < S::ahead; ++j)
                to[j * (S::sets * 32)] = make_uint4(w[0].word(j), w[1].word(j), w[2].word(j), w[3].word(j));
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(peer_addr(smem_addr(&s_sf_full[turn]), leader));
            c += 2;
            load();                                          // behind the fence
        }
    } else if (warp >= 8) {                                  // results
        bool ok = true;
        uint32_t n = 0;
        const int q = warp & 3;
        for (uint32_t t = first; ok && t < tiles; t += step, ++n) {
            uint32_t tl, tr;
            tile_at(t, p.tiles_l, p.tiles_r, tl, tr);
            const uint32_t buf = n & 1;
            if (!(ok = warp_agrees(wait(s_acc_full[buf], (n >> 1) & 1)))) break;
            tc_fence_after();
            const size_t row = (size_t)tl * (kRowsL * CG) + rank * kRowsL + q * 32 + lane;
            auto release = [&] {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(peer_addr(smem_addr(&s_acc_free), leader));
            };
            if (S::over == 0) release();
#pragma unroll 1
            for (int i = 0; i < BN; i += 32) {
                // the shared columns are the first accumulator's last ones and the second one's first
                const int c = buf == 0 && S::over ? (i + S::second) % BN : i;
                uint32_t v[32];
                tmem_ld32(v, tmem + buf * S::second + c + ((uint32_t)(q * 32) << 16));
                tmem_ld_wait();
                if (S::over && i + 32 == S::over) release();
                if constexpr (SPLIT) {                       // the stages are free: every product of theirs is done
                    float* part = reinterpret_cast<float*>(base_p) + q * 32 + lane;
#pragma unroll
                    for (int j = 0; j < 32; ++j) part[(c + j) * kRowsL] = __uint_as_float(v[j]);
                } else {
                    store_block<OUT>(p, v, row, (size_t)tr * BN + c, s_out + q * 32 * 33, lane);
                }
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    // A wait that gave up, in whichever warp, may have left copies under way: let those of this CTA land before its memory goes.
    if (s_gave_up) {
        const uint64_t began = global_ns();
        while (global_ns() - began < 1000ull * 1000) {}
        __syncthreads();
    }
    if constexpr (SPLIT) {                                   // this CTA's share of the columns, the parts in order
        static_assert(S::stages * S::stage >= BN * kRowsL * 4, "a part fits in the stages");
        cluster_sync();
        uint32_t tl, tr;
        tile_at(first, p.tiles_l, p.tiles_r, tl, tr);
        const size_t row = (size_t)tl * (kRowsL * CG) + rank * kRowsL + lane * 4;
        const uint32_t part = in_cluster / CG, c_hi = BN * (part + 1) / p.split;
        for (uint32_t c = BN * part / p.split + warp; c < c_hi; c += kThreads / 32) {
            const size_t col = (size_t)tr * BN + c;
            if (col >= p.rows_r) break;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (uint32_t i = 0; i < p.split; ++i) {
                const float4 v = ld_peer4(peer_addr(base + (c * kRowsL + lane * 4) * 4, i * CG + rank));
                sum.x += v.x;
                sum.y += v.y;
                sum.z += v.z;
                sum.w += v.w;
            }
            const size_t at = col * p.ld + row;
            if ((p.ld & 3) == 0) {
                if (row >= p.rows_l) continue;
                uint8_t* to = p.dst + at * OUT::size;
                MXQ_CHECKED(to, 4 * OUT::size, continue)
                if constexpr (OUT::size == 4) *reinterpret_cast<float4*>(to) = sum;
                else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(sum.x, sum.y), pack_bf16x2(sum.z, sum.w));
            } else {
                const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (row + j < p.rows_l) put<OUT>(p.dst, at + j, v[j]);
            }
        }
    }
    if constexpr (CG == 2 || SPLIT) cluster_sync();
    if (warp == 0) tmem_free<CG>(tmem, S::tmem_cols);
}

// ---- launchers --------------------------------------------------------------------------------------------

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder()
{
    static const EncodeFn fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

// [rows, k] bytes in boxes of `box_rows` x 128, zeros beyond the matrix
bool make_map(CUtensorMap* map, const uint8_t* p, size_t rows, size_t k, int box_rows)
{
    const EncodeFn enc = encoder();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)k};
    const cuuint32_t box[2] = {kTileK, (cuuint32_t)box_rows}, elem[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(p), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class OUT, int CG, int BN, int BLOCK, bool SPLIT>
int run_block(const MatmulArgs& m, uint32_t split, cudaStream_t stream)
{
    using S = Shape<CG, BN>;
    static std::atomic<uint64_t> done{0};
    auto kern = matmul_tc_kernel<OUT, CG, BN, BLOCK, SPLIT>;
    if (int rc = allow_smem(reinterpret_cast<const void*>(kern), S::smem, done)) return rc;
    TcArgs p;
    p.ls = SPLIT ? m.bs : m.as;
    p.rs = SPLIT ? m.as : m.bs;
    p.rows_l = SPLIT ? m.n : m.m;
    p.rows_r = SPLIT ? m.m : m.n;
    p.dst = m.dst;
    p.ld = m.n;
    p.split = split;
    p.kblocks = (uint32_t)(m.k / (size_t)m.block);
    p.ktiles = (uint32_t)((m.k + kTileK - 1) / kTileK);
    p.tiles_l = (uint32_t)((p.rows_l + kRowsL * CG - 1) / (kRowsL * CG));
    p.tiles_r = (uint32_t)((p.rows_r + BN - 1) / BN);
    if ((uint64_t)p.tiles_l * p.tiles_r > 0x7FFFFFFFull / (CG * split)) return MXQ_ERR_SIZE;
    CUtensorMap ml, mr;
    if (!make_map(&ml, SPLIT ? m.b : m.a, p.rows_l, m.k, kRowsL) || !make_map(&mr, SPLIT ? m.a : m.b, p.rows_r, m.k, S::rows_r)) return MXQ_ERR_CUDA;
    const uint32_t tiles = p.tiles_l * p.tiles_r, most = 148 / CG;
    const unsigned grid = SPLIT ? tiles * split * CG : (tiles < most ? tiles : most) * CG;
    return launch_grid(kern, dim3(grid), kThreads, S::smem, (int)(CG * split), stream, ml, mr, p);
}

template <class OUT, int CG, int BN, bool SPLIT>
int run(const MatmulArgs& m, uint32_t split, cudaStream_t stream)
{
    if (m.block == 32) return run_block<OUT, CG, BN, 32, SPLIT>(m, split, stream);
    if (m.block == 64) return run_block<OUT, CG, BN, 64, SPLIT>(m, split, stream);
    return run_block<OUT, CG, BN, 128, SPLIT>(m, split, stream);
}

// What a launch is expected to take, in microseconds: a fixed part per wave of CTAs (start, first loads, sums and stores of the
// results) and a time per k tile, as measured with blocks of 128 (device time, inputs of a few calls in turn):
//   single CTAs, 32 columns, k in S parts    512 x 512 x 4096 S = 1, 2, 4: 12.7 10.2 9.6;   13 x 14336 x 4096 S = 1: 14.9
//   single CTAs, 64 columns                  64 x 14336 x 4096 S = 1: 15.8 (32 columns 26.8: two waves);  1000 x 1111 x 1152: 8.8
//   pairs, 128 columns, k in S parts         200 x 4096 x 14336 S = 1, 2: 31.0 21.1
//   pairs, 128 columns, tiles in turn        512 x 4096 x 4096: 13.1 (256 columns 16.3);  4096 x 4096 x 4096: 67
//   pairs, 256 columns, tiles in turn        512 x 4096 x 4096: 16.3;  4096 x 4096 x 4096: 56
// The rule picks the smallest; beyond four CTAs a cluster finds too few free neighbours (S = 8: 17.7 against 7.9 us with S = 4 for
// one row of 4096 x 4096), so more parts are not offered.
struct Plan {
    int cg, bn, split;                                       // split 0: tiles in turn
    double us;
};

Plan plan(const MatmulArgs& m)
{
    auto tiles = [](size_t rows, size_t per) { return (double)((rows + per - 1) / per); };
    const double kt = tiles(m.k, kTileK);
    auto waves = [](double ctas) { return ctas <= 148 ? 1.0 : (double)(size_t)((ctas + 147) / 148); };
    Plan best{2, 256, 0, 4.0 + waves(2 * tiles(m.m, 256) * tiles(m.n, 256)) * (kt * 0.36 + 1.6)};
    auto offer = [&](int cg, int bn, int split, double us) {
        if (us < best.us) best = Plan{cg, bn, split, us};
    };
    offer(2, 128, 0, 4.0 + waves(2 * tiles(m.m, 256) * tiles(m.n, 128)) * (kt * 0.25 + 1.2));
    for (int s = 1; s <= 4; s *= 2) {
        if (s > kt) break;
        const double part = (double)(size_t)((kt + s - 1) / s);
        offer(1, 32, s, waves(tiles(m.n, 128) * tiles(m.m, 32) * s) * (6.2 + part * 0.2));
        offer(1, 64, s, waves(tiles(m.n, 128) * tiles(m.m, 64) * s) * (6.5 + part * 0.21));
        if (s <= 2) offer(2, 128, s, waves(2 * tiles(m.n, 256) * tiles(m.m, 128) * s) * (6.6 + part * 0.22));
    }
    return best;
}

#ifdef MXQ_DEBUG
__device__ unsigned int g_went_on;

// One warp whose even lanes wait for a phase that is over and whose odd lanes for one that nothing ends: which lanes went on.
__global__ void wait_kernel(uint64_t limit_ns)
{
    __shared__ __align__(8) uint64_t s_bar;
    __shared__ uint32_t s_gave_up;
    if (threadIdx.x == 0) {
        mbar_init(smem_addr(&s_bar), 1);
        s_gave_up = 0;
    }
    __syncwarp();
    const bool went_on = warp_agrees(mbar_wait(smem_addr(&s_bar), (threadIdx.x & 1) ^ 1, &s_gave_up, &g_status, limit_ns));
    const unsigned int lanes = __ballot_sync(0xFFFFFFFFu, went_on);
    if (threadIdx.x == 0) g_went_on = lanes;
}
#endif

template <class OUT>
int choose(const MatmulArgs& m, cudaStream_t stream)
{
    const Plan p = plan(m);
    if (p.split && p.bn == 32) return run<OUT, 1, 32, true>(m, (uint32_t)p.split, stream);
    if (p.split && p.bn == 64) return run<OUT, 1, 64, true>(m, (uint32_t)p.split, stream);
    if (p.split) return run<OUT, 2, 128, true>(m, (uint32_t)p.split, stream);
    if (p.bn == 128) return run<OUT, 2, 128, false>(m, 1, stream);
    return run<OUT, 2, 256, false>(m, 1, stream);
}

}  // namespace

double matmul_tc_us(const MatmulArgs& p) { return plan(p).us; }

int launch_matmul_tc(const MatmulArgs& p, int dst_dtype, cudaStream_t stream)
{
    return dst_dtype == MXQ_F32 ? choose<F32>(p, stream) : choose<BF16>(p, stream);
}

// Whether a bounded wait of these kernels gave up on the current device; waits for the device.
int tc_status(int reset)
{
    unsigned int v = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, g_status, sizeof v) != cudaSuccess) {
        (void)cudaGetLastError();
        return MXQ_ERR_CUDA;
    }
    if (v && reset) {
        const unsigned int zero = 0;
        if (cudaMemcpyToSymbol(g_status, &zero, sizeof zero) != cudaSuccess) {
            (void)cudaGetLastError();
            return MXQ_ERR_CUDA;
        }
    }
    return v ? MXQ_ERR_TIMEOUT : MXQ_OK;
}

}  // namespace mxq

#pragma GCC visibility push(default)
extern "C" int mxq_debug_wait(unsigned int milliseconds, unsigned int* lanes)
{
#ifdef MXQ_DEBUG
    if (!lanes) return MXQ_ERR_NULL;
    if (milliseconds > 1000) return MXQ_ERR_SIZE;
    mxq::wait_kernel<<<1, 32>>>((uint64_t)milliseconds * 1000000ull);
    if (cudaDeviceSynchronize() == cudaSuccess && cudaMemcpyFromSymbol(lanes, mxq::g_went_on, sizeof *lanes) == cudaSuccess) return 1;
    (void)cudaGetLastError();
    return MXQ_ERR_CUDA;
#else
    (void)milliseconds;
    (void)lanes;
    return 0;
#endif
}
#pragma GCC visibility pop