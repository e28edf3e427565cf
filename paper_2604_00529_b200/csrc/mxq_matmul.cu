// D = A^ B^T of two operands in the MXFP anchor's format, E4M3, with one E8M0 scale per block along k (Sec. 3.5; the lower formats have no
// product but mxq_moe's): D[i, j] = sum over blocks b of Xa[i, b] Xb[j, b] sum over k in b of Pa[i, k] Pb[j, k].
#include "mxq_kernels.cuh"
#include "mxq_launch.h"
#include "mxq_product.cuh"

namespace mxq {

namespace {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// ---- few rows of A ----------------------------------------------------------------------------------------
// Bound by reading B once.  A CTA of 16 warps covers 32 rows of B and up to eight of A; the warps share k out in chunks of 64 and
// meet in shared memory at the end, in a fixed order.  Codes go from global memory straight into the fragments of the warp's
// matrix instruction: widened to FP16, exactly, by the conversion instruction, and the block's two scales multiply the
// FP32 sum of the block.  (One row of A, B 4096 x 4096: 6.2 us; eight warps 9.7, 16 rows of B 8.6, one chunk under way per warp
// instead of two 6.8.  The variant for blocks of 32 spills 52 bytes per thread.)
//   BLK32: blocks of 32.  Two of the four lanes of a row then hold one block and two the other: a step is taken twice, with the other
//   lanes' elements of A zero (the matrix instructions are the least of this kernel's time).

constexpr int kFewWarps = 16;
constexpr int kFewTiles = 2;                                // 16-row tiles of B per CTA
constexpr int kFewDepth = 2;                                // chunks in flight per warp

struct Piece {                                              // a lane's 16 codes of one row in a chunk of 64; zeros beyond k
    uint32_t w[4];
    __device__ __forceinline__ void load(const uint8_t* row, uint32_t k0, uint32_t k, int t)
    {
        const uint32_t at = k0 + t * 16;
        const uint4 v = at < k ? ld_once(row + at) : make_uint4(0, 0, 0, 0);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
};

// The scale bytes of a row for a chunk: one, or with blocks of 32 two (127, a factor of 1, beyond k: what they scale is 0).
template <int SUB>
__device__ __forceinline__ void chunk_scales(const uint8_t* row, uint32_t k0, uint32_t k, uint32_t kblocks, int block_shift, uint32_t (&x)[SUB])
{
    const uint32_t kb = k0 >> block_shift;
    if constexpr (SUB == 1) {
        x[0] = k0 < k ? ld_u8(row + kb) : 127u;
    } else if ((kblocks & 1u) == 0) {                       // (the row then begins at an even address)
        const uint32_t w = k0 < k ? ld_u16(row + kb) : 0x7F7Fu;
        x[0] = w & 255u;
        x[1] = w >> 8;
    } else {
#pragma unroll
        for (int s = 0; s < SUB; ++s) x[s] = kb + s < kblocks ? ld_u8(row + kb + s) : 127u;
    }
}

// sum += acc 2^(xb + xa - 254), element e of rows (e >> 1) of B and (e & 1) of A.  The exponents are added before they become
// a factor, so that a large scale of one operand and a small one of the other do not overflow on the way.  A factor that
// is no normal FP32 number, or a poisoned block, takes the long way; zero blocks (byte 0, sums of 0) do not.
__device__ __forceinline__ void add_scaled(float (&sum)[4], const float (&acc)[4], uint32_t xb0, uint32_t xb1, uint32_t xa0, uint32_t xa1)
{
    const uint32_t xb[2] = {xb0, xb1}, xa[2] = {xa0, xa1};
    bool odd = max(max(xb0, xb1), max(xa0, xa1)) == 255u;
    int f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[e] = (int)(xb[e >> 1] + xa[e & 1]) - 127;
        odd |= f[e] > 254 || (f[e] < 1 && acc[e] != 0.f);
    }
    if (__any_sync(0xFFFFFFFFu, odd)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool poisoned = max(xb[e >> 1], xa[e & 1]) == 255u;
            sum[e] += poisoned ? __uint_as_float(0x7FC00000u) : ldexpf(acc[e], f[e] - 127);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(acc[e], __int_as_float(max(f[e], 1) << 23), sum[e]);
    }
}

template <class OUT>
__device__ __forceinline__ void store_out(uint8_t* dst, size_t i, float v)
{
    if constexpr (OUT::size == 4) {
        MXQ_CHECKED(dst + i * 4, 4, return)
        reinterpret_cast<float*>(dst)[i] = v;
    } else {
        st_u16(dst + i * 2, pack_bf16x2(v, 0.f) & 0xFFFFu);
    }
}

constexpr int kFewRows = 8;                                 // rows of A: the columns of a matrix step

template <class OUT, bool BLK32>
__global__ void __launch_bounds__(kFewWarps * 32)
matmul_few_kernel(const uint8_t* __restrict__ a, const uint8_t* __restrict__ as, const uint8_t* __restrict__ b,
                  const uint8_t* __restrict__ bs, size_t m, size_t n, uint32_t k, uint32_t kblocks, int block_shift, uint8_t* __restrict__ dst)
{
    constexpr int SUB = BLK32 ? 2 : 1;                      // blocks that a chunk of 64 touches
    __shared__ float s_sum[kFewWarps][kFewTiles][4][32];
    pdl_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const size_t j0 = (size_t)blockIdx.x * (16 * kFewTiles);
    // rows beyond the matrices read their last row; their results are not stored
    const uint8_t *br[kFewTiles][2], *bsr[kFewTiles][2], *ar = a + min((size_t)g, m - 1) * k, *asr[2];
#pragma unroll
    for (int u = 0; u < kFewTiles; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const size_t r = min(j0 + u * 16 + h * 8 + g, n - 1);
            br[u][h] = b + r * k;
            bsr[u][h] = bs + r * kblocks;
        }
#pragma unroll
    for (int h = 0; h < 2; ++h) asr[h] = as + min((size_t)(2 * t + h), m - 1) * kblocks;
    pdl_acquire();
    float sum[kFewTiles][4] = {};
    const uint32_t chunks = (k + 63) / 64;
    for (uint32_t c0 = warp; c0 < chunks; c0 += kFewWarps * kFewDepth) {
        Piece pb[kFewDepth][kFewTiles][2], pa[kFewDepth];
        uint32_t xb[kFewDepth][kFewTiles][2][SUB], xa[kFewDepth][2][SUB];
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) {
            const uint32_t k0 = (c0 + d * kFewWarps) * 64;         // a chunk beyond k loads nothing and adds zeros
#pragma unroll
            for (int u = 0; u < kFewTiles; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) pb[d][u][h].load(br[u][h], k0, k, t);
            pa[d].load(ar, k0, k, t);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int u = 0; u < kFewTiles; ++u) chunk_scales<SUB>(bsr[u][h], k0, k, kblocks, block_shift, xb[d][u][h]);
                chunk_scales<SUB>(asr[h], k0, k, kblocks, block_shift, xa[d][h]);
            }
        }
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) {
            uint32_t x[SUB][8];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t lo, hi;
                e4m3_word_to_f16(pa[d].w[w], lo, hi);
#pragma unroll
                for (int s = 0; s < SUB; ++s) {
                    const bool mine = !BLK32 || (t >> 1) == s;
                    x[s][2 * w] = mine ? lo : 0u;
                    x[s][2 * w + 1] = mine ? hi : 0u;
                }
            }
#pragma unroll
            for (int u = 0; u < kFewTiles; ++u) {
                uint32_t f0[8], f1[8];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    e4m3_word_to_f16(pb[d][u][0].w[w], f0[2 * w], f0[2 * w + 1]);
                    e4m3_word_to_f16(pb[d][u][1].w[w], f1[2 * w], f1[2 * w + 1]);
                }
#pragma unroll
                for (int s = 0; s < SUB; ++s) {
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < 4; ++w) F16Mma::mma(acc, f0[2 * w], f1[2 * w], f0[2 * w + 1], f1[2 * w + 1], x[s][2 * w], x[s][2 * w + 1]);
                    add_scaled(sum[u], acc, xb[d][u][0][s], xb[d][u][1][s], xa[d][0][s], xa[d][1][s]);
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kFewTiles; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) s_sum[warp][u][e][lane] = sum[u][e];
    __syncthreads();
    // element (row g + 8 (e >> 1) of a tile of B, row 2 t + (e & 1) of A) sits at [e][g * 4 + t]
    if (threadIdx.x >= kFewTiles * 128) return;
    const int row = threadIdx.x % (16 * kFewTiles), col = threadIdx.x / (16 * kFewTiles);
    const int e = (row >> 3 & 1) * 2 + (col & 1), ln = (row & 7) * 4 + (col >> 1);
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) v += s_sum[w][row >> 4][e][ln];
    const size_t j = j0 + row;
    if ((size_t)col < m && j < n) store_out<OUT>(dst, (size_t)col * n + j, v);
}

template <class OUT>
int run_few(const MatmulArgs& p, cudaStream_t stream)
{
    const size_t ctas = (p.n + 16 * kFewTiles - 1) / (16 * kFewTiles);
    const uint32_t kblocks = (uint32_t)(p.k / (size_t)p.block);
    const int shift = p.block == 32 ? 5 : p.block == 64 ? 6 : 7;
    auto go = [&](auto kern) {
        return launch_kernel(kern, (int)ctas, kFewWarps * 32, stream, p.a, p.as, p.b, p.bs, p.m, p.n, (uint32_t)p.k, kblocks, shift, p.dst);
    };
    return p.block == 32 ? go(matmul_few_kernel<OUT, true>) : go(matmul_few_kernel<OUT, false>);
}

// What a launch is expected to take, in microseconds: a time per wave of CTAs (one per SM) that grows with k.  As measured, one row of A:
// B 1024 x 1024 3.4 (tensor cores 4.7), 4096 x 4096 6.2 (7.9), 6144 x 4096 11.6 (two waves; 10.0), 14336 x 4096 22 (15.5); with
// blocks of 32, 4096 x 2048 5.7 (6.5) and 4096 x 4096 10.4 (8.0).
double few_us(const MatmulArgs& p)
{
    const size_t ctas = (p.n + 16 * kFewTiles - 1) / (16 * kFewTiles);
    return (double)((ctas + 147) / 148) * (2.1 + (p.block == 32 ? 0.002 : 0.001) * (double)p.k);
}

}  // namespace

int launch_matmul_few(const MatmulArgs& p, int dst_dtype, cudaStream_t stream)
{
    return dst_dtype == MXQ_F32 ? run_few<F32>(p, stream) : run_few<BF16>(p, stream);
}

}  // namespace mxq

using namespace mxq;

#pragma GCC visibility push(default)
extern "C" {

int mxq_matmul(const void* a_codes, const uint8_t* a_scales, const void* b_codes, const uint8_t* b_scales, size_t m, size_t n,
               size_t k, int fmt, int block, void* dst, int dst_dtype, mxq_stream stream)
{
    if (fmt != MXQ_FP8_E4M3 || (dst_dtype != MXQ_F32 && dst_dtype != MXQ_BF16)) return MXQ_ERR_FORMAT;
    if (block != 32 && block != 64 && block != 128) return MXQ_ERR_BLOCK;
    const size_t most = ((size_t)1 << 31) - 1;
    if (k % (size_t)block || m > most || n > most || k > most) return MXQ_ERR_SIZE;
    if (m == 0 || n == 0) return MXQ_OK;
    if (!dst || (k && (!a_codes || !a_scales || !b_codes || !b_scales))) return MXQ_ERR_NULL;
    if (!aligned(dst, 32) || !aligned(a_codes, 32) || !aligned(b_codes, 32) || !aligned(a_scales, 16) || !aligned(b_scales, 16))
        return MXQ_ERR_ALIGN;
    const size_t size = dst_dtype == MXQ_F32 ? 4u : 2u;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (k == 0) {                                            // an empty sum
        if (cudaMemsetAsync(dst, 0, m * n * size, s) == cudaSuccess) return MXQ_OK;
        (void)cudaGetLastError();
        return MXQ_ERR_CUDA;
    }
    MXQ_DEBUG_SCOPE();
    MXQ_DEBUG_EXPECT(a_codes, m * k);
    MXQ_DEBUG_EXPECT(a_scales, m * (k / (size_t)block));
    MXQ_DEBUG_EXPECT(b_codes, n * k);
    MXQ_DEBUG_EXPECT(b_scales, n * (k / (size_t)block));
    MXQ_DEBUG_EXPECT(dst, m * n * size);
    const MatmulArgs p{static_cast<const uint8_t*>(a_codes), a_scales, static_cast<const uint8_t*>(b_codes), b_scales, m, n, k, block,
                       static_cast<uint8_t*>(dst)};
    return m <= (size_t)kFewRows && few_us(p) <= matmul_tc_us(p) ? launch_matmul_few(p, dst_dtype, s) : launch_matmul_tc(p, dst_dtype, s);
}

int mxq_wait_status(int reset) { return tc_status(reset); }

}  // extern "C"
#pragma GCC visibility pop
