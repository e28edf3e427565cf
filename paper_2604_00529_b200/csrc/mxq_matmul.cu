// D = A^ B^T of two MXFP8 E4M3 operands with one E8M0 scale per block along k (the product that the converted weights are for,
// Sec. 3.5): D[i, j] = sum over blocks b of Xa[i, b] Xb[j, b] sum over k in b of Pa[i, k] Pb[j, k].
#include "mxq_kernels.cuh"
#include "mxq_launch.h"
#include "mxq_product.cuh"

namespace mxq {

namespace {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// ---- few rows of A ----------------------------------------------------------------------------------------
// Bound by reading B once.  A CTA of eight warps covers 16 rows of B and 8 NG rows of A; the warps share k out in chunks of 64
// and meet in shared memory at the end, in a fixed order.  Codes go from global memory straight into the fragments of the
// warp's matrix instruction: widened to FP16, exactly, by the conversion instruction, and the block's two scales
// multiply the FP32 sum of the block.
//   BLK32: blocks of 32; a lane's piece is then 8 bytes, so that a matrix step stays within a block (16 bytes otherwise).

constexpr int kFewWarps = 8;
constexpr int kFewDepth = 4;                                // chunks in flight per warp

template <bool BLK32>
struct Piece;                                               // the codes of one row in a chunk of 64: 16 bytes per lane
template <>
struct Piece<false> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const uint8_t* row, size_t k0, size_t k, int t)
    {
        const size_t at = k0 + (size_t)t * 16;
        const uint4 v = at < k ? ld_once(row + at) : make_uint4(0, 0, 0, 0);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
};
template <>
struct Piece<true> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const uint8_t* row, size_t k0, size_t k, int t)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const size_t at = k0 + 32 * h + (size_t)t * 8;
            const uint2 v = at < k ? ld_once8(row + at) : make_uint2(0, 0);
            w[2 * h] = v.x;
            w[2 * h + 1] = v.y;
        }
    }
};

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

template <class OUT, int NG, bool BLK32>
__global__ void __launch_bounds__(kFewWarps * 32)
matmul_few_kernel(const uint8_t* __restrict__ a, const uint8_t* __restrict__ as, const uint8_t* __restrict__ b,
                  const uint8_t* __restrict__ bs, size_t m, size_t n, size_t k, uint32_t tiles_n, uint32_t kblocks, int block_shift,
                  uint8_t* __restrict__ dst)
{
    constexpr int SUB = BLK32 ? 2 : 1;                      // blocks that a chunk of 64 touches
    __shared__ float s_sum[kFewWarps][NG][4][32];
    pdl_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const size_t j0 = (size_t)(blockIdx.x % tiles_n) * 16, i0 = (size_t)(blockIdx.x / tiles_n) * (8 * NG);
    pdl_acquire();
    // rows beyond the matrix read its last row; their results are not stored
    const size_t jr[2] = {min(j0 + g, n - 1), min(j0 + g + 8, n - 1)};
    size_t ir[NG], ic[NG][2];
#pragma unroll
    for (int q = 0; q < NG; ++q) {
        ir[q] = min(i0 + q * 8 + g, m - 1);
        ic[q][0] = min(i0 + q * 8 + 2 * t, m - 1);
        ic[q][1] = min(i0 + q * 8 + 2 * t + 1, m - 1);
    }
    float sum[NG][4] = {};
    const size_t chunks = (k + 63) / 64;
    for (size_t c0 = warp; c0 < chunks; c0 += kFewWarps * kFewDepth) {
        Piece<BLK32> pb[kFewDepth][2], pa[kFewDepth][NG];
        uint32_t xb[kFewDepth][2][SUB], xa[kFewDepth][NG][2][SUB];
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) {
            const size_t c = c0 + d * kFewWarps, k0 = c * 64;       // a chunk beyond k loads nothing and adds zeros
#pragma unroll
            for (int h = 0; h < 2; ++h) pb[d][h].load(b + jr[h] * k, k0, k, t);
#pragma unroll
            for (int q = 0; q < NG; ++q) pa[d][q].load(a + ir[q] * k, k0, k, t);
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                const size_t kk = k0 + 32 * s, kb = kk >> block_shift;
                const bool in = kk < k;
#pragma unroll
                for (int h = 0; h < 2; ++h) xb[d][h][s] = in ? ld_u8(bs + jr[h] * kblocks + kb) : 127u;
#pragma unroll
                for (int q = 0; q < NG; ++q)
#pragma unroll
                    for (int h = 0; h < 2; ++h) xa[d][q][h][s] = in ? ld_u8(as + ic[q][h] * kblocks + kb) : 127u;
            }
        }
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) {
            uint32_t f0[8], f1[8];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                e4m3_word_to_f16(pb[d][0].w[w], f0[2 * w], f0[2 * w + 1]);
                e4m3_word_to_f16(pb[d][1].w[w], f1[2 * w], f1[2 * w + 1]);
            }
#pragma unroll
            for (int q = 0; q < NG; ++q) {
                uint32_t x[8];
#pragma unroll
                for (int w = 0; w < 4; ++w) e4m3_word_to_f16(pa[d][q].w[w], x[2 * w], x[2 * w + 1]);
#pragma unroll
                for (int s = 0; s < SUB; ++s) {
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = s * (4 / SUB); w < (s + 1) * (4 / SUB); ++w)
                        F16Mma::mma(acc, f0[2 * w], f1[2 * w], f0[2 * w + 1], f1[2 * w + 1], x[2 * w], x[2 * w + 1]);
                    add_scaled(sum[q], acc, xb[d][0][s], xb[d][1][s], xa[d][q][0][s], xa[d][q][1][s]);
                }
            }
        }
    }
#pragma unroll
    for (int q = 0; q < NG; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) s_sum[warp][q][e][lane] = sum[q][e];
    __syncthreads();
    // element (row g + 8 (e >> 1) of B, row 2 t + (e & 1) of A) of group q sits at [q][e][g * 4 + t]
    for (int o = threadIdx.x; o < NG * 128; o += kFewWarps * 32) {
        const int q = o >> 7, col = (o >> 4) & 7, row = o & 15;
        const int e = (row >> 3) * 2 + (col & 1), ln = (row & 7) * 4 + (col >> 1);
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) v += s_sum[w][q][e][ln];
        const size_t i = i0 + q * 8 + col, j = j0 + row;
        if (i < m && j < n) store_out<OUT>(dst, i * n + j, v);
    }
}

template <class OUT, int NG>
int run_few(const MatmulArgs& p, cudaStream_t stream)
{
    const size_t gx = (p.n + 15) / 16, gy = (p.m + 8 * NG - 1) / (8 * NG);
    if (gx * gy > 0x7FFFFFFF) return MXQ_ERR_SIZE;
    const uint32_t kblocks = (uint32_t)(p.k / (size_t)p.block);
    const int shift = p.block == 32 ? 5 : p.block == 64 ? 6 : 7;
    auto go = [&](auto kern) {
        return launch_kernel(kern, (int)(gx * gy), kFewWarps * 32, stream, p.a, p.as, p.b, p.bs, p.m, p.n, p.k, (uint32_t)gx, kblocks, shift,
                             p.dst);
    };
    return p.block == 32 ? go(matmul_few_kernel<OUT, NG, true>) : go(matmul_few_kernel<OUT, NG, false>);
}

}  // namespace

int launch_matmul_few(const MatmulArgs& p, int dst_dtype, cudaStream_t stream)
{
    if (p.m <= 8) return dst_dtype == MXQ_F32 ? run_few<F32, 1>(p, stream) : run_few<BF16, 1>(p, stream);
    return dst_dtype == MXQ_F32 ? run_few<F32, 2>(p, stream) : run_few<BF16, 2>(p, stream);
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
    return m <= 4 ? launch_matmul_few(p, dst_dtype, s) : launch_matmul_tc(p, dst_dtype, s);
}

int mxq_wait_status(int reset) { return tc_status(reset); }

}  // extern "C"
#pragma GCC visibility pop
