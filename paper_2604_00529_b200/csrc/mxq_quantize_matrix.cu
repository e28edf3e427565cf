// Q_f (Eq. 1-3) of a matrix along its rows and of its transpose, from one read: the operands of a linear layer's three products
// (y = x w^T takes x and w along k, dx = dy w takes dy along n and w^T along n, dw = dy^T x takes both transposes along m).
//
// A CTA of 256 threads holds a tile of 128 x 128 elements in registers, eight columns of four consecutive rows, twice, per
// thread.  Blocks of 32, 64 or 128 elements never cross a tile.  Along the rows the block maximum is a shuffle over 4, 8 or
// 16 lanes; along the columns each thread's four rows meet in shared memory.  The transposed codes go through shared memory
// four rows to a word, words exchanged so that neither side has bank conflicts, and leave as whole 128-byte lines.
// Rows beyond the matrix, up to a whole block, are zeros: they add nothing to a product.
#include "mxq_kernels.cuh"
#include "mxq_launch.h"

namespace mxq {
namespace {

constexpr int kTile = 128;
constexpr int kMatThreads = 256;

// Eight consecutive elements of one row: BF16 as they lie in memory, two to a word (half the registers of FP32 values).
template <class T>
struct Eight;
template <>
struct Eight<BF16> {
    uint32_t w[4];
    __device__ __forceinline__ float at(int j) const { return __uint_as_float((j & 1) ? (w[j / 2] & 0xFFFF0000u) : (w[j / 2] << 16)); }
    __device__ __forceinline__ uint32_t upper2(int i) const { return w[i] & 0x7FFF7FFFu; }      // |patterns|' upper halves, elements 2 i, 2 i + 1
    __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
    __device__ __forceinline__ void load(const uint8_t* p)
    {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    }
    __device__ __forceinline__ void put(int j, const uint8_t* p) { w[j / 2] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(p)) << (16 * (j & 1)); }
};
template <>
struct Eight<F32> {
    uint32_t w[8];
    __device__ __forceinline__ float at(int j) const { return __uint_as_float(w[j]); }
    __device__ __forceinline__ uint32_t upper2(int i) const { return __byte_perm(w[2 * i], w[2 * i + 1], 0x7632) & 0x7FFF7FFFu; }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 0;
    }
    __device__ __forceinline__ void load(const uint8_t* p)
    {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p)), b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
    __device__ __forceinline__ void put(int j, const uint8_t* p) { w[j] = __ldg(reinterpret_cast<const uint32_t*>(p)); }
};

// Eight elements at p, the first `left` columns of them inside the matrix; zeros outside.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const uint8_t* __restrict__ p, size_t left, Eight<T>& v)
{
    v.zero();
    if constexpr (VEC) {                                     // cols % 8 == 0: a piece is inside or outside as a whole
        if (left == 0) return;
        MXQ_CHECKED(p, 8 * T::size, return)
        v.load(p);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if ((size_t)j >= left) continue;
            MXQ_CHECKED(p + j * T::size, T::size, continue)
            v.put(j, p + j * T::size);
        }
    }
}

struct MatrixShared {
    uint32_t max[2][8][kTile / 2];                           // [rows / 64][warp][column pair]
    uint8_t byte[4][kTile];                                  // scale byte per group of 32 rows and column
    alignas(16) float inv[4][kTile];                         // its multiplier
    alignas(16) uint32_t codes[kTile][32];                   // [column][four rows], exchanged
};

// FP32 bit patterns are ordered like the values, and only the exponent field of a maximum is used (0xFF: the block is
// poisoned): the patterns' upper halves are enough, two to a word.
//   WHOLE: the tile lies inside the matrix; nothing is compared with its edges.  (The kernel is bound by instructions: 14336 x 4096 BF16
//   took 25 per element and 55 us with every access compared and addressed for itself, 45 us like this: 5.2 TB/s.  The variants
//   without vector loads, for cols % 8 != 0, spill 8 to 68 bytes per thread.)
template <class T, class F, int BLOCK, bool VEC, bool WHOLE>
__device__ __forceinline__ void matrix_tile(const uint8_t* __restrict__ src, size_t rows, size_t cols, uint8_t* __restrict__ codes,
                                            uint8_t* __restrict__ scales, uint8_t* __restrict__ codes_t, uint8_t* __restrict__ scales_t, size_t tr, size_t tc, MatrixShared& sh)
{
    constexpr int LPB = BLOCK / 8;                           // lanes per block along a row
    constexpr int G = BLOCK / 32;                            // groups of 32 rows per block along a column
    auto& s_max = sh.max;
    auto& s_byte = sh.byte;
    auto& s_inv = sh.inv;
    auto& s_codes = sh.codes;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, l = lane & 15, rg = warp * 2 + (lane >> 4);
    const size_t r0 = tr * kTile, c0 = tc * kTile, c = c0 + l * 8;
    const size_t rows_p = (rows + BLOCK - 1) / BLOCK * BLOCK, cols_p = (cols + BLOCK - 1) / BLOCK * BLOCK;
    const size_t row = r0 + rg * 4;                          // the thread's rows: row + i and row + 64 + i

    Eight<T> v[2][4];
    {
        const size_t pitch = cols * T::size, left = WHOLE ? 8 : cols > c ? cols - c : 0;
        const uint8_t* p = src + row * pitch + c * T::size;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) load8<T, VEC>(p + (s * 64 + i) * pitch, WHOLE || row + s * 64 + i < rows ? left : 0, v[s][i]);
    }

    // along the columns: the thread's four rows, the two halves of the warp, then (below) the four warps of a group of 32 rows
    if (codes_t) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t m = __vmaxu2(__vmaxu2(v[s][0].upper2(j), v[s][1].upper2(j)), __vmaxu2(v[s][2].upper2(j), v[s][3].upper2(j)));
                m = __vmaxu2(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                if (lane < 16) s_max[s][warp][l * 4 + j] = m;
            }
    }

    if (codes) {                                             // along the rows: the maxima of two rows to a word
        uint32_t m[2][2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t a[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const Eight<T>& e = v[s][2 * h + i];
                    a[i] = __vmaxu2(__vmaxu2(e.upper2(0), e.upper2(1)), __vmaxu2(e.upper2(2), e.upper2(3)));
                }
                m[s][h] = __vmaxu2(__byte_perm(a[0], a[1], 0x5410), __byte_perm(a[0], a[1], 0x7632));
            }
#pragma unroll
        for (int o = 1; o < LPB; o <<= 1)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h) m[s][h] = __vmaxu2(m[s][h], __shfl_xor_sync(0xFFFFFFFFu, m[s][h], o));
        uint8_t* const pc = codes + row * cols_p + c;
        uint8_t* const ps = scales + row * (cols_p / BLOCK) + c / BLOCK;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Eight<T>& e = v[s][i];
                const BlockScale sc = block_scale<F>((i & 1) ? m[s][i / 2] & 0xFFFF0000u : m[s][i / 2] << 16);
                uint2 q;
                q.x = quantize_fp_hw_quad<F>(e.at(0) * sc.inv, e.at(1) * sc.inv, e.at(2) * sc.inv, e.at(3) * sc.inv);
                q.y = quantize_fp_hw_quad<F>(e.at(4) * sc.inv, e.at(5) * sc.inv, e.at(6) * sc.inv, e.at(7) * sc.inv);
                if (sc.byte == 255u) q = make_uint2(0, 0);
                if (WHOLE || (row + s * 64 + i < rows && c < cols_p)) {
                    uint8_t* p = pc + (s * 64 + i) * cols_p;
                    bool ok = true;
                    MXQ_CHECKED(p, 8, ok = false)
                    if (ok) *reinterpret_cast<uint2*>(p) = q;
                    if (l % LPB == 0) st_u8(ps + (s * 64 + i) * (cols_p / BLOCK), sc.byte);
                }
            }
    }
    if (!codes_t) return;
    __syncthreads();
    bool poison = false;
    {
        const int k0 = (tid >> 7) * 2, col = tid & 127;      // two groups of 32 rows of one column
        uint32_t g[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (G < 4 && (k >> 1) != (k0 >> 1)) continue;
            uint32_t m = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) m = max(m, (s_max[k >> 1][(k & 1) * 4 + w][col >> 1] >> (16 * (col & 1))) & 0xFFFFu);
            g[k] = m;
        }
        uint32_t lo = k0 ? g[2] : g[0], hi = k0 ? g[3] : g[1];
        if constexpr (G == 2) lo = hi = max(lo, hi);
        if constexpr (G == 4) lo = hi = max(max(g[0], g[1]), max(g[2], g[3]));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const BlockScale sc = block_scale<F>((h ? hi : lo) << 16);
            s_byte[k0 + h][col] = (uint8_t)sc.byte;
            s_inv[k0 + h][col] = sc.byte == 255u ? __uint_as_float(0x7FC00000u) : sc.inv;
            poison |= sc.byte == 255u;
        }
    }
    poison = __syncthreads_or(poison);
    if (tid < kTile && (WHOLE || c0 + tid < cols)) {         // a column's scale bytes: one store where they are aligned
        constexpr int N = 4 / G;
        const size_t per_col = rows_p / BLOCK;
        uint8_t* to = scales_t + (c0 + tid) * per_col + tr * N;
        const uint32_t a = s_byte[0][tid], b = s_byte[G == 1 ? 1 : 2][tid];
        if (N == 4 && per_col % 4 == 0) {
            st_u32(to, a | b << 8 | (uint32_t)s_byte[2][tid] << 16 | (uint32_t)s_byte[3][tid] << 24);
        } else if (N == 2 && per_col % 2 == 0) {
            st_u16(to, a | b << 8);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (WHOLE || r0 + k * BLOCK < rows_p) st_u8(to + k, s_byte[k * G][tid]);
        }
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const float* const from = &s_inv[s * 2 + (rg >> 3)][l * 8];
        const float4 f0 = *reinterpret_cast<const float4*>(from), f1 = *reinterpret_cast<const float4*>(from + 4);
        const float inv[8] = {f0.x, f0.y, f0.z, f0.w, f1.x, f1.y, f1.z, f1.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t q = quantize_fp_hw_quad<F>(v[s][0].at(j) * inv[j], v[s][1].at(j) * inv[j], v[s][2].at(j) * inv[j], v[s][3].at(j) * inv[j]);
            if (poison && inv[j] != inv[j]) q = 0;           // (`poison` is the CTA's)
            s_codes[l * 8 + j][(rg + 16 * s) ^ (2 * l)] = q;
        }
    }
    __syncthreads();
    // a column's 128 rows: 16 lanes of eight bytes each
    const size_t at = r0 + (size_t)l * 8;
    const int c1 = warp * 2 + (lane >> 4);
    uint8_t* to = codes_t + (c0 + c1) * rows_p + at;
    const size_t step = 16 * rows_p;
#pragma unroll
    for (int n = 0; n < kTile / 16; ++n, to += step) {
        const int cc = c1 + n * 16;
        const uint2 q = *reinterpret_cast<const uint2*>(&s_codes[cc][(2 * l) ^ (2 * (cc >> 3))]);
        if (!WHOLE && (c0 + cc >= cols || at >= rows_p)) continue;
        MXQ_CHECKED(to, 8, continue)
        *reinterpret_cast<uint2*>(to) = q;
    }
}

template <class T, class F, int BLOCK, bool VEC>
__global__ void __launch_bounds__(kMatThreads, T::size == 2 && VEC ? 4 : T::size == 2 ? 3 : 2)
quantize_matrix_kernel(const uint8_t* __restrict__ src, size_t rows, size_t cols, uint8_t* __restrict__ codes,
                       uint8_t* __restrict__ scales, uint8_t* __restrict__ codes_t, uint8_t* __restrict__ scales_t, uint32_t row_tiles, uint32_t col_tiles)
{
    __shared__ MatrixShared sh;
    pdl_release();
    // eight tiles of a column one after another: the transpose's lines then meet in L2 as longer runs
    const uint32_t band = blockIdx.x / (8 * col_tiles), height = min(8u, row_tiles - band * 8), in_band = blockIdx.x - band * 8 * col_tiles;
    const size_t tr = band * 8 + in_band % height, tc = in_band / height;
    pdl_acquire();
    if ((tr + 1) * kTile <= rows && (tc + 1) * kTile <= cols) matrix_tile<T, F, BLOCK, VEC, true>(src, rows, cols, codes, scales, codes_t, scales_t, tr, tc, sh);
    else matrix_tile<T, F, BLOCK, VEC, false>(src, rows, cols, codes, scales, codes_t, scales_t, tr, tc, sh);
}

template <class T, int BLOCK>
int run(const void* src, size_t rows, size_t cols, void* codes, uint8_t* scales, void* codes_t, uint8_t* scales_t, cudaStream_t stream)
{
    using F = Fmt<MXQ_FP8_E4M3>;
    const size_t rt = (rows + kTile - 1) / kTile, ct = (cols + kTile - 1) / kTile;
    if (ct > (1u << 28) || rt > 0x7FFFFFFF / ct) return MXQ_ERR_SIZE;
    auto go = [&](auto kern) {
        return launch_kernel(kern, (int)(rt * ct), kMatThreads, stream, static_cast<const uint8_t*>(src), rows, cols,
                             static_cast<uint8_t*>(codes), scales, static_cast<uint8_t*>(codes_t), scales_t, (uint32_t)rt, (uint32_t)ct);
    };
    return cols % 8 == 0 ? go(quantize_matrix_kernel<T, F, BLOCK, true>) : go(quantize_matrix_kernel<T, F, BLOCK, false>);
}

template <class T>
int by_block(int block, const void* src, size_t rows, size_t cols, void* codes, uint8_t* scales, void* codes_t, uint8_t* scales_t,
             cudaStream_t stream)
{
    switch (block) {
    case 32: return run<T, 32>(src, rows, cols, codes, scales, codes_t, scales_t, stream);
    case 64: return run<T, 64>(src, rows, cols, codes, scales, codes_t, scales_t, stream);
    default: return run<T, 128>(src, rows, cols, codes, scales, codes_t, scales_t, stream);
    }
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace

}  // namespace mxq

using namespace mxq;

#pragma GCC visibility push(default)
extern "C" {

size_t mxq_matrix_codes_bytes(size_t rows, size_t cols, int block)
{
    return block > 0 ? rows * ((cols + (size_t)block - 1) / (size_t)block) * (size_t)block : 0;
}

size_t mxq_matrix_scales_bytes(size_t rows, size_t cols, int block)
{
    return block > 0 ? rows * ((cols + (size_t)block - 1) / (size_t)block) : 0;
}

int mxq_quantize_matrix(const void* src, int src_dtype, size_t rows, size_t cols, int fmt, int block, void* codes, uint8_t* scales,
                        void* codes_t, uint8_t* scales_t, mxq_stream stream)
{
    if (fmt != MXQ_FP8_E4M3 || (src_dtype != MXQ_F32 && src_dtype != MXQ_BF16)) return MXQ_ERR_FORMAT;
    if (block != 32 && block != 64 && block != 128) return MXQ_ERR_BLOCK;
    if (rows == 0 || cols == 0) return MXQ_OK;
    if (rows > (SIZE_MAX / 8) / cols) return MXQ_ERR_SIZE;
    if (!src || (!codes && !codes_t) || !codes != !scales || !codes_t != !scales_t) return MXQ_ERR_NULL;
    if (!aligned(src, 32) || !aligned(codes, 32) || !aligned(codes_t, 32) || !aligned(scales, 16) || !aligned(scales_t, 16)) return MXQ_ERR_ALIGN;
    MXQ_DEBUG_SCOPE();
    MXQ_DEBUG_EXPECT(src, rows * cols * (src_dtype == MXQ_F32 ? 4u : 2u));
    MXQ_DEBUG_EXPECT(codes, mxq_matrix_codes_bytes(rows, cols, block));
    MXQ_DEBUG_EXPECT(scales, mxq_matrix_scales_bytes(rows, cols, block));
    MXQ_DEBUG_EXPECT(codes_t, mxq_matrix_codes_bytes(cols, rows, block));
    MXQ_DEBUG_EXPECT(scales_t, mxq_matrix_scales_bytes(cols, rows, block));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (src_dtype == MXQ_F32) return by_block<F32>(block, src, rows, cols, codes, scales, codes_t, scales_t, s);
    return by_block<BF16>(block, src, rows, cols, codes, scales, codes_t, scales_t, s);
}

}  // extern "C"
#pragma GCC visibility pop
