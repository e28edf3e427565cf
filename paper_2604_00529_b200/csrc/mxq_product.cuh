// What the kernels that multiply by stored codes share: the warp's matrix instruction on 16-bit operands, and the
// widening of packed element codes to 16-bit values in the fragment order of that instruction.
//
// A warp's m16n8k16 step takes from lane (g = lane / 4, t = lane % 4) two pairs of row g, two pairs of row g + 8 and two
// pairs of column g; which 16 of the k values the step covers, and in which order, is free as long as both
// operands agree.  So a lane reads 16 consecutive bytes of codes of its rows and uses them as they lie.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "mxq_access.cuh"
#include "mxq_codec.cuh"

namespace mxq {

struct F16Mma {
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
struct Bf16Mma {
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
    {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};

// 16 bytes of an operand that nothing writes while the kernel runs.
__device__ __forceinline__ uint4 ld_once(const uint8_t* p)
{
    uint4 v = make_uint4(0, 0, 0, 0);
    MXQ_CHECKED(p, 16, return v)
    asm volatile("ld.global.nc.L1::no_allocate.L2::128B.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// ---- codes to BF16 pairs, the block's scale multiplied in -------------------------------------------------
// Every element value of these formats has at most eight significant bits, and a scale is a power of two: the product is a BF16
// number, exactly, unless it leaves BF16's range (FP32's range: it then over- or underflows as FP32 would, to within a
// subnormal's rounding).  MXFP: the code's fields put in the places of BF16's stand for 2^-120 (E4M3) or 2^-126 (E2M1) times
// the element, subnormal elements being BF16 subnormals, and the scale's multiplier puts that back.  MXINT: the code under the
// exponent of 128 is 128 + its low bits.  E4M3's NaN codes (S.1111.111) would come out as 480 and are looked for by themselves
// (note_nan).
// Word w of a lane's 16 bytes gives NP = 2 (8 bits) or 4 (4 bits) pairs; pairs hold the word's elements in the order of order_pairs.

template <int FMT>
struct Widen {
    static constexpr int bits = fmt_info(FMT).bits;
    static constexpr bool fp = fmt_info(FMT).kind == KIND_FP;
    static constexpr int NP = bits == 8 ? 2 : 4;
    static constexpr int up = !fp ? 0 : FMT == MXQ_FP8_E4M3 ? 120 : 126;      // codes stand for 2^-up times the element
    static constexpr uint32_t limit = 254u - (uint32_t)up;                    // the largest byte whose multiplier is one BF16 number
    static_assert(FMT == MXQ_FP8_E4M3 || FMT == MXQ_FP4_E2M1 || FMT == MXQ_INT8 || FMT == MXQ_INT4, "8- and 4-bit formats");

    // the multiplier 2^(byte - 127 + up), as a pair; beyond BF16's range its first factor
    static __device__ __forceinline__ uint32_t factor(uint32_t byte)
    {
        uint32_t h;
        if constexpr (fp) h = min(byte + (uint32_t)up, 254u) << 7;
        else h = byte == 255u ? 0x7FC0u : byte ? byte << 7 : 0x0040u;
        return h * 0x10001u;
    }
    // the second factor (1 for bytes up to `limit`, NaN for 0xFF)
    static __device__ __forceinline__ uint32_t factor2(uint32_t byte)
    {
        const uint32_t h = byte == 255u ? 0x7FC0u : byte <= limit ? 0x3F80u : (byte - limit + 127u) << 7;
        return h * 0x10001u;
    }
    static constexpr bool has_nan = FMT == MXQ_FP8_E4M3;
    // Adding one to a byte flips its top bit exactly if the seven bits below are ones.  (The carry out of 0xFF may flip more; 0xFF is a
    // NaN code itself.)  Two instructions per four codes.
    static __device__ __forceinline__ void note_nan(const uint4& c, uint32_t& seen)
    {
        seen |= (c.x + 0x01010101u) ^ c.x;
        seen |= (c.y + 0x01010101u) ^ c.y;
        seen |= (c.z + 0x01010101u) ^ c.z;
        seen |= (c.w + 0x01010101u) ^ c.w;
    }
    static __device__ __forceinline__ bool saw_nan(uint32_t seen) { return (seen & 0x80808080u) != 0; }
    static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b)
    {
        uint32_t d;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
    static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t b)
    {
        uint32_t d;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        return d;
    }
    static __device__ __forceinline__ void pairs(uint32_t w, uint32_t f, uint32_t (&o)[NP])
    {
        if constexpr (FMT == MXQ_FP8_E4M3) {
            o[0] = ((w << 8) & 0x80008000u) | ((w << 4) & 0x07F007F0u);
            o[1] = (w & 0x80008000u) | ((w >> 4) & 0x07F007F0u);
        } else if constexpr (FMT == MXQ_FP4_E2M1) {
            // a nibble n, multiplied by 2^6 + 2^12, has its magnitude at bits 6 - 8 and its sign at bit 15
            const uint32_t h = w >> 8;
            o[0] = ((w & 0x000F000Fu) * 4160u) & 0x81C081C0u;
            o[1] = ((w & 0x00F000F0u) * 260u) & 0x81C081C0u;
            o[2] = ((h & 0x000F000Fu) * 4160u) & 0x81C081C0u;
            o[3] = ((h & 0x00F000F0u) * 260u) & 0x81C081C0u;
        } else if constexpr (FMT == MXQ_INT8) {
            const uint32_t h = w >> 8;
            o[0] = sub((w & 0x007F007Fu) | 0x43004300u, (w & 0x00800080u) | 0x43004300u);
            o[1] = sub((h & 0x007F007Fu) | 0x43004300u, (h & 0x00800080u) | 0x43004300u);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = sub(((w >> (4 * i)) & 0x000F000Fu) ^ 0x43084308u, 0x43084308u);
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) o[i] = mul(o[i], f);
    }
};

// The same order for the other operand: BF16 pairs of consecutive elements -> the pairs of Widen (NP words of a code word's
// elements: x[0 .. NP) in memory order).
template <int NP>
__device__ __forceinline__ void order_pairs(const uint32_t (&x)[NP], uint32_t (&o)[NP])
{
    if constexpr (NP == 2) {
        o[0] = __byte_perm(x[0], x[1], 0x5410);
        o[1] = __byte_perm(x[0], x[1], 0x7632);
    } else {
        o[0] = __byte_perm(x[0], x[2], 0x5410);
        o[1] = __byte_perm(x[0], x[2], 0x7632);
        o[2] = __byte_perm(x[1], x[3], 0x5410);
        o[3] = __byte_perm(x[1], x[3], 0x7632);
    }
}

}  // namespace mxq
