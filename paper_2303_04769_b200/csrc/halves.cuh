// FP32 operands as pairs of halves for tcgen05 kind::f16.
//
// A float x is x_hi + x_lo, two halves of 11 significant bits each after a power of two has brought the largest value of its row or tile to
// 2^14 .. 2^15, so nothing the sums can see is lost to half precision's range.  3xTF32 forms hi*hi + hi*lo + lo*hi, TF32 hi*hi alone: a half has
// TF32's 11 bits, and kind::f16 runs at twice kind::tf32's rate and reads half the bytes.
#pragma once

#include <cuda_fp16.h>

#include "entry.cuh"
#include "sm100.cuh"

namespace small {
namespace halves {
using namespace sm100;

constexpr int kTile = 128;               // rows of an operand tile

// The exponent that brings |x| <= most to below 2^15: x * lift(e) and back by drop(e).
__device__ __forceinline__ int top_exponent(float most) { return min(max((int)(__float_as_uint(most) >> 23), 15), 254); }     // most >= 0
__device__ __forceinline__ float lift(int e) { return __uint_as_float((uint32_t)(268 - e) << 23); }
__device__ __forceinline__ float drop(int e) { return __uint_as_float((uint32_t)(e - 14) << 23); }

// 2^e: 0 where it is less than any float, and no more than 2^127.
__device__ __forceinline__ float power(int e) {
    e = min(e, 127);
    return __uint_as_float(e >= -126 ? (uint32_t)(e + 127) << 23 : e >= -149 ? 1u << (e + 149) : 0u);
}

// |x|; what is not finite does not count: it stays what it is at any scale, and must not take its tile's other values with it.
__device__ __forceinline__ float magnitude(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.0f; }

__device__ __forceinline__ uint32_t pack_halves(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two operands -> the nearest halves (off by at most 2^-12 of the value) and what these leave.  What is left of a value that is not finite
// is 0, or it would turn infinities into NaN in every product.
__device__ __forceinline__ float nearest_half(float x) { return __uint_as_float((__float_as_uint(x) + 0x1000u) & 0xffffe000u); }        // |x| < 65488
__device__ __forceinline__ void split_finite(float a, float b, uint32_t &hi, uint32_t &lo) {
    const float ah = nearest_half(a), bh = nearest_half(b);
    hi = pack_halves(ah, bh);
    lo = pack_halves(a - ah, b - bh);
    const bool a_in = fabsf(a) < 65488.0f, b_in = fabsf(b) < 65488.0f;
    if (!a_in || !b_in) {
        hi = pack_halves(a_in ? ah : a, b_in ? bh : b);
        lo = pack_halves(a_in ? a - ah : 0.0f, b_in ? b - bh : 0.0f);
    }
}

// Byte of the 16-byte chunk that holds columns c .. c + 7 of row r: atoms of 64 columns, `rows` rows of 128 bytes each, swizzled.
__device__ __forceinline__ uint32_t chunk_at(int r, int c, int rows) {
    return (uint32_t)(c >> 6) * rows * 128 + r * 128 + ((((uint32_t)c >> 3 & 7) ^ (r & 7)) << 4);
}

__device__ __forceinline__ float magnitude(float4 v) { return fmaxf(fmaxf(magnitude(v.x), magnitude(v.y)), fmaxf(magnitude(v.z), magnitude(v.w))); }
// Their high and low parts to a tile of `DP` channels of high parts and as many of low ones.
template <int DP>
__device__ __forceinline__ void store4(char *tile, int r, int c, float4 v, float up) {
    uint2 hi, lo;
    split_finite(v.x * up, v.y * up, hi.x, lo.x);
    split_finite(v.z * up, v.w * up, hi.y, lo.y);
    *reinterpret_cast<uint2 *>(tile + chunk_at(r, c, kTile) + (c & 4) * 2) = hi;
    *reinterpret_cast<uint2 *>(tile + chunk_at(r, DP + c, kTile) + (c & 4) * 2) = lo;
}

// D[tmem] (+)= A * B^T in halves, FP32 accumulate, M = 128, K = 16; A from shared memory, or from tensor memory (two halves a column).
__device__ __forceinline__ void mma_f16(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}"
        ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(kDescHi), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_f16_tmem(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %3};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b_lo), "r"(kDescHi), "r"(idesc), "r"(accumulate) : "memory");
}
// Two floats as one operand of the packed FP32 instructions.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
          "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ uint32_t f16_desc(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24); }

}  // namespace halves
}  // namespace small
