// What the attention kernels share: the call's arguments, where a head's channels and an image's valid pixels lie.
#pragma once

#include <cfloat>
#include <cmath>

#include "entry.cuh"

namespace small {

struct AttnArgs {
    const float *q, *k, *v, *bias;
    const int32_t *q_ext, *k_ext;
    float *out;
    void *ws;
    int N, heads, kv_heads, D, QH, QW, KH, KW;
    int QP, KP, CB;                                      // pixels of the planes, channel blocks of q and out
    long long q_stride, k_stride, v_stride;              // floats between images
    float scale, cap;
    int pitch;                                           // of the bias table's rows as it is read: QW + KW - 1, or more where a copy of it is
};

#ifdef __CUDACC__
// An image's valid rows and columns.
__device__ __forceinline__ int2 extent(const int32_t *e, int n, int h, int w) {
    if (!e) return make_int2(h, w);
    return make_int2(min(max(e[2 * n], 0), h), min(max(e[2 * n + 1], 0), w));
}
// Float of channel c, pixel p in an image of `pixels`.
__device__ __forceinline__ size_t at(int c, int p, int pixels) { return ((size_t)(c >> 5) * pixels + p) * 32 + (c & 31); }

// Places in the bias table: of_query(i) - of_key(j) is that of the pair's displacement.
__device__ __forceinline__ int of_query(const AttnArgs &a, int i) { return (i / a.QW + a.KH - 1) * a.pitch + i % a.QW + a.KW - 1; }
__device__ __forceinline__ int of_key(const AttnArgs &a, int y, int x) { return y * a.pitch + x; }

constexpr float kLog2e = 1.4426950408889634f;

// A table entry for exponentials of two; finite values stay finite, those below -2.3e38 are taken as equally low.
__device__ __forceinline__ float powers_of_two(float b) {
    const float r = b * kLog2e;
    return fabsf(r) < INFINITY || !(fabsf(b) < INFINITY) ? r : copysignf(FLT_MAX, b);
}
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Four consecutive channels from c on of a head's `D` at pixel p, 0 behind the last.  Eight lanes take a row's 128 bytes together.
__device__ __forceinline__ float4 load4(const float *x, int first, int c, int D, int p, int pixels) {
    if (((first | D) & 3) == 0) return c < D ? *reinterpret_cast<const float4 *>(x + at(first + c, p, pixels)) : make_float4(0.f, 0.f, 0.f, 0.f);
    float4 v;
    v.x = c + 0 < D ? x[at(first + c + 0, p, pixels)] : 0.0f; v.y = c + 1 < D ? x[at(first + c + 1, p, pixels)] : 0.0f;
    v.z = c + 2 < D ? x[at(first + c + 2, p, pixels)] : 0.0f; v.w = c + 3 < D ? x[at(first + c + 3, p, pixels)] : 0.0f;
    return v;
}

__device__ __forceinline__ void copy16_or_clear(uint32_t to, const float *from, bool some) {        // 16 bytes to shared memory, zeros where there are none
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(some ? 16 : 0) : "memory");
}

// cap * tanh(x / cap).  Below 1/2 by Lambert's continued fraction x / (1 + x^2 / (3 + x^2 / (5 + x^2 / (7 + x^2 / 9)))), whose
// relative error there is some x^10 / 1e7, 1e-10; above as (e - 1) / (e + 1), e = exp(2 x), where neither is a small difference.
__device__ __forceinline__ float capped(float x, float cap, float over_cap) {
    const float t = x * over_cap, u = fminf(fabsf(t), 16.0f), s = u * u, e = __expf(2.0f * u);
    const float num = u < 0.5f ? u * fmaf(s, s + 105.0f, 945.0f) : e - 1.0f;
    const float den = u < 0.5f ? fmaf(s, fmaf(s, 15.0f, 420.0f), 945.0f) : e + 1.0f;
    return t == t ? copysignf(cap * __fdividef(num, den), t) : x;
}
#endif

// attention.cu
int launch_attention_fp32(small_ctx *, const AttnArgs &, cudaStream_t);
// attention_few.cu: few queries; a row is a query of a head that shares its keys
constexpr int kFewQueries = 16;
int launch_attention_few(small_ctx *, const AttnArgs &, cudaStream_t);
// attention_small.cu: a head's keys and values in a block's shared memory, and how much of it that takes
constexpr size_t kSmallShared = 220 * 1024;
size_t attention_small_bytes(int D, int KP);
int launch_attention_small(small_ctx *, const AttnArgs &, cudaStream_t);
// attention_tc.cu: the tensor-core form, and the workspace it takes
size_t attention_tc_workspace(int N, int kv_heads, int D, int KP);
int launch_attention_tc(small_ctx *, const AttnArgs &, bool x3, cudaStream_t);

}  // namespace small
