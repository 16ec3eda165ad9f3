// Attention over the pixels of a plane: entry points, the rule that picks the kernel, and the FP32 kernel.
//
// attention_fp32_kernel: a block takes 64 queries of one head and walks the keys 64 at a time.  Scores, maxima and sums of a row stay
// in the 16 lanes that share it; the exponentials cross shared memory once to become the second product's operand.  Bound by FP32
// multiply-adds: 4 x 4 scores a thread, then 4 rows x D / 16 columns of the result.
#include <algorithm>

#include "attention.cuh"

namespace small {
namespace {

constexpr int kRows = 64, kKeys = 64, kThreads = 256, kPitch = kRows + 4;

template <int DP>
__global__ void __launch_bounds__(kThreads) attention_fp32_kernel(const AttnArgs a) {
    extern __shared__ float smem[];
    float *Qs = smem, *Ks = Qs + DP * kPitch, *Ps = Ks + DP * kPitch, *Vs = Ps + kKeys * kPitch;      // [d][row], [d][key], [key][row], [key][d]
    __shared__ int koff[kKeys];
    grid_dep_sync();
    grid_dep_trigger();
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    const int n = blockIdx.z, h = blockIdx.y, hk = h / (a.heads / a.kv_heads), i0 = blockIdx.x * kRows;
    const float *q = a.q + n * a.q_stride, *k = a.k + n * a.k_stride, *v = a.v + n * a.v_stride;
    const int2 qe = extent(a.q_ext, n, a.QH, a.QW), ke = extent(a.k_ext, n, a.KH, a.KW);
    const int keys = ke.x * ke.y;
    const float *bias = a.bias ? a.bias + (size_t)h * (a.QH + a.KH - 1) * (a.QW + a.KW - 1) : nullptr;
    const float over_cap = a.cap > 0.0f ? 1.0f / a.cap : 0.0f;

    for (int i = tid; i < DP * kRows; i += kThreads) {
        const int r = i / DP, d = i % DP, p = i0 + r;
        Qs[d * kPitch + r] = p < a.QP && d < a.D ? q[at(h * a.D + d, p, a.QP)] : 0.0f;
    }
    int qoff[4];
    float m[4], l[4], o[4][DP / 16];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        qoff[r] = bias && i0 + ty * 4 + r < a.QP ? of_query(a, i0 + ty * 4 + r) : -1;
        m[r] = -INFINITY;
        l[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) o[r][c] = 0.0f;
    }
    for (int j0 = 0; j0 < keys; j0 += kKeys) {
        __syncthreads();
        for (int i = tid; i < DP * kKeys; i += kThreads) {
            const int r = i / DP, d = i % DP, j = j0 + r;
            const bool in = j < keys && d < a.D;
            const int p = in ? j / ke.y * a.KW + j % ke.y : 0;
            const size_t e = in ? at(hk * a.D + d, p, a.KP) : 0;
            Ks[d * kPitch + r] = in ? k[e] : 0.0f;
            Vs[r * DP + d] = in ? v[e] : 0.0f;
        }
        if (tid < kKeys) koff[tid] = j0 + tid < keys ? of_key(a, (j0 + tid) / ke.y, (j0 + tid) % ke.y) : 0;
        __syncthreads();
        float s[4][4] = {};
#pragma unroll 4
        for (int d = 0; d < DP; ++d) {
            const float4 x = *reinterpret_cast<const float4 *>(Qs + d * kPitch + ty * 4), y = *reinterpret_cast<const float4 *>(Ks + d * kPitch + tx * 4);
            const float xr[4] = {x.x, x.y, x.z, x.w}, yr[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[r][c] = fmaf(xr[r], yr[c], s[r][c]);
        }
        float shrink[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float top = m[r];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float x = s[r][c] * a.scale;
                if (a.cap > 0.0f) x = capped(x, a.cap, over_cap);
                if (qoff[r] >= 0) x += j0 + tx * 4 + c < keys ? bias[qoff[r] - koff[tx * 4 + c]] : 0.0f;
                s[r][c] = j0 + tx * 4 + c < keys ? x : -INFINITY;
                top = fmaxf(top, s[r][c]);
            }
#pragma unroll
            for (int w = 1; w < 16; w *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, w));
            const float base = top == -INFINITY ? 0.0f : top;       // nothing to weigh yet: exp(-inf) below
            shrink[r] = __expf(m[r] - base);
            m[r] = top;
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) { s[r][c] = __expf(s[r][c] - base); sum += s[r][c]; }
            l[r] = fmaf(l[r], shrink[r], sum);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) *reinterpret_cast<float4 *>(Ps + (tx * 4 + c) * kPitch + ty * 4) = make_float4(s[0][c], s[1][c], s[2][c], s[3][c]);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) o[r][c] *= shrink[r];
#pragma unroll 4
        for (int j = 0; j < kKeys; ++j) {
            const float4 x = *reinterpret_cast<const float4 *>(Ps + j * kPitch + ty * 4);
            const float xr[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
                const float y = Vs[j * DP + c * 16 + tx];
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r][c] = fmaf(xr[r], y, o[r][c]);
            }
        }
    }
    const int pad = h == a.heads - 1 ? a.CB * 32 - a.heads * a.D : 0;        // lanes behind the last channel, written as +0
    float *out = a.out + (size_t)n * a.CB * a.QP * 32;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int p = i0 + ty * 4 + r;
        float sum = l[r];
#pragma unroll
        for (int w = 1; w < 16; w *= 2) sum += __shfl_xor_sync(~0u, sum, w);
        if (p >= a.QP) continue;
        const bool live = p / a.QW < qe.x && p % a.QW < qe.y && sum != 0.0f;
        const float inv = 1.0f / sum;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c)
            if (c * 16 + tx < a.D) out[at(h * a.D + c * 16 + tx, p, a.QP)] = live ? o[r][c] * inv : 0.0f;
        for (int c = tx; c < pad; c += 16) out[at(a.heads * a.D + c, p, a.QP)] = 0.0f;
    }
}

template <int DP>
int launch_fp32(small_ctx *ctx, const AttnArgs &a, cudaStream_t st) {
    static std::atomic<unsigned long long> done{0};
    const size_t smem = sizeof(float) * (2 * DP * kPitch + kKeys * kPitch + kKeys * DP);
    if (int s = allow_shared_memory(ctx, attention_fp32_kernel<DP>, done, smem)) return s;
    launch_kernel(ctx, attention_fp32_kernel<DP>, dim3((unsigned)ceil_div(a.QP, kRows), (unsigned)a.heads, (unsigned)a.N), dim3(kThreads), smem, st, a);
    return check_launch(ctx);
}

bool attention_shape_ok(int N, int heads, int kv_heads, int D, int QH, int QW, int KH, int KW) {
    if (N < 1 || heads < 1 || kv_heads < 1 || D < 1 || D > 128 || QH < 1 || QW < 1 || KH < 1 || KW < 1 || heads % kv_heads) return false;
    if ((long long)QH * QW > (1ll << 24) || (long long)KH * KW > (1ll << 24)) return false;
    return N <= 65535 && heads <= 65535 && ((long long)QH + KH) * ((long long)QW + KW) <= (1ll << 30);
}

// Which kernel (us, 4 heads unless said, with a bias).
//   Few queries (8 heads of 64): where a row's keys are long, the kernel that streams them (196 keys, batch 2, 4 rows a key head 7.3, in shared
//   memory 8.7; batch 32 11.9 and 16.9; 7 heads of 96, 88 keys, one row, batch 8 7.3 and 11.2), with more rows or few keys shared memory (8 rows
//   9.8 and 8.9, 16 rows batch 32 44.7 and 17.9; one row of 100 keys 7.5 and 6.4).
//   More queries, FP32: shared memory wherever it holds the keys (144 keys of 128 channels, batch 128 708 and 312; of 64, batch 2 36 and 12).
//   In the tensor-core modes those kernels' two launches cost 10 at least.  Where queries and keys fit one of their tiles, half empty then, shared
//   memory at any batch (49 pixels, 64 channels: batch 2 11.0 and 6.2, 128 40.8 and 25.4); else up to some 48 M multiply-adds of whole tiles (72
//   pixels, 64 channels: batch 16, 38 M, 12.5 and 11.7, 32 16.7 and 16.8; 196 pixels: 64 channels batch 4, 51 M, 16.4 and 14.6, 32 channels
//   batch 8, 51 M, 13.1 and 14.5).
//   Beyond that, while the rows of all heads are few, the streaming kernel, which shares out the keys (us, FP32 kernel / tensor cores / it, 8 heads
//   of 64: 17 queries on 96 x 96, batch 4, 544 rows 1439 / 195 / 137; 64 queries on 56 x 56, 512 rows 458 / 60 / 39, 128 61 / 60; 64 queries on 96 x
//   96, batch 4, 2048 rows 1431 / 195 / 260, on 28 x 28, batch 11, 5632 rows 126 / 33 / 94).
enum class Kernel { few, small, tensor_cores, fp32 };

Kernel kernel_of(int N, int heads, int kv_heads, int D, int QP, int KP, unsigned math) {
    const bool holds = attention_small_bytes(D, KP) <= kSmallShared && (long long)QP * (heads / kv_heads) <= 1 << 30;      // rows are ints there
    const int lanes = D <= 32 ? 32 : D <= 64 ? 64 : 128;             // channels as the kernels hold them
    if (QP <= kFewQueries) return holds && ((KP <= 128 && KP * lanes <= 8192) || QP * (heads / kv_heads) > 4) ? Kernel::small : Kernel::few;
    const double work = (double)N * heads * QP * (ceil_div(KP, 64) * 64.0) * lanes;
    if (holds && (math == SMALL_MATH_FP32 || (QP <= 64 && KP <= 64) || work <= 48e6)) return Kernel::small;
    const long long rows = (long long)N * heads * QP;
    if (math != SMALL_MATH_FP32) return rows <= 768 && (D & 3) == 0 ? Kernel::few : Kernel::tensor_cores;
    return rows <= 6000 ? Kernel::few : Kernel::fp32;
}

}  // namespace

int launch_attention_fp32(small_ctx *ctx, const AttnArgs &a, cudaStream_t st) {
    return a.D <= 32 ? launch_fp32<32>(ctx, a, st) : a.D <= 64 ? launch_fp32<64>(ctx, a, st) : launch_fp32<128>(ctx, a, st);
}

}  // namespace small

using namespace small;

SMALL_API size_t small_attention_workspace_bytes(int N, int heads, int kv_heads, int D, int QH, int QW, int KH, int KW, unsigned math) {
    if (!attention_shape_ok(N, heads, kv_heads, D, QH, QW, KH, KW) || (math & ~SMALL_MATH_MASK) || !one_math_mode(math)) return 0;
    return kernel_of(N, heads, kv_heads, D, QH * QW, KH * KW, math) == Kernel::tensor_cores ? attention_tc_workspace(N, kv_heads, D, KH * KW) : 0;
}

SMALL_API int small_attention(small_ctx *ctx, const float *q, const float *k, const float *v, const float *bias, const int32_t *q_extents,
                              const int32_t *k_extents, float *out, void *workspace, size_t workspace_bytes, int N, int heads, int kv_heads,
                              int D, int QH, int QW, int KH, int KW, long long q_stride, long long k_stride, long long v_stride,
                              float scale, float cap, unsigned flags, void *stream) {
    if (!ctx) return SMALL_ERR_NOT_INIT;
    CallOfItsOwn call(ctx);
    if ((flags & ~SMALL_MATH_MASK) || !one_math_mode(flags)) return SMALL_ERR_INVALID_ARG;
    if (!std::isfinite(scale) || !std::isfinite(cap) || cap < 0.0f) return SMALL_ERR_INVALID_ARG;
    if (int s = check_pointers({q, k, v, out}, {bias, q_extents, k_extents, workspace})) return s;
    if (!attention_shape_ok(N, heads, kv_heads, D, QH, QW, KH, KW)) return SMALL_ERR_SHAPE;
    const int QP = QH * QW, KP = KH * KW;
    const long long q_image = (long long)packed_elems(1, heads * D, QH, QW), k_image = (long long)packed_elems(1, kv_heads * D, KH, KW);
    if (!q_stride) q_stride = q_image;
    if (!k_stride) k_stride = k_image;
    if (!v_stride) v_stride = k_image;
    if (q_stride < q_image || k_stride < k_image || v_stride < k_image) return SMALL_ERR_SHAPE;
    if ((q_stride | k_stride | v_stride) & 3) return SMALL_ERR_ALIGN;
    const long long far = 1ll << 59;                 // bytes of a tensor stay inside 64 bits
    if (q_stride > far / N || k_stride > far / N || v_stride > far / N) return SMALL_ERR_SHAPE;
    const size_t ws = small_attention_workspace_bytes(N, heads, kv_heads, D, QH, QW, KH, KW, flags);
    if (workspace_bytes < ws || (ws && !workspace)) return SMALL_ERR_WORKSPACE;
    const size_t table = sizeof(float) * (size_t)heads * (QH + KH - 1) * (QW + KW - 1);
    const struct { const void *p; size_t n; } read[] = {
        {q, sizeof(float) * (size_t)(q_stride * (N - 1) + q_image)}, {k, sizeof(float) * (size_t)(k_stride * (N - 1) + k_image)},
        {v, sizeof(float) * (size_t)(v_stride * (N - 1) + k_image)}, {bias, table}, {q_extents, sizeof(int32_t) * 2 * (size_t)N}, {k_extents, sizeof(int32_t) * 2 * (size_t)N}};
    const size_t out_bytes = sizeof(float) * (size_t)q_image * N;
    for (const auto &r : read)
        if (r.p && (ranges_overlap(r.p, r.n, out, out_bytes) || (ws && ranges_overlap(r.p, r.n, workspace, ws)))) return SMALL_ERR_OVERLAP;
    if (ws && ranges_overlap(out, out_bytes, workspace, ws)) return SMALL_ERR_OVERLAP;
    const OnDevice on(ctx);
    if (on.error != cudaSuccess) { ctx->last_cuda = (int)on.error; return SMALL_ERR_CUDA; }
    // The kernels take cap * log2(e) and 1 / cap: both stay ordinary numbers.  Scores below 2^80 lose less than 2^-41 of themselves to a cap above 2^100;
    // capped at 2^-60 or below, all scores weigh 1 to FP32's last bit.
    if (cap > 0x1p100f) cap = 0.0f;
    else if (cap > 0.0f) cap = std::max(cap, 0x1p-60f);
    const AttnArgs a{q, k, v, bias, q_extents, k_extents, out, workspace, N, heads, kv_heads, D, QH, QW, KH, KW, QP, KP, blocks_of(heads * D),
                     q_stride, k_stride, v_stride, scale, cap, QW + KW - 1};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (kernel_of(N, heads, kv_heads, D, QP, KP, flags)) {
    case Kernel::tensor_cores: return launch_attention_tc(ctx, a, (flags & SMALL_MATH_MASK) == SMALL_MATH_3XTF32, st);
    case Kernel::few: return launch_attention_few(ctx, a, st);
    case Kernel::small: return launch_attention_small(ctx, a, st);
    default: return launch_attention_fp32(ctx, a, st);
    }
}
