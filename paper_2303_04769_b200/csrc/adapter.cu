// 1 x 1 convolution with a low-rank adapter for each image, out = act(W x + b + s_a Up_a (Down_a x)): entry points, and the form for few
// pixels and for FP32 arithmetic - small_conv2d for the shared product, and two kernels for what the adapters add to it.
#include "adapter.cuh"

namespace small {
namespace {

constexpr int kMaxRank = 128, kThreads = 256;

bool adapter_shape_ok(int adapters, int C, int K, int R) {
    return adapters >= 1 && C >= 1 && K >= 1 && R >= 1 && R <= kMaxRank && C <= (1 << 20) && K <= (1 << 20) && adapters <= (1 << 20);
}

__global__ void __launch_bounds__(kThreads) pack_adapters_kernel(const float *__restrict__ down, const float *__restrict__ up, float *__restrict__ packed,
                                                                 int adapters, const AdapterShape s) {
    grid_dep_sync();
    grid_dep_trigger();
    const size_t stride = (size_t)gridDim.x * blockDim.x, first = blockIdx.x * (size_t)blockDim.x + threadIdx.x;
    for (size_t i = first; i < s.down * adapters; i += stride) {
        const size_t a = i / s.down, e = i % s.down;
        const int c = (int)(e / (s.RP * 32)) * 32 + (int)(e & 31), r = (int)(e / 32 % s.RP);
        packed[i] = c < s.C && r < s.R ? down[(a * s.R + r) * s.C + c] : 0.0f;
    }
    for (size_t i = first; i < s.up * adapters; i += stride) {
        const size_t a = i / s.up, e = i % s.up;
        const int k = (int)(e / (s.RP * 32)) * 32 + (int)(e & 31), r = (int)(e / 32 % s.RP);
        packed[s.down * adapters + i] = k < s.K && r < s.R ? up[(a * s.K + k) * s.R + r] : 0.0f;
    }
}

__device__ __forceinline__ bool adapter_of(const AdaptArgs &a, int n, int &id) {
    id = a.adapter[n];
    return id >= 0 && id < a.adapters;
}

// t[n][pixel][rank] = scale Down x.  A warp takes kPixels pixels of an image and eight ranks, a lane a channel of each block: every load is a
// whole line, and each serves kPixels or eight products.  The sums are dealt out over the lanes while they are added up.
template <int kPixels>
__global__ void __launch_bounds__(kThreads) adapter_down_kernel(const AdaptArgs a, const AdapterShape s) {
    grid_dep_sync();
    grid_dep_trigger();
    const int lane = threadIdx.x & 31, rows = s.RP / 8, runs = (a.HW + kPixels - 1) / kPixels;
    const long long tasks = (long long)a.N * runs * rows, stride = (long long)gridDim.x * (kThreads / 32);
    for (long long i = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); i < tasks; i += stride) {
        const int rg = (int)(i % rows), p0 = (int)(i / rows % runs) * kPixels, n = (int)(i / rows / runs);
        int id;
        if (!adapter_of(a, n, id)) continue;
        const float *x = a.in + (size_t)n * s.CB * a.HW * 32 + lane, *w = a.packed + id * s.down + rg * 256 + lane;
        float acc[kPixels * 8];
#pragma unroll
        for (int u = 0; u < kPixels * 8; ++u) acc[u] = 0.0f;
#pragma unroll 4
        for (int cb = 0; cb < s.CB; ++cb) {
            float v[kPixels];
#pragma unroll
            for (int q = 0; q < kPixels; ++q) v[q] = p0 + q < a.HW && cb * 32 + lane < s.C ? x[((size_t)cb * a.HW + p0 + q) * 32] : 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const float u = w[(cb * s.RP + r) * 32];
#pragma unroll
                for (int q = 0; q < kPixels; ++q) acc[q * 8 + r] = fmaf(v[q], u, acc[q * 8 + r]);
            }
        }
        // halves of the sums go to halves of the lanes, until a lane has kPixels / 4 of them left (or several lanes the same one)
        int have = kPixels * 8;
#pragma unroll
        for (int bit = 16; bit; bit /= 2) {
            const bool upper = lane & bit;
            if (have > 1) {
#pragma unroll
                for (int u = 0; u < kPixels * 4; ++u)
                    if (u < have / 2) {
                        const float give = upper ? acc[u] : acc[u + have / 2], keep = upper ? acc[u + have / 2] : acc[u];
                        acc[u] = keep + __shfl_xor_sync(~0u, give, bit);
                    }
                have /= 2;
            } else {
                acc[0] += __shfl_xor_sync(~0u, acc[0], bit);
            }
        }
        const float factor = a.scale ? a.scale[id] : 1.0f;
        const int e = kPixels == 4 ? lane : lane >> 2, p = p0 + e / 8;               // one pixel: four lanes have each rank's sum
        if ((kPixels == 4 || (lane & 3) == 0) && p < a.HW) static_cast<float *>(a.ws)[((size_t)n * a.HW + p) * s.RP + rg * 8 + e % 8] = factor * acc[0];
    }
}

// out = act(out + Up t).  A warp takes kPixels pixels and a block of filters, a lane a filter.
template <int kPixels>
__global__ void __launch_bounds__(kThreads) adapter_up_kernel(const AdaptArgs a, const AdapterShape s) {
    grid_dep_sync();
    grid_dep_trigger();
    const int lane = threadIdx.x & 31, runs = (a.HW + kPixels - 1) / kPixels;
    const long long tasks = (long long)a.N * s.KB * runs, stride = (long long)gridDim.x * (kThreads / 32);
    for (long long i = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); i < tasks; i += stride) {
        const int p0 = (int)(i % runs) * kPixels, kb = (int)(i / runs % s.KB), n = (int)(i / runs / s.KB);
        int id;
        const bool some = adapter_of(a, n, id);
        if (!some && !a.relu) continue;
        float *out = a.out + (((size_t)n * s.KB + kb) * a.HW + p0) * 32 + lane;
        float acc[kPixels];
#pragma unroll
        for (int q = 0; q < kPixels; ++q) acc[q] = p0 + q < a.HW ? out[q * 32] : 0.0f;
        if (some) {
            const float *w = a.packed + s.down * a.adapters + id * s.up + (size_t)kb * s.RP * 32 + lane;
            const float4 *t = reinterpret_cast<const float4 *>(static_cast<const float *>(a.ws) + ((size_t)n * a.HW + p0) * s.RP);
#pragma unroll 2
            for (int r = 0; r < s.RP; r += 4) {
                const float w0 = w[r * 32], w1 = w[r * 32 + 32], w2 = w[r * 32 + 64], w3 = w[r * 32 + 96];
#pragma unroll
                for (int q = 0; q < kPixels; ++q) {
                    const float4 v = p0 + q < a.HW ? t[(q * s.RP + r) / 4] : make_float4(0.f, 0.f, 0.f, 0.f);
                    acc[q] = fmaf(v.x, w0, fmaf(v.y, w1, fmaf(v.z, w2, fmaf(v.w, w3, acc[q]))));
                }
            }
        }
        if (kb * 32 + lane >= s.K) continue;             // pad lanes stay what the convolution has written
#pragma unroll
        for (int q = 0; q < kPixels; ++q)
            if (p0 + q < a.HW) out[q * 32] = a.relu && !(acc[q] > 0.0f) ? 0.0f : acc[q];
    }
}

unsigned task_blocks(const small_ctx *ctx, long long tasks) {
    const long long blocks = (tasks + kThreads / 32 - 1) / (kThreads / 32), most = (long long)ctx->sm_count * 16;
    return (unsigned)(blocks < most ? blocks : most);
}

}  // namespace
}  // namespace small

using namespace small;

SMALL_API size_t small_adapter_elems(int adapters, int C, int K, int R) {
    return adapter_shape_ok(adapters, C, K, R) ? AdapterShape(adapters, C, K, R).floats : 0;
}

SMALL_API int small_pack_adapters(small_ctx *ctx, const float *down, const float *up, float *packed, int adapters, int C, int K, int R, void *stream) {
    if (!ctx) return SMALL_ERR_NOT_INIT;
    CallOfItsOwn call(ctx);
    if (int s = check_pointers({down, up, packed})) return s;
    if (!adapter_shape_ok(adapters, C, K, R)) return SMALL_ERR_SHAPE;
    const size_t bytes = sizeof(float) * small_adapter_elems(adapters, C, K, R);
    if (ranges_overlap(down, sizeof(float) * adapters * (size_t)R * C, packed, bytes) || ranges_overlap(up, sizeof(float) * adapters * (size_t)K * R, packed, bytes))
        return SMALL_ERR_OVERLAP;
    const OnDevice on(ctx);
    if (on.error != cudaSuccess) { ctx->last_cuda = (int)on.error; return SMALL_ERR_CUDA; }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const AdapterShape s(adapters, C, K, R);
    launch_kernel(ctx, pack_adapters_kernel, dim3(task_blocks(ctx, (long long)((s.down + s.up) * adapters / 32))), dim3(kThreads), 0, st, down, up, packed, adapters, s);
    if (int e = check_launch(ctx)) return e;
    return launch_pack_halves(ctx, down, up, packed, adapters, s, st);
}

SMALL_API size_t small_adapted_conv2d_workspace_bytes(int N, int C, int K, int H, int W, int R) {
    if (N < 1 || H < 1 || W < 1 || (long long)H * W > (1ll << 24) || !adapter_shape_ok(1, C, K, R)) return 0;
    const size_t products = sizeof(float) * (size_t)N * H * W * AdapterShape(1, C, K, R).RP;
    const size_t whole = adapted_tc_preferred(N, C, K, H * W, R, kSmCount) ? adapted_tc_workspace(N, C, K, H * W, R) : 0;
    return whole > products ? whole : products;
}

SMALL_API int small_adapted_conv2d(small_ctx *ctx, const float *in, const float *w_blk, const float *bias, const float *packed,
                                   const int32_t *adapter, const float *scale, float *out, void *workspace, int N, int C, int K, int H, int W,
                                   int R, int adapters, unsigned flags, void *stream) {
    if (!ctx) return SMALL_ERR_NOT_INIT;
    CallOfItsOwn call(ctx);
    if (flags & ~(SMALL_RELU | SMALL_ACCUMULATE | SMALL_MATH_MASK) || !one_math_mode(flags)) return SMALL_ERR_INVALID_ARG;
    if (int s = check_pointers({in, w_blk, packed, adapter, out}, {bias, scale, workspace})) return s;
    Geom g;
    if (!adapter_shape_ok(adapters, C, K, R)) return SMALL_ERR_SHAPE;
    if (int s = make_geom(g, N, C, K, H, W, 1, 1, 1, 0, 0, 0, 0)) return s;
    const size_t ws = small_adapted_conv2d_workspace_bytes(N, C, K, H, W, R);
    if (!workspace) return SMALL_ERR_WORKSPACE;
    const unsigned math = flags & SMALL_MATH_MASK;
    const size_t in_b = sizeof(float) * packed_elems(N, C, H, W), out_b = sizeof(float) * packed_elems(N, K, H, W);
    const struct { const void *p; size_t n; } read[] = {
        {in, in_b}, {w_blk, sizeof(float) * small_conv_weight_elems(C, K, 1, 1, math)}, {bias, sizeof(float) * K},
        {packed, sizeof(float) * small_adapter_elems(adapters, C, K, R)}, {adapter, sizeof(int32_t) * N}, {scale, sizeof(float) * adapters}};
    for (const auto &r : read)
        if (r.p && (ranges_overlap(r.p, r.n, out, out_b) || ranges_overlap(r.p, r.n, workspace, ws))) return SMALL_ERR_OVERLAP;
    if (ranges_overlap(out, out_b, workspace, ws)) return SMALL_ERR_OVERLAP;
    const OnDevice on(ctx);
    if (on.error != cudaSuccess) { ctx->last_cuda = (int)on.error; return SMALL_ERR_CUDA; }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const AdapterShape s(adapters, C, K, R);
    const AdaptArgs a{in, w_blk, bias, packed, scale, adapter, out, workspace, N, H * W, adapters, (flags & SMALL_RELU) != 0, (flags & SMALL_ACCUMULATE) != 0};
    if (math != SMALL_MATH_FP32 && adapted_tc_preferred(N, C, K, H * W, R, kSmCount))
        return launch_adapted_tc(ctx, a, s, math == SMALL_MATH_3XTF32, st);
    if (int e = small_conv2d(ctx, in, w_blk, bias, out, N, C, K, H, W, 1, 1, 1, 0, 0, 0, 0, flags & ~SMALL_RELU, stream)) return e;
    const bool runs = H * W >= 4;                        // several pixels a warp where an image has them
    const long long rows = (long long)N * (s.RP / 8), blocks = (long long)N * s.KB;
    if (runs) launch_kernel(ctx, adapter_down_kernel<4>, dim3(task_blocks(ctx, rows * ceil_div(H * W, 4))), dim3(kThreads), 0, st, a, s);
    else launch_kernel(ctx, adapter_down_kernel<1>, dim3(task_blocks(ctx, rows * H * W)), dim3(kThreads), 0, st, a, s);
    if (int e = check_launch(ctx)) return e;
    if (runs) launch_kernel(ctx, adapter_up_kernel<8>, dim3(task_blocks(ctx, blocks * ceil_div(H * W, 8))), dim3(kThreads), 0, st, a, s);
    else launch_kernel(ctx, adapter_up_kernel<1>, dim3(task_blocks(ctx, blocks * H * W)), dim3(kThreads), 0, st, a, s);
    return check_launch(ctx);
}
