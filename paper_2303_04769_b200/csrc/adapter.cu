// 1 x 1 convolution with a low-rank adapter for each image, out = act(W x + b + s_a Up_a (Down_a x)): entry points, and the form for few
// pixels and for FP32 arithmetic - small_conv2d for the shared product, and a kernel for what the adapters add to it.
#include "adapter.cuh"

namespace small {
namespace {

constexpr int kMaxRank = 128, kThreads = 256, kWarps = kThreads / 32;

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

// out = act(out + scale Up (Down x)) behind the convolution that has written `out`: a block takes a run of up to 32 pixels of an image (kPoint: one) and a
// run of filter blocks.  The products with Down, t, come first, from what is older than the convolution: they are taken while it runs.
// For them a warp takes four pixels and eight ranks, a lane a channel of each block, so that every load is a whole line and serves four or
// eight products; one pixel's channel blocks are dealt out to the warps.  Then a warp takes a filter block, a lane a filter.
constexpr int kMostRun = 32;             // pixels of a block

// kAhead: channel blocks whose loads are on their way at once (left to the compiler they were not: 16.5 us for 11.9, four images 512 -> 512 on 7 x 7);
// two cost a block of three an SM, so one where blocks are many (64 images 64 -> 64 on 28 x 28: 24.3 for 26.6).
template <bool kPoint, int kAhead>
__global__ void __launch_bounds__(kThreads) adapter_add_kernel(const AdaptArgs a, const AdapterShape s, int run, int runs, int filter_blocks) {
    extern __shared__ float t_s[];                       // [pixels][RP], kPoint: [warps][RP]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = blockIdx.x / runs, p0 = blockIdx.x % runs * run;
    const int pixels = kPoint ? 1 : min(run, a.HW - p0), id = a.adapter[n];
    const bool some = id >= 0 && id < a.adapters;
    if (some) {
        const float *x = a.in + ((size_t)n * s.CB * a.HW + p0) * 32 + lane, *w = a.packed + id * s.down + lane;
        const float factor = a.scale ? a.scale[id] : 1.0f;
        constexpr int kPixels = kPoint ? 1 : 4, kSums = kPixels * 8;
        for (int i = kPoint ? 0 : warp; i < (kPoint ? 1 : (pixels + 3) / 4) * (s.RP / 8); i += kPoint ? 1 : kWarps) {
            const int rg = i % (s.RP / 8), q0 = i / (s.RP / 8) * 4;
            float acc[kSums];
#pragma unroll
            for (int u = 0; u < kSums; ++u) acc[u] = 0.0f;
            constexpr int kStep = kPoint ? kWarps : 1;
#pragma unroll 1
            for (int cb = kPoint ? warp : 0; cb < s.CB; cb += kAhead * kStep) {
                float v[kAhead][kPixels], u[kAhead][8];
#pragma unroll
                for (int h = 0; h < kAhead; ++h) {
                    const int b = cb + h * kStep;
#pragma unroll
                    for (int q = 0; q < kPixels; ++q) v[h][q] = q0 + q < pixels && b * 32 + lane < s.C ? __ldg(x + ((size_t)b * a.HW + q0 + q) * 32) : 0.0f;
#pragma unroll
                    for (int r = 0; r < 8; ++r) u[h][r] = b < s.CB ? __ldg(w + (b * s.RP + rg * 8 + r) * 32) : 0.0f;
                }
#pragma unroll
                for (int h = 0; h < kAhead; ++h)
#pragma unroll
                    for (int r = 0; r < 8; ++r)
#pragma unroll
                        for (int q = 0; q < kPixels; ++q) acc[q * 8 + r] = fmaf(v[h][q], u[h][r], acc[q * 8 + r]);
            }
            // halves of the sums go to halves of the lanes, until each lane has one (one pixel: four lanes the same one)
            int have = kSums;
#pragma unroll
            for (int bit = 16; bit; bit /= 2) {
                const bool upper = lane & bit;
                if (have > 1) {
#pragma unroll
                    for (int u = 0; u < kSums / 2; ++u)
                        if (u < have / 2) {
                            const float give = upper ? acc[u] : acc[u + have / 2], keep = upper ? acc[u + have / 2] : acc[u];
                            acc[u] = keep + __shfl_xor_sync(~0u, give, bit);
                        }
                    have /= 2;
                } else {
                    acc[0] += __shfl_xor_sync(~0u, acc[0], bit);
                }
            }
            if (kPoint) {
                if ((lane & 3) == 0) t_s[warp * s.RP + rg * 8 + lane / 4] = factor * acc[0];
            } else if (q0 + lane / 8 < pixels) {
                t_s[(q0 + lane / 8) * s.RP + rg * 8 + lane % 8] = factor * acc[0];
            }
        }
        __syncthreads();
        if (kPoint) {
            float sum = 0.0f;
            if (threadIdx.x < s.RP)
#pragma unroll
                for (int i = 0; i < kWarps; ++i) sum += t_s[i * s.RP + threadIdx.x];
            __syncthreads();
            if (threadIdx.x < s.RP) t_s[threadIdx.x] = sum;
            __syncthreads();
        }
    }
    grid_dep_sync();                                     // the convolution
    grid_dep_trigger();
    if (!some && !a.relu) return;
    constexpr int kPixels = kPoint ? 1 : 8;
    const int kb0 = blockIdx.y * filter_blocks, count = min(filter_blocks, s.KB - kb0), groups = kPoint ? 1 : (pixels + 7) / 8;
    for (int i = warp; i < count * groups; i += kWarps) {
        const int kb = kb0 + i / groups, q0 = i % groups * 8;
        float *out = a.out + (((size_t)n * s.KB + kb) * a.HW + p0 + q0) * 32 + lane;
        float acc[kPixels];
#pragma unroll
        for (int q = 0; q < kPixels; ++q) acc[q] = q0 + q < pixels ? out[q * 32] : 0.0f;
        if (some) {
            const float *w = a.packed + s.down * a.adapters + id * s.up + (size_t)kb * s.RP * 32 + lane;
#pragma unroll 2
            for (int r = 0; r < s.RP; r += 4) {
                const float w0 = w[r * 32], w1 = w[r * 32 + 32], w2 = w[r * 32 + 64], w3 = w[r * 32 + 96];
#pragma unroll
                for (int q = 0; q < kPixels; ++q) {
                    const float4 v = q0 + q < pixels ? *reinterpret_cast<const float4 *>(t_s + (q0 + q) * s.RP + r) : make_float4(0.f, 0.f, 0.f, 0.f);
                    acc[q] = fmaf(v.x, w0, fmaf(v.y, w1, fmaf(v.z, w2, fmaf(v.w, w3, acc[q]))));
                }
            }
        }
        if (kb * 32 + lane >= s.K) continue;             // pad lanes stay what the convolution has written
#pragma unroll
        for (int q = 0; q < kPixels; ++q)
            if (q0 + q < pixels) out[q * 32] = a.relu && !(acc[q] > 0.0f) ? 0.0f : acc[q];
    }
}

// The whole layer for few pixels, in FP32 whatever the mode: a block takes 32 filters and eight pixels.  The warps share out the filters' channel
// blocks, a lane a filter, each load serving eight products; before that each warp takes one pixel's t, a lane a channel of each block, and what
// Up makes of it, a lane a filter.  Bound by the launch and two trips to L2; two dependent launches cost half as much again.
constexpr int kFew = 8;                  // pixels of a block

__global__ void __launch_bounds__(kThreads) adapted_few_kernel(const AdaptArgs a, const AdapterShape s) {
    extern __shared__ float4 few_s[];
    float *x_s = reinterpret_cast<float *>(few_s), *part_s = x_s + s.CB * 32 * kFew, *t_s = part_s + kWarps * kFew * 32;      // [channel][pixel], [warp][pixel][filter], [pixel][RP]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, kb = blockIdx.x, m0 = blockIdx.y * kFew, M = a.N * a.HW;
    grid_dep_sync();
    grid_dep_trigger();
    const float *w = a.w + (size_t)kb * s.CB * 1024 + lane;
    float w_now[32];
    auto fetch = [&](int cb) {
#pragma unroll
        for (int c = 0; c < 32; ++c) w_now[c] = cb < s.CB ? w[(size_t)cb * 1024 + c * 32] : 0.0f;
    };
    fetch(warp);
    for (int i = threadIdx.x; i < s.CB * 8 * kFew; i += kThreads) {
        const int q = i % kFew, c = i / kFew * 4, m = m0 + q;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (m < M) v = *reinterpret_cast<const float4 *>(a.in + (((size_t)(m / a.HW) * s.CB + (c >> 5)) * a.HW + m % a.HW) * 32 + (c & 31));
        x_s[(c + 0) * kFew + q] = c + 0 < s.C ? v.x : 0.0f; x_s[(c + 1) * kFew + q] = c + 1 < s.C ? v.y : 0.0f;
        x_s[(c + 2) * kFew + q] = c + 2 < s.C ? v.z : 0.0f; x_s[(c + 3) * kFew + q] = c + 3 < s.C ? v.w : 0.0f;
    }
    // this warp's pixel: what its adapter adds to filter `lane`
    const int m = m0 + warp, n = m / a.HW, id = m < M ? a.adapter[n] : -1;
    float sum = 0.0f;
    if (id >= 0 && id < a.adapters) {
        const float *x = a.in + ((size_t)n * s.CB * a.HW + m % a.HW) * 32 + lane, *down = a.packed + id * s.down + lane;
        const float *up = a.packed + s.down * a.adapters + id * s.up + (size_t)kb * s.RP * 32 + lane;
        const float factor = a.scale ? a.scale[id] : 1.0f;
        float *t = t_s + warp * s.RP;
        constexpr int kAhead = 8;
        for (int rg = 0; rg < s.RP; rg += 8) {
            float acc[8] = {};
#pragma unroll 1
            for (int cb = 0; cb < s.CB; cb += kAhead) {  // all of these loads on their way at once (left to the compiler they were not: 14.4 us for 6.9)
                float v[kAhead], d[kAhead][8];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const bool in = cb + u < s.CB;
                    v[u] = in && (cb + u) * 32 + lane < s.C ? __ldg(x + (size_t)(cb + u) * a.HW * 32) : 0.0f;
#pragma unroll
                    for (int r = 0; r < 8; ++r) d[u][r] = in ? __ldg(down + ((cb + u) * s.RP + rg + r) * 32) : 0.0f;
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int r = 0; r < 8; ++r) acc[r] = fmaf(v[u], d[u][r], acc[r]);
            }
            // halves of the sums go to halves of the lanes; four lanes end with the same one
#pragma unroll
            for (int bit = 16, have = 8; bit; bit /= 2, have /= 2) {
                const bool upper = lane & bit;
                if (have > 1) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if (u < have / 2) {
                            const float give = upper ? acc[u] : acc[u + have / 2], keep = upper ? acc[u + have / 2] : acc[u];
                            acc[u] = keep + __shfl_xor_sync(~0u, give, bit);
                        }
                } else {
                    acc[0] += __shfl_xor_sync(~0u, acc[0], bit);
                }
            }
            if ((lane & 3) == 0) t[rg + lane / 4] = factor * acc[0];
        }
        __syncwarp();
#pragma unroll 8
        for (int r = 0; r < s.RP; ++r) sum = fmaf(t[r], up[r * 32], sum);
    }
    __syncthreads();
    float acc[kFew] = {};
    for (int cb = warp; cb < s.CB; cb += kWarps) {
        float now[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) now[c] = w_now[c];
        fetch(cb + kWarps);
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            const float4 lo = *reinterpret_cast<const float4 *>(x_s + (cb * 32 + c) * kFew), hi = *reinterpret_cast<const float4 *>(x_s + (cb * 32 + c) * kFew + 4);
            acc[0] = fmaf(now[c], lo.x, acc[0]); acc[1] = fmaf(now[c], lo.y, acc[1]); acc[2] = fmaf(now[c], lo.z, acc[2]); acc[3] = fmaf(now[c], lo.w, acc[3]);
            acc[4] = fmaf(now[c], hi.x, acc[4]); acc[5] = fmaf(now[c], hi.y, acc[5]); acc[6] = fmaf(now[c], hi.z, acc[6]); acc[7] = fmaf(now[c], hi.w, acc[7]);
        }
    }
#pragma unroll
    for (int q = 0; q < kFew; ++q) part_s[(warp * kFew + q) * 32 + lane] = acc[q];
    __syncthreads();
    if (m >= M) return;
    float *out = a.out + (((size_t)n * s.KB + kb) * a.HW + m % a.HW) * 32 + lane;
    const int k = kb * 32 + lane;
    if (k >= s.K) { *out = 0.0f; return; }
#pragma unroll
    for (int i = 0; i < kWarps; ++i) sum += part_s[(i * kFew + warp) * 32 + lane];
    if (a.bias) sum += a.bias[k];
    if (a.accumulate) sum += *out;
    *out = a.relu && !(sum > 0.0f) ? 0.0f : sum;
}
// While its blocks are no more than the SMs, and t is not taken from many rank groups one after the other (us, here / the layer in two launches: one
// vector or 7 x 7 of four images, 64 -> 64, rank 8 4.4 / 6.4; 128 vectors 256 -> 256, rank 8 5.3 / 6.5, 512 17.6 / 6.8; eight of 512 -> 512, rank 8
// 7.6 / 6.6, as a plane of 5 x 5 7.7 / 12.1, where the shared product takes longer; 64 -> 512, rank 32 7.0 / 6.5).
bool few_preferred(int N, int HW, const AdapterShape &s, int sms) {
    return s.RP <= 24 && s.CB * s.RP <= (HW < 4 ? 64 : 128) && ((long long)N * HW + kFew - 1) / kFew * s.KB <= sms;
}
size_t few_bytes(const AdapterShape &s) { return sizeof(float) * (size_t)(s.CB * 32 * kFew + kWarps * kFew * 32 + kFew * s.RP); }       // 26 KB at most

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
    return adapted_tc_preferred(N, C, K, H * W, R, kSmCount) ? adapted_tc_workspace(N, C, K, H * W, R) : 0;
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
    const unsigned math = flags & SMALL_MATH_MASK;
    const size_t ws = math == SMALL_MATH_FP32 ? 0 : small_adapted_conv2d_workspace_bytes(N, C, K, H, W, R);
    if (ws && !workspace) return SMALL_ERR_WORKSPACE;
    const size_t in_b = sizeof(float) * packed_elems(N, C, H, W), out_b = sizeof(float) * packed_elems(N, K, H, W);
    const struct { const void *p; size_t n; } read[] = {
        {in, in_b}, {w_blk, sizeof(float) * small_conv_weight_elems(C, K, 1, 1, math)}, {bias, sizeof(float) * K},
        {packed, sizeof(float) * small_adapter_elems(adapters, C, K, R)}, {adapter, sizeof(int32_t) * N}, {scale, sizeof(float) * adapters}};
    for (const auto &r : read)
        if (r.p && (ranges_overlap(r.p, r.n, out, out_b) || (ws && ranges_overlap(r.p, r.n, workspace, ws)))) return SMALL_ERR_OVERLAP;
    if (ws && ranges_overlap(out, out_b, workspace, ws)) return SMALL_ERR_OVERLAP;
    const OnDevice on(ctx);
    if (on.error != cudaSuccess) { ctx->last_cuda = (int)on.error; return SMALL_ERR_CUDA; }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const AdapterShape s(adapters, C, K, R);
    const AdaptArgs a{in, w_blk, bias, packed, scale, adapter, out, workspace, N, H * W, adapters, (flags & SMALL_RELU) != 0, (flags & SMALL_ACCUMULATE) != 0};
    if (ws)
        return launch_adapted_tc(ctx, a, s, math == SMALL_MATH_3XTF32, st);
    if (few_preferred(N, H * W, s, ctx->sm_count)) {
        launch_kernel(ctx, adapted_few_kernel, dim3((unsigned)s.KB, (unsigned)ceil_div(N * H * W, kFew)), dim3(kThreads), few_bytes(s), st, a, s);
        return check_launch(ctx);
    }
    const bool point = H * W < 4;
    if ((long long)N * ceil_div(H * W, point ? 1 : 8) > 0x7fffffff) return SMALL_ERR_SHAPE;
    if (int e = small_conv2d(ctx, in, w_blk, bias, out, N, C, K, H, W, 1, 1, 1, 0, 0, 0, 0, flags & ~SMALL_RELU, stream)) return e;
    // Blocks for the SMs: shorter runs while they are few, then, up to two a SM, fewer filter blocks each, at least eight apart, as each takes the products
    // with Down anew.  us, runs of 32 / 16 / 8: 93 -> 280, rank 43, 6 x 46, batch 6 26.7 / 17.9 / 15.6; 256 -> 256, rank 64, 14 x 14, batch 1 34.9 /
    // 19.5 / 11.8; 183 -> 237, rank 2, 5 x 5, batch 64 12.7 / 11.8 / 13.0.
    int run = point ? 1 : kMostRun;
    while (run > 8 && (long long)N * ceil_div(H * W, run) < ctx->sm_count * 3 / 4) run /= 2;
    const int runs = ceil_div(H * W, run), most = ceil_div(s.KB, 8), more = (int)std::max(1ll, 2ll * ctx->sm_count / ((long long)N * runs));
    const int filter_blocks = ceil_div(s.KB, more < most ? more : most);
    const dim3 grid((unsigned)(N * runs), (unsigned)ceil_div(s.KB, filter_blocks));
    const size_t t = sizeof(float) * s.RP * (point ? kWarps : run);
    if (point) launch_kernel(ctx, adapter_add_kernel<true, 4>, grid, dim3(kThreads), t, st, a, s, run, runs, filter_blocks);
    else if ((long long)N * runs > 4 * ctx->sm_count) launch_kernel(ctx, adapter_add_kernel<false, 1>, grid, dim3(kThreads), t, st, a, s, run, runs, filter_blocks);
    else launch_kernel(ctx, adapter_add_kernel<false, 2>, grid, dim3(kThreads), t, st, a, s, run, runs, filter_blocks);
    return check_launch(ctx);
}
