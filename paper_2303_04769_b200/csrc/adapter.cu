// 1 x 1 convolution with a low-rank adapter for each image: out = act(W x + b + s_a Up_a (Down_a x)).
// The shared product is small_conv2d; the adapters' part is added to its result by the kernels here.
//
// Packed adapters: Down as [adapters][CB][RP][32 channels], RP = R rounded up to 8 (rows of one channel block together, as
// activations are), behind them Up as [adapters][RB][KB * 32 filters][32 ranks]; whatever is behind R, C or K is 0.
#include "entry.cuh"

namespace small {
namespace {

constexpr int kMaxRank = 128;

struct AdapterShape {
    int C, K, R, CB, KB, RP, RB;
    size_t down, up;                     // floats of one adapter's Down and Up
    AdapterShape(int C, int K, int R) : C(C), K(K), R(R), CB(blocks_of(C)), KB(blocks_of(K)), RP((R + 7) / 8 * 8), RB(blocks_of(R)) {
        down = (size_t)CB * RP * 32;
        up = (size_t)RB * KB * 32 * 32;
    }
};

bool adapter_shape_ok(int adapters, int C, int K, int R) {
    return adapters >= 1 && C >= 1 && K >= 1 && R >= 1 && R <= kMaxRank && C <= (1 << 20) && K <= (1 << 20);
}

__global__ void __launch_bounds__(256) pack_adapters_kernel(const float *__restrict__ down, const float *__restrict__ up, float *__restrict__ packed,
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
        const size_t a = i / s.up, e = i % s.up, rows = (size_t)s.KB * 32;
        const int r = (int)(e / (rows * 32)) * 32 + (int)(e & 31), k = (int)(e / 32 % rows);
        packed[s.down * adapters + i] = k < s.K && r < s.R ? up[(a * s.K + k) * s.R + r] : 0.0f;
    }
}

struct AdaptArgs {
    const float *in, *packed, *scale;
    const int32_t *adapter;
    float *t, *out;                      // t: [N][pixels][RP], the products with Down
    int N, HW, adapters;
    bool relu;
};

// t = scale Down x, a thread for each pixel and row.
__global__ void __launch_bounds__(256) adapter_down_kernel(const AdaptArgs a, const AdapterShape s) {
    grid_dep_sync();
    grid_dep_trigger();
    const size_t total = (size_t)a.N * a.HW * s.RP, stride = (size_t)gridDim.x * blockDim.x;
    for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < total; i += stride) {
        const int r = (int)(i % s.RP);
        const size_t np = i / s.RP;
        const int p = (int)(np % a.HW), n = (int)(np / a.HW), id = a.adapter[n];
        if (id < 0 || id >= a.adapters) continue;
        const float4 *x = reinterpret_cast<const float4 *>(a.in) + ((size_t)n * s.CB * a.HW + p) * 8;
        const float4 *w = reinterpret_cast<const float4 *>(a.packed + id * s.down) + r * 8;
        float acc = 0.0f;
        for (int cb = 0; cb < s.CB; ++cb, x += (size_t)a.HW * 8, w += s.RP * 8)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float4 u = x[j], v = w[j];
                acc = fmaf(u.x, v.x, fmaf(u.y, v.y, fmaf(u.z, v.z, fmaf(u.w, v.w, acc))));
            }
        a.t[i] = a.scale ? a.scale[id] * acc : acc;
    }
}

// out = act(out + Up t), a thread for each pixel and filter.
__global__ void __launch_bounds__(256) adapter_up_kernel(const AdaptArgs a, const AdapterShape s) {
    grid_dep_sync();
    grid_dep_trigger();
    const size_t total = (size_t)a.N * s.KB * a.HW * 32, stride = (size_t)gridDim.x * blockDim.x;
    for (size_t i = blockIdx.x * (size_t)blockDim.x + threadIdx.x; i < total; i += stride) {
        const size_t line = i >> 5;
        const int p = (int)(line % a.HW), kb = (int)(line / a.HW % s.KB), n = (int)(line / a.HW / s.KB), id = a.adapter[n];
        const int k = kb * 32 + (int)(i & 31);
        const bool some = id >= 0 && id < a.adapters;
        if (k >= s.K || (!some && !a.relu)) continue;
        float v = a.out[i];
        if (some) {
            const float *t = a.t + ((size_t)n * a.HW + p) * s.RP;
            const float *w = a.packed + s.down * a.adapters + id * s.up + (size_t)k * 32;
            for (int r = 0; r < s.R; ++r) v = fmaf(t[r], w[(size_t)(r >> 5) * s.KB * 1024 + (r & 31)], v);
        }
        a.out[i] = a.relu && !(v > 0.0f) ? 0.0f : v;
    }
}

unsigned stream_blocks(size_t items) { return (unsigned)(items / 256 + 1 < 148 * 16 ? items / 256 + 1 : 148 * 16); }

}  // namespace
}  // namespace small

using namespace small;

SMALL_API size_t small_adapter_elems(int adapters, int C, int K, int R) {
    if (!adapter_shape_ok(adapters, C, K, R)) return 0;
    const AdapterShape s(C, K, R);
    return (s.down + s.up) * adapters;
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
    launch_kernel(ctx, pack_adapters_kernel, dim3(stream_blocks(bytes / 4)), dim3(256), 0, static_cast<cudaStream_t>(stream), down, up, packed, adapters,
                  AdapterShape(C, K, R));
    return check_launch(ctx);
}

SMALL_API size_t small_adapted_conv2d_workspace_bytes(int N, int C, int K, int H, int W, int R) {
    if (N < 1 || H < 1 || W < 1 || (long long)H * W > (1ll << 24) || !adapter_shape_ok(1, C, K, R)) return 0;
    return sizeof(float) * (size_t)N * H * W * AdapterShape(C, K, R).RP;
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
    const size_t in_b = sizeof(float) * packed_elems(N, C, H, W), out_b = sizeof(float) * packed_elems(N, K, H, W);
    const struct { const void *p; size_t n; } read[] = {
        {in, in_b}, {w_blk, sizeof(float) * small_conv_weight_elems(C, K, 1, 1, flags & SMALL_MATH_MASK)}, {bias, sizeof(float) * K},
        {packed, sizeof(float) * small_adapter_elems(adapters, C, K, R)}, {adapter, sizeof(int32_t) * N}, {scale, sizeof(float) * adapters}};
    for (const auto &r : read)
        if (r.p && (ranges_overlap(r.p, r.n, out, out_b) || ranges_overlap(r.p, r.n, workspace, ws))) return SMALL_ERR_OVERLAP;
    if (ranges_overlap(out, out_b, workspace, ws)) return SMALL_ERR_OVERLAP;
    const OnDevice on(ctx);
    if (on.error != cudaSuccess) { ctx->last_cuda = (int)on.error; return SMALL_ERR_CUDA; }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (int s = small_conv2d(ctx, in, w_blk, bias, out, N, C, K, H, W, 1, 1, 1, 0, 0, 0, 0, flags & ~SMALL_RELU, stream)) return s;
    const AdapterShape s(C, K, R);
    const AdaptArgs a{in, packed, scale, adapter, static_cast<float *>(workspace), out, N, H * W, adapters, (flags & SMALL_RELU) != 0};
    launch_kernel(ctx, adapter_down_kernel, dim3(stream_blocks((size_t)N * H * W * s.RP)), dim3(256), 0, st, a, s);
    if (int e = check_launch(ctx)) return e;
    launch_kernel(ctx, adapter_up_kernel, dim3(stream_blocks((size_t)N * H * W * s.KB * 32)), dim3(256), 0, st, a, s);
    return check_launch(ctx);
}
