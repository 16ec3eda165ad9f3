// Group normalisation with an activation on blocked tensors:
//     out = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c]),   mean and var over a group of channels and the plane.
// Bound by memory: x has to be read once and the result written once.  The unit of work is one image's smallest run of channels
// that is both whole groups and whole channel blocks (lcm(channels of a group, 32), cut off at C), so that every 128-byte line is
// read by one unit only.  A cluster of 1 to 8 thread blocks shares out the unit's pixels and keeps them in shared memory: sums,
// then deviations from the mean, then the result are all taken from there, and only sums of groups cross the cluster.  Units
// too large for that are summed block by block (each block's mean and deviations, in shared memory too) and merged and
// normalised by a second kernel, which reads the tensor again.
#include <cmath>

#include "entry.cuh"

namespace small {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxGroups = 32;          // groups of a unit: lcm(c, 32) / c is at most 32

struct NormArgs {
    const float *in, *gamma, *beta;
    float *out, *stats;                 // stats: [N][units][splits][kMaxGroups][2], of the form in two kernels
    int C, CB, cpg, HW;                 // channels, channel blocks, channels of a group, pixels
    int unit_blocks, units;             // channel blocks of a unit (the last one's may be fewer), units of an image
    int splits;                         // thread blocks that share a unit's pixels
    int warps_per_block;                // warps that share a channel block
    float eps;
    unsigned act;
};

__device__ __forceinline__ float activate(float y, unsigned act) {
    if (act == SMALL_RELU) return y > 0.0f ? y : 0.0f;
    if (act == SMALL_SILU) return __fdividef(y, 1.0f + __expf(-y));      // exp to inf: -0, as the limit has it
    return y;
}

// The unit of this thread block and the part of its pixels that the block holds.
struct Part {
    int n, unit, split, b0, blocks, c0, channels, groups, p0, pixels;
    __device__ Part(const NormArgs &a, int block) {
        split = block % a.splits;
        const int u = block / a.splits;
        unit = u % a.units;
        n = u / a.units;
        b0 = unit * a.unit_blocks;
        blocks = min(a.unit_blocks, a.CB - b0);
        c0 = b0 * 32;
        channels = min(blocks * 32, a.C - c0);
        groups = channels / a.cpg;
        p0 = (int)((long long)a.HW * split / a.splits);
        pixels = (int)((long long)a.HW * (split + 1) / a.splits) - p0;
    }
};

// Sums over the part's pixels of f(value, channel of the unit), by channel and share of a channel block's warps.
template <typename F>
__device__ __forceinline__ void channel_sums(const Part &p, int wpb, const float4 *tile, float *sums, F f) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 7;
    for (int i = warp; i < p.blocks * wpb; i += kWarps) {
        const int b = i / wpb, share = i % wpb;
        const float4 *x = tile + (size_t)b * p.pixels * 8 + j;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int q = share * 4 + (lane >> 3); q < p.pixels; q += wpb * 4) {
            const float4 v = f(x[(size_t)q * 8], b * 32 + j * 4);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
#pragma unroll
        for (int o = 8; o < 32; o *= 2) {
            s.x += __shfl_xor_sync(~0u, s.x, o); s.y += __shfl_xor_sync(~0u, s.y, o);
            s.z += __shfl_xor_sync(~0u, s.z, o); s.w += __shfl_xor_sync(~0u, s.w, o);
        }
        if (lane < 8) reinterpret_cast<float4 *>(sums)[(share * p.blocks + b) * 8 + j] = s;
    }
}

// Sums by channel -> sums by group, a warp for each group.
__device__ __forceinline__ void group_sums(const Part &p, int cpg, int wpb, const float *sums, float *out) {
    const int lane = threadIdx.x & 31;
    for (int g = threadIdx.x >> 5; g < p.groups; g += kWarps) {
        float s = 0.0f;
        for (int share = 0; share < wpb; ++share)
            for (int c = lane; c < cpg; c += 32) s += sums[share * p.blocks * 32 + g * cpg + c];
#pragma unroll
        for (int o = 16; o; o /= 2) s += __shfl_xor_sync(~0u, s, o);
        if (lane == 0) out[g] = s;
    }
}

// kApply: a cluster holds the whole unit and writes the result; else a block writes its part's mean and deviations by group.
template <bool kApply>
__global__ void __launch_bounds__(kThreads) group_norm_kernel(const NormArgs a) {
    extern __shared__ float4 tile[];                     // [blocks][pixels][8]
    __shared__ float total[kMaxGroups], dev[kMaxGroups], mean_s[kMaxGroups], rstd_s[kMaxGroups];
    grid_dep_sync();
    const Part p(a, blockIdx.x);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 7, wpb = a.warps_per_block;
    const size_t plane4 = (size_t)a.HW * 8;
    const size_t first4 = ((size_t)p.n * a.CB + p.b0) * plane4 + (size_t)p.p0 * 8;
    const float4 *in = reinterpret_cast<const float4 *>(a.in) + first4;
    const int most = (a.HW + a.splits - 1) / a.splits;
    float *sums = reinterpret_cast<float *>(tile + (size_t)a.unit_blocks * most * 8);      // [warps of a block][blocks * 32]
    float *cmean = sums + wpb * a.unit_blocks * 32, *cscale = cmean + a.unit_blocks * 32, *cshift = cscale + a.unit_blocks * 32;

    // each warp copies what it sums, so that its own wait is enough
    for (int i = warp; i < p.blocks * wpb; i += kWarps) {
        const int b = i / wpb, share = i % wpb;
        for (int q = share * 4 + (lane >> 3); q < p.pixels; q += wpb * 4)
            copy16_async(tile + ((size_t)b * p.pixels + q) * 8 + j, in + (size_t)b * plane4 + (size_t)q * 8 + j);
    }
    copy_commit();
    grid_dep_trigger();
    if (kApply)
        for (int c = threadIdx.x; c < p.blocks * 32; c += kThreads) {
            cscale[c] = c >= p.channels ? 0.0f : a.gamma ? a.gamma[p.c0 + c] : 1.0f;
            cshift[c] = c >= p.channels ? 0.0f : a.beta ? a.beta[p.c0 + c] : 0.0f;
        }
    copy_wait<0>();
    __syncwarp();
    channel_sums(p, wpb, tile, sums, [](float4 v, int) { return v; });
    __syncthreads();
    group_sums(p, a.cpg, wpb, sums, total);
    if (kApply) { cluster_arrive(); cluster_wait(); } else __syncthreads();

    if (threadIdx.x < p.groups) {
        float s = 0.0f;
        if (kApply)
            for (int r = 0; r < a.splits; ++r) s += cluster_read(total + threadIdx.x, r);
        else
            s = total[threadIdx.x];
        mean_s[threadIdx.x] = s / ((float)a.cpg * (float)(kApply ? a.HW : p.pixels));
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.blocks * 32; c += kThreads) cmean[c] = c < p.channels ? mean_s[c / a.cpg] : 0.0f;
    __syncthreads();
    channel_sums(p, wpb, tile, sums, [&](float4 v, int c) {
        const float4 m = *reinterpret_cast<const float4 *>(cmean + c);
        v.x -= m.x; v.y -= m.y; v.z -= m.z; v.w -= m.w;
        return make_float4(v.x * v.x, v.y * v.y, v.z * v.z, v.w * v.w);
    });
    __syncthreads();
    group_sums(p, a.cpg, wpb, sums, dev);
    if (!kApply) {
        __syncthreads();
        if (threadIdx.x < p.groups) {
            float *s = a.stats + ((size_t)blockIdx.x * kMaxGroups + threadIdx.x) * 2;
            s[0] = mean_s[threadIdx.x];
            s[1] = dev[threadIdx.x];
        }
        return;
    }
    cluster_arrive();
    cluster_wait();
    if (threadIdx.x < p.groups) {
        float s = 0.0f;
        for (int r = 0; r < a.splits; ++r) s += cluster_read(dev + threadIdx.x, r);
        rstd_s[threadIdx.x] = 1.0f / sqrtf(s / ((float)a.cpg * (float)a.HW) + a.eps);
    }
    cluster_arrive();                                    // the others' sums are read: waited for before the block ends
    __syncthreads();
    for (int c = threadIdx.x; c < p.channels; c += kThreads) cscale[c] *= rstd_s[c / a.cpg];
    __syncthreads();
    float4 *out = reinterpret_cast<float4 *>(a.out) + first4;
    for (int i = warp; i < p.blocks * wpb; i += kWarps) {
        const int b = i / wpb, share = i % wpb, c = b * 32 + j * 4;
        const float4 m = *reinterpret_cast<const float4 *>(cmean + c), s = *reinterpret_cast<const float4 *>(cscale + c),
                     t = *reinterpret_cast<const float4 *>(cshift + c);
        for (int q = share * 4 + (lane >> 3); q < p.pixels; q += wpb * 4) {
            float4 v = tile[((size_t)b * p.pixels + q) * 8 + j];
            v.x = activate(fmaf(v.x - m.x, s.x, t.x), a.act); v.y = activate(fmaf(v.y - m.y, s.y, t.y), a.act);
            v.z = activate(fmaf(v.z - m.z, s.z, t.z), a.act); v.w = activate(fmaf(v.w - m.w, s.w, t.w), a.act);
            if (c + 4 > p.channels) {                    // pad lanes: +0 whatever lies there
                if (c + 0 >= p.channels) v.x = 0.0f;
                if (c + 1 >= p.channels) v.y = 0.0f;
                if (c + 2 >= p.channels) v.z = 0.0f;
                v.w = 0.0f;
            }
            __stcs(out + (size_t)b * plane4 + (size_t)q * 8 + j, v);
        }
    }
    cluster_wait();
}

// The second kernel: merges the parts' statistics (count-weighted means; deviations plus those of the means) and normalises.
__global__ void __launch_bounds__(kThreads) group_norm_apply_kernel(const NormArgs a) {
    extern __shared__ float4 tile[];
    __shared__ float mean_s[kMaxGroups], rstd_s[kMaxGroups];
    grid_dep_sync();
    grid_dep_trigger();
    const Part p(a, gridDim.x - 1 - blockIdx.x);         // what the first kernel read last is the likeliest to be in L2
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 7, wpb = a.warps_per_block;
    float *cmean = reinterpret_cast<float *>(tile), *cscale = cmean + a.unit_blocks * 32, *cshift = cscale + a.unit_blocks * 32;
    if (threadIdx.x < p.groups) {
        const float *s = a.stats + ((size_t)((size_t)p.n * a.units + p.unit) * a.splits * kMaxGroups + threadIdx.x) * 2;
        float mean = s[0], dev = s[1], count = (float)(int)((long long)a.HW / a.splits);
        for (int r = 1; r < a.splits; ++r) {
            const float n = (float)((int)((long long)a.HW * (r + 1) / a.splits) - (int)((long long)a.HW * r / a.splits));
            const float m = s[(size_t)r * kMaxGroups * 2], d = m - mean, all = count + n;
            dev += s[(size_t)r * kMaxGroups * 2 + 1] + d * d * (count * n / all) * (float)a.cpg;
            mean += d * (n / all);
            count = all;
        }
        mean_s[threadIdx.x] = mean;
        rstd_s[threadIdx.x] = 1.0f / sqrtf(dev / ((float)a.cpg * (float)a.HW) + a.eps);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.blocks * 32; c += kThreads) {
        const bool real = c < p.channels;
        cmean[c] = real ? mean_s[c / a.cpg] : 0.0f;
        cscale[c] = !real ? 0.0f : (a.gamma ? a.gamma[p.c0 + c] : 1.0f) * rstd_s[c / a.cpg];
        cshift[c] = real && a.beta ? a.beta[p.c0 + c] : 0.0f;
    }
    __syncthreads();
    const size_t plane4 = (size_t)a.HW * 8;
    const size_t first4 = ((size_t)p.n * a.CB + p.b0) * plane4 + (size_t)p.p0 * 8;
    const float4 *in = reinterpret_cast<const float4 *>(a.in) + first4;
    float4 *out = reinterpret_cast<float4 *>(a.out) + first4;
    for (int i = warp; i < p.blocks * wpb; i += kWarps) {
        const int b = i / wpb, share = i % wpb, c = b * 32 + j * 4;
        const float4 m = *reinterpret_cast<const float4 *>(cmean + c), s = *reinterpret_cast<const float4 *>(cscale + c),
                     t = *reinterpret_cast<const float4 *>(cshift + c);
        const float4 *x = in + (size_t)b * plane4 + j;
        float4 *y = out + (size_t)b * plane4 + j;
        constexpr int kAhead = 4;
        for (int q = share * 4 + (lane >> 3); q < p.pixels; q += wpb * 4 * kAhead) {
            float4 v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (q + u * wpb * 4 < p.pixels) v[u] = __ldcs(x + (size_t)(q + u * wpb * 4) * 8);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (q + u * wpb * 4 >= p.pixels) break;
                float4 r;
                r.x = activate(fmaf(v[u].x - m.x, s.x, t.x), a.act); r.y = activate(fmaf(v[u].y - m.y, s.y, t.y), a.act);
                r.z = activate(fmaf(v[u].z - m.z, s.z, t.z), a.act); r.w = activate(fmaf(v[u].w - m.w, s.w, t.w), a.act);
                if (c + 4 > p.channels) {
                    if (c + 0 >= p.channels) r.x = 0.0f;
                    if (c + 1 >= p.channels) r.y = 0.0f;
                    if (c + 2 >= p.channels) r.z = 0.0f;
                    r.w = 0.0f;
                }
                __stcs(y + (size_t)(q + u * wpb * 4) * 8, r);
            }
        }
    }
}

struct NormPlan {
    int unit_blocks, units, splits, warps_per_block;
    bool on_chip;
    size_t smem;
};

int gcd(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }

constexpr size_t kBlockBytes = 104u << 10;        // shared memory where two blocks share an SM
constexpr size_t kMostBytes = 220u << 10;         // at all

size_t block_bytes(const NormPlan &p, int HW) {   // the tile, the sums of channels, their means, scales and shifts
    return (size_t)p.unit_blocks * 128 * ((HW + p.splits - 1) / p.splits + p.warps_per_block + 3);
}

NormPlan plan_norm(int N, int C, int HW, int groups) {
    NormPlan p;
    const int cpg = C / groups, CB = blocks_of(C);
    const long long unit = (long long)cpg / gcd(cpg, 32) * 32;
    p.unit_blocks = unit / 32 < CB ? (int)(unit / 32) : CB;
    p.units = ceil_div(CB, p.unit_blocks);
    p.warps_per_block = p.unit_blocks < kWarps ? kWarps / p.unit_blocks : 1;
    const size_t bytes = (size_t)p.unit_blocks * HW * 128;
    p.splits = 1;
    while (p.splits < 8 && block_bytes(p, HW) > kBlockBytes) p.splits *= 2;
    p.on_chip = block_bytes(p, HW) <= kMostBytes;
    if (p.on_chip) {
        // few units: more blocks, down to 16 KB each
        while (p.splits < 8 && (long long)N * p.units * p.splits * 2 <= kSmCount && block_bytes(p, HW) > (16u << 10)) p.splits *= 2;
    } else {
        p.splits = (int)((bytes + kBlockBytes / 2 - 1) / (kBlockBytes / 2));
        if (p.splits > HW) p.splits = HW;
    }
    p.smem = block_bytes(p, HW);
    return p;
}

bool norm_shape_ok(int N, int C, int H, int W, int groups) {
    return N >= 1 && C >= 1 && H >= 1 && W >= 1 && groups >= 1 && groups <= C && C % groups == 0 && C <= (1 << 16) &&
           (long long)H * W <= (1ll << 24) && (long long)N * blocks_of(C) <= (1ll << 24);
}

}  // namespace
}  // namespace small

using namespace small;

SMALL_API size_t small_group_norm_workspace_bytes(int N, int C, int H, int W, int groups) {
    if (!norm_shape_ok(N, C, H, W, groups)) return 0;
    const NormPlan p = plan_norm(N, C, H * W, groups);
    return p.on_chip ? 0 : sizeof(float) * 2 * kMaxGroups * (size_t)N * p.units * p.splits;
}

SMALL_API int small_group_norm(small_ctx *ctx, const float *in, const float *gamma, const float *beta, float *out, void *workspace,
                               int N, int C, int H, int W, int groups, float eps, unsigned flags, void *stream) {
    if (!ctx) return SMALL_ERR_NOT_INIT;
    CallOfItsOwn call(ctx);
    if ((flags & ~(SMALL_RELU | SMALL_SILU)) || flags == (SMALL_RELU | SMALL_SILU)) return SMALL_ERR_INVALID_ARG;
    if (!std::isfinite(eps) || eps < 0.0f) return SMALL_ERR_INVALID_ARG;
    if (int s = check_pointers({in, out}, {gamma, beta, workspace})) return s;
    if (!norm_shape_ok(N, C, H, W, groups)) return SMALL_ERR_SHAPE;
    const NormPlan p = plan_norm(N, C, H * W, groups);
    const long long blocks = (long long)N * p.units * p.splits;
    if (blocks > 0x7fffffffLL) return SMALL_ERR_SHAPE;
    const size_t bytes = sizeof(float) * packed_elems(N, C, H, W), ws = small_group_norm_workspace_bytes(N, C, H, W, groups);
    if (in != out && ranges_overlap(in, bytes, out, bytes)) return SMALL_ERR_OVERLAP;
    for (const float *q : {gamma, beta})
        if (q && ranges_overlap(q, sizeof(float) * C, out, bytes)) return SMALL_ERR_OVERLAP;
    if (ws) {
        if (!workspace) return SMALL_ERR_WORKSPACE;
        if (ranges_overlap(workspace, ws, in, bytes) || ranges_overlap(workspace, ws, out, bytes)) return SMALL_ERR_OVERLAP;
        for (const float *q : {gamma, beta})
            if (q && ranges_overlap(q, sizeof(float) * C, workspace, ws)) return SMALL_ERR_OVERLAP;
    }
    const OnDevice on(ctx);
    if (on.error != cudaSuccess) { ctx->last_cuda = (int)on.error; return SMALL_ERR_CUDA; }
    const NormArgs a{in, gamma, beta, out, static_cast<float *>(workspace), C, blocks_of(C), C / groups, H * W,
                     p.unit_blocks, p.units, p.splits, p.warps_per_block, eps, flags};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    static std::atomic<unsigned long long> whole{0}, part{0};
    const size_t most = ctx->max_smem_optin - 2048;              // the kernels have static shared memory too
    if (p.smem > most) return SMALL_ERR_UNSUPPORTED;
    if (p.on_chip) {
        if (int s = allow_shared_memory(ctx, group_norm_kernel<true>, whole, most)) return s;
        launch_clusters(ctx, group_norm_kernel<true>, dim3((unsigned)blocks), dim3(kThreads), p.splits, p.smem, st, a);
        return check_launch(ctx);
    }
    if (int s = allow_shared_memory(ctx, group_norm_kernel<false>, part, most)) return s;
    launch_kernel(ctx, group_norm_kernel<false>, dim3((unsigned)blocks), dim3(kThreads), p.smem, st, a);
    if (int s = check_launch(ctx)) return s;
    launch_kernel(ctx, group_norm_apply_kernel, dim3((unsigned)blocks), dim3(kThreads), 3 * (size_t)p.unit_blocks * 128, st, a);
    return check_launch(ctx);
}
