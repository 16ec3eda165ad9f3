// Group normalisation with an activation on blocked tensors:
//     out = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c]),   mean and var over a group of channels and the plane.
// Bound by memory: x has to be read once and the result written once.  The unit of work is one image's smallest run of channels
// that is both whole groups and whole channel blocks (lcm(channels of a group, 32), cut off at C), so that every 128-byte line is
// read by one unit only.  A cluster of 1 to 8 thread blocks shares out the unit's pixels and keeps them in shared memory: sums,
// then deviations from the mean, then the result are all taken from there, and only sums of groups cross the cluster.  Units
// too large for that are summed block by block (each block's mean and deviations, in shared memory too) and merged and
// normalised by a second kernel, which reads the tensor again.  128 images of 256 channels, 56 x 56, 32 groups: 822 MB in 188 us with
// SiLU, 164 without; what waits most are the barriers of the two sums.  64 images of 128 channels, 28 x 28: 13.6 us, 3.8 TB/s.
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
    int splits, part;                   // thread blocks that share a unit's pixels, pixels of each (the last ones' may be fewer)
    int warps_per_block;                // warps that share a channel block
    int fold;                           // 1 << fold channels of a group where those are lanes of a warp, else -1
    float eps, over_count;              // 1 / (channels of a group * pixels)
};

template <unsigned kAct>
__device__ __forceinline__ float activate(float y) {
    if (kAct == SMALL_RELU) return y > 0.0f ? y : 0.0f;
    if (kAct == SMALL_SILU) return __fdividef(y, 1.0f + __expf(-y));     // exp to inf: -0, as the limit has it
    return y;
}
template <unsigned kAct>
__device__ __forceinline__ float4 normalise(float4 v, float4 m, float4 s, float4 t) {
    return make_float4(activate<kAct>(fmaf(v.x - m.x, s.x, t.x)), activate<kAct>(fmaf(v.y - m.y, s.y, t.y)), activate<kAct>(fmaf(v.z - m.z, s.z, t.z)),
                       activate<kAct>(fmaf(v.w - m.w, s.w, t.w)));
}
__device__ __forceinline__ float4 clear_pad(float4 v, int c, int channels) {         // pad lanes: +0 whatever lies there
    if (c + 4 <= channels) return v;
    return make_float4(c < channels ? v.x : 0.0f, c + 1 < channels ? v.y : 0.0f, c + 2 < channels ? v.z : 0.0f, 0.0f);
}
// 1 / sqrt(x): the approximation and one step of Newton's, which has nothing to add to the 0 of an infinite variance (inf * 0).
__device__ __forceinline__ float over_sqrt(float x) {
    const float r = rsqrtf(x);
    return x < INFINITY ? r * fmaf(-0.5f * x * r, r, 1.5f) : r;
}

// The unit of this thread block and the part of its pixels that the block holds.
struct Part {
    int n, unit, split, b0, blocks, c0, channels, groups, p0, pixels;
    __device__ Part(const NormArgs &a, int block, int y) {
        n = a.splits == 1 ? block : block / a.splits;
        split = block - n * a.splits;
        unit = y;
        b0 = unit * a.unit_blocks;
        blocks = min(a.unit_blocks, a.CB - b0);
        c0 = b0 * 32;
        channels = min(blocks * 32, a.C - c0);
        groups = a.fold >= 0 ? channels >> a.fold : channels / a.cpg;
        p0 = min(a.HW, split * a.part);
        pixels = min(a.HW - p0, a.part);
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
#pragma unroll 4
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

// Sums by channel and share -> use(channel of the unit, the sum of its group), called by one thread for each channel; groups whose channels are
// neighbouring lanes need no memory for it.  kCluster: summed over the cluster's blocks too, through `total`, which the others read until the next
// cluster_wait().  A barrier of the block is behind `sums` already; use() is followed by none.
template <bool kCluster, typename U>
__device__ __forceinline__ void group_sums(const NormArgs &a, const Part &p, const float *sums, float *total, U use) {
    const int lane = threadIdx.x & 31, wpb = a.warps_per_block, channels = p.blocks * 32;
    if (a.fold >= 0 && (!kCluster || a.splits == 1)) {
        for (int c = threadIdx.x; c < channels; c += kThreads) {
            float s = 0.0f;
#pragma unroll
            for (int share = 0; share < kWarps; ++share) s += share < wpb ? sums[share * channels + c] : 0.0f;
            for (int o = 1; o < 1 << a.fold; o *= 2) s += __shfl_xor_sync(~0u, s, o);
            use(c, s);
        }
        return;
    }
    for (int g = threadIdx.x >> 5; g < p.groups; g += kWarps) {          // a warp a group
        float s = 0.0f;
        for (int c = lane; c < a.cpg; c += 32) {
            float t = 0.0f;
#pragma unroll
            for (int share = 0; share < kWarps; ++share) t += share < wpb ? sums[share * channels + g * a.cpg + c] : 0.0f;
            s += t;
        }
#pragma unroll
        for (int o = 16; o; o /= 2) s += __shfl_xor_sync(~0u, s, o);
        if (lane == 0) total[g] = s;
    }
    if (kCluster && a.splits > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
    for (int c = threadIdx.x; c < channels; c += kThreads) {
        const int g = a.fold >= 0 ? c >> a.fold : c / a.cpg;
        float s = 0.0f;
        if (g < p.groups) {
            if (kCluster && a.splits > 1) {
                float part[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) part[r] = r < a.splits ? cluster_read(total + g, r) : 0.0f;         // all on their way at once
#pragma unroll
                for (int r = 0; r < 8; ++r) s += part[r];
            } else {
                s = total[g];
            }
        }
        use(c, s);
    }
}

// kApply: a cluster holds the whole unit and writes the result; else a block writes its part's mean and deviations by group.
template <bool kApply, unsigned kAct>
__global__ void __launch_bounds__(kThreads) group_norm_kernel(const NormArgs a) {
    extern __shared__ float4 tile[];                     // [blocks][pixels][8]
    __shared__ float total[kMaxGroups], dev[kMaxGroups];
    grid_dep_sync();
    const Part p(a, blockIdx.x, blockIdx.y);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 7, wpb = a.warps_per_block;
    const size_t plane4 = (size_t)a.HW * 8;
    const size_t first4 = ((size_t)p.n * a.CB + p.b0) * plane4 + (size_t)p.p0 * 8;
    const float4 *in = reinterpret_cast<const float4 *>(a.in) + first4;
    float *sums = reinterpret_cast<float *>(tile + (size_t)a.unit_blocks * a.part * 8);      // [warps of a block][blocks * 32]
    float *cmean = sums + wpb * a.unit_blocks * 32, *cscale = cmean + a.unit_blocks * 32, *cshift = cscale + a.unit_blocks * 32;

    // each warp copies what it sums, so that its own wait is enough
    for (int i = warp; i < p.blocks * wpb; i += kWarps) {
        const int b = i / wpb, share = i % wpb;
#pragma unroll 4
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
    const float over = kApply ? a.over_count : 1.0f / ((float)a.cpg * (float)p.pixels);
    group_sums<kApply>(a, p, sums, total, [&](int c, float s) { cmean[c] = s * over; });
    __syncthreads();
    channel_sums(p, wpb, tile, sums, [&](float4 v, int c) {
        const float4 m = *reinterpret_cast<const float4 *>(cmean + c);
        v.x -= m.x; v.y -= m.y; v.z -= m.z; v.w -= m.w;
        return make_float4(v.x * v.x, v.y * v.y, v.z * v.z, v.w * v.w);
    });
    __syncthreads();
    if (!kApply) {
        float *stats = a.stats + (((size_t)p.n * a.units + p.unit) * a.splits + p.split) * kMaxGroups * 2;
        group_sums<false>(a, p, sums, dev, [&](int c, float s) {
            const int g = a.fold >= 0 ? c >> a.fold : c / a.cpg;
            if (c >= p.channels || c != g * a.cpg) return;               // the group's first channel
            stats[g * 2] = cmean[c];
            stats[g * 2 + 1] = s;
        });
        return;
    }
    group_sums<true>(a, p, sums, dev, [&](int c, float s) { cscale[c] *= over_sqrt(fmaf(s, over, a.eps)); });
    if (a.splits > 1) cluster_arrive_relaxed();          // the others' sums are read: waited for before the block ends
    __syncthreads();
    float4 *out = reinterpret_cast<float4 *>(a.out) + first4;
    for (int i = warp; i < p.blocks * wpb; i += kWarps) {
        const int b = i / wpb, share = i % wpb, c = b * 32 + j * 4;
        const float4 m = *reinterpret_cast<const float4 *>(cmean + c), s = *reinterpret_cast<const float4 *>(cscale + c),
                     t = *reinterpret_cast<const float4 *>(cshift + c);
        const float4 *x = tile + (size_t)b * p.pixels * 8 + j;
        float4 *y = out + (size_t)b * plane4 + j;
#pragma unroll 4
        for (int q = share * 4 + (lane >> 3); q < p.pixels; q += wpb * 4) __stcs(y + (size_t)q * 8, clear_pad(normalise<kAct>(x[(size_t)q * 8], m, s, t), c, p.channels));
    }
    if (a.splits > 1) cluster_wait();
}

// The second kernel: merges the parts' statistics (count-weighted means; deviations plus those of the means) and normalises.
template <unsigned kAct>
__global__ void __launch_bounds__(kThreads) group_norm_apply_kernel(const NormArgs a) {
    extern __shared__ float4 tile[];
    __shared__ float mean_s[kMaxGroups], rstd_s[kMaxGroups];
    grid_dep_sync();
    grid_dep_trigger();
    const Part p(a, gridDim.x - 1 - blockIdx.x, gridDim.y - 1 - blockIdx.y);         // what the first kernel read last is the likeliest to be in L2
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 7, wpb = a.warps_per_block;
    float *cmean = reinterpret_cast<float *>(tile), *cscale = cmean + a.unit_blocks * 32, *cshift = cscale + a.unit_blocks * 32;
    // a warp a group, a lane the parts l, l + 32, ...; then the lanes' parts two by two
    for (int g = warp; g < p.groups; g += kWarps) {
        const float2 *s = reinterpret_cast<const float2 *>(a.stats) + ((size_t)p.n * a.units + p.unit) * a.splits * kMaxGroups + g;
        float mean = 0.0f, dev = 0.0f, count = 0.0f;
        auto join = [&](float m, float d2, float n) {
            if (n == 0.0f) return;
            if (count == 0.0f) { mean = m; dev = d2; count = n; return; }        // (below, 0 * the square of a far mean: of one beyond 1.8e19 NaN)
            const float d = m - mean, all = count + n, share = n / all;
            dev += d2 + d * d * (count * share) * (float)a.cpg;
            mean += d * share;
            count = all;
        };
        for (int r = lane; r < a.splits; r += 32) {
            const float2 v = s[(size_t)r * kMaxGroups];
            join(v.x, v.y, (float)min(a.HW - r * a.part, a.part));
        }
#pragma unroll
        for (int o = 16; o; o /= 2) {
            const float m = __shfl_down_sync(~0u, mean, o), d2 = __shfl_down_sync(~0u, dev, o), n = __shfl_down_sync(~0u, count, o);
            if (lane < o) join(m, d2, n);
        }
        if (lane == 0) {
            mean_s[g] = mean;
            rstd_s[g] = over_sqrt(fmaf(dev, a.over_count, a.eps));
        }
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
            for (int u = 0; u < kAhead; ++u)
                if (q + u * wpb * 4 < p.pixels) __stcs(y + (size_t)(q + u * wpb * 4) * 8, clear_pad(normalise<kAct>(v[u], m, s, t), c, p.channels));
        }
    }
}

struct NormPlan {
    int unit_blocks, units, splits, warps_per_block;
    bool on_chip;
    size_t smem;
};

int gcd(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }

// Shared memory of a block: a unit that leaves room for two blocks on an SM stays whole (28 x 28, 100 KB: 12.7 us, as two halves 14.1), a larger
// one is cut until three share one (56 x 56, 400 KB, batch 128, 256 channels: 181 us in eighths or in parts of 70 KB, 208 in quarters).
constexpr size_t kBlockBytes = 104u << 10, kSplitBytes = 70u << 10;
constexpr size_t kMostBytes = 220u << 10;         // at all
constexpr size_t kMostShared = (227u << 10) - 2048;         // what a block can have, less the kernels' static shared memory

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
    if (block_bytes(p, HW) > kBlockBytes)
        while (p.splits < 8 && block_bytes(p, HW) > kSplitBytes) p.splits *= 2;
    p.on_chip = block_bytes(p, HW) <= kMostBytes;
    if (p.on_chip) {
        // few units: more blocks, down to 16 KB each
        while (p.splits < 8 && (long long)N * p.units * p.splits * 2 <= kSmCount && block_bytes(p, HW) > (16u << 10)) p.splits *= 2;
    } else {
        p.splits = (int)((bytes + kBlockBytes / 2 - 1) / (kBlockBytes / 2));
        if (p.splits > HW) p.splits = HW;
        p.splits = ceil_div(HW, ceil_div(HW, p.splits));         // none without a pixel
        for (int part = ceil_div(HW, p.splits); part > 1 && block_bytes(p, HW) > kMostShared;) p.splits = ceil_div(HW, --part);
    }
    p.smem = block_bytes(p, HW);
    return p;
}

template <unsigned kAct>
int launch_norm(small_ctx *ctx, const NormArgs &a, const NormPlan &p, int N, cudaStream_t st) {
    static std::atomic<unsigned long long> whole{0}, part{0}, applied{0};
    const size_t most = kMostShared;
    const dim3 grid((unsigned)(N * p.splits), (unsigned)p.units), block(kThreads);
    if (p.on_chip) {
        if (int s = allow_shared_memory(ctx, group_norm_kernel<true, kAct>, whole, most)) return s;
        if (p.splits > 1) launch_clusters(ctx, group_norm_kernel<true, kAct>, grid, block, p.splits, p.smem, st, a);
        else launch_kernel(ctx, group_norm_kernel<true, kAct>, grid, block, p.smem, st, a);
        return check_launch(ctx);
    }
    if (int s = allow_shared_memory(ctx, group_norm_kernel<false, 0>, part, most)) return s;
    launch_kernel(ctx, group_norm_kernel<false, 0>, grid, block, p.smem, st, a);
    if (int s = check_launch(ctx)) return s;
    // means, scales and shifts of some more than 4000 channels pass the 48 KB that need not be asked for (with the kernel's static 256 bytes)
    const size_t channels = 3 * (size_t)p.unit_blocks * 128;
    if (channels > (47u << 10))
        if (int s = allow_shared_memory(ctx, group_norm_apply_kernel<kAct>, applied, most)) return s;
    launch_kernel(ctx, group_norm_apply_kernel<kAct>, grid, block, channels, st, a);
    return check_launch(ctx);
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
    if (p.smem > kMostShared) return SMALL_ERR_UNSUPPORTED;
    const long long blocks = (long long)N * p.units * p.splits;
    if (blocks > 0x7fffffffLL || p.units > 65535) return SMALL_ERR_SHAPE;
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
    const int cpg = C / groups, part = ceil_div(H * W, p.splits);
    const NormArgs a{in, gamma, beta, out, static_cast<float *>(workspace), C, blocks_of(C), cpg, H * W, p.unit_blocks, p.units, p.splits, part, p.warps_per_block,
                     cpg <= 32 && (cpg & (cpg - 1)) == 0 ? __builtin_ctz(cpg) : -1, eps, (float)(1.0 / ((double)cpg * H * W))};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return flags == SMALL_RELU ? launch_norm<SMALL_RELU>(ctx, a, p, N, st) : flags == SMALL_SILU ? launch_norm<SMALL_SILU>(ctx, a, p, N, st) : launch_norm<0>(ctx, a, p, N, st);
}
