// Attention of few queries (attention pooling: one), FP32 multiply-adds in every math mode: bound by reading keys and values, once.
//
// The rows that share a key head - its query heads times the queries, R of them a block - are held in registers, and so are their sums.  Eight
// lanes take a key's channels, 128 bytes a load; a warp's four such groups and a block's eight warps walk the keys side by side, each
// group with a running maximum of its own.  Loads go through shared memory, where each thread copies what it will read itself: two of three
// stages of 128 bytes a thread are under way while it works on the third, without a register or a barrier for them, in two blocks an SM (six
// stages in one block: 30 us for the 75 MB below, loads held in registers 57).  A cluster of up to 16 blocks shares out the keys; what groups, warps
// and blocks have found is joined by their maxima.  Batch 4, 4 key heads of 64 for 8 heads, 96 x 96: 75 MB in 23 us, 3.3 TB/s; 16 of 56 x 56: 4.5 TB/s.
#include "attention.cuh"

namespace small {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

constexpr int kStages = 3;
constexpr int kMostSplits = 16;
constexpr size_t kRing = (size_t)kWarps * kStages * 8 * 32 * sizeof(float4);

struct FewArgs {
    AttnArgs a;
    int rows, groups, splits;                            // rows of a key head, groups of R of them, blocks of a cluster
};

// kGeneral: a bias table, a cap or padded images.  The loop is kept short: unrolled over the stages it missed the instruction cache more
// than anything else.
template <int DP, int R, bool kGeneral>
__global__ void __launch_bounds__(kThreads, R * DP >= 512 ? 1 : 2) attention_few_kernel(const FewArgs f) {
    constexpr int kVec = DP / 32, kAhead = 4 / kVec;     // keys of a stage: 64 bytes of keys and 64 of values
    extern __shared__ float4 ring[];                     // [warp][stage][key or value][kAhead][kVec][lane]
    __shared__ float top_s[kWarps][R], sum_s[kWarps][R];
    __shared__ float4 out_s[kWarps][R][DP / 4];
    __shared__ float top_b[R], sum_b[R], out_b[R][DP];
    const AttnArgs &a = f.a;
    grid_dep_sync();
    grid_dep_trigger();
    const int split = blockIdx.x, hk = blockIdx.y / f.groups, r0 = blockIdx.y % f.groups * R, n = blockIdx.z;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = (lane & 7) * 4, share = a.heads / a.kv_heads;
    const int2 qe = extent(a.q_ext, n, a.QH, a.QW), ke = extent(a.k_ext, n, a.KH, a.KW);
    const int keys = ke.x * ke.y, from = (int)((long long)keys * split / f.splits), to = (int)((long long)keys * (split + 1) / f.splits);
    const float *k = a.k + n * a.k_stride, *v = a.v + n * a.v_stride;
    const bool whole = ke.y == a.KW, capping = a.cap > 0.0f;
    const size_t table = (size_t)(a.QH + a.KH - 1) * (a.QW + a.KW - 1);
    const float cap2 = a.cap * kLog2e, over_cap = capping ? 1.0f / a.cap : 0.0f, unit = capping ? a.scale : a.scale * kLog2e;

    float4 q[R][kVec], o[R][kVec];
    const float *bias[R];
    float m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool real = r0 + r < f.rows;
        const int row = real ? r0 + r : 0, h = hk * share + row / a.QP, i = row % a.QP;
        bias[r] = kGeneral && a.bias ? a.bias + h * table + of_query(a, i) : nullptr;
        m[r] = -INFINITY;
        l[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < kVec; ++c) {
            q[r][c] = real ? load4(a.q + n * a.q_stride, h * a.D, c * 32 + c0, a.D, i, a.QP) : make_float4(0.f, 0.f, 0.f, 0.f);
            q[r][c].x *= unit; q[r][c].y *= unit; q[r][c].z *= unit; q[r][c].w *= unit;
            o[r][c] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    const float4 *mine = ring + warp * kStages * 8 * 32 + lane;
    const uint32_t mine_s = (uint32_t)__cvta_generic_to_shared(mine);
    const int step = kAhead * kWarps * 4, rounds = (to - from + step - 1) / step;        // the same for all of the block
    const float *kc[kVec], *vc[kVec];                    // this lane's channels at pixel 0
#pragma unroll
    for (int c = 0; c < kVec; ++c) {
        const size_t e = c * 32 + c0 < a.D ? at(hk * a.D + c * 32 + c0, 0, a.KP) : 0;
        kc[c] = k + e;
        vc[c] = v + e;
    }
    int next = from + warp * 4 + (lane >> 3);            // this group's first key of the round that is fetched next
    // rows and columns of the keys to be fetched and of those to be weighed; a block's groups are kWarps * 4 keys apart
    struct Walk {
        int y, x;
        __device__ void on(int dy, int dx, int width) {
            y += dy;
            x += dx;
            if (x >= width) { x -= width; ++y; }
        }
    };
    const int width = kGeneral ? max(ke.y, 1) : 1, dy = kWarps * 4 / width, dx = kWarps * 4 % width;
    Walk ahead{next / width, next % width}, here = ahead;
    auto fetch = [&](int stage) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u, next += kWarps * 4) {
            const bool in = next < to;
            const int p = !in ? 0 : kGeneral && !whole ? ahead.y * a.KW + ahead.x : next;
            if (kGeneral && !whole) ahead.on(dy, dx, width);
#pragma unroll
            for (int c = 0; c < kVec; ++c) {
                const bool some = in && c * 32 + c0 < a.D;
                copy16_or_clear(mine_s + ((stage * 2 + 0) * 4 + u * kVec + c) * 512, kc[c] + (size_t)p * 32, some);
                copy16_or_clear(mine_s + ((stage * 2 + 1) * 4 + u * kVec + c) * 512, vc[c] + (size_t)p * 32, some);
            }
        }
        copy_commit();
    };
#pragma unroll 1
    for (int x = 0; x < kStages - 1; ++x) fetch(x);
    int j = from + warp * 4 + (lane >> 3);
#pragma unroll 1
    for (int round = 0, stage = 0; round < rounds; ++round, stage = stage == kStages - 1 ? 0 : stage + 1, j += step) {
        fetch(stage == 0 ? kStages - 1 : stage - 1);
        copy_wait<kStages - 1>();
        float4 x[kAhead][kVec], y[kAhead][kVec];
        float bias_of[R][kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (kGeneral && a.bias) {                    // on their way while the products are taken
                const bool in = j + u * kWarps * 4 < to;
                const int place = of_key(a, here.y, here.x);
                here.on(dy, dx, width);
#pragma unroll
                for (int r = 0; r < R; ++r) bias_of[r][u] = in ? __ldg(bias[r] - place) : 0.0f;
            }
#pragma unroll
            for (int c = 0; c < kVec; ++c) {
                x[u][c] = mine[((stage * 2 + 0) * 4 + u * kVec + c) * 32];
                y[u][c] = mine[((stage * 2 + 1) * 4 + u * kVec + c) * 32];
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s[kAhead], top = m[r];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                s[u] = 0.0f;
#pragma unroll
                for (int c = 0; c < kVec; ++c)
                    s[u] = fmaf(q[r][c].x, x[u][c].x, fmaf(q[r][c].y, x[u][c].y, fmaf(q[r][c].z, x[u][c].z, fmaf(q[r][c].w, x[u][c].w, s[u]))));
#pragma unroll
                for (int w = 1; w < 8; w *= 2) s[u] += __shfl_xor_sync(~0u, s[u], w);
                if (kGeneral && capping) s[u] = capped(s[u], cap2, over_cap);
                const bool in = j + u * kWarps * 4 < to;
                if (kGeneral && a.bias) s[u] += powers_of_two(bias_of[r][u]);
                if (!in) s[u] = -INFINITY;
                top = fmaxf(top, s[u]);
            }
            const float base = top == -INFINITY ? 0.0f : top, shrink = exp2_fast(m[r] - base);       // -inf: nothing to weigh yet
            m[r] = top;
            l[r] *= shrink;
#pragma unroll
            for (int c = 0; c < kVec; ++c) { o[r][c].x *= shrink; o[r][c].y *= shrink; o[r][c].z *= shrink; o[r][c].w *= shrink; }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const float w = exp2_fast(s[u] - base);
                l[r] += w;
#pragma unroll
                for (int c = 0; c < kVec; ++c) {
                    o[r][c].x = fmaf(w, y[u][c].x, o[r][c].x); o[r][c].y = fmaf(w, y[u][c].y, o[r][c].y);
                    o[r][c].z = fmaf(w, y[u][c].z, o[r][c].z); o[r][c].w = fmaf(w, y[u][c].w, o[r][c].w);
                }
            }
        }
    }
    copy_wait<0>();
    // the warp's four groups, then the block's warps, then the cluster's blocks
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float top = m[r];
#pragma unroll
        for (int w = 8; w < 32; w *= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, w));
        const float shrink = exp2_fast(m[r] - (top == -INFINITY ? 0.0f : top));
        l[r] *= shrink;
#pragma unroll
        for (int w = 8; w < 32; w *= 2) l[r] += __shfl_xor_sync(~0u, l[r], w);
#pragma unroll
        for (int c = 0; c < kVec; ++c) {
            float4 z = make_float4(o[r][c].x * shrink, o[r][c].y * shrink, o[r][c].z * shrink, o[r][c].w * shrink);
#pragma unroll
            for (int w = 8; w < 32; w *= 2) {
                z.x += __shfl_xor_sync(~0u, z.x, w); z.y += __shfl_xor_sync(~0u, z.y, w);
                z.z += __shfl_xor_sync(~0u, z.z, w); z.w += __shfl_xor_sync(~0u, z.w, w);
            }
            if (lane < 8) out_s[warp][r][c * 8 + lane] = z;
        }
        if (lane == 0) { top_s[warp][r] = top; sum_s[warp][r] = l[r]; }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < R * DP; e += kThreads) {
        const int r = e / DP, d = e % DP;
        float top = top_s[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top = fmaxf(top, top_s[w][r]);
        const float base = top == -INFINITY ? 0.0f : top;
        float z = 0.0f, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float shrink = exp2_fast(top_s[w][r] - base);
            z = fmaf(reinterpret_cast<const float *>(out_s[w][r])[d], shrink, z);
            sum = fmaf(sum_s[w][r], shrink, sum);
        }
        out_b[r][d] = z;
        if (d == 0) { top_b[r] = top; sum_b[r] = sum; }
    }
    cluster_arrive();
    cluster_wait();
    // Reads of other blocks' memory take some hundred cycles each: all of them at once, first what each block's share weighs, then the sums.
    __shared__ float weight_s[R][kMostSplits], total_s[R][kMostSplits];
    static_assert(R * kMostSplits <= kThreads && R * kMostSplits % 16 == 0, "a thread each");
    if (const int e = threadIdx.x; e < R * kMostSplits) {
        const int r = e / kMostSplits, b = e % kMostSplits;          // the blocks of a cluster are neighbouring lanes
        const float top = b < f.splits ? cluster_read(&top_b[r], b) : -INFINITY;
        float most = top;
#pragma unroll
        for (int w = 1; w < kMostSplits; w *= 2) most = fmaxf(most, __shfl_xor_sync(0xffffu << (threadIdx.x & 16), most, w));
        const float weight = exp2_fast(top - (most == -INFINITY ? 0.0f : most));
        weight_s[r][b] = weight;
        total_s[r][b] = b < f.splits ? cluster_read(&sum_b[r], b) * weight : 0.0f;
    }
    __syncthreads();
    float *out = a.out + (size_t)n * a.CB * a.QP * 32;
    for (int e = split * kThreads + threadIdx.x; e < R * DP; e += f.splits * kThreads) {
        const int r = e / DP, d = e % DP, row = r0 + r;
        if (row >= f.rows || d >= a.D) continue;
        float part[kMostSplits], z = 0.0f, sum = 0.0f;
#pragma unroll
        for (int b = 0; b < kMostSplits; ++b) part[b] = b < f.splits ? cluster_read(&out_b[r][d], b) : 0.0f;
#pragma unroll
        for (int b = 0; b < kMostSplits; ++b) {
            z = fmaf(part[b], b < f.splits ? weight_s[r][b] : 0.0f, z);
            sum += total_s[r][b];
        }
        const int i = row % a.QP;
        const bool live = i / a.QW < qe.x && i % a.QW < qe.y && sum != 0.0f;
        out[at((hk * share + row / a.QP) * a.D + d, i, a.QP)] = live ? z / sum : 0.0f;
    }
    if (split == 0 && hk == a.kv_heads - 1 && r0 == 0) {             // pad lanes
        const int first = a.heads * a.D, pad = a.CB * 32 - first;
        for (int e = threadIdx.x; e < pad * a.QP; e += kThreads) out[at(first + e % pad, e / pad, a.QP)] = 0.0f;
    }
    cluster_arrive();                                    // the others may still read this block's sums
    cluster_wait();
}

template <int DP, int R, bool kGeneral>
int launch(small_ctx *ctx, FewArgs f, cudaStream_t st) {
    static std::atomic<unsigned long long> done{0};
    const unsigned long long bit = 1ull << (ctx->device & 63);
    if (!(done.load(std::memory_order_relaxed) & bit)) {
        const cudaError_t e = cudaFuncSetAttribute(attention_few_kernel<DP, R, kGeneral>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) { ctx->last_cuda = (int)e; return SMALL_ERR_CUDA; }
        done.fetch_or(bit, std::memory_order_relaxed);
    }
    static std::atomic<unsigned long long> roomy{0};
    if (int s = allow_shared_memory(ctx, attention_few_kernel<DP, R, kGeneral>, roomy, kRing)) return s;
    f.groups = ceil_div(f.rows, R);
    if ((long long)f.a.kv_heads * f.groups > 65535) return launch_attention_fp32(ctx, f.a, st);          // a grid's limit
    // up to eight blocks a cluster while they are fewer than the SMs and have some rounds each, sixteen where even so most SMs would be idle: those
    // start together only where an eighth of the GPU is free (us, 8 / 16: batch 2, 8 heads of 64, 56 x 56 12.6 / 16.3, batch 4, 4 heads, 96 x 96 23.0 / 24.7,
    // one image and head 15.2 / 10.4)
    f.splits = 1;
    auto blocks = [&] { return (long long)f.a.N * f.a.kv_heads * f.groups * f.splits; };
    while (f.splits < kMostSplits && blocks() <= (f.splits < 8 ? kSmCount : kSmCount / 4) && f.a.KP >= f.splits * 2 * 64) f.splits *= 2;
    launch_clusters(ctx, attention_few_kernel<DP, R, kGeneral>, dim3((unsigned)f.splits, (unsigned)(f.a.kv_heads * f.groups), (unsigned)f.a.N), dim3(kThreads), f.splits, kRing, st, f);
    return check_launch(ctx);
}

template <int DP, int R>
int launch(small_ctx *ctx, const FewArgs &f, cudaStream_t st) {
    return f.a.bias || f.a.cap > 0.0f || f.a.k_ext ? launch<DP, R, true>(ctx, f, st) : launch<DP, R, false>(ctx, f, st);
}

template <int DP>
int launch_rows(small_ctx *ctx, const FewArgs &f, cudaStream_t st) {
    if (f.rows == 1) return launch<DP, 1>(ctx, f, st);
    if (f.rows == 2) return launch<DP, 2>(ctx, f, st);
    if (f.rows <= 4 || DP == 128) return launch<DP, 4>(ctx, f, st);
    return launch<DP, DP == 128 ? 4 : 8>(ctx, f, st);
}

}  // namespace

int launch_attention_few(small_ctx *ctx, const AttnArgs &a, cudaStream_t st) {
    if (a.D & 3) return launch_attention_fp32(ctx, a, st);           // heads that begin inside a 16-byte vector
    const FewArgs f{a, a.QP * (a.heads / a.kv_heads), 1, 1};
    return a.D <= 32 ? launch_rows<32>(ctx, f, st) : a.D <= 64 ? launch_rows<64>(ctx, f, st) : launch_rows<128>(ctx, f, st);
}

}  // namespace small
