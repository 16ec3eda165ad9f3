// 1 x 1 convolution with an adapter for each image as one product on the tensor cores (tcgen05, kind::f16): the products t = Down_a x stand
// behind an image's channels, and s_a Up_a behind the filters, so that the adapter costs some more steps of the reduction and the result is
// written once.  Operands are pairs of halves (halves.cuh).
//
// adapter_filters_kernel: the filters as halves, 64 channels a chunk, one exponent for the layer (a cluster finds it).
// adapter_pixels_kernel: 128 pixels of an image a block: each one's largest value in one pass over them (from memory), halves in a second (from
//   L2), which pass through shared memory, where the product with Down is taken from them.  t shares the pixels' accumulator later, so its
//   exponent follows from theirs, the filters' and the adapter's; where t could pass half precision's range - it is at most the largest value
//   times the largest sum of a Down row's magnitudes - the pixel takes a smaller scale, 2 to 5 powers of two as a rule, of 17 that halves of both
//   kinds have to spare.
// adapter_product_kernel: a block walks tiles of 128 pixels x 256 filters; warps for loading (plain bulk copies, two stages of 96 KB), MMAs
//   and the epilogue (bias, previous output, ReLU), two accumulators in tensor memory so that the epilogue of a tile runs beside the next.
//   256 filters a tile: 96 KB of operands for 1536 cycles of MMAs (62 bytes a cycle and SM from L2).
//
// Batch 64, 256 -> 768, 28 x 28, rank 16: 111 to 124 us (operands from L2 or not).  Pixels 37 (the filters, 12, beside them): the largest values, while
// memory still takes the result before, then four chunks that wait for their loads.  Product 72: MMAs 58 % of the time, the rest a stage
// waits for its load.  Floor 33 for the bytes, 37 for three products.
#include "adapter.cuh"
#include "halves.cuh"

namespace small {
namespace {
using namespace halves;

constexpr int kThreads = 256;
constexpr int kChunk = 64;               // channels
constexpr int kDownRun = 4;              // chunks whose products with Down one accumulator takes (see kRun)
constexpr uint32_t kPixelBytes = kTile * 256, kRankBytes = kTile * 128;          // of a chunk of channels, of 32 ranks
constexpr int kCluster = 8, kTeams = 4, kKept = 6;       // blocks of adapter_filters_kernel, teams of 256 threads of a block, items of a team in registers

struct Layout {
    int tiles, filter_tiles;             // pixel tiles of an image
    size_t ranks_at, filters_at, scales_at, bytes;
    Layout(int N, int C, int K, int HW, int R)
        : tiles(ceil_div(HW, kTile)), filter_tiles(ceil_div(blocks_of(K), kFilterTile)) {
        const int chunks = ceil_div(C, kChunk);
        ranks_at = (size_t)N * tiles * chunks * kPixelBytes;
        filters_at = ranks_at + (size_t)N * tiles * blocks_of(R) * kRankBytes;
        scales_at = filters_at + (size_t)chunks * blocks_of(K) * 32 * 256;
        bytes = scales_at + sizeof(int) * ((size_t)N * tiles * kTile + 4);       // exponents: the filters', three words unused, each pixel's
    }
};

struct TcArgs {
    AdaptArgs a;
    AdapterShape s;
    Layout at;
    int *status;
    uint32_t limit;
};

__device__ __forceinline__ char *ws_of(const TcArgs &c) { return static_cast<char *>(c.a.ws); }
__device__ __forceinline__ int *exponents(const TcArgs &c) { return reinterpret_cast<int *>(ws_of(c) + c.at.scales_at); }
__device__ __forceinline__ int tile_rows(const TcArgs &c, int kt) { return min(kFilterTile, c.s.KB - kt * kFilterTile) * 32; }
__device__ __forceinline__ float block_max(float v, float *s) {
#pragma unroll
    for (int o = 16; o; o /= 2) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = s[0];
#pragma unroll
    for (int i = 1; i < (int)blockDim.x / 32; ++i) v = fmaxf(v, s[i]);
    return v;
}

// The FP32 section of the packed filters, [KB][CB][32 channels][32 filters], as halves [filter tile][chunk]{high: rows x 128 bytes, low: the same}.
__global__ void __launch_bounds__(kThreads *kTeams) adapter_filters_kernel(const TcArgs c) {
    __shared__ float most_s[kThreads * kTeams / 32], top, blocks[kTeams][32][33];
    grid_dep_sync();
    grid_dep_trigger();
    const int items = c.s.KB * c.s.chunks * 2, tid = threadIdx.x % kThreads, team = blockIdx.x * kTeams + threadIdx.x / kThreads;
    const float4 *w = reinterpret_cast<const float4 *>(c.a.w);
    auto fetch = [&](int i) {
        const int kb = i / (c.s.chunks * 2), cb = i % (c.s.chunks * 2);
        return i < items && cb < c.s.CB ? __ldg(w + ((size_t)kb * c.s.CB + cb) * 256 + tid) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    float most = 0.0f;
    float4 kept[kKept];                                  // the first ones stay in registers
#pragma unroll
    for (int e = 0; e < kKept; ++e) kept[e] = fetch(team + e * kCluster * kTeams);
#pragma unroll
    for (int e = 0; e < kKept; ++e) most = fmaxf(most, magnitude(kept[e]));
    for (int i = team + kKept * kCluster * kTeams; i < items; i += 4 * kCluster * kTeams) {
        float4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fetch(i + e * kCluster * kTeams);
#pragma unroll
        for (int e = 0; e < 4; ++e) most = fmaxf(most, magnitude(v[e]));
    }
    most = block_max(most, most_s);
    if (threadIdx.x == 0) top = most;
    cluster_arrive();
    cluster_wait();
#pragma unroll
    for (int b = 0; b < kCluster; ++b) most = fmaxf(most, cluster_read(&top, b));
    cluster_arrive();
    const int ex = top_exponent(most);
    const float up = lift(ex);
    if (blockIdx.x == 0 && threadIdx.x == 0) exponents(c)[0] = ex;
    char *out = ws_of(c) + c.at.filters_at;
    float (*block)[33] = blocks[threadIdx.x / kThreads];
    auto lay_out = [&](int i, const float4 &v, auto ahead) {
        const int kb = i / (c.s.chunks * 2), cb = i % (c.s.chunks * 2), kt = kb / kFilterTile;
        __syncthreads();
        const int ch = tid >> 3, f0 = (tid & 7) * 4;
        block[f0][ch] = v.x; block[f0 + 1][ch] = v.y; block[f0 + 2][ch] = v.z; block[f0 + 3][ch] = v.w;
        ahead();
        __syncthreads();
        if (i >= items) return;
        const int f = tid >> 3, c0 = (tid & 7) * 4, rows = tile_rows(c, kt), row = kb % kFilterTile * 32 + f, col = (cb & 1) * 32 + c0;
        const bool real = kb * 32 + f < c.s.K;
        uint2 hi, lo;
        split_finite(real ? block[f][c0] * up : 0.0f, real ? block[f][c0 + 1] * up : 0.0f, hi.x, lo.x);
        split_finite(real ? block[f][c0 + 2] * up : 0.0f, real ? block[f][c0 + 3] * up : 0.0f, hi.y, lo.y);
        char *to = out + ((size_t)kt * c.s.chunks * kFilterTile * 32 + (size_t)(cb >> 1) * rows) * 256;
        *reinterpret_cast<uint2 *>(to + chunk_at(row, col, rows) + (col & 4) * 2) = hi;
        *reinterpret_cast<uint2 *>(to + chunk_at(row, kChunk + col, rows) + (col & 4) * 2) = lo;
    };
#pragma unroll
    for (int e = 0; e < kKept; ++e)
        if (e * kCluster * kTeams < items) lay_out(team + e * kCluster * kTeams, kept[e], [] {});
    float4 v = fetch(team + kKept * kCluster * kTeams);
    for (int i0 = kKept * kCluster * kTeams; i0 < items; i0 += kCluster * kTeams) {
        const float4 now = v;
        lay_out(i0 + team, now, [&] { v = fetch(i0 + team + kCluster * kTeams); });
    }
    cluster_wait();                                      // the others have read this block's maximum
}

__device__ __forceinline__ void bulk_store(void *to, uint32_t from, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\tcp.async.bulk.commit_group;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
}
template <int kLeft>
__device__ __forceinline__ void bulk_store_wait() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kLeft) : "memory"); }

__device__ __forceinline__ float4 clear_from(float4 v, int n) {          // the values from the n-th on: 0
    return make_float4(n > 0 ? v.x : 0.0f, n > 1 ? v.y : 0.0f, n > 2 ? v.z : 0.0f, n > 3 ? v.w : 0.0f);
}

__global__ void __launch_bounds__(kThreads, 4) adapter_pixels_kernel(const TcArgs c) {
    extern __shared__ char raw[];                        // a chunk of pixels and one of Down: four blocks a SM hide what each waits for
    __shared__ int ex_s[kTile], full_s[kTile];           // the pixels' exponents, and what they would be without t
    __shared__ uint64_t down_s, used_s;
    __shared__ uint32_t tmem_s;
    __shared__ int gave_up;
    const AdaptArgs &a = c.a;
    const AdapterShape &s = c.s;
    const int n = blockIdx.x / c.at.tiles, pt = blockIdx.x % c.at.tiles, p0 = pt * kTile, pixels = min(kTile, a.HW - p0);
    const int warp = warp_index(), lane = threadIdx.x & 31;
    char *chunk = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u), *down_chunk = chunk + kPixelBytes;
    float *t_sums = reinterpret_cast<float *>(down_chunk + s.RQ * 256);          // [rank][row], of runs of chunks, where there are several
    const uint32_t down_bytes = s.RQ * 256, down = smem_u32(&down_s), used = smem_u32(&used_s);
    const uint32_t columns = s.RQ <= 32 ? 32 : s.RQ <= 64 ? 64 : 128;
    // What is read here is older than the kernel in front of this one, which has waited for all before itself; its result comes after the wait.
    const float *x = a.in + (size_t)n * s.CB * a.HW * 32 + (size_t)p0 * 32;
    const int id = a.adapter[n];
    const bool some = id >= 0 && id < a.adapters;
    const char *halves = reinterpret_cast<const char *>(a.packed + s.down_halves_at + (some ? id : 0) * s.down_halves);
    auto load_down = [&](int k) {
        if (elect_one()) {
            mbar_expect_tx(down, down_bytes);
            bulk_load(smem_u32(down_chunk), halves + (size_t)k * down_bytes, down_bytes, down);
        }
        __syncwarp();
    };
    if (warp == 0) {
        if (elect_one()) {
            gave_up = 0;
            mbar_init(down, 1);
            mbar_init(used, 1);
            mbar_fence_init();
        }
        __syncwarp();
        if (some) {
            tmem_alloc(smem_u32(&tmem_s), columns);
            load_down(0);
        } else {                                         // a block that could still ask for tensor memory keeps the next one off its SM
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    // the largest value of each pixel: eight lanes take a pixel's 128 bytes, a thread four pixels
    const int r0 = threadIdx.x >> 3, c0 = (threadIdx.x & 7) * 4;
    float most[kTile / 32] = {};
#pragma unroll 1
    for (int cb = 0; cb < s.CB; cb += 2) {
        float4 v[2][kTile / 32];
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < kTile / 32; ++i)
                v[g][i] = r0 + i * 32 < pixels && cb + g < s.CB ? __ldg(reinterpret_cast<const float4 *>(x + ((size_t)(cb + g) * a.HW + r0 + i * 32) * 32 + c0)) : make_float4(0.f, 0.f, 0.f, 0.f);
        if ((cb + 2) * 32 > s.C)                         // pad lanes, whatever lies there, here and below
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < kTile / 32; ++i) v[g][i] = clear_from(v[g][i], s.C - (cb + g) * 32 - c0);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < kTile / 32; ++i) most[i] = fmaxf(most[i], magnitude(v[g][i]));
    }
#pragma unroll
    for (int i = 0; i < kTile / 32; ++i)
#pragma unroll
        for (int o = 1; o < 8; o *= 2) most[i] = fmaxf(most[i], __shfl_xor_sync(~0u, most[i], o));
    __syncthreads();                                     // (tensor memory is allocated)
    grid_dep_sync();                                     // the filters' exponent
    grid_dep_trigger();
    const float *info = a.packed + s.info_at + 4 * (size_t)(some ? id : 0);
    const float by = some && a.scale ? a.scale[id] : 1.0f, sums = info[2] * magnitude(by);
    const int ew = exponents(c)[0], eu = __float_as_int(info[0]), ed = __float_as_int(info[1]);
    float up[kTile / 32];
    int shrunk = 0;                                      // by how much a pixel's scale is smaller for t's sake
#pragma unroll
    for (int i = 0; i < kTile / 32; ++i) {
        int ex = top_exponent(most[i]);
        if (some) {
            const int room = min(max(ex, top_exponent(most[i] * sums) + eu - ew), 254);
            shrunk = max(shrunk, room - ex);
            ex = room;
        }
        up[i] = lift(ex);
        if (c0 == 0) {
            ex_s[r0 + i * 32] = ex;
            full_s[r0 + i * 32] = top_exponent(most[i]);
            exponents(c)[4 + (size_t)blockIdx.x * kTile + r0 + i * 32] = ex;
        }
    }
    // t is taken from the halves that are written - unless so little is left of them (an adapter far larger than the filters) that t would suffer:
    // then from halves of their own, at the pixels' full scale, in a pass in front.
    const bool apart = __syncthreads_or(shrunk > 8);
    const int steps = apart ? 2 * s.chunks : s.chunks;
    char *out = ws_of(c) + (size_t)blockIdx.x * s.chunks * kPixelBytes;
    const uint32_t tmem = tmem_s, desc = f16_desc(s.RQ);
    for (int step = 0, k = 0; step < steps; ++step, k = k == s.chunks - 1 ? 0 : k + 1) {
        const bool multiply = some && step < s.chunks, keep = step >= steps - s.chunks;
        if (multiply && step && step % kDownRun == 0) {  // a run's products join the sums, as in adapter_product_kernel
            if (warp == 0) mbar_wait_uniform(used, step - 1 & 1, &gave_up, c.status, c.limit);
            __syncthreads();
            tc_fence_after();
            for (int rb = warp >> 2; rb < s.RB; rb += 2) {
                float v[32];
                tmem_ld32(tmem + rb * 32 + ((uint32_t)(warp & 3) << 21), v);
                float *t = t_sums + rb * 32 * kTile + (warp & 3) * 32 + lane;
#pragma unroll
                for (int u = 0; u < 32; ++u)
                    if (rb * 32 + u < s.RQ) t[u * kTile] = step == kDownRun ? v[u] : t[u * kTile] + v[u];
            }
            tc_fence_before();
        }
        float4 v2[2][kTile / 32];                        // on its way while the chunk before is written out and multiplied
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < kTile / 32; ++i)
                v2[g][i] = r0 + i * 32 < pixels && k * 2 + g < s.CB ? __ldg(reinterpret_cast<const float4 *>(x + ((size_t)(k * 2 + g) * a.HW + r0 + i * 32) * 32 + c0)) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (step) {
            if (warp == 0) {
                bulk_store_wait<0>();
                if (some && step <= s.chunks) mbar_wait_uniform(used, step - 1 & 1, &gave_up, c.status, c.limit);
                if (multiply) load_down(k);
            }
            __syncthreads();
        }
        if ((k * 2 + 2) * 32 > s.C)
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < kTile / 32; ++i) v2[g][i] = clear_from(v2[g][i], s.C - (k * 2 + g) * 32 - c0);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < kTile / 32; ++i) store4<kChunk>(chunk, r0 + i * 32, g * 32 + c0, v2[g][i], keep ? up[i] : lift(top_exponent(most[i])));
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        if (warp == 0) {
            if (multiply) mbar_wait_uniform(down, k & 1, &gave_up, c.status, c.limit);
            tc_fence_after();
            if (elect_one()) {
                if (keep) bulk_store(out + (size_t)k * kPixelBytes, smem_u32(chunk), kPixelBytes);
                if (multiply) {
                    const uint32_t xa = smem_desc_lo(smem_u32(chunk)), wa = smem_desc_lo(smem_u32(down_chunk));
                    for (int term = 0; term < 3; ++term)             // small terms first
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            mma_f16(tmem, xa + e * 2 + (term == 0 ? kPixelBytes / 32 : 0), wa + e * 2 + (term == 1 ? s.RQ * 8 : 0), desc, k % kDownRun > 0 || e > 0 || term > 0);
                    mma_commit(used);
                }
            }
            __syncwarp();
        }
    }
    if (some) {
        mbar_wait_uniform(used, s.chunks - 1 & 1, &gave_up, c.status, c.limit);
        tc_fence_after();
        const int row = (warp & 3) * 32 + lane, ex = ex_s[row];
        const int et = ex + ew - eu;                     // t * lift(et) beside halves of Up meets the pixel's scale beside halves of the filters
        const float x_drop = drop(apart ? full_s[row] : ex);
        const float factor = et <= 254 ? by * drop(ed) : 0.0f, up_t = lift(min(max(et, 15), 254));       // (beyond: 2^-100 of the sum and less, nothing)
        for (int rb = warp >> 2; rb < s.RB; rb += 2) {   // a thread a pixel and 32 ranks
            char *to = ws_of(c) + c.at.ranks_at + ((size_t)blockIdx.x * s.RB + rb) * kRankBytes;
            float v[32];
            tmem_ld32(tmem + rb * 32 + ((uint32_t)(warp & 3) << 21), v);
            if (s.chunks > kDownRun)
#pragma unroll
                for (int u = 0; u < 32; ++u)
                    if (rb * 32 + u < s.RQ) v[u] += t_sums[(rb * 32 + u) * kTile + row];
#pragma unroll
            for (int u = 0; u < 32; u += 4) {
                // columns behind RQ have no product in them
                const bool real = rb * 32 + u < s.RQ && row < pixels;
                const float4 t = real ? make_float4(v[u] * x_drop * factor, v[u + 1] * x_drop * factor, v[u + 2] * x_drop * factor, v[u + 3] * x_drop * factor)
                                      : make_float4(0.f, 0.f, 0.f, 0.f);
                store4<32>(to, row, u, t, up_t);
            }
        }
    }
    if (warp == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    if (!some) return;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) {
        if (gave_up) {                                   // what is still on its way must land before the block ends
            mbar_wait(down, s.chunks - 1 & 1, kDefaultWaitIters);
            mbar_wait(used, s.chunks - 1 & 1, kDefaultWaitIters);
        }
        tmem_dealloc(tmem, columns);
    }
}

// The tensor core cuts its accumulator off at 24 bits at each step, on the average by 0.36 * 2^-23 of what stands there: what a result loses that way
// grows with the steps of a sum and is lost on one side.  So an accumulator takes a run of chunks, and the epilogue adds the runs' products in FP32
// registers, where sums are rounded; sums that lose nothing stay exact.
template <bool kX3> constexpr int kRun = kX3 ? 2 : 8;        // chunks

constexpr int kStages = 2, kStageBytes = kPixelBytes + kFilterTile * 32 * 256, kProductThreads = 320;

template <bool kX3>
__global__ void __launch_bounds__(kProductThreads, 1) adapter_product_kernel(const TcArgs c) {
    extern __shared__ char raw[];
    __shared__ uint64_t full_s[kStages * 2], empty_s[kStages],        // a stage: what the first term takes, the rest
                         done_s[2], free_s[2], drained;
    __shared__ uint32_t tmem_s;
    __shared__ int gave_up;
    const AdaptArgs &a = c.a;
    const AdapterShape &s = c.s;
    const int warp = warp_index();
    char *stages = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t full = smem_u32(full_s), empty = smem_u32(empty_s), done = smem_u32(done_s), free = smem_u32(free_s);
    if (warp == 9) tmem_alloc(smem_u32(&tmem_s), 512);
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int i = 0; i < kStages; ++i) { mbar_init(full + i * 16, 1); mbar_init(full + i * 16 + 8, 1); mbar_init(empty + i * 8, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(done + i * 8, 1); mbar_init(free + i * 8, 256); }
        mbar_init(smem_u32(&drained), 1);
        mbar_fence_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dep_sync();
    grid_dep_trigger();
    const uint32_t tmem = tmem_s;
    volatile int *stop = &gave_up;
    const int pixel_tiles = a.N * c.at.tiles, work = pixel_tiles * c.at.filter_tiles;
    auto ranks_of = [&](int np) {                        // rank blocks of a pixel tile
        const int id = a.adapter[np / c.at.tiles];
        return id >= 0 && id < a.adapters ? s.RB : 0;
    };
    int issued = 0;                                      // stages, by warp 8
    if (warp == 8) {
        int slot = 0, phase = 1;
        bool ok = true;
        for (int i = blockIdx.x; i < work && ok; i += gridDim.x) {
            const int np = i / c.at.filter_tiles, kt = i % c.at.filter_tiles, rows = tile_rows(c, kt), ranks = ranks_of(np);
            const int id = ranks ? a.adapter[np / c.at.tiles] : 0;
            const char *x = ws_of(c) + (size_t)np * c.s.chunks * kPixelBytes, *t = ws_of(c) + c.at.ranks_at + (size_t)np * s.RB * kRankBytes;
            const char *w = ws_of(c) + c.at.filters_at + (size_t)kt * c.s.chunks * kFilterTile * 32 * 256;
            const char *u = reinterpret_cast<const char *>(a.packed + s.up_halves_at + id * s.up_halves) + (size_t)kt * s.RB * kFilterTile * 32 * 128;
            for (int k = 0; k < c.s.chunks + ranks; ++k) {
                if (issued >= kStages && !(ok = mbar_wait_uniform(empty + slot * 8, phase, stop, c.status, c.limit))) break;
                const int rb = k - c.s.chunks;
                if (elect_one()) {
                    const uint32_t to = smem_u32(stages + slot * kStageBytes), bar = full + slot * 16;
                    auto load = [&](uint32_t at, const char *from, uint32_t bytes, uint32_t b) {
                        for (uint32_t e = 0; e < bytes; e += 8192) bulk_load(to + at + e, from + e, min(8192u, bytes - e), b);
                    };
                    if (rb >= 0) {                       // 32 ranks have both parts in a row
                        mbar_expect_tx(bar, kRankBytes + rows * 128);
                        load(0, t + (size_t)rb * kRankBytes, kRankBytes, bar);
                        load(kPixelBytes, u + (size_t)rb * rows * 128, rows * 128, bar);
                        if (kX3) mbar_arrive(bar + 8);
                    } else {                             // high parts lie in front; the terms begin with low pixels and high filters
                        const char *fx = x + (size_t)k * kPixelBytes, *fw = w + (size_t)k * rows * 256;
                        const uint32_t half = kPixelBytes / 2;
                        mbar_expect_tx(bar, half + rows * 128);
                        load(kX3 ? half : 0, kX3 ? fx + half : fx, half, bar);
                        load(kPixelBytes, fw, rows * 128, bar);
                        if (kX3) {
                            mbar_expect_tx(bar + 8, half + rows * 128);
                            load(0, fx, half, bar + 8);
                            load(kPixelBytes + rows * 128, fw + rows * 128, rows * 128, bar + 8);
                        }
                    }
                }
                __syncwarp();
                ++issued;
                if (++slot == kStages) { slot = 0; phase ^= 1; }
            }
        }
    } else if (warp == 9) {
        const uint32_t first = smem_desc_lo(smem_u32(stages));
        int slot = 0, phase = 0, buffer = 0, buffer_phase = 1, turn = 0;
        bool ok = true;
        for (int i = blockIdx.x; i < work && ok; i += gridDim.x) {
            const int np = i / c.at.filter_tiles, rows = tile_rows(c, i % c.at.filter_tiles), ranks = ranks_of(np);
            const uint32_t desc = f16_desc(rows);
            for (int k = 0, in_run = 0; k < c.s.chunks + ranks; ++k) {
                if (in_run == 0 && turn >= 2 && !(ok = mbar_wait_uniform(free + buffer * 8, buffer_phase, stop, c.status, c.limit))) break;
                const uint32_t d = tmem + buffer * 256;
                const uint32_t x = first + slot * (kStageBytes >> 4), w = x + (kPixelBytes >> 4);
                if (!(ok = mbar_wait_uniform(full + slot * 16, phase, stop, c.status, c.limit))) break;
                tc_fence_after();
                if (kX3) {                               // small terms first: low pixels and high filters while the rest is on its way
                    if (k < c.s.chunks && elect_one())
#pragma unroll
                        for (int e = 0; e < 4; ++e) mma_f16(d, x + e * 2 + kPixelBytes / 32, w + e * 2, desc, in_run > 0 || e > 0);
                    __syncwarp();
                    if (!(ok = mbar_wait_uniform(full + slot * 16 + 8, phase, stop, c.status, c.limit))) break;
                    tc_fence_after();
                }
                // the ranks' steps belong to the last run of channels
                const bool last = k == c.s.chunks + ranks - 1 || (in_run == kRun<kX3> - 1 && k < c.s.chunks - 1);
                if (elect_one()) {
                    if (k < c.s.chunks) {
#pragma unroll
                        for (int term = kX3 ? 1 : 2; term < 3; ++term)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                mma_f16(d, x + e * 2, w + e * 2 + (term == 1 ? rows * 8 : 0), desc, kX3 || in_run > 0 || e > 0);
                    } else {
                        const int steps = (min(s.R - (k - c.s.chunks) * 32, 32) + 15) / 16;
#pragma unroll
                        for (int term = kX3 ? 0 : 2; term < 3; ++term)
                            for (int e = 0; e < steps; ++e) mma_f16(d, x + e * 2 + (term == 0 ? 4 : 0), w + e * 2 + (term == 1 ? 4 : 0), desc, 1);
                    }
                    mma_commit(empty + slot * 8);
                    if (last) mma_commit(done + buffer * 8);
                }
                __syncwarp();
                if (++slot == kStages) { slot = 0; phase ^= 1; }
                ++in_run;
                if (last) {
                    in_run = 0;
                    ++turn;
                    if (++buffer == 2) { buffer = 0; buffer_phase ^= 1; }
                }
            }
        }
        if (!ok) {
            if (elect_one()) mma_commit(smem_u32(&drained));
            __syncwarp();
            mbar_wait(smem_u32(&drained), 0, kDefaultWaitIters);
        }
    } else {
        const int lane = threadIdx.x & 31, half = warp >> 2;
        const int w_exponent = exponents(c)[0];
        float4 *rows = reinterpret_cast<float4 *>(stages + kStages * kStageBytes) + warp * 256;
        int buffer = 0, phase = 0;
        for (int i = blockIdx.x; i < work; i += gridDim.x) {
            const int np = i / c.at.filter_tiles, kt = i % c.at.filter_tiles, n = np / c.at.tiles, p0 = np % c.at.tiles * kTile + (warp & 3) * 32;
            // undoes both operands' scaling: the pixel's and the filters' parts may each pass FP32's range where the result does not
            const TwoFactors back(exponents(c)[4 + (size_t)np * kTile + (warp & 3) * 32 + lane] + w_exponent - 2 * 141);
            const int blocks = tile_rows(c, kt) / 32;
            float sum[kFilterTile / 2][32] = {};         // of this warp's blocks of filters
            bool given_up = false;
#pragma unroll 1
            for (int k = 0; k < c.s.chunks; k += kRun<kX3>) {
                if ((given_up = !mbar_wait_uniform(done + buffer * 8, phase, stop, c.status, c.limit))) break;
                tc_fence_after();
#pragma unroll
                for (int e = 0; e < kFilterTile / 2; ++e) {
                    if (half + e * 2 >= blocks) continue;
#pragma unroll
                    for (int g = 0; g < 32; g += 16) {
                        float v[16];
                        tmem_ld16(tmem + buffer * 256 + (half + e * 2) * 32 + g + ((uint32_t)(warp & 3) << 21), v);
#pragma unroll
                        for (int u = 0; u < 16; ++u) sum[e][g + u] += v[u];
                    }
                }
                tc_fence_before();
                mbar_arrive(free + buffer * 8);
                if (++buffer == 2) { buffer = 0; phase ^= 1; }
            }
            if (given_up) break;
#pragma unroll
            for (int e = 0; e < kFilterTile / 2; ++e) {
                const int b = half + e * 2;
                if (b >= blocks) continue;
                const float (&v)[32] = sum[e];
                // through shared memory, so that a store is whole lines: eight lanes a pixel
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    rows[lane * 8 + (u ^ (lane & 7))] = make_float4(v[u * 4] * back.a * back.b, v[u * 4 + 1] * back.a * back.b, v[u * 4 + 2] * back.a * back.b,
                                                                    v[u * 4 + 3] * back.a * back.b);
                __syncwarp();
                const int k0 = (kt * kFilterTile + b) * 32 + (lane & 7) * 4;
                float4 add = make_float4(0.f, 0.f, 0.f, 0.f);
                if (a.bias) {
                    if (k0 + 4 <= s.K) add = *reinterpret_cast<const float4 *>(a.bias + k0);
                    else add = make_float4(k0 < s.K ? a.bias[k0] : 0.0f, k0 + 1 < s.K ? a.bias[k0 + 1] : 0.0f, k0 + 2 < s.K ? a.bias[k0 + 2] : 0.0f, 0.0f);
                }
                float4 *out = reinterpret_cast<float4 *>(a.out) + (((size_t)n * s.KB + kt * kFilterTile + b) * a.HW + p0) * 8 + lane;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int r = u * 4 + (lane >> 3);
                    float4 y = rows[r * 8 + ((lane & 7) ^ (r & 7))];
                    y.x += add.x; y.y += add.y; y.z += add.z; y.w += add.w;
                    if (p0 + r >= a.HW) continue;
                    if (a.accumulate) {
                        const float4 before = out[u * 32];
                        y.x += before.x; y.y += before.y; y.z += before.z; y.w += before.w;
                    }
                    if (a.relu) y = make_float4(fmaxf(y.x, 0.0f), fmaxf(y.y, 0.0f), fmaxf(y.z, 0.0f), fmaxf(y.w, 0.0f));
                    if (k0 + 4 > s.K) y = make_float4(k0 < s.K ? y.x : 0.0f, k0 + 1 < s.K ? y.y : 0.0f, k0 + 2 < s.K ? y.z : 0.0f, 0.0f);       // +0 in pad lanes
                    __stcs(out + u * 32, y);             // operands are read again, results here not: they leave L2 first (131 -> 128 us)
                }
                __syncwarp();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (gave_up && warp == 8)                            // what is still on its way must land before the block ends
        for (int x = max(0, issued - kStages); x < issued; ++x)
            for (int y = 0; y < (kX3 ? 2 : 1); ++y) mbar_wait(full + x % kStages * 16 + y * 8, (x / kStages) & 1, kDefaultWaitIters);
    if (warp == 9) tmem_dealloc(tmem, 512);
}

// Up and Down as halves, a block an adapter each.
__global__ void __launch_bounds__(kThreads) pack_halves_kernel(const float *__restrict__ down, const float *__restrict__ up, float *__restrict__ packed, const AdapterShape s) {
    __shared__ float most_s[kThreads / 32], sum_s[kThreads / 32];
    grid_dep_sync();
    grid_dep_trigger();
    const int a = blockIdx.x, cols = blockIdx.y ? s.C : s.R;             // of a row: Up is [K][R], Down [R][C]
    const float *w = blockIdx.y ? down + (size_t)a * s.R * s.C : up + (size_t)a * s.K * s.R;
    float most = 0.0f, sums = 0.0f;
    for (size_t i = threadIdx.x; i < (size_t)(blockIdx.y ? s.C : s.K) * s.R; i += kThreads) most = fmaxf(most, magnitude(w[i]));
    const int ex = top_exponent(block_max(most, most_s));
    const float by = lift(ex);
    if (blockIdx.y) {
        for (int r = threadIdx.x >> 5; r < s.R; r += kThreads / 32) {    // a warp a row
            float sum = 0.0f;
            for (int ch = threadIdx.x & 31; ch < s.C; ch += 32) sum += magnitude(w[(size_t)r * s.C + ch]);
#pragma unroll
            for (int o = 16; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
            sums = fmaxf(sums, sum);
        }
        sums = block_max(sums, sum_s);
    }
    if (threadIdx.x == 0) {
        float *info = packed + s.info_at + 4 * (size_t)a;
        info[blockIdx.y] = __int_as_float(ex);
        if (blockIdx.y) info[2] = sums;
    }
    char *out = reinterpret_cast<char *>(blockIdx.y ? packed + s.down_halves_at + a * s.down_halves : packed + s.up_halves_at + a * s.up_halves);
    // four columns at a time; a row of 128 bytes holds 64 channels' high (or low) halves, or both of 32 ranks
    const int wide = blockIdx.y ? 64 : 32, runs = blockIdx.y ? s.chunks : s.RB, all = blockIdx.y ? s.RQ : s.KB * 32;
    for (size_t i = threadIdx.x; i < (size_t)all * runs * (wide / 4); i += kThreads) {
        const int e = (int)(i % (wide / 4)) * 4, run = (int)(i / (wide / 4) % runs), r = (int)(i / (wide / 4) / runs);
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = r < (blockIdx.y ? s.R : s.K) && run * wide + e + u < cols ? w[(size_t)r * cols + run * wide + e + u] * by : 0.0f;
        uint2 hi, lo;
        split_finite(v[0], v[1], hi.x, lo.x);
        split_finite(v[2], v[3], hi.y, lo.y);
        const int kt = blockIdx.y ? 0 : r / (kFilterTile * 32), row = blockIdx.y ? r : r % (kFilterTile * 32);
        const int rows = blockIdx.y ? s.RQ : min(kFilterTile, s.KB - kt * kFilterTile) * 32;
        char *to = blockIdx.y ? out + (size_t)run * rows * 256 : out + ((size_t)kt * s.RB * kFilterTile * 32 + (size_t)run * rows) * 128;
        *reinterpret_cast<uint2 *>(to + chunk_at(row, e, rows) + (e & 4) * 2) = hi;
        *reinterpret_cast<uint2 *>(to + chunk_at(row, wide + e, rows) + (e & 4) * 2) = lo;
    }
}

}  // namespace

// The other form writes the result twice and takes the adapter's products in FP32, which costs the more the larger the rank; this one lays the
// pixels out first.  us, here / there, rank 8 and 32, batch 64 unless said: 256 -> 768 on 28 x 28 110 / 209 and 114 / 338; 256 -> 256 74 / 92 and 74 /
// 173; 128 -> 128 37 / 38 and 38 / 78; 64 -> 64 27 / 24 and 27 / 47; 256 -> 256 on 14 x 14 30 / 33 and 30 / 61; 512 -> 128 on 28 x 28 119 / 104 and 119 /
// 236; batch 128, 512 -> 512 on 14 x 14 94 / 136 and 95 / 224, on 8 x 8 56 / 46 and 57 / 82; batch 4, 320 -> 960 on 32 x 32 40 / 35 and 40 / 61.  Few
// channels, ranks 16 and 32: batch 95, 11 -> 52 on 11 x 19 20.2 / 14.4 and 20.4 / 20.5, batch 41, 41 -> 17 on 32 x 8 15.3 / 10.2 and 15.4 / 14.1.  Few
// tiles, many operations: batch 31, 390 -> 135, rank 31 on 11 x 20 35.4 / 58.6.
bool adapted_tc_preferred(int N, int C, int K, int HW, int R, int sms) {
    const long long tiles = (long long)N * ceil_div(HW, kTile) * ceil_div(blocks_of(K), kFilterTile);
    if (HW < 64 || tiles >= (1 << 28)) return false;
    if (R <= 8) return K > 128 && tiles >= 2 * sms;
    const int blocks = blocks_of(C) + blocks_of(K);
    const double apart = (double)N * HW * blocks * 32 * ceil_div(R, 8) * 8;          // the adapter's multiply-adds in FP32
    return tiles >= sms / 2 ? blocks > 4 || apart >= 40e6 : tiles >= sms / 4 && apart >= 100e6;
}

size_t adapted_tc_workspace(int N, int C, int K, int HW, int R) { return Layout(N, C, K, HW, R).bytes; }

int launch_pack_halves(small_ctx *ctx, const float *down, const float *up, float *packed, int adapters, const AdapterShape &s, cudaStream_t st) {
    launch_kernel(ctx, pack_halves_kernel, dim3((unsigned)adapters, 2), dim3(kThreads), 0, st, down, up, packed, s);
    return check_launch(ctx);
}

int launch_adapted_tc(small_ctx *ctx, const AdaptArgs &a, const AdapterShape &s, bool x3, cudaStream_t st) {
    const TcArgs c{a, s, Layout(a.N, s.C, s.K, a.HW, s.R), ctx->dev_status, ctx->wait_iters};
    launch_clusters(ctx, adapter_filters_kernel, dim3(kCluster), dim3(kThreads * kTeams), kCluster, 0, st, c);
    if (int e = check_launch(ctx)) return e;
    static std::atomic<unsigned long long> pixels{0}, exact{0}, fast{0};
    const size_t passing = 1024 + (size_t)kPixelBytes + (size_t)s.RQ * (256 + (s.chunks > kDownRun ? kTile * sizeof(float) : 0)), stages = 1024 + (size_t)kStages * kStageBytes + 8 * 4096;
    if (int e = allow_shared_memory(ctx, adapter_pixels_kernel, pixels, 1024 + kPixelBytes + 128 * (256 + kTile * sizeof(float)))) return e;
    launch_kernel(ctx, adapter_pixels_kernel, dim3((unsigned)(a.N * c.at.tiles)), dim3(kThreads), passing, st, c);
    if (int e = check_launch(ctx)) return e;
    const int work = a.N * c.at.tiles * c.at.filter_tiles;
    const dim3 grid((unsigned)(work < ctx->sm_count ? work : ctx->sm_count));
    if (x3) {
        if (int e = allow_shared_memory(ctx, adapter_product_kernel<true>, exact, stages)) return e;
        launch_kernel(ctx, adapter_product_kernel<true>, grid, dim3(kProductThreads), stages, st, c);
    } else {
        if (int e = allow_shared_memory(ctx, adapter_product_kernel<false>, fast, stages)) return e;
        launch_kernel(ctx, adapter_product_kernel<false>, grid, dim3(kProductThreads), stages, st, c);
    }
    return check_launch(ctx);
}

}  // namespace small
