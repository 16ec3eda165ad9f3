// 1 x 1 convolution with an adapter for each image as one product on the tensor cores (tcgen05, kind::f16): the products t = Down_a x stand
// behind an image's channels, and s_a Up_a behind the filters, so that the adapter costs some more steps of the reduction and the result is
// written once.  Operands are pairs of halves (halves.cuh).
//
// adapter_filters_kernel: the filters as halves, 64 channels a chunk, each filter brought to the same size by a power of two.
// adapter_pixels_kernel: 128 pixels of an image a block: each one's largest value in one pass over them (from memory), halves in a second (from
//   L2), which pass through shared memory, where the product with Down is taken from them.  t becomes halves by pixel, too.
// adapter_product_kernel: a block walks tiles of 128 pixels x 256 filters; warps for loading (plain bulk copies, two stages of 96 KB), MMAs
//   and the epilogue (scales, sums, bias, previous output, ReLU), two accumulators in tensor memory so that the epilogue of a run runs beside the
//   next.  t times Up is a run of its own, because rows of Up are brought to one size whatever the filters' is.
//   256 filters a tile: 96 KB of operands for 1536 cycles of MMAs (62 bytes a cycle and SM from L2).
//
// Batch 64, 256 -> 768, 28 x 28, rank 16: 134 us.  Pixels 36 (the filters, 5, beside them): the largest values, while memory still takes the result
// before, then four chunks that wait for their loads.  Product 83: MMAs half of the time; what a stage takes to load, and the epilogue's sums, scales
// and stores, fill the rest.  With an accumulator for all of a tile's steps 72, see kRun; of 168 registers a thread for all roles 94, as the epilogue's sums spill.
// Floor 33 for the bytes, 37 for three products.
#include "adapter.cuh"
#include "halves.cuh"

namespace small {
namespace {
using namespace halves;

constexpr int kThreads = 256;
constexpr int kChunk = 64;               // channels
constexpr int kDownRun = 4;              // chunks whose products with Down one accumulator takes (see kRun)
constexpr uint32_t kPixelBytes = kTile * 256, kRankBytes = kTile * 128;          // of a chunk of channels, of 32 ranks
constexpr int kTeams = 4, kKept = 4;     // teams of 256 threads of adapter_filters_kernel, channel blocks of a team in registers

struct Layout {
    int tiles, filter_tiles;             // pixel tiles of an image
    size_t ranks_at, filters_at, scales_at, bytes;
    Layout(int N, int C, int K, int HW, int R)
        : tiles(ceil_div(HW, kTile)), filter_tiles(ceil_div(blocks_of(K), kFilterTile)) {
        const int chunks = ceil_div(C, kChunk);
        ranks_at = (size_t)N * tiles * chunks * kPixelBytes;
        filters_at = ranks_at + (size_t)N * tiles * blocks_of(R) * kRankBytes;
        scales_at = filters_at + (size_t)chunks * blocks_of(K) * 32 * 256;
        bytes = scales_at + sizeof(float) * (size_t)blocks_of(K) * 32 + sizeof(int2) * (size_t)N * tiles * kTile;
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
// What undoes the scaling: each filter's factor; the exponents of each pixel's x (+ 141) and t.
__device__ __forceinline__ float *filter_factors(const TcArgs &c) { return reinterpret_cast<float *>(ws_of(c) + c.at.scales_at); }
__device__ __forceinline__ int2 *pixel_exponents(const TcArgs &c) { return reinterpret_cast<int2 *>(filter_factors(c) + c.s.KB * 32); }
// Of an adapter's packed scales: the first word, Down's exponent; Up's factors from the fifth on.
template <typename T> __device__ __forceinline__ T *info_of(T *packed, const AdapterShape &s, int id) { return packed + s.info_at + id * s.info; }
__device__ __forceinline__ int tile_rows(const TcArgs &c, int kt) { return min(kFilterTile, c.s.KB - kt * kFilterTile) * 32; }
// The FP32 section of the packed filters, [KB][CB][32 channels][32 filters], as halves [filter tile][chunk]{high: rows x 128 bytes, low: the same}, a
// block 32 filters: each one's largest value, then its halves.
__global__ void __launch_bounds__(kThreads *kTeams) adapter_filters_kernel(const TcArgs c) {
    __shared__ float most_s[kThreads * kTeams / 32][32], blocks[kTeams][32][33];
    __shared__ int ex_s[32];
    grid_dep_sync();
    grid_dep_trigger();
    const int items = c.s.chunks * 2, tid = threadIdx.x % kThreads, team = threadIdx.x / kThreads, lane = threadIdx.x & 31, kb = blockIdx.x, kt = kb / kFilterTile;
    const int rows = tile_rows(c, kt);
    const float4 *w = reinterpret_cast<const float4 *>(c.a.w) + (size_t)kb * c.s.CB * 256 + tid;
    auto fetch = [&](int cb) { return cb < c.s.CB ? __ldg(w + (size_t)cb * 256) : make_float4(0.f, 0.f, 0.f, 0.f); };
    float4 most = make_float4(0.f, 0.f, 0.f, 0.f);       // of filters (tid & 7) * 4 and the next three
    auto count = [&](const float4 &v) {
        most = make_float4(fmaxf(most.x, magnitude(v.x)), fmaxf(most.y, magnitude(v.y)), fmaxf(most.z, magnitude(v.z)), fmaxf(most.w, magnitude(v.w)));
    };
    float4 kept[kKept];                                  // the first ones stay in registers
#pragma unroll
    for (int e = 0; e < kKept; ++e) kept[e] = fetch(team + e * kTeams);
#pragma unroll
    for (int e = 0; e < kKept; ++e) count(kept[e]);
    for (int i = team + kKept * kTeams; i < items; i += 4 * kTeams) {
        float4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fetch(i + e * kTeams);
#pragma unroll
        for (int e = 0; e < 4; ++e) count(v[e]);
    }
#pragma unroll
    for (int o = 8; o < 32; o *= 2) {
        most.x = fmaxf(most.x, __shfl_xor_sync(~0u, most.x, o)); most.y = fmaxf(most.y, __shfl_xor_sync(~0u, most.y, o));
        most.z = fmaxf(most.z, __shfl_xor_sync(~0u, most.z, o)); most.w = fmaxf(most.w, __shfl_xor_sync(~0u, most.w, o));
    }
    if (lane < 8) *reinterpret_cast<float4 *>(&most_s[threadIdx.x >> 5][lane * 4]) = most;
    __syncthreads();
    if (threadIdx.x < 32) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < kThreads * kTeams / 32; ++i) m = fmaxf(m, most_s[i][lane]);
        ex_s[lane] = top_exponent(m);
        filter_factors(c)[kb * 32 + lane] = drop(ex_s[lane]);
    }
    __syncthreads();
    // a thread's four channels of filter f
    const int f = tid >> 3, c0 = (tid & 7) * 4, row = kb % kFilterTile * 32 + f;
    const float up = lift(ex_s[f]);
    const bool real = kb * 32 + f < c.s.K;
    char *out = ws_of(c) + c.at.filters_at + (size_t)kt * c.s.chunks * kFilterTile * 32 * 256;
    float (*block)[33] = blocks[team];
    auto lay_out = [&](int cb, const float4 &v, auto ahead) {
        __syncthreads();
        const int ch = tid >> 3, f0 = (tid & 7) * 4;
        block[f0][ch] = v.x; block[f0 + 1][ch] = v.y; block[f0 + 2][ch] = v.z; block[f0 + 3][ch] = v.w;
        ahead();
        __syncthreads();
        if (cb >= items) return;
        const int col = (cb & 1) * 32 + c0;
        uint2 hi, lo;
        split_finite(real ? block[f][c0] * up : 0.0f, real ? block[f][c0 + 1] * up : 0.0f, hi.x, lo.x);
        split_finite(real ? block[f][c0 + 2] * up : 0.0f, real ? block[f][c0 + 3] * up : 0.0f, hi.y, lo.y);
        char *to = out + (size_t)(cb >> 1) * rows * 256;
        *reinterpret_cast<uint2 *>(to + chunk_at(row, col, rows) + (col & 4) * 2) = hi;
        *reinterpret_cast<uint2 *>(to + chunk_at(row, kChunk + col, rows) + (col & 4) * 2) = lo;
    };
#pragma unroll
    for (int e = 0; e < kKept; ++e)
        if (e * kTeams < items) lay_out(team + e * kTeams, kept[e], [] {});
    float4 v = fetch(team + kKept * kTeams);
    for (int i0 = kKept * kTeams; i0 < items; i0 += kTeams) {
        const float4 now = v;
        lay_out(i0 + team, now, [&] { v = fetch(i0 + team + kTeams); });
    }
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
    __shared__ int ex_s[kTile];                          // the pixels' exponents
    __shared__ float t_most_s[2][kTile];
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
    grid_dep_sync();                                     // what follows is written where an earlier call may still read
    grid_dep_trigger();
    float up[kTile / 32];
#pragma unroll
    for (int i = 0; i < kTile / 32; ++i) {
        const int ex = top_exponent(most[i]);
        up[i] = lift(ex);
        if (c0 == 0) {
            ex_s[r0 + i * 32] = ex;
            pixel_exponents(c)[(size_t)blockIdx.x * kTile + r0 + i * 32].x = ex;
        }
    }
    char *out = ws_of(c) + (size_t)blockIdx.x * s.chunks * kPixelBytes;
    const uint32_t tmem = tmem_s, desc = f16_desc(s.RQ);
    for (int k = 0; k < s.chunks; ++k) {
        if (some && k && k % kDownRun == 0) {            // a run's products join the sums, as in adapter_product_kernel
            if (warp == 0) mbar_wait_uniform(used, k - 1 & 1, &gave_up, c.status, c.limit);
            __syncthreads();
            tc_fence_after();
            for (int rb = warp >> 2; rb < s.RB; rb += 2) {
                float v[32];
                tmem_ld32(tmem + rb * 32 + ((uint32_t)(warp & 3) << 21), v);
                float *t = t_sums + rb * 32 * kTile + (warp & 3) * 32 + lane;
#pragma unroll
                for (int u = 0; u < 32; ++u)
                    if (rb * 32 + u < s.RQ) t[u * kTile] = k == kDownRun ? v[u] : t[u * kTile] + v[u];
            }
            tc_fence_before();
        }
        float4 v2[2][kTile / 32];                        // on its way while the chunk before is written out and multiplied
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < kTile / 32; ++i)
                v2[g][i] = r0 + i * 32 < pixels && k * 2 + g < s.CB ? __ldg(reinterpret_cast<const float4 *>(x + ((size_t)(k * 2 + g) * a.HW + r0 + i * 32) * 32 + c0)) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (k) {
            if (warp == 0) {
                bulk_store_wait<0>();
                if (some) {
                    mbar_wait_uniform(used, k - 1 & 1, &gave_up, c.status, c.limit);
                    load_down(k);
                }
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
            for (int i = 0; i < kTile / 32; ++i) store4<kChunk>(chunk, r0 + i * 32, g * 32 + c0, v2[g][i], up[i]);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        if (warp == 0) {
            if (some) mbar_wait_uniform(down, k & 1, &gave_up, c.status, c.limit);
            tc_fence_after();
            if (elect_one()) {
                bulk_store(out + (size_t)k * kPixelBytes, smem_u32(chunk), kPixelBytes);
                if (some) {
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
        // a thread a pixel and 16 of each 32 ranks: the pixel's largest t, then halves of them
        const int row = (warp & 3) * 32 + lane, half = warp >> 2;
        float by = a.scale ? a.scale[id] : 1.0f;
        int far = 0;                                     // exponent of a scale that is taken in parts
        if (fabsf(by) < 0x1p-60f) { by *= 0x1p100f; far = -100; }
        if (fabsf(by) > 0x1p60f && fabsf(by) < INFINITY) { by *= 0x1p-100f; far = 100; }
        auto ranks = [&](int rb, float (&t)[16]) {
            tmem_ld16(tmem + rb * 32 + half * 16 + ((uint32_t)(warp & 3) << 21), t);
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                const int r = rb * 32 + half * 16 + u;
                if (s.chunks > kDownRun && r < s.RQ) t[u] += t_sums[r * kTile + row];
                t[u] = r < s.RQ && row < pixels ? t[u] * by : 0.0f;              // (columns behind RQ have no product in them)
            }
        };
        float most_t = 0.0f;
        for (int rb = 0; rb < s.RB; ++rb) {
            float t[16];
            ranks(rb, t);
#pragma unroll
            for (int u = 0; u < 16; ++u) most_t = fmaxf(most_t, magnitude(t[u]));
        }
        t_most_s[half][row] = most_t;
        __syncthreads();
        const int et = top_exponent(fmaxf(most_t, t_most_s[half ^ 1][row]));
        const float up_t = lift(et);
        if (half == 0)
            pixel_exponents(c)[(size_t)blockIdx.x * kTile + row].y = et + ex_s[row] + __float_as_int(*info_of(a.packed, s, id)) - 3 * 141 + far;
        for (int rb = 0; rb < s.RB; ++rb) {
            char *to = ws_of(c) + c.at.ranks_at + ((size_t)blockIdx.x * s.RB + rb) * kRankBytes;
            float t[16];
            ranks(rb, t);
#pragma unroll
            for (int u = 0; u < 16; u += 4) store4<32>(to, row, half * 16 + u, make_float4(t[u], t[u + 1], t[u + 2], t[u + 3]), up_t);
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
// registers, where sums are rounded; sums that lose nothing stay exact.  (Four chunks in 3xTF32: 131 us for 134, errors of 256 channels 1.1e-6 for 5e-7.)
template <bool kX3> constexpr int kRun = kX3 ? 2 : 8;        // chunks

constexpr int kPassing = 4096;           // bytes of shared memory that a warp's results pass through
constexpr int kStages = 2, kStageBytes = kPixelBytes + kFilterTile * 32 * 256, kEpilogueWarps = 8, kProductThreads = kEpilogueWarps * 32 + 128;
constexpr int kRolesRegs = 56, kEpilogueRegs = 224;     // a thread, of the 168 that each is launched with
static_assert(kRolesRegs * 128 + kEpilogueRegs * kEpilogueWarps * 32 <= 168 * kProductThreads, "more than the launch brings is waited for without an end");

// mbar_wait_uniform without a call: a kernel that deals out its registers by role must not have any.
__device__ __forceinline__ bool wait_here(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *status, uint32_t limit) {
    return __all_sync(0xffffffffu, mbar_wait<64>(bar, parity, abort_flag, status, limit));
}

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
    constexpr int kLoader = kEpilogueWarps, kIssuer = kLoader + 1;
    if (warp == kIssuer) tmem_alloc(smem_u32(&tmem_s), 512);
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int i = 0; i < kStages; ++i) { mbar_init(full + i * 16, 1); mbar_init(full + i * 16 + 8, 1); mbar_init(empty + i * 8, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(done + i * 8, 1); mbar_init(free + i * 8, kEpilogueWarps * 32); }
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
    int issued = 0;                                      // stages, by the loading warp
    if (warp >= kLoader) {                               // two roles, two idle warps
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRolesRegs));
        if (warp == kLoader) {
            int slot = 0, phase = 1;
            bool ok = true;
            for (int i = blockIdx.x; i < work && ok; i += gridDim.x) {
                const int np = i / c.at.filter_tiles, kt = i % c.at.filter_tiles, rows = tile_rows(c, kt), ranks = ranks_of(np);
                const int id = ranks ? a.adapter[np / c.at.tiles] : 0;
                const char *x = ws_of(c) + (size_t)np * c.s.chunks * kPixelBytes, *t = ws_of(c) + c.at.ranks_at + (size_t)np * s.RB * kRankBytes;
                const char *w = ws_of(c) + c.at.filters_at + (size_t)kt * c.s.chunks * kFilterTile * 32 * 256;
                const char *u = reinterpret_cast<const char *>(a.packed + s.up_halves_at + id * s.up_halves) + (size_t)kt * s.RB * kFilterTile * 32 * 128;
                for (int k = 0; k < c.s.chunks + ranks; ++k) {
                    if (issued >= kStages && !(ok = wait_here(empty + slot * 8, phase, stop, c.status, c.limit))) break;
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
        } else if (warp == kIssuer) {
            const uint32_t first = smem_desc_lo(smem_u32(stages));
            int slot = 0, phase = 0, buffer = 0, buffer_phase = 1, turn = 0;
            bool ok = true;
            for (int i = blockIdx.x; i < work && ok; i += gridDim.x) {
                const int np = i / c.at.filter_tiles, rows = tile_rows(c, i % c.at.filter_tiles), ranks = ranks_of(np);
                const uint32_t desc = f16_desc(rows);
                for (int k = 0, in_run = 0; k < c.s.chunks + ranks; ++k) {
                    if (in_run == 0 && turn >= 2 && !(ok = wait_here(free + buffer * 8, buffer_phase, stop, c.status, c.limit))) break;
                    const uint32_t d = tmem + buffer * 256;
                    const uint32_t x = first + slot * (kStageBytes >> 4), w = x + (kPixelBytes >> 4);
                    if (!(ok = wait_here(full + slot * 16, phase, stop, c.status, c.limit))) break;
                    tc_fence_after();
                    if (kX3) {                               // small terms first: low pixels and high filters while the rest is on its way
                        if (k < c.s.chunks && elect_one())
#pragma unroll
                            for (int e = 0; e < 4; ++e) mma_f16(d, x + e * 2 + kPixelBytes / 32, w + e * 2, desc, in_run > 0 || e > 0);
                        __syncwarp();
                        if (!(ok = wait_here(full + slot * 16 + 8, phase, stop, c.status, c.limit))) break;
                        tc_fence_after();
                    }
                    // the ranks' steps are a run of their own: their product has another scale
                    const bool last = k == c.s.chunks - 1 || k == c.s.chunks + ranks - 1 || (in_run == kRun<kX3> - 1 && k < c.s.chunks);
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
                                for (int e = 0; e < steps; ++e) mma_f16(d, x + e * 2 + (term == 0 ? 4 : 0), w + e * 2 + (term == 1 ? 4 : 0), desc, in_run > 0 || e > 0 || term > (kX3 ? 0 : 2));
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
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEpilogueRegs));
        // a warp takes 32 pixels of every other block of filters, a thread a pixel
        constexpr int kShares = kEpilogueWarps / 4, kBlocks = kFilterTile / kShares;
        const int lane = threadIdx.x & 31, part = warp >> 2;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        float4 *rows = reinterpret_cast<float4 *>(stages + kStages * kStageBytes) + warp * kPassing / 16;
        // What undoes a filter's scaling, of W and of Up, and its bias; what undoes a pixel's.  Asked for while the tile before is stored.
        float w_factor[kBlocks], u_factor[kBlocks], bias[kBlocks];
        int2 ex;
        int id;
        bool some;
        auto fetch_id = [&](int i) { id = a.adapter[i / c.at.filter_tiles / c.at.tiles]; };
        auto fetch = [&](int i) {
            const int np = i / c.at.filter_tiles, kt = i % c.at.filter_tiles;
            some = id >= 0 && id < a.adapters;
            ex = pixel_exponents(c)[(size_t)np * kTile + (warp & 3) * 32 + lane];
#pragma unroll
            for (int e = 0; e < kBlocks; ++e) {
                const int k = (kt * kFilterTile + part + e * kShares) * 32 + lane;
                w_factor[e] = k < s.KB * 32 ? filter_factors(c)[k] : 0.0f;
                bias[e] = a.bias && k < s.K ? a.bias[k] : 0.0f;
                u_factor[e] = some && k < s.KB * 32 ? info_of(a.packed, s, id)[4 + k] : 0.0f;
            }
        };
        int buffer = 0, phase = 0;
        fetch_id(blockIdx.x);                            // (no block without work is launched)
        fetch(blockIdx.x);
        for (int i = blockIdx.x; i < work; i += gridDim.x) {
            const int np = i / c.at.filter_tiles, kt = i % c.at.filter_tiles, n = np / c.at.tiles, p0 = np % c.at.tiles * kTile + (warp & 3) * 32;
            const int blocks = tile_rows(c, kt) / 32;
            const int next = min(i + (int)gridDim.x, work - 1);          // (asked for at the end, too: values kept instead would take registers all along)
            fetch_id(next);
            uint64_t sum[kBlocks][16] = {};              // of this warp's blocks of filters, by twos
            // the next accumulator's columns, a block at a time
            auto take = [&](auto before, auto use) -> bool {
                if (!wait_here(done + buffer * 8, phase, stop, c.status, c.limit)) return false;
                tc_fence_after();
#pragma unroll
                for (int e = 0; e < kBlocks; ++e) {
                    if (part + e * kShares >= blocks) continue;
                    before(e);
                    float v[32];
                    tmem_ld32(tmem + buffer * 256 + (part + e * kShares) * 32 + lanes, v);
                    use(e, v);
                }
                tc_fence_before();
                mbar_arrive(free + buffer * 8);
                if (++buffer == 2) { buffer = 0; phase ^= 1; }
                return true;
            };
            bool ok = true;
#pragma unroll 1
            for (int k = 0; k < c.s.chunks && ok; k += kRun<kX3>)
                ok = take([](int) {}, [&](int e, const float (&v)[32]) {
#pragma unroll
                    for (int u = 0; u < 32; u += 2) sum[e][u / 2] = add2(sum[e][u / 2], pair(v[u], v[u + 1]));
                });
            if (!ok) break;
            // A filter's three go to all lanes, where the results pass through later: [block]{32 of each}
            __syncwarp();
#pragma unroll
            for (int e = 0; e < kBlocks; ++e) {
                float *to = reinterpret_cast<float *>(rows) + e * 96 + lane;
                to[0] = w_factor[e];
                to[32] = u_factor[e];
                to[64] = bias[e];
            }
            __syncwarp();
            // sums are kept smaller by 2^(64 - exponent) where a pixel's scale would let them pass FP32's range in front of the filter's
            const int kept_back = min(max((some ? max(ex.x - 141, ex.y) : ex.x - 141) - 64, 0), 127);
            const float x_back = power(ex.x - 141 - kept_back), t_back = some ? power(ex.y - kept_back) : 0.0f, down = power(-kept_back), up = power(kept_back);
            // scales and bias, while the adapter's part is on its way
            float4 f[8], add[8];
#pragma unroll
            for (int e = 0; e < kBlocks; ++e) {
#pragma unroll
                for (int u = 0; u < 8; ++u) { f[u] = rows[e * 24 + u]; add[u] = rows[e * 24 + 16 + u]; }
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    uint64_t *y = &sum[e][u * 2];
                    y[0] = fma2(mul2(y[0], pair(x_back, x_back)), pair(f[u].x, f[u].y), mul2(pair(add[u].x, add[u].y), pair(down, down)));
                    y[1] = fma2(mul2(y[1], pair(x_back, x_back)), pair(f[u].z, f[u].w), mul2(pair(add[u].z, add[u].w), pair(down, down)));
                }
            }
            if (some && !take([&](int e) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) f[u] = rows[e * 24 + 8 + u];
                }, [&](int e, const float (&v)[32]) {
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        uint64_t *y = &sum[e][u * 2];
                        y[0] = fma2(mul2(pair(v[u * 4], v[u * 4 + 1]), pair(t_back, t_back)), pair(f[u].x, f[u].y), y[0]);
                        y[1] = fma2(mul2(pair(v[u * 4 + 2], v[u * 4 + 3]), pair(t_back, t_back)), pair(f[u].z, f[u].w), y[1]);
                    }
                })) break;
            const int left = a.HW - p0;                  // pixels
            fetch(next);
#pragma unroll
            for (int e = 0; e < kBlocks; ++e) {
                const int b = part + e * kShares;
                if (b >= blocks) continue;
                float4 y[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    unpair(mul2(sum[e][u * 2], pair(up, up)), y[u].x, y[u].y);
                    unpair(mul2(sum[e][u * 2 + 1], pair(up, up)), y[u].z, y[u].w);
                }
                float4 *out = reinterpret_cast<float4 *>(a.out) + (((size_t)n * s.KB + kt * kFilterTile + b) * a.HW + p0) * 8 + lane;
                // through shared memory, so that a store is whole lines: eight lanes a pixel
                __syncwarp();
#pragma unroll
                for (int u = 0; u < 8; ++u) rows[lane * 8 + (u ^ (lane & 7))] = y[u];
                __syncwarp();
#pragma unroll
                for (int u = 0; u < 8; ++u) y[u] = rows[(u * 4 + (lane >> 3)) * 8 + ((lane & 7) ^ ((u * 4 + (lane >> 3)) & 7))];
                if (a.accumulate) {
                    float4 before[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) before[u] = u * 4 + (lane >> 3) < left ? out[u * 32] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int u = 0; u < 8; ++u) { y[u].x += before[u].x; y[u].y += before[u].y; y[u].z += before[u].z; y[u].w += before[u].w; }
                }
                if (a.relu)
#pragma unroll
                    for (int u = 0; u < 8; ++u) y[u] = make_float4(fmaxf(y[u].x, 0.0f), fmaxf(y[u].y, 0.0f), fmaxf(y[u].z, 0.0f), fmaxf(y[u].w, 0.0f));
                const int filters = s.K - (kt * kFilterTile + b) * 32;
                if (filters < 32)                        // +0 in pad lanes
#pragma unroll
                    for (int u = 0; u < 8; ++u) y[u] = clear_from(y[u], filters - (lane & 7) * 4);
                // operands are read again, results here not: they leave L2 first (131 -> 128 us)
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (left >= 32 || u * 4 + (lane >> 3) < left) __stcs(out + u * 32, y[u]);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (gave_up && warp == kLoader)                            // what is still on its way must land before the block ends
        for (int x = max(0, issued - kStages); x < issued; ++x)
            for (int y = 0; y < (kX3 ? 2 : 1); ++y) mbar_wait(full + x % kStages * 16 + y * 8, (x / kStages) & 1, kDefaultWaitIters);
    if (warp == kIssuer) tmem_dealloc(tmem, 512);
}

// Up and Down as halves, a block an adapter each.  Each row of Down (a rank) is brought to the same size; what that takes from some ranks beside the
// largest one, Up's columns get, in front of each of its rows being brought to one size, too.
__global__ void __launch_bounds__(kThreads) pack_halves_kernel(const float *__restrict__ down, const float *__restrict__ up, float *__restrict__ packed, const AdapterShape s) {
    __shared__ int rank_s[128];
    grid_dep_sync();
    grid_dep_trigger();
    const int a = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float *d = down + (size_t)a * s.R * s.C, *u = up + (size_t)a * s.K * s.R;
    for (int r = warp; r < s.R; r += kThreads / 32) {
        float most = 0.0f;
        for (int ch = lane; ch < s.C; ch += 32) most = fmaxf(most, magnitude(d[(size_t)r * s.C + ch]));
#pragma unroll
        for (int o = 16; o; o /= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
        if (lane == 0) rank_s[r] = top_exponent(most);
    }
    __syncthreads();
    int ed = 0;
    for (int r = 0; r < s.R; ++r) ed = max(ed, rank_s[r]);
    float *info = info_of(packed, s, a);
    if (blockIdx.y) {                                    // Down: rows of 128 bytes hold 64 channels' high (or low) halves
        if (threadIdx.x == 0) info[0] = __int_as_float(ed);
        char *out = reinterpret_cast<char *>(packed + s.down_halves_at + a * s.down_halves);
        for (size_t i = threadIdx.x; i < (size_t)s.RQ * s.chunks * 16; i += kThreads) {
            const int e = (int)(i % 16) * 4, run = (int)(i / 16 % s.chunks), r = (int)(i / 16 / s.chunks), ch = run * 64 + e;
            const float by = r < s.R ? lift(rank_s[r]) : 0.0f;
            float v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = r < s.R && ch + x < s.C ? d[(size_t)r * s.C + ch + x] * by : 0.0f;
            uint2 hi, lo;
            split_finite(v[0], v[1], hi.x, lo.x);
            split_finite(v[2], v[3], hi.y, lo.y);
            char *to = out + (size_t)run * s.RQ * 256;
            *reinterpret_cast<uint2 *>(to + chunk_at(r, e, s.RQ) + (e & 4) * 2) = hi;
            *reinterpret_cast<uint2 *>(to + chunk_at(r, 64 + e, s.RQ) + (e & 4) * 2) = lo;
        }
        return;
    }
    // Up: rows of 128 bytes hold both halves of 32 ranks; a warp a row, a lane a rank of each 32
    char *out = reinterpret_cast<char *>(packed + s.up_halves_at + a * s.up_halves);
    for (int k = warp; k < s.KB * 32; k += kThreads / 32) {
        int ex = 15;                                     // of the row's largest value
        for (int r = lane; k < s.K && r < s.R; r += 32) {
            const float m = magnitude(u[(size_t)k * s.R + r]);
            if (m > 0.0f) ex = max(ex, (int)(__float_as_uint(m) >> 23) + rank_s[r] - ed);
        }
#pragma unroll
        for (int o = 16; o; o /= 2) ex = max(ex, __shfl_xor_sync(~0u, ex, o));
        if (lane == 0) info[4 + k] = drop(ex);
        const int kt = k / (kFilterTile * 32), row = k % (kFilterTile * 32), rows = min(kFilterTile, s.KB - kt * kFilterTile) * 32;
        for (int rb = 0; rb < s.RB; ++rb) {
            const int r = rb * 32 + lane;
            const float v = k < s.K && r < s.R ? ldexpf(u[(size_t)k * s.R + r], 141 - ex + rank_s[r] - ed) : 0.0f, w = __shfl_down_sync(~0u, v, 1);
            uint32_t hi, lo;
            split_finite(v, w, hi, lo);
            char *to = out + ((size_t)kt * s.RB * kFilterTile * 32 + (size_t)rb * rows) * 128;
            if ((lane & 1) == 0) {
                *reinterpret_cast<uint32_t *>(to + chunk_at(row, lane, rows) + (lane & 7) * 2) = hi;
                *reinterpret_cast<uint32_t *>(to + chunk_at(row, 32 + lane, rows) + (lane & 7) * 2) = lo;
            }
        }
    }
}

}  // namespace

// The other form writes the result twice and takes the adapter's products in FP32, which costs the more the larger the rank; this one lays the
// pixels out first.  us, here / there, back to back on three sets of tensors in turn, rank 8 and 32, batch 64 unless said: 256 -> 768 on 28 x 28 124 / 220
// and 125 / 369; 256 -> 256 77 / 100 and 78 / 192; 128 -> 128 44 / 44 and 44 / 88; 64 -> 64 33 / 26 and 33 / 51; 256 -> 256 on 14 x 14 30 / 34 and 30 /
// 68; 512 -> 128 on 28 x 28 121 / 115 and 119 / 263; batch 128, 512 -> 512 on 14 x 14 100 / 143 and 101 / 236, on 8 x 8 54 / 51 and 54 / 88; batch 4, 320 ->
// 960 on 32 x 32 32 / 36 and 33 / 63.  Few channels, ranks 16 and 32: batch 95, 11 -> 52 on 11 x 19 20.0 / 14.7 and 20.0 / 20.8, batch 41, 41 -> 17 on
// 32 x 8 14.2 / 10.7 and 14.1 / 15.4.  Few tiles, many operations: batch 31, 390 -> 135, rank 31 on 11 x 20 37.0 / 59.0; batch 20, 256 -> 512, rank 24 on
// 14 x 14 26.1 / 38.4.  Near the line: batch 64, 64 -> 64, rank 16 on 28 x 28 33 / 34, batch 80, 96 -> 160, rank 16 on 9 x 10 17.8 / 17.6, 64 -> 96, rank 9
// on 8 x 8 14.3 / 11.3.
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
    launch_kernel(ctx, adapter_filters_kernel, dim3((unsigned)s.KB), dim3(kThreads * kTeams), 0, st, c);
    if (int e = check_launch(ctx)) return e;
    static std::atomic<unsigned long long> pixels{0}, exact{0}, fast{0};
    // a role's share of the registers is waited for without an end if the launch brings fewer than all shares together
    static std::atomic<unsigned long long> counted{0};
    const unsigned long long bit = 1ull << (ctx->device & 63);
    if (!(counted.load(std::memory_order_relaxed) & bit)) {
        for (const void *kern : {reinterpret_cast<const void *>(adapter_product_kernel<true>), reinterpret_cast<const void *>(adapter_product_kernel<false>)}) {
            cudaFuncAttributes f;
            const cudaError_t e = cudaFuncGetAttributes(&f, kern);
            if (e != cudaSuccess) { ctx->last_cuda = (int)e; return SMALL_ERR_CUDA; }
            if (f.numRegs * kProductThreads < kRolesRegs * 128 + kEpilogueRegs * kEpilogueWarps * 32) return SMALL_ERR_UNSUPPORTED;
        }
        counted.fetch_or(bit, std::memory_order_relaxed);
    }
    const size_t passing = 1024 + (size_t)kPixelBytes + (size_t)s.RQ * (256 + (s.chunks > kDownRun ? kTile * sizeof(float) : 0)), stages = 1024 + (size_t)kStages * kStageBytes + kEpilogueWarps * kPassing;
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
