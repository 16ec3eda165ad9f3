// Attention over the pixels of a plane on the tensor cores (tcgen05, kind::f16), at TF32's or FP32's accuracy.
//
// Operands are pairs of halves (halves.cuh); weights exp(x - m) are scaled by 2^14 so that theirs are exact far down, and the sum of
// weights too, so that it cancels.
//
// attention_tiles_kernel lays the valid keys and values of each image out once, 128 keys a tile, as the MMAs read them: keys
// [key][hi | lo channels], values transposed [channel][hi keys | lo keys], rows of 128 bytes swizzled, so that a tile is two plain
// bulk copies.  Every block of queries (QP / 256 a head, times the heads that share them) reads them so; converting in each
// block instead would repeat it that many times beside the softmax, which is what bounds the main kernel.
//
// attention_tc_kernel: a block takes one or two tiles of 128 queries of a head.  One warp loads tiles, one issues MMAs, four (eight)
// do the softmax of each query tile.  Scores lie in three rotating buffers of tensor memory (128 lanes x 128 columns); a thread takes a
// row (two share it where the result has 128 channels) and writes the weights as halves over the scores, where they are the second
// product's A operand.  While one tile's softmax runs, the tensor cores work on the other's.  Each key tile's product with the values
// starts from zero and is added to the thread's own FP32 sums: the tensor core's accumulator is cut off, not rounded, at each step, which over
// thousands of keys would add up (5e-8 a step), and no rescaling of tensor memory is needed when the maximum grows.
//
// Bound by the softmax: a table entry, an exponential, the split into halves and two crossings of tensor memory a score.  Batch 4, 8 heads of 64,
// 56 x 56 with a bias: 356 us (tiles 19 of them), 227 TFLOP/s of the formula's operations; the three products alone would take 148.
#include <type_traits>

#include "attention.cuh"
#include "halves.cuh"

namespace small {
namespace {
using namespace halves;

constexpr float kLift = 14.0f;           // weights are scaled by 2^14

// Workspace: [N][kv_heads][tiles]{keys: DP * 512 bytes, values: DP * 512 bytes}; int[N][tiles][128 + 16], the keys' places in the bias table
// (of_key), and of each eight keys the last one's if they are neighbours there, else -1; float[N][kv_heads][tiles][2], how to undo the scaling.
constexpr int kRun = 8, kPlaceInts = kTile + kTile / kRun;
__device__ __forceinline__ int *key_places(const AttnArgs &a, int tiles, int tile_bytes) {
    return reinterpret_cast<int *>(static_cast<char *>(a.ws) + (size_t)a.N * a.kv_heads * tiles * 2 * tile_bytes);
}
__device__ __forceinline__ float *undo_scaling(const AttnArgs &a, int tiles, int tile_bytes) {
    return reinterpret_cast<float *>(key_places(a, tiles, tile_bytes) + (size_t)a.N * tiles * kPlaceInts);
}
template <int DP>
__global__ void __launch_bounds__(256) attention_tiles_kernel(const AttnArgs a, int tiles) {
    constexpr int kBytes = DP * 512;
    __shared__ float most_s[8];
    extern __shared__ float values[];                    // [128][DP + 1]
    grid_dep_sync();
    grid_dep_trigger();
    const int t = blockIdx.x >> 1, hk = blockIdx.y, n = blockIdx.z;
    const bool is_v = blockIdx.x & 1;
    const int2 e = extent(a.k_ext, n, a.KH, a.KW);
    const int keys = e.x * e.y;
    if (t * kTile >= keys) return;
    const size_t tile = ((size_t)n * a.kv_heads + hk) * tiles + t;
    char *out = static_cast<char *>(a.ws) + tile * 2 * kBytes + (is_v ? kBytes : 0);
    const float *x = is_v ? a.v + n * a.v_stride : a.k + n * a.k_stride;
    // eight lanes a key, four channels of every 32 each; a warp takes keys 16 w .. 16 w + 15
    const int lane = threadIdx.x & 31, first = (threadIdx.x >> 5) * 16 + (lane >> 3), c0 = (lane & 7) * 4;
    float4 v[4][DP / 32];
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = t * kTile + first + 4 * i, p = j < keys ? j / e.y * a.KW + j % e.y : -1;
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) v[i][k] = p >= 0 ? load4(x, hk * a.D, k * 32 + c0, a.D, p, a.KP) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < DP / 32; ++k) most = fmaxf(most, magnitude(v[i][k]));
#pragma unroll
    for (int o = 16; o; o /= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    if (lane == 0) most_s[threadIdx.x >> 5] = most;
    if (is_v)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < DP / 32; ++k) {
                float *w = values + (first + 4 * i) * (DP + 1) + k * 32 + c0;
                w[0] = v[i][k].x; w[1] = v[i][k].y; w[2] = v[i][k].z; w[3] = v[i][k].w;
            }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, most_s[i]);
    const int ex = top_exponent(most);
    const float up = lift(ex);
    if (threadIdx.x == 0) undo_scaling(a, tiles, kBytes)[tile * 2 + is_v] = drop(ex);
    if (!is_v) {
        if (hk == 0 && threadIdx.x < kTile) {
            const int j = t * kTile + threadIdx.x;
            int *places = key_places(a, tiles, kBytes) + ((size_t)n * tiles + t) * kPlaceInts;
            const int place = j < keys ? of_key(a, j / e.y, j % e.y) : 0, first_of = __shfl_sync(~0u, place, threadIdx.x & 24);
            places[threadIdx.x] = place;
            if (threadIdx.x % kRun == kRun - 1) places[kTile + threadIdx.x / kRun] = place - first_of == kRun - 1 ? place : -1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < DP / 32; ++k) store4<DP>(out, first + 4 * i, k * 32 + c0, v[i][k], up);
        return;
    }
    for (int i = threadIdx.x; i < DP * 16; i += 256) {   // eight lanes a channel's 128 bytes
        const int d = (i >> 3) % DP, k0 = (i & 7) * 8 + i / (8 * DP) * 64;
        float w[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) w[u] = values[(k0 + u) * (DP + 1) + d] * up;
        uint4 hi, lo;
        split_finite(w[0], w[1], hi.x, lo.x); split_finite(w[2], w[3], hi.y, lo.y);
        split_finite(w[4], w[5], hi.z, lo.z); split_finite(w[6], w[7], hi.w, lo.w);
        *reinterpret_cast<uint4 *>(out + chunk_at(d, k0, DP)) = hi;
        *reinterpret_cast<uint4 *>(out + chunk_at(d, kTile + k0, DP)) = lo;
    }
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_st4(uint32_t taddr, const uint32_t (&r)[4]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// A load that is waited for later; the wait takes the values, so that nothing uses them in front of it.
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
          "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]),
          "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]),
          "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
          "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
        :: "memory");
}

// v = cap * tanh(v * over_cap), as `capped` in attention.cuh: both quotients with the argument's sign, one reciprocal.
__device__ __forceinline__ void capped(float &v0, float &v1, float cap, float over_cap) {
    const uint64_t t = fma2(pair(v0, v1), pair(over_cap, over_cap), 0), s = fma2(t, t, 0);
    const uint64_t num = fma2(t, fma2(s, add2(s, pair(105.0f, 105.0f)), pair(945.0f, 945.0f)), 0);
    const uint64_t den = fma2(s, fma2(s, pair(15.0f, 15.0f), pair(420.0f, 420.0f)), pair(945.0f, 945.0f));
    float a0, a1, s0, s1, n0, n1, d0, d1, p0, p1, q0, q1;
    unpair(fma2(t, pair(2.0f * kLog2e, 2.0f * kLog2e), 0), a0, a1);
    const uint64_t e = pair(exp2_fast(fminf(a0, 64.0f)), exp2_fast(fminf(a1, 64.0f)));
    unpair(s, s0, s1);
    unpair(num, n0, n1);
    unpair(den, d0, d1);
    unpair(add2(e, pair(-1.0f, -1.0f)), p0, p1);
    unpair(add2(e, pair(1.0f, 1.0f)), q0, q1);
    const bool far0 = s0 >= 0.25f, far1 = s1 >= 0.25f;               // (a NaN goes with the near ones, and through)
    float r0, r1;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(far0 ? q0 : d0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(far1 ? q1 : d1));
    unpair(fma2(fma2(pair(far0 ? p0 : n0, far1 ? p1 : n1), pair(r0, r1), 0), pair(cap, cap), 0), v0, v1);
}

constexpr int kMaxRing = 4;
constexpr int kPlaces = 8;               // tiles: one is used no longer when the keys of the eighth behind it are asked for
// Threads of a row: one has registers for 64 sums and for scores under way; the table's reads want twice as many warps to hide behind.
template <int DP, bool kGeneral> constexpr int kRowThreads = DP == 128 || kGeneral ? 2 : 1;
template <int DP, bool kGeneral> constexpr int kBlock = (DP == 128 ? 1 : 2) * kTile * kRowThreads<DP, kGeneral> + 64;

struct TcArgs {
    AttnArgs a;
    int tiles;                           // key tiles of a whole plane, as the workspace counts them
    int q_tiles;                         // tiles of queries that a block takes: 1 or 2
    int ring;                            // shared-memory slots for key and value tiles
    int table_floats;                    // of the bias table's part in shared memory; 0: read where it lies
    int *status;
    uint32_t limit;
};

struct Shared {
    uint64_t full[kMaxRing], empty[kMaxRing];            // a slot has its tile; its last product is done
    uint64_t scores[3], weights[3];                      // a buffer has a tile's scores; 256 threads have written their weights
    uint64_t part[2], taken[2];                          // a query tile's product with the values is there; 256 threads have added it
    uint64_t placed[kPlaces];                            // a tile's keys' places in the bias table are there
    uint64_t drained;                                    // after a wait that ran out: all MMAs are done
    uint32_t tmem;
    int gave_up;
    float exchange[2][2][2][kTile];                      // [parity of the key tile][query tile][half of the keys][row]: maxima; at last sums
    float q_drop[2][kTile];
    alignas(16) int places[kPlaces][kPlaceInts];
};

// kGeneral: scores pass through the cap and the bias table.
template <int DP, bool kX3, bool kGeneral>
__global__ void __launch_bounds__(kBlock<DP, kGeneral>, 1) attention_tc_kernel(const TcArgs c) {
    constexpr int kBytes = DP * 512;                     // of a tile of queries, keys or values
    constexpr int kShare = kRowThreads<DP, kGeneral>;            // threads of a row
    constexpr int kKeys = kTile / kShare, kOut = DP / kShare;            // a thread's keys of a tile, and its channels of the result
    constexpr int kWarps = 4 * kShare;                   // softmax warps of a query tile
    extern __shared__ char raw[];
    __shared__ Shared sh;
    const AttnArgs &a = c.a;
    const int n = blockIdx.z, h = blockIdx.y, hk = h / (a.heads / a.kv_heads);
    const int i0 = blockIdx.x * c.q_tiles * kTile, nq = min(c.q_tiles, (a.QP - i0 + kTile - 1) / kTile);
    const int warp = warp_index(), loader = c.q_tiles * kWarps, issuer = loader + 1;
    char *base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    char *queries = base, *slots = base + c.q_tiles * kBytes;
    float *table = reinterpret_cast<float *>(slots + c.ring * kBytes);
    if (warp == issuer) tmem_alloc(smem_u32(&sh.tmem), 512);
    const uint32_t full = smem_u32(sh.full), empty = smem_u32(sh.empty), scores = smem_u32(sh.scores), weights = smem_u32(sh.weights),
                   part = smem_u32(sh.part), taken = smem_u32(sh.taken), placed = smem_u32(sh.placed);
    // What this kernel reads besides the tiles is older than the kernel in front of it, which has waited for all before itself.
    const int2 qe = extent(a.q_ext, n, a.QH, a.QW), ke = extent(a.k_ext, n, a.KH, a.KW);
    const int keys = ke.x * ke.y, tiles = (keys + kTile - 1) / kTile, steps = tiles * nq;
    const int wg = warp / kWarps, half = warp / 4 % kShare, row = threadIdx.x & (kTile - 1);         // of the softmax warps: query tile, share of the keys, row
    const int TW = a.QW + a.KW - 1;
    const float *bias = a.bias ? a.bias + (size_t)h * (a.QH + a.KH - 1) * TW : nullptr;
    int qoff = 0;
    const int i = i0 + wg * kTile + row;
    // The tiles, keys before values; without the low parts: values' lie in the second half of their tile, keys' too but for 32 channels, whose
    // rows hold both.
    const uint32_t k_bytes = kX3 || DP == 32 ? kBytes : kBytes / 2, v_bytes = kX3 ? kBytes : kBytes / 2;
    const char *from_tiles = static_cast<const char *>(a.ws) + ((size_t)n * a.kv_heads + hk) * c.tiles * 2 * kBytes;
    const int *from_places = key_places(a, c.tiles, kBytes) + (size_t)n * c.tiles * kPlaceInts;
    int issued = 0;                                      // by the loading warp
    auto load = [&](int slot) {
        if (elect_one()) {
            const uint32_t bytes = issued & 1 ? v_bytes : k_bytes;
            mbar_expect_tx(full + slot * 8, bytes);
            bulk_load(smem_u32(slots + slot * kBytes), from_tiles + (size_t)issued * kBytes, bytes, full + slot * 8);
            if (kGeneral && bias && !(issued & 1)) {           // (whoever asks waits: nothing may arrive behind a block's end)
                const int t = issued >> 1, at = t % kPlaces;
                mbar_expect_tx(placed + at * 8, kPlaceInts * sizeof(int));
                bulk_load(smem_u32(sh.places[at]), from_places + t * kPlaceInts, kPlaceInts * sizeof(int), placed + at * 8);
            }
        }
        __syncwarp();
        ++issued;
    };
    if (warp == loader) {                                // on their way before the queries are converted
        if (elect_one()) {
            sh.gave_up = 0;
            for (int i = 0; i < kMaxRing; ++i) { mbar_init(full + i * 8, 1); mbar_init(empty + i * 8, 1); }
            for (int i = 0; i < 3; ++i) { mbar_init(scores + i * 8, 1); mbar_init(weights + i * 8, kShare * kTile); }
            for (int i = 0; i < 2; ++i) { mbar_init(part + i * 8, 1); mbar_init(taken + i * 8, kShare * kTile); }
            for (int i = 0; i < kPlaces; ++i) mbar_init(placed + i * 8, 1);
            mbar_init(smem_u32(&sh.drained), 1);
            mbar_fence_init();
        }
        __syncwarp();
        grid_dep_sync();
        while (issued < min(2 * tiles, c.ring)) load(issued);
    }
    if (wg < nq) {                                       // eight lanes a row
        char *mine = queries + wg * kBytes;
        constexpr int kRows = kTile / kWarps / 4;        // of a lane
        const int lane = threadIdx.x & 31, c0 = (lane & 7) * 4, r0 = (warp % kWarps) * (kTile / kWarps) + (lane >> 3);
        const float *q = a.q + n * a.q_stride;
#pragma unroll 1
        for (int i4 = 0; i4 < kRows; i4 += 4) {
            float4 v[4][DP / 32];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int p = i0 + wg * kTile + r0 + 4 * (i4 + k);
#pragma unroll
                for (int ch = 0; ch < DP / 32; ++ch) v[k][ch] = p < a.QP ? load4(q, h * a.D, ch * 32 + c0, a.D, p, a.QP) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = r0 + 4 * (i4 + k);
                float most = 0.0f;
#pragma unroll
                for (int ch = 0; ch < DP / 32; ++ch) most = fmaxf(most, magnitude(v[k][ch]));
#pragma unroll
                for (int o = 1; o < 8; o *= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
                const int ex = top_exponent(most);
                const float up = a.scale < 0.0f ? -lift(ex) : lift(ex);          // the scale's sign goes with the queries: what is left is >= 0
                if (c0 == 0) sh.q_drop[wg][r] = fabsf(a.scale) * drop(ex);
#pragma unroll
                for (int ch = 0; ch < DP / 32; ++ch) store4<DP>(mine, r, ch * 32 + c0, v[k][ch], up);
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (kGeneral && bias && warp < loader) {
        qoff = of_query(a, min(i, a.QP - 1));
        if (c.table_floats) {                            // the table's rows that these queries meet
            const int y0 = i0 / a.QW, y1 = min(i0 + nq * kTile, a.QP) - 1;
            const int rows = y1 / a.QW - y0 + a.KH;
            const float *from = bias + (size_t)y0 * TW;
            for (int r = warp; r < rows; r += loader)
#pragma unroll 4
                for (int e = threadIdx.x & 31; e < TW; e += 32) table[r * a.pitch + e] = powers_of_two(from[r * TW + e]);
            qoff -= y0 * a.pitch;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    volatile int *stop = &sh.gave_up;
    auto s_at = [&](int buffer) { return tmem + buffer * kTile; };
    auto o_at = [&](int tile) { return tmem + 3 * kTile + tile * DP; };

    // Not before this block has its tensor memory: a block of the next kernel could take it, and wait for this kernel's end with it.
    if (warp == loader) grid_dep_trigger();
    if (warp == loader) {
        for (int slot = 0, phase = 0; issued < 2 * tiles;) {
            if (!mbar_wait_uniform(empty + slot * 8, phase, stop, c.status, c.limit)) break;
            load(slot);
            if (++slot == c.ring) { slot = 0; phase ^= 1; }
        }
    } else if (warp == issuer) {
        const uint32_t q_lo = smem_desc_lo(smem_u32(queries)), slot_lo = smem_desc_lo(smem_u32(slots));
        auto column = [&](int col, int rows) { return (uint32_t)(((col >> 6) * rows * 128 + (col & 63) * 2) >> 4); };
        // Step s + 2's scores go in front of step s's product, so that the softmax finds its next scores at hand - unless their keys
        // have to wait for a slot that this product gives free: with one query tile step s + 2 is two key tiles on.
        const bool early = nq == 2 || c.ring >= 4;
        // Places in the rings, kept as they go: a division in front of an MMA is time the tensor cores wait.  Steps go by query tile first.
        const int two = nq - 1;
        struct Place {
            int at, phase;
            __device__ void on(int by, int of) { if ((at += by) >= of) { at -= of; phase ^= 1; } }
        } k_slot{0, 0}, v_slot{1, 0}, to{0, 0}, from{0, 0};              // slots of keys and values, buffers of scores and of weights
        auto score = [&](int s) -> bool {                // queries x keys of step s
            const int j = s & two;
            if (j == 0 && !mbar_wait_uniform(full + k_slot.at * 8, k_slot.phase, stop, c.status, c.limit)) return false;
            // the buffer's last weights, those of step s - 3, are used up (else `taken` has said so in front of step s - 2's product)
            if (early && s >= 3 && !mbar_wait_uniform(part + ((s - 3) & two) * 8, (s - 3) >> two & 1, stop, c.status, c.limit)) return false;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t d = s_at(to.at), qa = q_lo + j * (kBytes >> 4), kb = slot_lo + k_slot.at * (kBytes >> 4), desc = f16_desc(kTile);
#pragma unroll
                for (int term = kX3 ? 0 : 2; term < 3; ++term)           // small terms first
#pragma unroll
                    for (int k = 0; k < DP; k += 16)
                        mma_f16(d, qa + column(k + (term == 0 ? DP : 0), kTile), kb + column(k + (term == 1 ? DP : 0), kTile), desc, k > 0 || term > (kX3 ? 0 : 2));
                mma_commit(scores + to.at * 8);
                if (j == two) mma_commit(empty + k_slot.at * 8);
            }
            __syncwarp();
            to.on(1, 3);
            if (j == two) k_slot.on(2, c.ring);
            return true;
        };
        bool ok = true;
        for (int s = 0; s < min(2, steps) && ok; ++s) ok = score(s);
        for (int s = 0; s < steps && ok; ++s) {
            const int j = s & two, t = s >> two;
            if (early && s + 2 < steps && !(ok = score(s + 2))) break;
            ok = mbar_wait_uniform(weights + from.at * 8, from.phase, stop, c.status, c.limit);
            if (ok && t > 0) ok = mbar_wait_uniform(taken + j * 8, (t - 1) & 1, stop, c.status, c.limit);
            if (ok && j == 0) ok = mbar_wait_uniform(full + v_slot.at * 8, v_slot.phase, stop, c.status, c.limit);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t d = o_at(j), pa = s_at(from.at), vb = slot_lo + v_slot.at * (kBytes >> 4), desc = f16_desc(DP);
#pragma unroll
                for (int term = kX3 ? 0 : 2; term < 3; ++term)
#pragma unroll
                    for (int k = 0; k < kTile; k += 16)
                        mma_f16_tmem(d, pa + (k >> 5) * 32 + (k & 16) / 2 + (term == 0 ? 16 : 0), vb + column(k + (term == 1 ? kTile : 0), DP), desc,
                                     k > 0 || term > (kX3 ? 0 : 2));
                mma_commit(part + j * 8);
                if (j == two) mma_commit(empty + v_slot.at * 8);
            }
            __syncwarp();
            from.on(1, 3);
            if (j == two) v_slot.on(2, c.ring);
            if (!early && s + 2 < steps) ok = score(s + 2);
        }
        if (!ok) {
            if (elect_one()) mma_commit(smem_u32(&sh.drained));
            __syncwarp();
            mbar_wait(smem_u32(&sh.drained), 0, kDefaultWaitIters);
        }
    } else if (wg < nq) {
        grid_dep_sync();
        const float *undo = undo_scaling(a, c.tiles, kBytes) + ((size_t)n * a.kv_heads + hk) * c.tiles * 2;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;               // this warp's 32 lanes of tensor memory
        const float q_drop = sh.q_drop[wg][row], cap2 = a.cap * kLog2e, over_cap = a.cap > 0.0f ? 1.0f / a.cap : 0.0f;
        const float *at_copy = table + qoff;             // (a pointer of its own: one that could be either place is read the slow way)
        uint64_t o[kOut / 2];
        float l = 0.0f, m = INFINITY;                    // m: 14 less the running maximum, in powers of two
        float2 drops = tiles ? *reinterpret_cast<const float2 *>(undo) : make_float2(0.f, 0.f), next = drops;
        int buffer = wg, phase = 0;
#pragma unroll
        for (int d = 0; d < kOut / 2; ++d) o[d] = 0;
        // Adds a tile's product with the values: after the next tile's weights are on their way, when it has long been there.
        auto take_part = [&](int t, float v_drop) {
            v_drop *= 1.0f / (1 << (int)kLift);
            mbar_wait_uniform(part + wg * 8, t & 1, stop, c.status, c.limit);
            tc_fence_after();
#pragma unroll
            for (int d = 0; d < kOut; d += 16) {
                float x[16];
                tmem_ld16(o_at(wg) + lanes + half * kOut + d, x);
#pragma unroll
                for (int u = 0; u < 16; u += 2) o[(d + u) / 2] = fma2(pair(x[u], x[u + 1]), pair(v_drop, v_drop), o[(d + u) / 2]);
            }
            tc_fence_before();
            mbar_arrive(taken + wg * 8);
        };
        // A wait that runs out ends the waits behind it at once; the loop goes on, so that the barrier of these 256 threads is met.
        auto tile = [&](int t, auto last) {              // last: keys may be missing (code of its own: the tests cost as much as the rest)
            constexpr bool kLast = decltype(last)::value;
            const int left = keys - t * kTile - half * kKeys;
            const float last_v = drops.y;
            drops = next;
            if (!kLast) next = *reinterpret_cast<const float2 *>(undo + 2 * t + 2);
            if (kGeneral && bias) mbar_wait_uniform(placed + t % kPlaces * 8, t / kPlaces & 1, stop, c.status, c.limit);
            mbar_wait_uniform(scores + buffer * 8, phase, stop, c.status, c.limit);
            tc_fence_after();
            const uint32_t st = s_at(buffer) + lanes + half * kKeys;
            const float f = q_drop * drops.x, scale2 = f * kLog2e;
            // The scores, in chunks of 32 keys: the last two stay in registers between the maximum and the exponentials.
            constexpr int kChunks = kKeys / 32;
            float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, one[32], two[32];
            auto take = [&](float (&v)[32], int g) {     // scores as the softmax takes them; the largest of each in `top`
                if (kGeneral) {
                    if (a.cap > 0.0f) {
                        const float to_cap = fminf(f * over_cap, FLT_MAX);           // (an infinite one would make NaN of a score of 0)
#pragma unroll
                        for (int u = 0; u < 32; u += 2) capped(v[u], v[u + 1], cap2, to_cap);
                    }
                    if (bias) {
                        const float f1 = a.cap > 0.0f ? 1.0f : scale2;
                        const int *place = sh.places[t % kPlaces] + half * kKeys + g;
                        if (c.table_floats) {
                            const int4 runs = *reinterpret_cast<const int4 *>(sh.places[t % kPlaces] + kTile + (half * kKeys + g) / kRun);
                            const int run[4] = {runs.x, runs.y, runs.z, runs.w};
#pragma unroll
                            for (int u = 0; u < 32; u += kRun) {
                                if (run[u / kRun] >= 0) {            // one row of the plane: neighbours in the table
                                    const float *b = at_copy - run[u / kRun];
#pragma unroll
                                    for (int w = 0; w < kRun; ++w) v[u + w] = fmaf(v[u + w], f1, b[kRun - 1 - w]);
                                } else {
#pragma unroll
                                    for (int w = 0; w < kRun; ++w) v[u + w] = fmaf(v[u + w], f1, at_copy[-place[u + w]]);
                                }
                            }
                        } else {
#pragma unroll
                            for (int u = 0; u < 32; ++u) v[u] = fmaf(v[u], f1, powers_of_two(bias[qoff - place[u]]));
                        }
                    }
                }
                if (kLast)
#pragma unroll
                    for (int u = 0; u < 32; ++u) v[u] = g + u < left ? v[u] : -INFINITY;
#pragma unroll
                for (int u = 0; u < 32; u += 2) top[u >> 1 & 3] = max3(top[u >> 1 & 3], v[u], v[u + 1]);
            };
            auto keep = [&](const float (&v)[32], int g) {           // where the scores were, until their turn comes
                uint32_t w[32];
#pragma unroll
                for (int u = 0; u < 32; ++u) w[u] = __float_as_uint(v[u]);
                tmem_st32(st + g, w);
            };
            tmem_ld32_async(st, one);
            if (kChunks == 4) {
                tmem_ld32_async(st + 32, two);
                tmem_ld_wait(one);
                take(one, 0);
                tmem_ld32_async(st + 64, one);
                tmem_ld_wait(two);
                take(two, 32);
                tmem_ld32_async(st + 96, two);
                tmem_ld_wait(one);
                take(one, 64);
                tmem_ld_wait(two);
                take(two, 96);
            } else {
                tmem_ld_wait(one);
                take(one, 0);
                if (kGeneral) keep(one, 0);
                tmem_ld32_async(st + 32, two);
                tmem_ld_wait(two);
                take(two, 32);
            }
            const float mine = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            float most = mine;
            if (kShare == 2) {
                sh.exchange[t & 1][wg][half][row] = mine;
                asm volatile("bar.sync %0, 256;" ::"r"(1 + wg) : "memory");
                most = fmaxf(mine, sh.exchange[t & 1][wg][half ^ 1][row]);
            }
            // weights are exp2(v * scale2 + m), or exp2(v + m) where the scale is already in
            const float now = fminf(m, kGeneral ? kLift - most : fmaf(-most, scale2, kLift)), add = kGeneral && now == INFINITY ? 0.0f : now;       // nothing to weigh yet
            const float shrink = kGeneral && now == INFINITY ? 1.0f : exp2_fast(now - m);
            m = now;
            uint64_t sum[2] = {0, 0};
            auto weigh = [&](float (&v)[32], int g) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int u = 0; u < 32; u += 2) {
                    uint64_t x = pair(v[u], v[u + 1]);
                    x = kGeneral ? add2(x, pair(add, add)) : fma2(x, pair(scale2, scale2), pair(add, add));
                    float x0, x1;
                    unpair(x, x0, x1);
                    x0 = exp2_fast(x0);
                    x1 = exp2_fast(x1);
                    if (!kGeneral && kLast) {             // -inf * 0, where the scores have no scale
                        x0 = g + u < left ? x0 : 0.0f;
                        x1 = g + u + 1 < left ? x1 : 0.0f;
                    }
                    const uint64_t e = pair(x0, x1);
                    sum[u >> 1 & 1] = add2(sum[u >> 1 & 1], e);
                    if (kX3) {
                        const float h0 = __uint_as_float(__float_as_uint(x0) & 0xffffe000u), h1 = __uint_as_float(__float_as_uint(x1) & 0xffffe000u);
                        float r0, r1;
                        unpair(fma2(pair(h0, h1), pair(-1.0f, -1.0f), e), r0, r1);
                        hi[u / 2 & 3] = pack_halves(h0, h1);
                        lo[u / 2 & 3] = pack_halves(r0, r1);
                    } else {
                        hi[u / 2 & 3] = pack_halves(x0, x1);
                    }
                    if ((u & 7) == 6) {                  // 16 keys are 8 columns of high parts and 8 of low ones, 16 columns on; four at a time: fewer registers (362 -> 356 us)
                        tmem_st4(st + g + (u & 24) / 2, hi);
                        if (kX3) tmem_st4(st + g + 16 + (u & 24) / 2, lo);
                    }
                }
            };
            if (kChunks == 4) {
                weigh(one, 64);
                tmem_ld32_async(st, one);
                weigh(two, 96);
                tmem_ld32_async(st + 32, two);
                tmem_ld_wait(one);
                weigh(one, 0);
                tmem_ld_wait(two);
                weigh(two, 32);
            } else {
                weigh(two, 32);
                if (kGeneral) tmem_st_wait();
                tmem_ld32_async(st, one);
                tmem_ld_wait(one);
                weigh(one, 0);
            }
            tmem_st_wait();
            tc_fence_before();
            mbar_arrive(weights + buffer * 8);
            float s0, s1;
            unpair(add2(sum[0], sum[1]), s0, s1);
            l = fmaf(l, shrink, s0 + s1);
            if (t) take_part(t - 1, last_v);
            if ((buffer += nq) >= 3) { buffer -= 3; phase ^= 1; }
            if (__any_sync(~0u, shrink != 1.0f))
#pragma unroll
                for (int d = 0; d < kOut / 2; ++d) o[d] = fma2(o[d], pair(shrink, shrink), 0);
        };
        for (int t = 0; t < tiles - 1; ++t) tile(t, std::false_type());
        if (tiles) {
            tile(tiles - 1, std::true_type());
            take_part(tiles - 1, drops.y);
        }
        if (kShare == 2) {
            sh.exchange[tiles & 1][wg][half][row] = l;
            asm volatile("bar.sync %0, 256;" ::"r"(1 + wg) : "memory");
            l += sh.exchange[tiles & 1][wg][half ^ 1][row];
        }
        // Rows of the result where the queries were (all products with them are done), and out from there, eight lanes a row.
        const bool live = i < a.QP && i / a.QW < qe.x && i % a.QW < qe.y && l != 0.0f;
        const float inv = live ? (1 << (int)kLift) / l : 0.0f;
        float4 *rows = reinterpret_cast<float4 *>(queries + wg * kBytes);
#pragma unroll
        for (int d = 0; d < kOut; d += 4) {
            float4 x;
            unpair(o[d / 2], x.x, x.y);
            unpair(o[d / 2 + 1], x.z, x.w);
            rows[row * (DP / 4) + ((half * kOut + d) / 4 ^ (row & 7))] =
                live ? make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        asm volatile("bar.sync %0, %1;" ::"r"(1 + wg), "n"(kWarps * 32) : "memory");
        float *out = a.out + (size_t)n * a.CB * a.QP * 32;
        const int lane = threadIdx.x & 31, c0 = (lane & 7) * 4, first = h * a.D;
#pragma unroll 4
        for (int r = (warp % kWarps) * 4 + (lane >> 3); r < kTile; r += kWarps * 4) {
            const int p = i0 + wg * kTile + r;
            if (p >= a.QP) break;
#pragma unroll
            for (int ch = c0; ch < DP; ch += 32) {
                const float4 x = rows[r * (DP / 4) + (ch / 4 ^ (r & 7))];
                if ((a.D & 3) == 0) {
                    if (ch < a.D) *reinterpret_cast<float4 *>(out + at(first + ch, p, a.QP)) = x;
                } else {
                    if (ch + 0 < a.D) out[at(first + ch + 0, p, a.QP)] = x.x;
                    if (ch + 1 < a.D) out[at(first + ch + 1, p, a.QP)] = x.y;
                    if (ch + 2 < a.D) out[at(first + ch + 2, p, a.QP)] = x.z;
                    if (ch + 3 < a.D) out[at(first + ch + 3, p, a.QP)] = x.w;
                }
            }
            if (h == a.heads - 1)
                for (int ch = a.heads * a.D + (lane & 7); ch < a.CB * 32; ch += 8) out[at(ch, p, a.QP)] = 0.0f;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (sh.gave_up && warp == loader) {                  // what is still on its way must land before the block ends
        for (int x = max(0, issued - c.ring); x < issued; ++x) mbar_wait(full + x % c.ring * 8, (x / c.ring) & 1, kDefaultWaitIters);
        for (int t = max(0, (issued + 1) / 2 - kPlaces); kGeneral && bias && t < (issued + 1) / 2; ++t) mbar_wait(placed + t % kPlaces * 8, t / kPlaces & 1, kDefaultWaitIters);
    }
    if (warp == issuer) tmem_dealloc(tmem, 512);
}

int padded(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : 128; }

template <int DP>
int launch(small_ctx *ctx, const AttnArgs &a, bool x3, cudaStream_t st) {
    static std::atomic<unsigned long long> tiled{0}, done[4] = {};
    const int tiles = ceil_div(a.KP, kTile);
    TcArgs c{a, tiles, 1, kMaxRing, 0, ctx->dev_status, ctx->wait_iters};
    const size_t most = ctx->max_smem_optin - 12288, tile = (size_t)DP * 512;
    // One tile a block where that still fits the SMs (batch 1, 8 heads of 64, 28 x 28: 31.5 -> 24.3 us; batch 4, 4 heads, 32 x 32 47.9 -> 38.8)
    if (DP < 128 && (long long)a.N * a.heads * ceil_div(a.QP, kTile) > ctx->sm_count) c.q_tiles = 2;
    while (c.ring > 2 && 1024 + (c.q_tiles + c.ring) * tile > most) --c.ring;
    if (a.bias) {
        // Rows of the copy lie so far apart that a warp's queries read different banks where their row of the plane ends, too.
        const int pitch = a.QW + (a.KW - 1 + 31) / 32 * 32;
        const int rows = c.q_tiles * kTile, y = (rows + a.QW - 2) / a.QW + 1;        // rows of the plane that such a run of pixels can touch
        const size_t table = sizeof(float) * ((size_t)(y < a.QH ? y : a.QH) + a.KH - 1) * pitch;
        const int fewest = 3 < c.ring ? 3 : c.ring;
        if (1024 + (c.q_tiles + fewest) * tile + table <= most) {
            while (1024 + (c.q_tiles + c.ring) * tile + table > most) --c.ring;
            c.table_floats = (int)(table / 4);
            c.a.pitch = pitch;
        }
    }
    const size_t values = sizeof(float) * kTile * (DP + 1);
    if (int s = allow_shared_memory(ctx, attention_tiles_kernel<DP>, tiled, values)) return s;
    launch_kernel(ctx, attention_tiles_kernel<DP>, dim3((unsigned)(2 * tiles), (unsigned)a.kv_heads, (unsigned)a.N), dim3(256), values, st, c.a, tiles);
    if (int s = check_launch(ctx)) return s;
    const size_t smem = 1024 + (c.q_tiles + c.ring) * tile + sizeof(float) * c.table_floats;
    const bool general = a.bias || a.cap > 0.0f;
    auto run = [&](auto *kern, int row_threads, std::atomic<unsigned long long> &d) {
        if (int s = allow_shared_memory(ctx, kern, d, most)) return s;
        launch_kernel(ctx, kern, dim3((unsigned)ceil_div(a.QP, c.q_tiles * kTile), (unsigned)a.heads, (unsigned)a.N), dim3(c.q_tiles * kTile * row_threads + 64), smem, st, c);
        return check_launch(ctx);
    };
    constexpr int kG = kRowThreads<DP, true>, kP = kRowThreads<DP, false>;
    return x3 ? general ? run(attention_tc_kernel<DP, true, true>, kG, done[0]) : run(attention_tc_kernel<DP, true, false>, kP, done[1])
              : general ? run(attention_tc_kernel<DP, false, true>, kG, done[2]) : run(attention_tc_kernel<DP, false, false>, kP, done[3]);
}

}  // namespace

size_t attention_tc_workspace(int N, int kv_heads, int D, int KP) {
    return (size_t)N * kv_heads * ceil_div(KP, kTile) * ((size_t)padded(D) * 1024 + 2 * sizeof(float)) + (size_t)N * ceil_div(KP, kTile) * kPlaceInts * sizeof(int);
}

int launch_attention_tc(small_ctx *ctx, const AttnArgs &a, bool x3, cudaStream_t st) {
    return padded(a.D) == 32 ? launch<32>(ctx, a, x3, st) : padded(a.D) == 64 ? launch<64>(ctx, a, x3, st) : launch<128>(ctx, a, x3, st);
}

}  // namespace small
