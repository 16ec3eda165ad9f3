// Attention whose keys and values of a head fit a block's shared memory, FP32 multiply-adds in every math mode: bound by the launch, then by
// what shared memory hands out.
//
// A block holds the keys and values of one key head and takes a share of its rows (queries of the heads that read them).  A warp takes four
// rows at a time: two keys a lane for the scores, which go through shared memory; then eight keys of each row for the bias, the cap, the
// maximum and the weights, every score being known; then eight lanes a key's channels for the sums, four keys at a time.  Few instructions matter
// more than any of this: what a block runs once it fetches from L2 first (2 x 3 planes: four rows' cap and
// bias unrolled 10 us, now 4.6).  8 heads of 64, 7 x 7 with a bias: batch 8 6.7 us, 64 25.6.
#include "attention.cuh"

namespace small {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kRows = 4;       // rows a warp takes at a time

struct SmallArgs {
    AttnArgs a;
    int rows, share;                                     // rows of a key head, rows of a block
    int held, scored;                                    // keys held: a multiple of 4; scores held: of 64
};

__host__ __device__ constexpr int key_pitch(int DP) { return DP + 4; }       // eight neighbouring keys' vectors in different banks

template <int DP, bool kGeneral>
__global__ void __launch_bounds__(kThreads, 2) attention_small_kernel(const SmallArgs f) {
    constexpr int kVec = DP / 32, kPitch = key_pitch(DP);
    extern __shared__ float4 held[];
    const AttnArgs &a = f.a;
    float *Ks = reinterpret_cast<float *>(held), *Vs = Ks + f.held * kPitch, *Qs = Vs + f.held * DP, *Ps = Qs + kWarps * kRows * DP;
    int *koff = reinterpret_cast<int *>(Ps + kWarps * f.scored * kRows);
    grid_dep_sync();
    grid_dep_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = lane >> 3, c0 = (lane & 7) * 4;
    const int hk = blockIdx.y, n = blockIdx.z, share = a.heads / a.kv_heads;
    const int2 qe = extent(a.q_ext, n, a.QH, a.QW), ke = extent(a.k_ext, n, a.KH, a.KW);
    const int keys = ke.x * ke.y;
    const float *q = a.q + n * a.q_stride, *k = a.k + n * a.k_stride, *v = a.v + n * a.v_stride;
    const bool capping = a.cap > 0.0f, biased = kGeneral && a.bias;
    const float cap2 = a.cap * kLog2e, over_cap = capping ? 1.0f / a.cap : 0.0f, unit = capping ? a.scale : a.scale * kLog2e;

    for (int i = tid; i < f.held * (DP / 4); i += kThreads) {
        const int j = i / (DP / 4), c = i % (DP / 4) * 4;
        const bool in = j < keys;
        int p = in ? j : 0;
        if (kGeneral && in && ke.y != a.KW) p = j / ke.y * a.KW + j % ke.y;
        float *ks = Ks + j * kPitch + c, *vs = Vs + j * DP + c;
        if ((a.D & 3) == 0) {
            const bool some = in && c < a.D;
            const size_t e = some ? at(hk * a.D + c, p, a.KP) : 0;
            copy16_or_clear((uint32_t)__cvta_generic_to_shared(ks), k + e, some);
            copy16_or_clear((uint32_t)__cvta_generic_to_shared(vs), v + e, some);
        } else {
            *reinterpret_cast<float4 *>(ks) = load4(k, hk * a.D, in ? c : DP, a.D, p, a.KP);
            *reinterpret_cast<float4 *>(vs) = load4(v, hk * a.D, in ? c : DP, a.D, p, a.KP);
        }
    }
    copy_commit();
    if (biased)
        for (int j = tid; j < keys; j += kThreads) koff[j] = of_key(a, j / ke.y, j % ke.y);

    float *qs = Qs + warp * kRows * DP, *ps = Ps + warp * f.scored * kRows;
    const int first = blockIdx.x * f.share, last = min(first + f.share, f.rows), mine = lane & 3;
    float *out = a.out + (size_t)n * a.CB * a.QP * 32;
    bool waited = false;
#pragma unroll 1
    for (int r0 = first + warp * kRows; r0 < last || !waited; r0 += kWarps * kRows) {
        // this group's row; those behind the last are computed as the last and not written
        const int row = min(r0 + group, last - 1), h = hk * share + row / a.QP, i = row % a.QP;
#pragma unroll
        for (int c = 0; c < kVec; ++c) {
            float4 z = load4(q, h * a.D, c * 32 + c0, a.D, i, a.QP);
            z.x *= unit; z.y *= unit; z.z *= unit; z.w *= unit;
            *reinterpret_cast<float4 *>(qs + group * DP + c * 32 + c0) = z;
        }
        const float *bias = nullptr;                     // of row `mine`
        if (biased) {
            const long long place = (long long)h * (a.QH + a.KH - 1) * (a.QW + a.KW - 1) + of_query(a, i);
            bias = a.bias + __shfl_sync(~0u, place, mine * 8);
        }
        if (!waited) { copy_wait<0>(); __syncthreads(); waited = true; } else __syncwarp();
        if (r0 >= last) break;
#pragma unroll 1
        for (int j0 = 0; j0 < f.scored; j0 += 64) {
            float s[2][kRows] = {};
            const float *ks[2] = {Ks + min(j0 + lane, f.held - 1) * kPitch, Ks + min(j0 + 32 + lane, f.held - 1) * kPitch};
#pragma unroll 4
            for (int d = 0; d < DP; d += 4) {
                const float4 x0 = *reinterpret_cast<const float4 *>(ks[0] + d), x1 = *reinterpret_cast<const float4 *>(ks[1] + d);
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const float4 y = *reinterpret_cast<const float4 *>(qs + r * DP + d);
                    s[0][r] = fmaf(x0.x, y.x, fmaf(x0.y, y.y, fmaf(x0.z, y.z, fmaf(x0.w, y.w, s[0][r]))));
                    s[1][r] = fmaf(x1.x, y.x, fmaf(x1.y, y.y, fmaf(x1.z, y.z, fmaf(x1.w, y.w, s[1][r]))));
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) *reinterpret_cast<float4 *>(ps + (j0 + u * 32 + lane) * kRows) = make_float4(s[u][0], s[u][1], s[u][2], s[u][3]);
        }
        __syncwarp();
        float m = -INFINITY, total = 0.0f;               // of row `mine`, eight keys of it at a time
#pragma unroll 1
        for (int j = lane >> 2; j < f.scored; j += 32) {
            float s[4], b[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                s[u] = ps[(j + u * 8) * kRows + mine];
                if (biased) b[u] = j + u * 8 < keys ? bias[-koff[j + u * 8]] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (kGeneral && capping) s[u] = capped(s[u], cap2, over_cap);
                if (biased) s[u] += powers_of_two(b[u]);
                if (j + u * 8 >= keys) s[u] = -INFINITY;
                m = fmaxf(m, s[u]);
                ps[(j + u * 8) * kRows + mine] = s[u];
            }
        }
#pragma unroll
        for (int w = 4; w < 32; w *= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, w));
        if (m == -INFINITY) m = 0.0f;                    // no key has any weight
#pragma unroll 1
        for (int j = lane >> 2; j < f.scored; j += 32) {
            float w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) w[u] = exp2_fast(ps[(j + u * 8) * kRows + mine] - m);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                ps[(j + u * 8) * kRows + mine] = w[u];
                total += w[u];
            }
        }
#pragma unroll
        for (int w = 4; w < 32; w *= 2) total += __shfl_xor_sync(~0u, total, w);
        total = __shfl_sync(~0u, total, group);
        __syncwarp();
        float4 o[kRows][kVec] = {};
#pragma unroll 2
        for (int j = group; j < f.held; j += 4) {        // a group's own keys
            const float4 w4 = *reinterpret_cast<const float4 *>(ps + j * kRows);
            const float w[kRows] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
            for (int c = 0; c < kVec; ++c) {
                const float4 y = *reinterpret_cast<const float4 *>(Vs + j * DP + c * 32 + c0);
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    o[r][c].x = fmaf(w[r], y.x, o[r][c].x); o[r][c].y = fmaf(w[r], y.y, o[r][c].y);
                    o[r][c].z = fmaf(w[r], y.z, o[r][c].z); o[r][c].w = fmaf(w[r], y.w, o[r][c].w);
                }
            }
        }
        // the four groups' sums: two of the rows to the other half of the warp, then one of those to the neighbouring group
        const bool up = group >> 1, odd = group & 1;
        auto halve = [](float low, float high, bool keep_high, int w) { return (keep_high ? high : low) + __shfl_xor_sync(~0u, keep_high ? low : high, w); };
        auto halve4 = [&](const float4 &low, const float4 &high, bool keep_high, int w) {
            return make_float4(halve(low.x, high.x, keep_high, w), halve(low.y, high.y, keep_high, w), halve(low.z, high.z, keep_high, w), halve(low.w, high.w, keep_high, w));
        };
        const bool real = r0 + group < last, live = i / a.QW < qe.x && i % a.QW < qe.y && total != 0.0f;
        const float inv = live ? 1.0f / total : 0.0f;
#pragma unroll
        for (int c = 0; c < kVec; ++c) {
            const float4 z = halve4(halve4(o[0][c], o[2][c], up, 16), halve4(o[1][c], o[3][c], up, 16), odd, 8);
            const float part[4] = {z.x, z.y, z.z, z.w};
            const int d = c * 32 + c0;
            if (real && d < a.D) {
                if ((a.D & 3) == 0) {
                    *reinterpret_cast<float4 *>(out + at(h * a.D + d, i, a.QP)) = live ? make_float4(z.x * inv, z.y * inv, z.z * inv, z.w * inv) : make_float4(0.f, 0.f, 0.f, 0.f);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (d + e < a.D) out[at(h * a.D + d + e, i, a.QP)] = live ? part[e] * inv : 0.0f;
                }
            }
        }
        if (real && h == a.heads - 1)                    // pad lanes
            for (int c = a.heads * a.D + (lane & 7); c < a.CB * 32; c += 8) out[at(c, i, a.QP)] = 0.0f;
        __syncwarp();                                    // the next rows overwrite these
    }
}

int up(int x, int unit) { return ceil_div(x, unit) * unit; }

template <int DP>
size_t shared_bytes(int KP) {
    const size_t held = up(KP, 4), scored = up(KP, 64);
    return sizeof(float) * (held * (key_pitch(DP) + DP) + kWarps * kRows * DP + kWarps * scored * kRows + held);
}

template <int DP, bool kGeneral>
int launch(small_ctx *ctx, const SmallArgs &f, cudaStream_t st) {
    static std::atomic<unsigned long long> done{0};
    const size_t smem = shared_bytes<DP>(f.a.KP);
    if (int s = allow_shared_memory(ctx, attention_small_kernel<DP, kGeneral>, done, kSmallShared)) return s;
    launch_kernel(ctx, attention_small_kernel<DP, kGeneral>, dim3((unsigned)ceil_div(f.rows, f.share), (unsigned)f.a.kv_heads, (unsigned)f.a.N), dim3(kThreads), smem, st, f);
    return check_launch(ctx);
}

template <int DP>
int launch(small_ctx *ctx, const AttnArgs &a, cudaStream_t st) {
    SmallArgs f{a, a.QP * (a.heads / a.kv_heads), 0, up(a.KP, 4), up(a.KP, 64)};
    // two blocks an SM, where the rows are that many
    const int parts = (int)std::min<long long>(ceil_div(f.rows, kWarps * kRows), std::max<long long>(1, 2ll * kSmCount / ((long long)a.N * a.kv_heads)));
    f.share = up(ceil_div(f.rows, parts), kRows);
    return a.bias || a.cap > 0.0f || a.k_ext ? launch<DP, true>(ctx, f, st) : launch<DP, false>(ctx, f, st);
}

}  // namespace

size_t attention_small_bytes(int D, int KP) {
    return D <= 32 ? shared_bytes<32>(KP) : D <= 64 ? shared_bytes<64>(KP) : shared_bytes<128>(KP);
}

int launch_attention_small(small_ctx *ctx, const AttnArgs &a, cudaStream_t st) {
    return a.D <= 32 ? launch<32>(ctx, a, st) : a.D <= 64 ? launch<64>(ctx, a, st) : launch<128>(ctx, a, st);
}

}  // namespace small
