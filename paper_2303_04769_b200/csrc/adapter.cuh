// What the kernels of adapted 1 x 1 convolutions share: sizes of the packed adapters and the call's arguments.
#pragma once

#include "entry.cuh"

namespace small {

// Packed adapters (small_pack_adapters), whatever is behind R, C or K being 0:
//   Down   float[adapters][CB][RP][32 channels]            RP = R rounded up to 8: rows of a channel block together, as activations are
//   Up     float[adapters][KB][RP][32 filters]
//   Up     [adapters][filter tiles][RB]{filters of the tile: 128 bytes, 32 high halves and 32 low ones of 32 ranks, swizzled}
//   Down   [adapters][chunks of 64 channels]{RQ rows of 128 bytes of high halves, the same of low ones, swizzled}     RQ = R rounded up to 16
//   [adapters]{int: Down's exponent; 3 unused; KB * 32 floats: what undoes the scaling of each row of Up}
// Filter tiles have eight channel blocks, the last one what is left.
struct AdapterShape {
    int C, K, R, CB, KB, RP, RB, RQ, chunks;
    size_t down, up, up_halves, down_halves;             // floats of one adapter
    size_t up_halves_at, down_halves_at, info_at, info, floats;
    AdapterShape(int adapters, int C, int K, int R) : C(C), K(K), R(R), CB(blocks_of(C)), KB(blocks_of(K)), RP((R + 7) / 8 * 8), RB(blocks_of(R)),
          RQ((R + 15) / 16 * 16), chunks((C + 63) / 64) {
        down = (size_t)CB * RP * 32;
        up = (size_t)KB * RP * 32;
        up_halves = (size_t)RB * KB * 32 * 32;
        down_halves = (size_t)chunks * RQ * 64;
        up_halves_at = (down + up) * adapters;
        down_halves_at = up_halves_at + up_halves * adapters;
        info_at = down_halves_at + down_halves * adapters;
        info = 4 + (size_t)KB * 32;
        floats = info_at + info * adapters;
    }
};
constexpr int kFilterTile = 8;           // channel blocks of filters

struct AdaptArgs {
    const float *in, *w, *bias, *packed, *scale;
    const int32_t *adapter;
    float *out;
    void *ws;
    int N, HW, adapters;
    bool relu, accumulate;
};

// adapter_tc.cu: the whole layer on the tensor cores, whether it pays, its workspace, and its operands
bool adapted_tc_preferred(int N, int C, int K, int HW, int R, int sms);
size_t adapted_tc_workspace(int N, int C, int K, int HW, int R);
int launch_adapted_tc(small_ctx *, const AdaptArgs &, const AdapterShape &, bool x3, cudaStream_t);
int launch_pack_halves(small_ctx *, const float *down, const float *up, float *packed, int adapters, const AdapterShape &, cudaStream_t);

}  // namespace small
