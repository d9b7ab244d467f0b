// ssm.hpp -- how the selective scan's channels and states lie on lanes and
// workgroups, forward (ssm.hip) and backward (ssm_back.hip).
#pragma once

#include "../../include/libscan.h"
#include "lm.hpp"

namespace ls {

constexpr int kSsmBlock = 16;  // steps between checkpoints

// LN lanes share a channel, each with SPL of its NP = LN * SPL states (indices
// past n are padding: A = B = C = 0).  With LN = 4 a quad is a channel, and a wave
// holds 16 channels; with LN = 16 the four lanes of a quad are four channels and
// the 16 quads hold the states.  Four waves to a workgroup.
template <int LN_, int SPL_>
struct SsmLanes {
    static_assert(LN_ == 4 || LN_ == 16, "a channel lies on a quad or across the quads");
    static constexpr int LN = LN_, SPL = SPL_, NP = LN * SPL, CPW = 64 / LN, CH = 4 * CPW;
    __device__ static __forceinline__ int channel(int lane) { return LN == 4 ? lane >> 2 : lane & 3; }
    __device__ static __forceinline__ int part(int lane) { return LN == 4 ? lane & 3 : lane >> 2; }
    // v[t], t < 16: this lane's share of a sum over its channel's states at step
    // t.  Calls put(t, sum) for the steps whose sums end up in this lane.
    template <class F>
    __device__ static __forceinline__ void sum_states(float (&v)[kSsmBlock], int lane, F put) {
        if constexpr (LN == 4) {
            quad_reduce<kSsmBlock>(v, lane);
#pragma unroll
            for (int j = 0; j < kSsmBlock / 4; ++j) put(quad_index<kSsmBlock>(lane, j), v[j]);
        } else {
            put(lane >> 2, quads_reduce16(v, lane));
        }
    }
    // The same for sums over the wave's channels, of one state index.
    template <class F>
    __device__ static __forceinline__ void sum_channels(float (&v)[kSsmBlock], int lane, F put) {
        if constexpr (LN == 4) {
            put(lane >> 2, quads_reduce16(v, lane));
        } else {
            quad_reduce<kSsmBlock>(v, lane);
#pragma unroll
            for (int j = 0; j < kSsmBlock / 4; ++j) put(quad_index<kSsmBlock>(lane, j), v[j]);
        }
    }
};

// The workgroup's row, group and channels c0 .. c0 + lim (all of one group).
struct SsmBlock {
    int b, g, k, c0, lim;
};
__device__ __forceinline__ SsmBlock ssm_block(const libscan_ssm& p, int nb, int ch,
                                              uint32_t index) {
    SsmBlock r;
    const int groups = (int)p.groups, per = (int)p.dim / groups;
    r.k = index % nb;
    const int bg = index / nb;
    r.g = bg % groups;
    r.b = bg / groups;
    r.c0 = r.g * per + r.k * ch;
    const int left = per - r.k * ch;
    r.lim = left < ch ? left : ch;
    return r;
}
inline int ssm_blocks(const libscan_ssm& p, int ch) {
    return (int)((p.dim / p.groups + ch - 1) / ch);
}

__device__ __forceinline__ int ssm_len(const libscan_ssm& p, int b) {
    if (!p.lengths) return (int)p.steps;
    const int n = p.lengths[b];
    return n < 0 ? 0 : n < (int)p.steps ? n : (int)p.steps;
}

}  // namespace ls
