// ssm.hpp -- how the selective scan's channels and states lie on lanes and
// workgroups, forward (ssm.hip) and backward (ssm_back.hip).
#pragma once

#include "../../include/libscan.h"
#include "lm.hpp"

namespace ls {

constexpr int kSsmBlock = 16;  // steps between checkpoints

// LN lanes share a channel, each with SPL of its NP = LN * SPL states (indices
// past n are padding: A = B = C = 0); the other lanes of the wave hold other
// channels.  Four waves to a workgroup.  Sums over the lanes of one kind are
// shared out over them (share_sums), which is cheapest over the high bits of
// the lane, so the larger number of lanes lies there.
template <int LN_, int SPL_>
struct SsmLanes {
    static_assert(LN_ == 8 || LN_ == 16, "lanes of a channel");
    static constexpr int LN = LN_, SPL = SPL_, NP = LN * SPL, CPW = 64 / LN, CH = 4 * CPW;
    __device__ static __forceinline__ int channel(int lane) {
        return LN == 16 ? lane & 3 : lane / LN;
    }
    __device__ static __forceinline__ int part(int lane) {
        return LN == 16 ? lane >> 2 : lane % LN;
    }
    // v[t], t < 16: this lane's share of a sum over its channel's states at step
    // t.  Calls put(t, sum) for the steps whose sums end up in this lane.
    template <class F>
    __device__ static __forceinline__ void sum_states(float (&v)[kSsmBlock], int lane, F put) {
        if constexpr (LN == 8)
            share<2, 1, 0>(v, lane, put);
        else
            share<5, 4, 3, 2>(v, lane, put);
    }
    // The same for sums over the wave's channels, of one state index.
    template <class F>
    __device__ static __forceinline__ void sum_channels(float (&v)[kSsmBlock], int lane, F put) {
        if constexpr (LN == 8)
            share<5, 4, 3>(v, lane, put);
        else
            share<0, 1>(v, lane, put);
    }

private:
    template <int... BITS, class F>
    __device__ static __forceinline__ void share(float (&v)[kSsmBlock], int lane, F put) {
        share_sums<kSsmBlock, BITS...>(v, lane);
        const int t = share_index<kSsmBlock, BITS...>(lane);
#pragma unroll
        for (int j = 0; j < kSsmBlock >> sizeof...(BITS); ++j) put(t + j, v[j]);
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
