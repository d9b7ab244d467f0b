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

// ------------------------------------------------ a channel to a lane

typedef const __attribute__((address_space(4))) float* ScalarPtr;

// B and C as fp32, in groups of GP states (GP of B, then GP of C; padding and the
// steps past a row's tokens are 0), as the scanning waves read them with scalar
// loads: one group at a time, the next one on its way while the last is used.
template <int NP>
struct LaneGroups {
    static constexpr int GP = NP < 16 ? NP : 16, NG = NP / GP;
    float v[2 * GP];
    template <int COUNT>
    __device__ __forceinline__ void load(ScalarPtr p) {
        asm volatile("" : "+s"(p));  // not earlier than here
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = p[i];
    }
};

// Waits for the scalar loads in flight, which return in no order, before new
// ones start, and keeps the compiler from mixing the two.
__device__ __forceinline__ void scalar_loads_done() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
}

// Waves of a workgroup: neighbours in channels, on the same steps, so that all
// but the first to get there find B and C in the scalar cache.
constexpr int kLaneWaves = 8;

// The channel block and chunk of steps of a wave.
struct LaneBlock {
    SsmBlock k;
    int c, t0, end, len;  // steps t0 .. end of chunk c are this wave's; end <= len
    uint32_t lo;          // this lane's channel after k.c0; lanes past the last channel double
                          // it, and store what it stores
};
__device__ __forceinline__ LaneBlock lane_block(const libscan_ssm& p, int nb, int chunk, int c) {
    LaneBlock r;
    r.k = ssm_block(p, nb, kWave, blockIdx.x * kLaneWaves + uni(threadIdx.x / kWave));
    r.c = c;
    r.len = ssm_len(p, r.k.b);
    r.t0 = r.c * chunk;
    r.end = r.t0 + chunk < r.len ? r.t0 + chunk : r.len;
    const int lane = threadIdx.x % kWave;
    r.lo = (uint32_t)(lane < r.k.lim ? lane : r.k.lim - 1);
    return r;
}

// A row of a tensor at one step after the other: the address is uniform and
// stays in one pair of scalar registers (the empty asm keeps the compiler from
// holding the multiples of the stride instead), the lanes add their channel.
template <class T>
struct StepPtr {
    __attribute__((address_space(1))) T* p;
    int64_t stride;
    __device__ __forceinline__ StepPtr(T* first, int64_t step)
        : p((__attribute__((address_space(1))) T*)first), stride(step) {}
    __device__ __forceinline__ void next() {
        p += stride;
        asm("" : "+s"(p));
    }
};

// The step sizes of COUNT steps, in the lane that owns the channel (one branch
// for all of them: branches between the steps would keep them apart).
template <int COUNT, class T>
__device__ __forceinline__ void step_sizes(const libscan_ssm& p, const T (&dt)[COUNT], float bias,
                                           float (&delta)[COUNT]) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) delta[i] = to_f32(dt[i]) + bias;
    if (p.softplus) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) delta[i] = softplus(delta[i]);
    }
}

constexpr int kAhead = 8;  // steps whose inputs a lane loads together

// A lane's states (or rates): `have` consecutive floats, 0 after them.
template <int NP>
__device__ __forceinline__ void load_states(const float* p, int have, float (&v)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; i += 4) {
        Pack<float, 4> w;
        w.load(p + i, have - i);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i + j] = w.v[j];
    }
}
template <int NP>
__device__ __forceinline__ void store_states(float* p, int have, const float (&v)[NP]) {
#pragma unroll
    for (int i = 0; i < NP; i += 4) {
        Pack<float, 4> w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w.v[j] = v[i + j];
        w.store(p + i, have - i);
    }
}

// B and C of the whole call for the scalar loads: `np` states (8, 16, 32 or 64) and
// ssm_bc_bytes of memory.
size_t ssm_bc_bytes(const libscan_ssm& p, int np);
void launch_ssm_bc(const libscan_ssm& p, int np, float* bc, hipStream_t stream);

// The states that chunks start from, in the place of what they end in (chunk x
// batch x dim x np; `sums`: their sums of delta): forward from init (nullable, batch x
// dim x n) through chunk 0, 1, ..., or backward through the last, the one before, ...
// The chunk that comes last in that order has no end to read.
void launch_ssm_starts(const libscan_ssm& p, int np, const float* init, float* ends,
                       const float* sums, int chunks, bool backward, hipStream_t stream);

}  // namespace ls
