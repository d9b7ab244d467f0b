// lm.hpp -- element types, activations and wave reductions shared by the
// kernels of the language model operators (conv.hip, ssm.hip, logits.hip).
#pragma once

#include "device.hpp"

namespace ls {

// Elements are read as fp32 and rounded once (to nearest even) when stored.
template <class T>
__device__ __forceinline__ float to_f32(T v) {
    return (float)v;
}
template <class T>
__device__ __forceinline__ T from_f32(float v) {
    return (T)v;
}

// V consecutive elements: one wide access when all of them exist (global
// memory takes it at any element's alignment), else one by one up to `count`;
// the rest are 0.
template <class T, int V>
struct Pack {
    typedef T Vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    Vec v;
    __device__ __forceinline__ void load(const T* p, int count) {
        if (count >= V) {
            v = *reinterpret_cast<const Vec*>(p);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = i < count ? p[i] : T(0);
        }
    }
    __device__ __forceinline__ void store(T* p, int count) const {
        if (count >= V) {
            *reinterpret_cast<Vec*>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < count) p[i] = v[i];
        }
    }
};
template <class T>
struct Pack<T, 1> {
    T v[1];
    __device__ __forceinline__ void load(const T* p, int count) { v[0] = count > 0 ? *p : T(0); }
    __device__ __forceinline__ void store(T* p, int count) const {
        if (count > 0) *p = v[0];
    }
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float rcp_fast(float v) { return __builtin_amdgcn_rcpf(v); }

// 1 / (1 + e^-v), by the exponential and reciprocal instructions (1 ulp each).
__device__ __forceinline__ float sigmoid(float v) {
    return rcp_fast(1.0f + exp2_fast(-v * kLog2e));
}

// log(1 + e^v) = max(v, 0) + log(1 + e), e = e^-|v|.  w = 1 + e is rounded; what it
// lost, c = e - (w - 1), is put back as log(w + c) = log(w) + c / w, with c for c / w
// (c <= 2^-24, and w is near 1 where c counts).  Step sizes near e^-7 would
// otherwise lose half their bits.  A NaN, which the maximum drops, stays in e.
__device__ __forceinline__ float softplus(float v) {
    const float e = exp2_fast(-__builtin_fabsf(v) * kLog2e);
    const float w = 1.0f + e;
    const float c = e - (w - 1.0f);
    return __builtin_fmaf(__builtin_amdgcn_logf(w), kLn2, c) + __builtin_fmaxf(v, 0.0f);
}

// ------------------------------------------------ reductions inside a wave

template <int CTRL>
__device__ __forceinline__ float dpp_f(float v) {
    const int b = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, b, CTRL, 0xf, 0xf, true));
}

__device__ __forceinline__ float as_f32(unsigned b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ unsigned as_u32(float v) { return __builtin_bit_cast(unsigned, v); }

// Two sums over the pairs of lanes that differ in bit BIT, one to a lane of the
// pair: p's where the bit is 0, q's where it is 1.  Rows of 32 and of 16 lanes
// exchange halves by the swap instructions, lanes inside a row by DPP.
template <int BIT>
__device__ __forceinline__ float pair_sum(float p, float q, int lane) {
    if constexpr (BIT == 5) {
        const auto r = __builtin_amdgcn_permlane32_swap(as_u32(p), as_u32(q), false, false);
        return as_f32(r[0]) + as_f32(r[1]);
    } else if constexpr (BIT == 4) {
        const auto r = __builtin_amdgcn_permlane16_swap(as_u32(p), as_u32(q), false, false);
        return as_f32(r[0]) + as_f32(r[1]);
    } else {
        // row_ror:8; row_ror:12 and :4 (from four lanes up, and down); quad_perm
        constexpr int kP = BIT == 3 ? 0x128 : BIT == 2 ? 0x12C : BIT == 1 ? 0x4E : 0xB1;
        constexpr int kQ = BIT == 2 ? 0x124 : kP;
        p += dpp_f<kP>(p);
        q += dpp_f<kQ>(q);
        return (lane & (1 << BIT)) ? q : p;
    }
}

// Sums of K values over the lanes that differ in the given bits, shared out: a
// lane is left with v[j] = the sum of the former v[share_index<K, BITS...>(lane) + j],
// j < K / 2^(number of bits).
template <int K, int BIT, int... REST>
__device__ __forceinline__ int share_index(int lane) {
    int i = ((lane >> BIT) & 1) * (K / 2);
    if constexpr (sizeof...(REST) > 0) i += share_index<K / 2, REST...>(lane);
    return i;
}
template <int K, int BIT, int... REST, int N>
__device__ __forceinline__ void share_sums(float (&v)[N], int lane) {
    static_assert(K % 2 == 0 && K <= N, "every bit halves the sums");
#pragma unroll
    for (int i = 0; i < K / 2; ++i) v[i] = pair_sum<BIT>(v[i], v[i + K / 2], lane);
    if constexpr (sizeof...(REST) > 0) share_sums<K / 2, REST...>(v, lane);
}

// ------------------------------------------------ sums over partial results

// A workgroup of kSumThreads adds sums of `count` parts, part[k * stride + i] over k:
// each by SLICES threads, which take every SLICES-th part, joined in order.  The sum
// is returned to the threads of the first slice; all threads of the workgroup
// call.  Eight slices for long sums (of 306 parts: 38 us by one thread, 8 by eight),
// one for short ones, which would leave the others idle.
constexpr int kSumThreads = 256;
template <int SLICES>
constexpr int kSumOuts = kSumThreads / SLICES;
inline bool long_sum(int64_t count) { return count > 16; }

__device__ __forceinline__ float2 add_values(float2 a, float2 b) {
    return float2{a.x + b.x, a.y + b.y};
}
__device__ __forceinline__ float add_values(float a, float b) { return a + b; }

template <int SLICES, class V>
__device__ __forceinline__ V sum_parts(const V* part, int64_t count, int64_t stride, int64_t i) {
    constexpr int OUTS = kSumOuts<SLICES>;
    const int out = threadIdx.x % OUTS, slice = threadIdx.x / OUTS;
    V sum{};
#pragma unroll 8
    for (int64_t k = slice; k < count; k += SLICES) sum = add_values(sum, part[k * stride + i]);
    if constexpr (SLICES > 1) {
        __shared__ V s_part[SLICES][OUTS];
        s_part[slice][out] = sum;
        __syncthreads();
        if (slice == 0) {
#pragma unroll
            for (int j = 1; j < SLICES; ++j) sum = add_values(sum, s_part[j][out]);
        }
        __syncthreads();  // before a next call writes there
    }
    return sum;
}

}  // namespace ls
