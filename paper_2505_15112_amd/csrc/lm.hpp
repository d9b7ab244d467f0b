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

// Sums of K values over the four lanes of a quad, shared out: lane q of the
// quad is left with v[j] = the sum of the former v[quad_index(q, j)], j < K / 4.
template <int K>
__device__ __forceinline__ int quad_index(int lane, int j) {
    return (lane & 1) * (K / 2) + ((lane >> 1) & 1) * (K / 4) + j;
}
template <int K>
__device__ __forceinline__ void quad_reduce(float (&v)[K], int lane) {
    static_assert(K % 4 == 0, "a quad shares out multiples of four sums");
#pragma unroll
    for (int i = 0; i < K / 2; ++i) {
        const float p = v[i] + dpp_f<0xB1>(v[i]);                  // quad_perm 1,0,3,2
        const float q = v[i + K / 2] + dpp_f<0xB1>(v[i + K / 2]);
        v[i] = (lane & 1) ? q : p;
    }
#pragma unroll
    for (int i = 0; i < K / 4; ++i) {
        const float p = v[i] + dpp_f<0x4E>(v[i]);                  // quad_perm 2,3,0,1
        const float q = v[i + K / 4] + dpp_f<0x4E>(v[i + K / 4]);
        v[i] = (lane & 2) ? q : p;
    }
}

__device__ __forceinline__ float as_f32(unsigned b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ unsigned as_u32(float v) { return __builtin_bit_cast(unsigned, v); }

// Sums of 16 values over the 16 quads of the wave (lanes of one place in
// their quads), shared out: the returned value is the sum of v[lane >> 2].
// Halves are exchanged by the two swap instructions (rows of 32 and 16 lanes),
// then inside rows by rotations.
__device__ __forceinline__ float quads_reduce16(float (&v)[16], int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(as_u32(v[i]), as_u32(v[i + 8]), false,
                                                        false);
        v[i] = as_f32(r[0]) + as_f32(r[1]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(as_u32(v[i]), as_u32(v[i + 4]), false,
                                                        false);
        v[i] = as_f32(r[0]) + as_f32(r[1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float p = v[i] + dpp_f<0x128>(v[i]);  // row_ror:8
        const float q = v[i + 2] + dpp_f<0x128>(v[i + 2]);
        v[i] = (lane & 8) ? q : p;
    }
    const float p = v[0] + dpp_f<0x12C>(v[0]);  // row_ror:12: from four lanes up
    const float q = v[1] + dpp_f<0x124>(v[1]);  // row_ror:4: from four lanes down
    return (lane & 4) ? q : p;
}

}  // namespace ls
