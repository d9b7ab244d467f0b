// norm.hip -- layer norm over groups of channels, with the residual sum in front
// of it, and its gradients.
//
// y = (x - mean) rstd weight + bias over each group of a row's channels.  With
// w = dy weight and xhat = (x - mean) rstd,
//   dx = rstd (w - mean(w) - xhat mean(w xhat)) + dsum,
//   dweight = sum over rows of dy xhat, dbias = sum over rows of dy.
#include "launch.hpp"
#include "lm.hpp"

namespace ls {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v, float* s) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    __syncthreads();
    if (threadIdx.x % 64 == 0) s[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) v += s[i];
    return v;
}

// The workgroup's row and group.
struct Place {
    int64_t row, x, residual;
    int c0, per;
};
__device__ __forceinline__ Place place(const libscan_norm& p) {
    Place r;
    r.row = blockIdx.x / p.groups;
    r.per = (int)(p.dim / p.groups);
    r.c0 = (int)(blockIdx.x % p.groups) * r.per;
    const int64_t b = r.row / p.steps, t = r.row % p.steps;
    r.x = b * p.x_batch + t * p.x_step + r.c0;
    r.residual = b * p.residual_batch + t * p.residual_step + r.c0;
    return r;
}

template <class T, class W>
__global__ void __launch_bounds__(kThreads) k_norm(libscan_norm p, T* y, T* sum, float* stats) {
    __shared__ float s[kThreads / 64];
    const Place at = place(p);
    const T* x = (const T*)p.x + at.x;
    const T* res = p.residual ? (const T*)p.residual + at.residual : nullptr;
    const auto value = [&](int c) {
        const float v = to_f32(x[c]);
        return res ? to_f32(from_f32<T>(v + to_f32(res[c]))) : v;
    };
    float mean = 0.0f, var = 0.0f;
    for (int c = threadIdx.x; c < at.per; c += kThreads) mean += value(c);
    mean = block_sum(mean, s) / at.per;
    for (int c = threadIdx.x; c < at.per; c += kThreads) {
        const float d = value(c) - mean;
        var = __builtin_fmaf(d, d, var);
    }
    var = block_sum(var, s) / at.per;
    const float rstd = 1.0f / __builtin_sqrtf(var + (float)p.eps);
    const int64_t out = at.row * p.dim + at.c0;
    for (int c = threadIdx.x; c < at.per; c += kThreads) {
        const float v = value(c);
        float n = (v - mean) * rstd;
        if (p.weight) n *= to_f32(((const W*)p.weight)[at.c0 + c]);
        if (p.bias) n += to_f32(((const W*)p.bias)[at.c0 + c]);
        if (sum) sum[out + c] = from_f32<T>(v);
        y[out + c] = from_f32<T>(n);
    }
    if (stats && threadIdx.x == 0) {
        stats[2 * (int64_t)blockIdx.x] = mean;
        stats[2 * (int64_t)blockIdx.x + 1] = rstd;
    }
}

struct Grad {
    const void* dy;
    int64_t dy_batch, dy_step;
    const void* dsum;
    int64_t dsum_batch, dsum_step;
    const float* stats;
};

template <class T, class W>
__global__ void __launch_bounds__(kThreads) k_norm_dx(libscan_norm p, Grad g, T* dx) {
    __shared__ float s[kThreads / 64];
    const Place at = place(p);
    const int64_t b = at.row / p.steps, t = at.row % p.steps;
    const T* x = (const T*)p.x + at.x;
    const T* dy = (const T*)g.dy + b * g.dy_batch + t * g.dy_step + at.c0;
    const T* dsum = g.dsum ? (const T*)g.dsum + b * g.dsum_batch + t * g.dsum_step + at.c0 : nullptr;
    const float mean = g.stats[2 * (int64_t)blockIdx.x], rstd = g.stats[2 * (int64_t)blockIdx.x + 1];
    const auto weighted = [&](int c) {
        const float d = to_f32(dy[c]);
        return p.weight ? d * to_f32(((const W*)p.weight)[at.c0 + c]) : d;
    };
    float m0 = 0.0f, m1 = 0.0f;
    for (int c = threadIdx.x; c < at.per; c += kThreads) {
        const float w = weighted(c);
        m0 += w;
        m1 = __builtin_fmaf(w, (to_f32(x[c]) - mean) * rstd, m1);
    }
    m0 = block_sum(m0, s) / at.per;
    m1 = block_sum(m1, s) / at.per;
    T* out = dx + at.row * p.dim + at.c0;
    for (int c = threadIdx.x; c < at.per; c += kThreads) {
        float d = rstd * (weighted(c) - m0 - (to_f32(x[c]) - mean) * rstd * m1);
        if (dsum) d += to_f32(dsum[c]);
        out[c] = from_f32<T>(d);
    }
}

// Partial sums of dweight and dbias over `rows` rows, a column to a thread:
// part[block][2][dim].
template <class T>
__global__ void __launch_bounds__(kThreads)
    k_norm_dw(libscan_norm p, Grad g, int64_t rows, float* part) {
    const int c = blockIdx.y * kThreads + threadIdx.x;
    if (c >= p.dim) return;
    const int64_t all = p.batch * p.steps, lo = blockIdx.x * rows;
    const int64_t hi = lo + rows < all ? lo + rows : all;
    const int group = (int)(c / (p.dim / p.groups));
    float dw = 0.0f, db = 0.0f;
    for (int64_t r = lo; r < hi; ++r) {
        const int64_t b = r / p.steps, t = r % p.steps;
        const float d = to_f32(((const T*)g.dy)[b * g.dy_batch + t * g.dy_step + c]);
        const float x = to_f32(((const T*)p.x)[b * p.x_batch + t * p.x_step + c]);
        const float* st = g.stats + 2 * (r * p.groups + group);
        dw = __builtin_fmaf(d, (x - st[0]) * st[1], dw);
        db += d;
    }
    part[(2 * (int64_t)blockIdx.x) * p.dim + c] = dw;
    part[(2 * (int64_t)blockIdx.x + 1) * p.dim + c] = db;
}

template <int SLICES>
__global__ void __launch_bounds__(kSumThreads)
    k_norm_sum(const float* part, int64_t count, int64_t dim, float* dweight, float* dbias) {
    const int64_t i = blockIdx.x * (int64_t)kSumOuts<SLICES> + threadIdx.x % kSumOuts<SLICES>;
    const bool on = i < 2 * dim;
    const float v = sum_parts<SLICES>(part, on ? count : 0, 2 * dim, i);
    if (!on || threadIdx.x >= kSumOuts<SLICES>) return;
    float* out = i < dim ? dweight : dbias;
    if (out) out[i < dim ? i : i - dim] = v;
}

constexpr int64_t kPartRows = 64;
int64_t parts(const libscan_norm& p) {
    const int64_t rows = p.batch * p.steps;
    return (rows + kPartRows - 1) / kPartRows;
}

template <class F>
hipError_t by_type(const libscan_norm& p, F f) {
    const bool wide = p.weight_type == LIBSCAN_F32;
    if (p.type == LIBSCAN_F32) f(float(), float());
    else if (p.type == LIBSCAN_F16) wide ? f(_Float16(), float()) : f(_Float16(), _Float16());
    else wide ? f(__bf16(), float()) : f(__bf16(), __bf16());
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const libscan_norm& p, void* y, void* sum, float* stats,
                       hipStream_t stream) {
    const int64_t grid = p.batch * p.steps * p.groups;
    if (grid == 0 || p.dim == 0) return hipSuccess;
    return by_type(p, [&](auto t, auto w) {
        using T = decltype(t);
        k_norm<T, decltype(w)><<<(uint32_t)grid, kThreads, 0, stream>>>(p, (T*)y, (T*)sum, stats);
    });
}

size_t norm_scratch_bytes(const libscan_norm& p) { return (size_t)(parts(p) * 2 * p.dim * 4); }

hipError_t launch_norm_back(const libscan_norm& p, const void* dy, int64_t dy_batch,
                            int64_t dy_step, const void* dsum, int64_t dsum_batch,
                            int64_t dsum_step, const float* stats, void* dx, float* dweight,
                            float* dbias, void* scratch, hipStream_t stream) {
    const Grad g{dy, dy_batch, dy_step, dsum, dsum_batch, dsum_step, stats};
    const int64_t grid = p.batch * p.steps * p.groups;
    if (p.dim == 0) return hipSuccess;
    float* part = (float*)scratch;
    return by_type(p, [&](auto t, auto w) {
        using T = decltype(t);
        if (grid) {
            k_norm_dx<T, decltype(w)><<<(uint32_t)grid, kThreads, 0, stream>>>(p, g, (T*)dx);
            k_norm_dw<T><<<dim3((uint32_t)parts(p), (uint32_t)((p.dim + kThreads - 1) / kThreads)),
                           kThreads, 0, stream>>>(p, g, kPartRows, part);
        }
        k_norm_sum<8><<<(uint32_t)((2 * p.dim + kSumOuts<8> - 1) / kSumOuts<8>), kSumThreads, 0,
                        stream>>>(part, parts(p), p.dim, dweight, dbias);
    });
}

}  // namespace ls
