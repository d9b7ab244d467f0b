// conv.hip -- the causal depthwise convolution in front of the selective scan.
//
// y[t] = f(bias + sum_j w[j] x[t - (W-1) + j]) per channel, W = 2..4.  HBM bounds
// it: a thread owns 8 bytes of channels and a run of steps, so that every
// input is loaded once (but for the W-1 in front of a run) and the window
// slides through registers.  The window is the inputs themselves, in their type;
// sums and the weights' gradients are fp32, and a result is rounded once.
#include "launch.hpp"
#include "lm.hpp"

#include "../../include/libscan.h"

namespace ls {

namespace {

constexpr int kThreads = 256;
constexpr int kRun = 8;       // steps a thread owns, forward
// Backward: a thread's run is W-1 steps that only open the window, and these.
constexpr int kSteady = 28;
constexpr int kAhead = 4;     // steps a thread loads ahead, backward
constexpr int kBackV = 4;     // channels of a thread, backward
constexpr int kBackSide = 32; // threads of a workgroup over channels, backward
constexpr int kBackRuns = kThreads / kBackSide;

__host__ __device__ constexpr int back_run(int width) { return kSteady + width - 1; }
// workgroups over the steps of a row, backward (one even where there are none,
// for the gradient of the first state)
__host__ __device__ inline int back_runs(int64_t steps, int width) {
    const int per = back_run(width) * kBackRuns;
    return steps ? (int)((steps + per - 1) / per) : 1;
}

__device__ __forceinline__ int conv_len(const libscan_conv& p, int b) {
    if (!p.lengths) return (int)p.steps;
    const int n = p.lengths[b];
    return n < 0 ? 0 : n < (int)p.steps ? n : (int)p.steps;
}

// weight and bias of V channels from c0 on, which lie together in memory
template <class P, int W, int V>
__device__ __forceinline__ void load_weights_as(const P* weight, const P* b, int c0, int count,
                                                float (&w)[W][V], float (&bias)[V]) {
    Pack<P, V> row[W], br;
#pragma unroll
    for (int k = 0; k < W; ++k)
        row[k].load(weight + (int64_t)c0 * W + k * V, count >= V ? V : count * W - k * V);
    br.load(b + c0, b ? count : 0);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][i] = to_f32(row[(i * W + j) / V].v[(i * W + j) % V]);
        bias[i] = to_f32(br.v[i]);
    }
}
template <class T, int W, int V>
__device__ __forceinline__ void load_weights(const libscan_conv& p, int c0, int count,
                                             float (&w)[W][V], float (&bias)[V]) {
    if (p.weight_type == LIBSCAN_F32)
        load_weights_as<float, W, V>((const float*)p.weight, (const float*)p.bias, c0, count, w,
                                     bias);
    else
        load_weights_as<T, W, V>((const T*)p.weight, (const T*)p.bias, c0, count, w, bias);
}

// x of step t, which may lie in the first state (t >= -(W-1)), or past the end (0)
template <class T, int W, int V>
__device__ __forceinline__ void load_step(const libscan_conv& p, const T* px, const T* ps, int t,
                                          int len, int count, Pack<T, V>& v) {
    if (t >= 0)
        v.load(px + t * p.x_step, t < len ? count : 0);
    else
        v.load(ps + (t + W - 1) * p.dim, ps ? count : 0);
}

// bf16, W = 4: 1 x 2048 x 4096 in 12 us, 4 x 2048 x 4096 in 35 us (134 MB: 3.9 TB/s).
// Runs of 4, 8 and 16 steps by 8 and 16 bytes of channels were measured: longer
// runs and wider threads leave too few waves, shorter runs load the W-1 inputs in
// front of them too often.
template <class T, int W>
__global__ __launch_bounds__(kThreads) void k_conv(libscan_conv p, T* y, T* state_out) {
    constexpr int V = 8 / sizeof(T);
    const int dim = (int)p.dim, steps = (int)p.steps;
    const int64_t nc = (dim + V - 1) / V, nr = steps ? (steps + kRun - 1) / kRun : 1;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= nc * nr * p.batch) return;
    const int c0 = (int)(id % nc) * V, r = (int)(id / nc % nr), b = (int)(id / (nc * nr));
    const int count = dim - c0, len = conv_len(p, b), t0 = r * kRun;
    const T* px = (const T*)p.x + b * p.x_batch + c0;
    const T* ps = p.state ? (const T*)p.state + (int64_t)b * (W - 1) * dim + c0 : nullptr;
    T* py = y + (int64_t)b * steps * dim + c0;
    float w[W][V], bias[V];
    load_weights<T, W, V>(p, c0, count, w, bias);
    Pack<T, V> x[kRun + W - 1];
#pragma unroll
    for (int i = 0; i < kRun + W - 1; ++i)
        load_step<T, W, V>(p, px, ps, t0 + i - (W - 1), len, count, x[i]);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
        const int t = t0 + i;
        if (t < steps) {
            Pack<T, V> out;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                float u = bias[c];
#pragma unroll
                for (int j = 0; j < W; ++j) u = __builtin_fmaf(w[j][c], to_f32(x[i + j].v[c]), u);
                if (p.silu) u *= sigmoid(u);
                out.v[c] = from_f32<T>(t < len ? u : 0.0f);
            }
            out.store(py + (int64_t)t * dim, count);
        }
    }
    // the last W-1 inputs, by the thread of the row's last token
    if (state_out && (len > 0 ? (len - 1) / kRun : 0) == r) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            Pack<T, V> v;
            load_step<T, W, V>(p, px, ps, len - (W - 1) + j, len, count, v);
            v.store(state_out + ((int64_t)b * (W - 1) + j) * dim + c0, count);
        }
    }
}

// One token against the pool: 64 rows of 4096 channels in 4 us, launch and latency.
template <class T, int W>
__global__ __launch_bounds__(kThreads) void k_conv_step(libscan_conv p, T* states,
                                                        int64_t n_states, const int32_t* slots,
                                                        T* y) {
    constexpr int V = 8 / sizeof(T);
    const int dim = (int)p.dim;
    const int64_t nc = (dim + V - 1) / V;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= nc * p.batch) return;
    const int c0 = (int)(id % nc) * V, b = (int)(id / nc), count = dim - c0;
    const int64_t slot = slots ? slots[b] : b;
    T* py = y + (int64_t)b * dim + c0;
    Pack<T, V> out;
    if (slot < 0 || slot >= n_states) {
#pragma unroll
        for (int c = 0; c < V; ++c) out.v[c] = T(0);
        out.store(py, count);
        return;
    }
    T* ps = states + slot * (W - 1) * dim + c0;
    Pack<T, V> x[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) x[j].load(ps + (int64_t)j * dim, count);
    x[W - 1].load((const T*)p.x + b * p.x_batch + c0, count);
    float w[W][V], bias[V];
    load_weights<T, W, V>(p, c0, count, w, bias);
#pragma unroll
    for (int c = 0; c < V; ++c) {
        float u = bias[c];
#pragma unroll
        for (int j = 0; j < W; ++j) u = __builtin_fmaf(w[j][c], to_f32(x[j].v[c]), u);
        if (p.silu) u *= sigmoid(u);
        out.v[c] = from_f32<T>(u);
    }
    out.store(py, count);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) x[j + 1].store(ps + (int64_t)j * dim, count);
}

struct BackArgs {
    const void* dy;
    int64_t dy_batch, dy_step;
    const void* dstate_out;
    void *dx, *dstate;
    float* part;  // [row of blocks][W + 1][dim]: sums of dweight's columns and of dbias
};

// Gradients.  g[t] = dy[t] f'(u[t]), u formed again; dx[t] = sum_j w[j] g[t + W-1 - j],
// so a thread forms g of its run and of the W-1 steps behind it.  4 x 2048 x 4096,
// bf16, W = 4: 55 us for 201 MB, 3.7 TB/s; the inner loop has no branches (73 us
// with them), and loads kAhead steps ahead of what it uses.
template <class T, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void k_conv_back(libscan_conv p, BackArgs o) {
    constexpr int V = kBackV;
    __shared__ float s_sum[kBackRuns][W + 1][kBackSide * V];
    const int dim = (int)p.dim, steps = (int)p.steps;
    const int side = threadIdx.x % kBackSide, run = threadIdx.x / kBackSide;
    const int nc = (dim + kBackSide * V - 1) / (kBackSide * V);
    const int nr = back_runs(steps, W);
    const int cb = blockIdx.x % nc, part = blockIdx.x / nc;  // part = b * nr + rb
    const int b = part / nr, rb = part % nr;
    const int c0 = (cb * kBackSide + side) * V, count = dim - c0, len = conv_len(p, b);
    const int t0 = (rb * kBackRuns + run) * back_run(W);
    const T* px = (const T*)p.x + b * p.x_batch + c0;
    const T* ps = p.state ? (const T*)p.state + (int64_t)b * (W - 1) * dim + c0 : nullptr;
    const T* pdy = (const T*)o.dy + b * o.dy_batch + c0;
    const T* pso = o.dstate_out ? (const T*)o.dstate_out + (int64_t)b * (W - 1) * dim + c0 : nullptr;
    T* pdx = (T*)o.dx + (int64_t)b * steps * dim + c0;
    float w[W][V], bias[V], dw[W][V], db[V];
    load_weights<T, W, V>(p, c0, count, w, bias);
#pragma unroll
    for (int c = 0; c < V; ++c) {
        db[c] = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][c] = 0.0f;
    }
    if (count > 0 && (t0 < steps || t0 == 0)) {
        float x[W][V];        // x[t - (W-1)] .. x[t]
        float g[W][V] = {};   // g[t - (W-1)] .. g[t]
        // (no output of an empty row reads its first state)
        const int open = len > 0 ? count : 0;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            Pack<T, V> v;
            load_step<T, W, V>(p, px, ps, t0 - (W - 1) + j, len, open, v);
#pragma unroll
            for (int c = 0; c < V; ++c) x[j][c] = to_f32(v.v[c]);
        }
        auto load = [&](int t, Pack<T, V>& xt, Pack<T, V>& dy) {
            const int has = t < len ? count : 0;
            xt.load(px + t * p.x_step, has);
            dy.load(pdy + t * o.dy_step, has);
        };
        // g of step t, and what it gives the weights
        auto form = [&](int t, const Pack<T, V>& xt, const Pack<T, V>& dy, bool own) {
#pragma unroll
            for (int c = 0; c < V; ++c) {
                x[W - 1][c] = to_f32(xt.v[c]);
                float gv = to_f32(dy.v[c]);
                if (SILU) {
                    float u = bias[c];
#pragma unroll
                    for (int j = 0; j < W; ++j) u = __builtin_fmaf(w[j][c], x[j][c], u);
                    const float sig = sigmoid(u);
                    gv *= sig * __builtin_fmaf(u, 1.0f - sig, 1.0f);
                }
                g[W - 1][c] = t < len ? gv : 0.0f;
                // Past the row's end g is 0, and inputs that are infinite or NaN must not meet
                // it.  (With the silu they have made NaN of the last outputs' g already, and
                // with it of all that they could spoil.)
                if (own) {
                    db[c] += g[W - 1][c];
#pragma unroll
                    for (int j = 0; j < W; ++j)
                        dw[j][c] = __builtin_fmaf(g[W - 1][c], SILU || t < len ? x[j][c] : 0.0f,
                                                  dw[j][c]);
                }
            }
        };
        // the gradient of input t - (W-1), which the W outputs up to t read
        auto gather = [&](int t, Pack<T, V>& out) {
            const int ti = t - (W - 1);
            float v[V];
#pragma unroll
            for (int c = 0; c < V; ++c) {
                v[c] = w[0][c] * g[W - 1][c];
#pragma unroll
                for (int j = 1; j < W; ++j) v[c] = __builtin_fmaf(w[j][c], g[W - 1 - j][c], v[c]);
            }
            const int j0 = ti - (len - (W - 1));  // its place in the last state
            if (pso && j0 >= 0 && ti < len) {
                Pack<T, V> so;
                so.load(pso + (int64_t)j0 * dim, count);
#pragma unroll
                for (int c = 0; c < V; ++c) v[c] += to_f32(so.v[c]);
            }
#pragma unroll
            for (int c = 0; c < V; ++c) out.v[c] = from_f32<T>(ti < len ? v[c] : 0.0f);
        };
        auto move = [&]() {
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    x[j][c] = x[j + 1][c];
                    g[j][c] = g[j + 1][c];
                }
        };
        auto store = [&](int t, const Pack<T, V>& out) {
            if (t < steps) out.store(pdx + (int64_t)t * dim, count);
        };

        Pack<T, V> ox[W - 1], ody[W - 1], nx[kAhead], ndy[kAhead];
#pragma unroll
        for (int i = 0; i < W - 1; ++i) load(t0 + i, ox[i], ody[i]);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(t0 + W - 1 + i, nx[i], ndy[i]);
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            form(t0 + i, ox[i], ody[i], true);
            if (t0 == 0 && o.dstate) {
                Pack<T, V> out;
                gather(i, out);
                out.store((T*)o.dstate + ((int64_t)b * (W - 1) + i) * dim + c0, count);
            }
            move();
        }
        int t = t0 + W - 1;
#pragma unroll 1
        for (int k = 0; k < kSteady; k += kAhead, t += kAhead) {
            Pack<T, V> cx[kAhead], cdy[kAhead], out[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                cx[i] = nx[i];
                cdy[i] = ndy[i];
                load(t + kAhead + i, nx[i], ndy[i]);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                form(t + i, cx[i], cdy[i], true);
                gather(t + i, out[i]);
                move();
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) store(t + i - (W - 1), out[i]);
        }
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {  // of the run behind: not this thread's own
            Pack<T, V> out;
            form(t + i, nx[i], ndy[i], false);
            gather(t + i, out);
            store(t + i - (W - 1), out);
            move();
        }
    }
#pragma unroll
    for (int c = 0; c < V; ++c) {
#pragma unroll
        for (int j = 0; j < W; ++j) s_sum[run][j][side * V + c] = dw[j][c];
        s_sum[run][W][side * V + c] = db[c];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < (W + 1) * kBackSide * V; e += kThreads) {
        const int j = e / (kBackSide * V), c = e % (kBackSide * V);
        if (cb * kBackSide * V + c < dim) {
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < kBackRuns; ++r) sum += s_sum[r][j][c];
            o.part[((int64_t)part * (W + 1) + j) * dim + cb * kBackSide * V + c] = sum;
        }
    }
}

// dweight and dbias: the workgroups' sums, added in order: 5 us for 4096 channels.
template <int SLICES>
__global__ __launch_bounds__(kSumThreads) void k_conv_sum(const float* part, int64_t parts,
                                                          int64_t dim, int width, float* dweight,
                                                          float* dbias) {
    const int64_t i = (int64_t)blockIdx.x * kSumOuts<SLICES> + threadIdx.x % kSumOuts<SLICES>;
    const int64_t total = dim * (width + 1);
    const float sum = sum_parts<SLICES>(part, i < total ? parts : 0, total, i);
    if (threadIdx.x >= kSumOuts<SLICES> || i >= total) return;
    const int j = (int)(i / dim);
    const int64_t c = i % dim;
    if (j < width)
        dweight[c * width + j] = sum;
    else if (dbias)
        dbias[c] = sum;
}

int64_t back_parts(const libscan_conv& p) {
    return p.batch * back_runs(p.steps, (int)p.width);
}

unsigned groups_of(int64_t n, int64_t per) { return (unsigned)((n + per - 1) / per); }

template <class T, int W>
hipError_t conv_as(const libscan_conv& p, void* y, void* state_out, hipStream_t s) {
    constexpr int V = 8 / sizeof(T);
    const int64_t nr = p.steps ? (p.steps + kRun - 1) / kRun : 1;
    const int64_t n = (p.dim + V - 1) / V * nr * p.batch;
    k_conv<T, W><<<groups_of(n, kThreads), kThreads, 0, s>>>(p, (T*)y, (T*)state_out);
    return hipGetLastError();
}

template <class T, int W>
hipError_t step_as(const libscan_conv& p, void* states, int64_t n_states, const int32_t* slots,
                   void* y, hipStream_t s) {
    constexpr int V = 8 / sizeof(T);
    const int64_t n = (p.dim + V - 1) / V * p.batch;
    k_conv_step<T, W><<<groups_of(n, kThreads), kThreads, 0, s>>>(p, (T*)states, n_states, slots,
                                                                 (T*)y);
    return hipGetLastError();
}

template <class T, int W>
hipError_t back_as(const libscan_conv& p, const BackArgs& o, float* dweight, float* dbias,
                   hipStream_t s) {
    const int64_t parts = back_parts(p);
    const int64_t nc = (p.dim + kBackSide * kBackV - 1) / (kBackSide * kBackV);
    auto* back = p.silu ? k_conv_back<T, W, true> : k_conv_back<T, W, false>;
    if (parts > 0) back<<<(unsigned)(parts * nc), kThreads, 0, s>>>(p, o);
    const int64_t outs = p.dim * (W + 1);
    if (long_sum(parts))
        k_conv_sum<8><<<groups_of(outs, kSumOuts<8>), kSumThreads, 0, s>>>(o.part, parts, p.dim, W,
                                                                         dweight, dbias);
    else
        k_conv_sum<1><<<groups_of(outs, kSumOuts<1>), kSumThreads, 0, s>>>(o.part, parts, p.dim, W,
                                                                         dweight, dbias);
    return hipGetLastError();
}

template <class F>
hipError_t by_type_width(const libscan_conv& p, F f) {
    auto width = [&](auto t) {
        switch (p.width) {
            case 2: return f(t, std::integral_constant<int, 2>());
            case 3: return f(t, std::integral_constant<int, 3>());
            default: return f(t, std::integral_constant<int, 4>());
        }
    };
    switch (p.type) {
        case LIBSCAN_F16: return width(_Float16());
        case LIBSCAN_BF16: return width(__bf16());
        default: return width(float());
    }
}

}  // namespace

hipError_t launch_conv(const libscan_conv& p, void* y, void* state_out, hipStream_t stream) {
    if (p.batch == 0 || p.dim == 0) return hipSuccess;
    return by_type_width(p, [&](auto t, auto w) {
        return conv_as<decltype(t), decltype(w)::value>(p, y, state_out, stream);
    });
}

hipError_t launch_conv_step(const libscan_conv& p, void* states, int64_t n_states,
                            const int32_t* slots, void* y, hipStream_t stream) {
    if (p.batch == 0 || p.dim == 0) return hipSuccess;
    return by_type_width(p, [&](auto t, auto w) {
        return step_as<decltype(t), decltype(w)::value>(p, states, n_states, slots, y, stream);
    });
}

size_t conv_scratch_bytes(const libscan_conv& p) {
    return (size_t)back_parts(p) * (p.width + 1) * p.dim * 4;
}

hipError_t launch_conv_back(const libscan_conv& p, const void* dy, int64_t dy_batch,
                            int64_t dy_step, const void* dstate_out, void* dx, float* dweight,
                            float* dbias, void* dstate, void* scratch, hipStream_t stream) {
    if (p.dim == 0) return hipSuccess;
    const BackArgs o{dy, dy_batch, dy_step, dstate_out, dx, dstate, (float*)scratch};
    return by_type_width(p, [&](auto t, auto w) {
        return back_as<decltype(t), decltype(w)::value>(p, o, dweight, dbias, stream);
    });
}

}  // namespace ls
