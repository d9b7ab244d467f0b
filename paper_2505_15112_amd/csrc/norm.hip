// norm.hip -- layer norm over groups of channels, with the residual sum in front
// of it, and its gradients.
//
// y = (x - mean) rstd weight + bias over each group of a row's channels.  With
// w = dy weight and xhat = (x - mean) rstd,
//   dx = rstd (w - mean(w) - xhat mean(w xhat)) + dsum,
//   dweight = sum over rows of dy xhat, dbias = sum over rows of dy.
#include <type_traits>

#include "launch.hpp"
#include "lm.hpp"

namespace ls {
namespace {

// A lane's vector of 16 bytes of T.
template <class T>
constexpr int kVec = 16 / sizeof(T);

// Keeps what was computed from a vector from being held until later uses: it is computed
// again from the 4 registers of the vector.
template <class P>
__device__ __forceinline__ void forget(P& x) {
    if constexpr (sizeof(P) == 16) {
        typedef unsigned U __attribute__((ext_vector_type(4)));
        U u = __builtin_bit_cast(U, x.v);
        asm volatile("" : "+v"(u));
        x.v = __builtin_bit_cast(decltype(x.v), u);
    }
}

// Sums over the LANES threads of a team (a power of two; a workgroup's teams all call).
// Calls take turns with two buffers `s` of N floats for each wave: what a buffer holds is
// read before the other's barrier, so one barrier a call will do.
template <int LANES, int N>
__device__ __forceinline__ void team_sums(float (&v)[N], float* s) {
#pragma unroll
    for (int m = (LANES < 64 ? LANES : 64) / 2; m > 0; m >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], m);
    if constexpr (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        float* mine = s + threadIdx.x / LANES * WAVES * N;
        if (threadIdx.x % 64 == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) mine[threadIdx.x % LANES / 64 * N + k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = mine[k];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) v[k] += mine[i * N + k];
        }
    }
}
template <int LANES>
__device__ __forceinline__ float team_sum(float v, float* s) {
    float one[1] = {v};
    team_sums<LANES>(one, s);
    return one[0];
}

// Row `row`'s elements of a batch x steps x dim operand.
__device__ __forceinline__ int64_t row_at(const libscan_norm& p, int64_t row, int64_t batch,
                                          int64_t step) {
    if (p.batch == 1) return row * step;
    return row / p.steps * batch + row % p.steps * step;
}

// A vector of weights or biases, as they are stored; `fill` where there are none.
template <class W, int V>
__device__ __forceinline__ Pack<W, V> load_weights(const void* w, int at, int count, float fill) {
    Pack<W, V> x;
    if (w) {
        x.load((const W*)w + at, count);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) x.v[e] = from_f32<W>(fill);
    }
    return x;
}

// ------------------------------------------------ rows in registers

// A team of LANES threads to a group of a row, with NV vectors a thread: one read of the
// row, the mean, then the sum of the squared differences.  Bound by memory: 8192 x 4096,
// bf16, with the sum: 51 us for 268 MB, 5.2 TB/s.
constexpr int kFrontThreads = 256;
template <class T, class W, int LANES, int NV>
__global__ void __launch_bounds__(LANES > kFrontThreads ? LANES : kFrontThreads, 8)
    k_norm(libscan_norm p, T* y, T* sum, float* stats) {
    constexpr int V = kVec<T>, THREADS = LANES > kFrontThreads ? LANES : kFrontThreads;
    constexpr int TEAMS = THREADS / LANES;
    __shared__ float s[2][THREADS / 64];
    const int lane = threadIdx.x % LANES, per = (int)(p.dim / p.groups);
    const int64_t all = p.batch * p.steps * p.groups;
    for (int64_t first = blockIdx.x * (int64_t)TEAMS; first < all;
         first += (int64_t)gridDim.x * TEAMS) {
        const int64_t seg = first + threadIdx.x / LANES;
        const bool on = seg < all;
        const int64_t row = seg / p.groups;
        const int c0 = (int)(seg % p.groups) * per;
        const T* x = (const T*)p.x + row_at(p, row, p.x_batch, p.x_step) + c0;
        const T* res = p.residual ? (const T*)p.residual +
                                        row_at(p, row, p.residual_batch, p.residual_step) + c0
                                  : nullptr;
        Pack<T, V> a[NV], b[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LANES + lane) * V, left = on ? per - c : 0;
            a[i].load(x + c, left);
            if (res) b[i].load(res + c, left);
        }
        float mean = 0.0f, var = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                if (res) a[i].v[e] = from_f32<T>(to_f32(a[i].v[e]) + to_f32(b[i].v[e]));
                mean += to_f32(a[i].v[e]);
            }
        mean = team_sum<LANES>(mean, s[0]) / per;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            forget(a[i]);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = to_f32(a[i].v[e]) - mean;
                if ((i * LANES + lane) * V + e < per) var = __builtin_fmaf(d, d, var);
            }
        }
        var = team_sum<LANES>(var, s[1]) / per;
        const float rstd = 1.0f / __builtin_sqrtf(var + (float)p.eps);
        if (!on) continue;
        const int64_t out = row * p.dim + c0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LANES + lane) * V, left = per - c;
            if (left <= 0) continue;
            forget(a[i]);
            const auto w = load_weights<W, V>(p.weight, c0 + c, left, 1.0f);
            const auto bias = load_weights<W, V>(p.bias, c0 + c, left, 0.0f);
            if (sum) a[i].store(sum + out + c, left);
#pragma unroll
            for (int e = 0; e < V; ++e)
                a[i].v[e] = from_f32<T>(__builtin_fmaf((to_f32(a[i].v[e]) - mean) * rstd, to_f32(w.v[e]),
                                                       to_f32(bias.v[e])));
            a[i].store(y + out + c, left);
        }
        if (stats && lane == 0) *(float2*)(stats + 2 * seg) = float2{mean, rstd};
    }
}

struct Grad {
    const void* dy;
    int64_t dy_batch, dy_step;
    const void* dsum;
    int64_t dsum_batch, dsum_step;
    const float* stats;
};

// The gradients likewise: the teams of a workgroup take rows of one group of channels,
// the next row's elements on their way while one is worked on, and add up dweight
// and dbias of their columns in registers, then over the teams in order.  Block i of a
// group has its sums at dweight + i * apart and dbias + i * apart (nullable).  A launch takes
// `some` groups from the first on.  8192 x 4096, bf16, with dsum: 62 us for 268 MB, 4.3
// TB/s.
constexpr int kBackThreads = 1024;
template <class T, class W, int LANES, int NV>
__global__ void __launch_bounds__(kBackThreads)
    k_norm_back(libscan_norm p, Grad g, T* dx, float* dweight, float* dbias, int64_t apart,
                int first, int some) {
    constexpr int V = kVec<T>, TEAMS = kBackThreads / LANES;
    // teams within a wave are joined by shifts, those left take turns in LDS
    constexpr int TURNS = LANES < 64 ? kBackThreads / 64 : TEAMS, COLS = LANES * NV * V;
    __shared__ float s[2][kBackThreads / 64 * 2], s_sum[TURNS > 1 ? 2 : 1][TURNS > 1 ? COLS : 1];
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    const int per = (int)(p.dim / p.groups), groups = (int)p.groups;
    const int group = first + blockIdx.x % some, block = blockIdx.x / some;
    const int64_t rows = p.batch * p.steps, every = (int64_t)(gridDim.x / some) * TEAMS;
    const int c0 = group * per;
    Pack<W, V> w[NV];
    float dw[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * LANES + lane) * V;
        w[i] = load_weights<W, V>(p.weight, c0 + c, per - c, 1.0f);
#pragma unroll
        for (int e = 0; e < V; ++e) dw[i][e] = db[i][e] = 0.0f;
    }
    struct Row {
        Pack<T, V> x[NV], dy[NV];
        float2 stats;
    };
    const auto load = [&](Row& r, int64_t row) {
        const bool on = row < rows;
        const T* x = (const T*)p.x + row_at(p, row, p.x_batch, p.x_step) + c0;
        const T* dy = (const T*)g.dy + row_at(p, row, g.dy_batch, g.dy_step) + c0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LANES + lane) * V, left = on ? per - c : 0;
            r.x[i].load(x + c, left);
            r.dy[i].load(dy + c, left);
        }
        r.stats = on ? *(const float2*)(g.stats + 2 * (row * groups + group)) : float2{0.0f, 0.0f};
    };
    Row now;
    int64_t row = (int64_t)block * TEAMS + team;
    load(now, row);
    // the teams of a workgroup stay together
    int turn = 0;
    for (int64_t at = (int64_t)block * TEAMS; at < rows; at += every, row += every, turn ^= 1) {
        const bool on = row < rows;
        Pack<T, V> dsum[NV];
        if (g.dsum) {
            const T* ds = (const T*)g.dsum + row_at(p, row, g.dsum_batch, g.dsum_step) + c0;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * LANES + lane) * V;
                dsum[i].load(ds + c, on ? per - c : 0);
            }
        }
        Row next;
        if (at + every < rows) load(next, row + every);
        const float mean = now.stats.x, rstd = now.stats.y;
        float m[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int left = per - (i * LANES + lane) * V;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                // behind the group's end dy is 0, but (0 - mean) rstd may be an infinity
                const float d = to_f32(now.dy[i].v[e]);
                const float hat = e < left ? (to_f32(now.x[i].v[e]) - mean) * rstd : 0.0f;
                const float u = d * to_f32(w[i].v[e]);
                m[0] += u;
                m[1] = __builtin_fmaf(u, hat, m[1]);
                dw[i][e] = __builtin_fmaf(d, hat, dw[i][e]);
                db[i][e] += d;
            }
        }
        team_sums<LANES>(m, s[turn]);
        const float m0 = m[0] / per, m1 = m[1] / per;
        if (on) {
            T* out = dx + row * p.dim + c0;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * LANES + lane) * V, left = per - c;
                if (left <= 0) continue;
                forget(now.x[i]), forget(now.dy[i]), forget(w[i]);
                Pack<T, V> o;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float hat = (to_f32(now.x[i].v[e]) - mean) * rstd;
                    const float u = to_f32(now.dy[i].v[e]) * to_f32(w[i].v[e]);
                    float v = rstd * (u - m0 - hat * m1);
                    if (g.dsum) v += to_f32(dsum[i].v[e]);
                    o.v[e] = from_f32<T>(v);
                }
                o.store(out + c, left);
            }
        }
        now = next;
    }
    if constexpr (LANES < 64) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e)
#pragma unroll
                for (int m = LANES; m < 64; m <<= 1) {
                    dw[i][e] += __shfl_xor(dw[i][e], m);
                    db[i][e] += __shfl_xor(db[i][e], m);
                }
    }
    constexpr int TURN = LANES < 64 ? 64 : LANES;
    const bool mine = LANES >= 64 || threadIdx.x % 64 < LANES;
    if constexpr (TURNS > 1) {
        for (int next = 0; next < TURNS; ++next) {
            __syncthreads();
            if (threadIdx.x / TURN == next && mine) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int c = (i * V + e) * LANES + lane;  // lanes next to each other
                        if (next > 0) {
                            dw[i][e] += s_sum[0][c];
                            db[i][e] += s_sum[1][c];
                        }
                        s_sum[0][c] = dw[i][e];
                        s_sum[1][c] = db[i][e];
                    }
            }
        }
        __syncthreads();
    }
    // the last turn's threads have the sums
    if (threadIdx.x / TURN != TURNS - 1 || !mine) return;
    const int64_t to = block * apart + c0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * LANES + lane) * V;
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (c + e < per) {
                if (dweight) dweight[to + c + e] = dw[i][e];
                if (dbias) dbias[to + c + e] = db[i][e];
            }
    }
}

// ------------------------------------------------ rows that do not fit registers

constexpr int kThreads = 1024;

// A workgroup to a group of a row, which is read three times, twice from the L2 cache.  501
// x 16389, fp16: 17 us; with three vectors a thread in registers 15, but some of them
// spilled, with four, one workgroup to a CU, 19.
template <class T, class W>
__global__ void __launch_bounds__(kThreads)
    k_norm_long(libscan_norm p, T* y, T* sum, float* stats) {
    constexpr int V = kVec<T>;
    __shared__ float s[2][kThreads / 64];
    const int per = (int)(p.dim / p.groups);
    const int64_t all = p.batch * p.steps * p.groups;
    for (int64_t seg = blockIdx.x; seg < all; seg += gridDim.x) {
        const int64_t row = seg / p.groups;
        const int c0 = (int)(seg % p.groups) * per;
        const T* x = (const T*)p.x + row_at(p, row, p.x_batch, p.x_step) + c0;
        const T* res = p.residual ? (const T*)p.residual +
                                        row_at(p, row, p.residual_batch, p.residual_step) + c0
                                  : nullptr;
        // f(c, the vector at c, elements there) over the group; behind its end they are 0
        const auto each = [&](auto f) {
            for (int c = threadIdx.x * V; c < per; c += kThreads * V) {
                Pack<T, V> a, b;
                a.load(x + c, per - c);
                if (res) {
                    b.load(res + c, per - c);
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        a.v[e] = from_f32<T>(to_f32(a.v[e]) + to_f32(b.v[e]));
                }
                f(c, a, per - c);
            }
        };
        float mean = 0.0f, var = 0.0f;
        each([&](int, const Pack<T, V>& a, int) {
#pragma unroll
            for (int e = 0; e < V; ++e) mean += to_f32(a.v[e]);
        });
        mean = team_sum<kThreads>(mean, s[0]) / per;
        each([&](int, const Pack<T, V>& a, int left) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = to_f32(a.v[e]) - mean;
                if (e < left) var = __builtin_fmaf(d, d, var);
            }
        });
        var = team_sum<kThreads>(var, s[1]) / per;
        const float rstd = 1.0f / __builtin_sqrtf(var + (float)p.eps);
        const int64_t out = row * p.dim + c0;
        each([&](int c, Pack<T, V>& a, int left) {
            const auto w = load_weights<W, V>(p.weight, c0 + c, left, 1.0f);
            const auto bias = load_weights<W, V>(p.bias, c0 + c, left, 0.0f);
            if (sum) a.store(sum + out + c, left);
#pragma unroll
            for (int e = 0; e < V; ++e)
                a.v[e] = from_f32<T>(__builtin_fmaf((to_f32(a.v[e]) - mean) * rstd, to_f32(w.v[e]),
                                                    to_f32(bias.v[e])));
            a.store(y + out + c, left);
        });
        if (stats && threadIdx.x == 0) *(float2*)(stats + 2 * seg) = float2{mean, rstd};
    }
}

template <class T, class W>
__global__ void __launch_bounds__(kThreads) k_norm_long_dx(libscan_norm p, Grad g, T* dx) {
    constexpr int V = kVec<T>;
    __shared__ float s[2][kThreads / 64];
    const int per = (int)(p.dim / p.groups);
    const int64_t all = p.batch * p.steps * p.groups;
    for (int64_t seg = blockIdx.x; seg < all; seg += gridDim.x) {
        const int64_t row = seg / p.groups;
        const int c0 = (int)(seg % p.groups) * per;
        const T* x = (const T*)p.x + row_at(p, row, p.x_batch, p.x_step) + c0;
        const T* dy = (const T*)g.dy + row_at(p, row, g.dy_batch, g.dy_step) + c0;
        const T* ds = (const T*)g.dsum + row_at(p, row, g.dsum_batch, g.dsum_step) + c0;
        const float2 st = *(const float2*)(g.stats + 2 * seg);
        // f(c, elements there, dy weight, xhat) over the group
        const auto each = [&](auto f) {
            for (int c = threadIdx.x * V; c < per; c += kThreads * V) {
                const int left = per - c;
                Pack<T, V> a, b;
                a.load(dy + c, left);
                b.load(x + c, left);
                const auto w = load_weights<W, V>(p.weight, c0 + c, left, 1.0f);
                float u[V], hat[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    u[e] = to_f32(a.v[e]) * to_f32(w.v[e]);
                    hat[e] = (to_f32(b.v[e]) - st.x) * st.y;
                }
                f(c, left, u, hat);
            }
        };
        float m0 = 0.0f, m1 = 0.0f;
        each([&](int, int left, const float (&u)[V], const float (&hat)[V]) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                m0 += u[e];  // 0 behind the end
                if (e < left) m1 = __builtin_fmaf(u[e], hat[e], m1);
            }
        });
        m0 = team_sum<kThreads>(m0, s[0]) / per;
        m1 = team_sum<kThreads>(m1, s[1]) / per;
        T* out = dx + row * p.dim + c0;
        each([&](int c, int left, const float (&u)[V], const float (&hat)[V]) {
            Pack<T, V> d, o;
            if (g.dsum) d.load(ds + c, left);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float v = st.y * (u[e] - m0 - hat[e] * m1);
                if (g.dsum) v += to_f32(d.v[e]);
                o.v[e] = from_f32<T>(v);
            }
            o.store(out + c, left);
        });
    }
}

// Partial sums of dweight and dbias over `rows` rows, four columns to a thread.
constexpr int kPartThreads = 256, kPartCols = 4 * kPartThreads;
template <class T>
__global__ void __launch_bounds__(kPartThreads)
    k_norm_long_dw(libscan_norm p, Grad g, int64_t rows, float* part) {
    const int blocks = (int)((p.dim + kPartCols - 1) / kPartCols);
    const int c = blockIdx.x % blocks * kPartCols + threadIdx.x * 4, block = blockIdx.x / blocks;
    if (c >= p.dim) return;
    const int64_t all = p.batch * p.steps, lo = block * rows;
    const int64_t hi = lo + rows < all ? lo + rows : all;
    const int per = (int)(p.dim / p.groups), left = (int)p.dim - c;
    float dw[4]{}, db[4]{};
#pragma unroll 4
    for (int64_t r = lo; r < hi; ++r) {
        Pack<T, 4> d, x;
        d.load((const T*)g.dy + row_at(p, r, g.dy_batch, g.dy_step) + c, left);
        x.load((const T*)p.x + row_at(p, r, p.x_batch, p.x_step) + c, left);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e >= left) break;
            const float2 st = *(const float2*)(g.stats + 2 * (r * p.groups + (c + e) / per));
            dw[e] = __builtin_fmaf(to_f32(d.v[e]), (to_f32(x.v[e]) - st.x) * st.y, dw[e]);
            db[e] += to_f32(d.v[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) {
            part[2 * (int64_t)block * p.dim + c + e] = dw[e];
            part[(2 * (int64_t)block + 1) * p.dim + c + e] = db[e];
        }
}

// ------------------------------------------------ the sums' last step

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

// ------------------------------------------------ launches

template <class F>
hipError_t by_type(const libscan_norm& p, F f) {
    const bool wide = p.weight_type == LIBSCAN_F32;
    if (p.type == LIBSCAN_F32) f(float(), float());
    else if (p.type == LIBSCAN_F16) wide ? f(_Float16(), float()) : f(_Float16(), _Float16());
    else wide ? f(__bf16(), float()) : f(__bf16(), __bf16());
    return hipGetLastError();
}

// The smallest team and number of vectors that hold a group's channels; no lanes if none
// does.  A second vector of eight elements would take the gradients more registers than
// there are.
struct Team {
    int lanes, vectors;
};
Team team(const libscan_norm& p, bool gradients) {
    const int64_t per = p.dim / p.groups, vec = p.type == LIBSCAN_F32 ? 4 : 8;
    const Team all[] = {{16, 1}, {32, 1}, {64, 1}, {128, 1}, {256, 1}, {512, 1}, {1024, 1}, {1024, 2}};
    const int most = gradients && vec == 8 ? 1 : 2;
    for (const Team& t : all)
        if (t.vectors <= most && t.lanes * t.vectors * vec >= per) return t;
    return {0, 0};
}
template <class F>
void by_team(const Team& t, F f) {
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 1024> all;
    if (t.lanes == 16) f(std::integral_constant<int, 16>(), one);
    else if (t.lanes == 32) f(std::integral_constant<int, 32>(), one);
    else if (t.lanes == 64) f(std::integral_constant<int, 64>(), one);
    else if (t.lanes == 128) f(std::integral_constant<int, 128>(), one);
    else if (t.lanes == 256) f(std::integral_constant<int, 256>(), one);
    else if (t.lanes == 512) f(std::integral_constant<int, 512>(), one);
    else if (t.vectors == 1) f(all, one);
    else f(all, std::integral_constant<int, 2>());
}

constexpr int64_t kMostBlocks = 1 << 20;  // the rest in further turns or launches
uint32_t capped(int64_t blocks) { return (uint32_t)(blocks < kMostBlocks ? blocks : kMostBlocks); }

// Rows of a block of k_norm_long_dw: 64 blocks, unless that is a few rows each.
int64_t part_rows(const libscan_norm& p) {
    const int64_t rows = (p.batch * p.steps + 63) / 64;
    return rows > 8 ? rows : 8;
}

// Blocks of rows that dweight and dbias are added up over first.
int64_t parts(const libscan_norm& p) {
    const int64_t rows = p.batch * p.steps;
    const Team t = team(p, true);
    if (!t.lanes) return (rows + part_rows(p) - 1) / part_rows(p);
    const int64_t teams = kBackThreads / t.lanes, blocks = (rows + teams - 1) / teams;
    // a workgroup to a CU: twice as many take turns (8192 x 4096, bf16: 70 us, not 60)
    const int64_t most = p.groups >= 256 ? 1 : 256 / p.groups;
    return blocks < most ? blocks : most;
}

}  // namespace

hipError_t launch_norm(const libscan_norm& p, void* y, void* sum, float* stats,
                       hipStream_t stream) {
    const int64_t all = p.batch * p.steps * p.groups;
    if (all == 0 || p.dim == 0) return hipSuccess;
    const Team t = team(p, false);
    return by_type(p, [&](auto type, auto weights) {
        using T = decltype(type);
        using W = decltype(weights);
        if (!t.lanes) {
            k_norm_long<T, W><<<capped(all), kThreads, 0, stream>>>(p, (T*)y, (T*)sum, stats);
            return;
        }
        by_team(t, [&](auto lanes, auto vectors) {
            constexpr int L = lanes.value, THREADS = L > kFrontThreads ? L : kFrontThreads;
            constexpr int TEAMS = THREADS / L;
            k_norm<T, W, L, vectors.value><<<capped((all + TEAMS - 1) / TEAMS), THREADS, 0, stream>>>(
                p, (T*)y, (T*)sum, stats);
        });
    });
}

size_t norm_scratch_bytes(const libscan_norm& p) { return (size_t)(parts(p) * 2 * p.dim * 4); }

hipError_t launch_norm_back(const libscan_norm& p, const void* dy, int64_t dy_batch,
                            int64_t dy_step, const void* dsum, int64_t dsum_batch,
                            int64_t dsum_step, const float* stats, void* dx, float* dweight,
                            float* dbias, void* scratch, hipStream_t stream) {
    const Grad g{dy, dy_batch, dy_step, dsum, dsum_batch, dsum_step, stats};
    const int64_t all = p.batch * p.steps * p.groups, count = parts(p);
    if (p.dim == 0) return hipSuccess;
    float* part = (float*)scratch;
    const Team t = team(p, true);
    return by_type(p, [&](auto type, auto weights) {
        using T = decltype(type);
        using W = decltype(weights);
        // one block's sums are the sums
        const bool whole = t.lanes && count == 1;
        if (all && t.lanes)
            by_team(t, [&](auto lanes, auto vectors) {
                if constexpr (vectors.value == 1 || sizeof(T) == 4)
                    // (more than one block to a group only up to 256 groups)
                    for (int64_t first = 0; first < p.groups; first += kMostBlocks) {
                        const int64_t left = p.groups - first;
                        const int some = (int)(left < kMostBlocks ? left : kMostBlocks);
                        k_norm_back<T, W, lanes.value, vectors.value>
                            <<<(uint32_t)(count * some), kBackThreads, 0, stream>>>(
                                p, g, (T*)dx, whole ? dweight : part, whole ? dbias : part + p.dim,
                                2 * p.dim, (int)first, some);
                    }
            });
        if (all && !t.lanes) {
            k_norm_long_dx<T, W><<<capped(all), kThreads, 0, stream>>>(p, g, (T*)dx);
            k_norm_long_dw<T><<<(uint32_t)(count * ((p.dim + kPartCols - 1) / kPartCols)),
                                kPartThreads, 0, stream>>>(p, g, part_rows(p), part);
        }
        if (whole || (!dweight && !dbias)) return;
        if (long_sum(count))
            k_norm_sum<8><<<(uint32_t)((2 * p.dim + kSumOuts<8> - 1) / kSumOuts<8>), kSumThreads, 0,
                            stream>>>(part, count, p.dim, dweight, dbias);
        else
            k_norm_sum<1><<<(uint32_t)((2 * p.dim + kSumOuts<1> - 1) / kSumOuts<1>), kSumThreads, 0,
                            stream>>>(part, count, p.dim, dweight, dbias);
    });
}

}  // namespace ls
