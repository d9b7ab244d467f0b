// attend.hip -- linear attention with a decay for each head: the walk over a
// row's tokens (attend.hpp), the gradients made of it, and the single token.
#include "attend.hpp"
#include "launch.hpp"

namespace ls {
namespace {

constexpr int kCols = 64;  // columns of a step's workgroup

// Gradients by head, batch x steps x heads x width fp32, to those of the groups.
template <class T>
__global__ void __launch_bounds__(256) k_join_heads(const float* in, T* out, int64_t count, int per,
                                                    int width) {
    const int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x;
    if (i >= count) return;
    const int64_t group = i / width, at = group * per * width + i % width;
    float sum = 0.0f;
    for (int j = 0; j < per; ++j) sum += in[at + (int64_t)j * width];
    out[i] = from_f32<T>(sum);
}

// The decays' gradients: dg[t] = sum over s >= t of (q.dq - k.dk)[s], and the part
// of the last state, <dS, S>.  A workgroup to a row and head.
constexpr int kGateThreads = 256;
__device__ double block_sum(double v, double* s) {
    const int tid = threadIdx.x;
    s[tid] = v;
    __syncthreads();
    for (int m = kGateThreads / 2; m > 0; m >>= 1) {
        if (tid < m) s[tid] += s[tid + m];
        __syncthreads();
    }
    const double r = s[0];
    __syncthreads();
    return r;
}

__global__ void __launch_bounds__(kGateThreads)
    k_gates(Walk w, const float* dq_dots, int dq_blocks, const float* dk_dots, int dk_blocks,
            const float* dstate_out, const float* last, int64_t state, float* out) {
    __shared__ double s[kGateThreads];
    const int h = blockIdx.x % w.heads, b = blockIdx.x / w.heads, tid = threadIdx.x;
    const int len = walk_len(w, b);
    const int64_t all = (int64_t)w.batch * w.steps * w.heads;
    double carry = 0.0;
    if (dstate_out) {
        for (int64_t i = tid; i < state; i += kGateThreads)
            carry += (double)dstate_out[blockIdx.x * state + i] * last[blockIdx.x * state + i];
        carry = block_sum(carry, s);
    }
    for (int end = w.steps; end > 0; end -= kGateThreads) {
        const int t = end - 1 - tid;  // thread 0 has the last token
        double v = 0.0;
        const int64_t at = ((int64_t)b * w.steps + t) * w.heads + h;
        if (t >= 0 && t < len) {
            for (int i = 0; i < dq_blocks; ++i) v += dq_dots[i * all + at];
            for (int i = 0; i < dk_blocks; ++i) v -= dk_dots[i * all + at];
        }
        s[tid] = v;
        __syncthreads();
        for (int m = 1; m < kGateThreads; m <<= 1) {
            const double more = tid >= m ? s[tid - m] : 0.0;
            __syncthreads();
            s[tid] += more;
            __syncthreads();
        }
        // a decay of -infinity leaves nothing to change
        if (t >= 0)
            out[at] = t < len && w.g[b * w.g_batch + t * w.g_step + h] != -__builtin_inff()
                          ? (float)(carry + s[tid]) : 0.0f;
        carry += s[kGateThreads - 1];
        __syncthreads();
    }
}

// One decay for all tokens of a head: the sum of their gradients.
__global__ void __launch_bounds__(kGateThreads) k_gate_sum(const float* in, float* out,
                                                           int64_t tokens, int heads) {
    __shared__ double s[kGateThreads];
    double v = 0.0;
    for (int64_t i = threadIdx.x; i < tokens; i += kGateThreads) v += in[i * heads + blockIdx.x];
    v = block_sum(v, s);
    if (threadIdx.x == 0) out[blockIdx.x] = (float)v;
}

// dS_0 = e^g[0] G[0], in place; a row without tokens keeps dS.
__global__ void __launch_bounds__(256) k_first_decay(Walk w, float* state, int64_t each) {
    const int h = blockIdx.x % w.heads, b = blockIdx.x / w.heads;
    if (walk_len(w, b) == 0) return;
    const float a = exp2_fast(w.g[b * w.g_batch + h] * kLog2e);
    for (int64_t i = threadIdx.x; i < each; i += 256) state[blockIdx.x * each + i] *= a;
}

// The states before every piece from what each adds, in place: a workgroup to 256
// elements of a row and head; piece i of element x is states[i * each + x].
__global__ void __launch_bounds__(256)
    k_carry(float* states, const float* whole, int pieces, int64_t each, const float* first,
            float* last) {
    const int64_t groups = (each + 255) / 256, bh = blockIdx.x / groups;
    const int64_t x = blockIdx.x % groups * 256 + threadIdx.x;
    if (x >= each) return;
    float* at = states + bh * pieces * each + x;
    float run = first ? first[bh * each + x] : 0.0f;
#pragma unroll 8
    for (int i = 0; i < pieces; ++i) {
        const float more = at[i * each];
        at[i * each] = run;
        run = __builtin_fmaf(whole[bh * pieces + i], run, more);
    }
    if (last) last[bh * each + x] = run;
}

// ------------------------------------------------ a single token

// A workgroup to 64 columns of a row's head.
template <class T>
__global__ void __launch_bounds__(kCols)
    k_attend_step(libscan_attend p, float* states, int64_t n_states, const int32_t* slots, T* y) {
    const int blocks = ((int)p.dv + kCols - 1) / kCols;
    const int block = blockIdx.x % blocks, bh = blockIdx.x / blocks;
    const int h = bh % (int)p.heads, b = bh / (int)p.heads;
    const int c = block * kCols + threadIdx.x;
    if (c >= p.dv) return;
    T* out = y + (int64_t)bh * p.dv + c;
    const int64_t slot = slots ? slots[b] : b;
    if (slot < 0 || slot >= n_states) {
        *out = T(0);
        return;
    }
    const int share = (int)(p.heads / p.groups);
    const T* q = (const T*)p.q + b * p.q_batch + (h / share) * p.q_head;
    const T* k = (const T*)p.k + b * p.k_batch + (h / share) * p.k_head;
    const float v = to_f32(((const T*)p.v + b * p.v_batch + h * p.v_head)[c]);
    const float g = p.fixed ? p.log_decay[h] : p.log_decay[b * p.decay_batch + h];
    const float a = exp2_fast(g * kLog2e);
    float* s = states + (slot * p.heads + h) * p.dk * p.dv + c;
    float o = 0.0f;
    for (int r = 0; r < p.dk; ++r) {
        const float x = __builtin_fmaf(to_f32(k[r]), v, a * s[r * p.dv]);
        s[r * p.dv] = x;
        o = __builtin_fmaf(to_f32(q[r]), x, o);
    }
    *out = from_f32<T>(o * (float)p.scale);
}

// ------------------------------------------------ launches

hipError_t run(int64_t type, const Walk& w, bool states, hipStream_t stream) {
    return type == LIBSCAN_F32   ? launch_walk<float>(w, states, stream)
           : type == LIBSCAN_F16 ? launch_walk<_Float16>(w, states, stream)
                                 : launch_walk<__bf16>(w, states, stream);
}

// What all walks of a call have in common.
Walk base(const libscan_attend& p) {
    Walk w{};
    w.batch = (int)p.batch, w.steps = (int)p.steps, w.heads = (int)p.heads;
    w.g = p.log_decay;
    w.g_batch = p.fixed ? 0 : p.decay_batch;
    w.g_step = p.fixed ? 0 : p.decay_step;
    w.lengths = p.lengths;
    w.pieces = 1, w.piece = w.steps;
    w.inner = w.outer = 1.0f;
    return w;
}
WalkSide side_q(const libscan_attend& p) {
    return {p.q, p.q_batch, p.q_step, p.q_head, (int)(p.heads / p.groups)};
}
WalkSide side_k(const libscan_attend& p) {
    return {p.k, p.k_batch, p.k_step, p.k_head, (int)(p.heads / p.groups)};
}
WalkSide side_v(const libscan_attend& p) { return {p.v, p.v_batch, p.v_step, p.v_head, 1}; }

// Rows are cut into pieces where they alone do not fill the GPU: a first run over k and
// v gives what each piece adds to the state.
struct Pieces {
    int count, places;
};
Pieces pieces(const libscan_attend& p) {
    const int64_t chunk = 64, chunks = (p.steps + chunk - 1) / chunk;
    const int64_t groups = p.batch * p.heads * walk_blocks((int)p.dk, (int)p.dv);
    int64_t count = groups ? 512 / groups : 1;
    if (count > chunks / 2) count = chunks / 2;
    if (count < 2) return {1, (int)p.steps};
    const int64_t each = (chunks + count - 1) / count;
    return {(int)((chunks + each - 1) / each), (int)(each * chunk)};
}

// Scratch in bytes from its start.
struct Room {
    int64_t at = 0;
    int64_t floats(int64_t n) {
        const int64_t here = at;
        at += (n * 4 + 255) / 256 * 256;
        return here;
    }
};
// What each piece adds to the states, and then the states before it.
struct Cut {
    int64_t states, whole;
    Cut(const libscan_attend& p, Room& room) {
        const int64_t n = pieces(p).count, all = n > 1 ? p.batch * p.heads * n : 0;
        states = room.floats(all * p.dk * p.dv);
        whole = room.floats(all);
    }
};
struct FrontPlan {
    Room room;
    Cut cut;
    FrontPlan(const libscan_attend& p) : cut(p, room) {}
};
struct BackPlan {
    Room room;
    Cut cut, back;  // of S, and of its gradient
    int64_t dq_dots, dk_dots, gates, last, dq, dk;
    BackPlan(const libscan_attend& p) : cut(p, room), back(p, room) {
        const int64_t tokens = p.batch * p.steps * p.heads;
        const int64_t blocks = walk_blocks((int)p.dv, (int)p.dk);
        const bool shared = p.groups < p.heads;
        dq_dots = room.floats(tokens * blocks);
        dk_dots = room.floats(tokens * blocks);
        gates = room.floats(p.fixed ? tokens : 0);
        last = room.floats(p.batch * p.heads * p.dk * p.dv);
        dq = room.floats(shared ? tokens * p.dk : 0);
        dk = room.floats(shared ? tokens * p.dk : 0);
    }
};

// The states before every piece of the walk w, whose first and last states are its
// rows'; w then takes them.
hipError_t cut_rows(int64_t type, Walk& w, const libscan_attend& p, const Cut& cut, char* mem,
                    hipStream_t stream) {
    const Pieces n = pieces(p);
    w.pieces = n.count, w.piece = n.places;
    if (n.count == 1) return hipSuccess;
    Walk states = w;
    states.first = {};
    states.last = {(float*)(mem + cut.states), p.dv, 1};
    states.whole = (float*)(mem + cut.whole);
    const hipError_t e = run(type, states, true, stream);
    if (e != hipSuccess) return e;
    const int64_t each = p.dk * p.dv, rows = p.batch * p.heads;
    k_carry<<<(uint32_t)(rows * ((each + 255) / 256)), 256, 0, stream>>>(
        states.last.p, states.whole, n.count, each, w.first.p, w.last.p);
    w.first = states.last;
    w.last = {};
    return hipGetLastError();
}

}  // namespace

size_t attend_scratch_bytes(const libscan_attend& p) { return (size_t)FrontPlan(p).room.at; }
size_t attend_back_scratch_bytes(const libscan_attend& p) { return (size_t)BackPlan(p).room.at; }

hipError_t launch_attend(const libscan_attend& p, void* y, float* state_out, void* scratch,
                         hipStream_t stream) {
    Walk w = base(p);
    w.dk = (int)p.dk, w.dv = (int)p.dv;
    w.q = side_q(p), w.k = side_k(p), w.v = side_v(p);
    w.outer = (float)p.scale;
    w.first = {const_cast<float*>(p.state), p.dv, 1};
    w.last = {state_out, p.dv, 1};
    w.out = y;
    const hipError_t e = cut_rows(p.type, w, p, FrontPlan(p).cut, (char*)scratch, stream);
    return e != hipSuccess ? e : run(p.type, w, false, stream);
}

hipError_t launch_attend_back(const libscan_attend& p, const void* dy, int64_t dy_batch,
                              int64_t dy_step, int64_t dy_head, const float* dstate_out, void* dq,
                              void* dk, void* dv, float* dlog_decay, float* dstate, void* scratch,
                              hipStream_t stream) {
    const BackPlan plan(p);
    char* mem = (char*)scratch;
    const auto floats = [&](int64_t at) { return (float*)(mem + at); };
    const bool shared = p.groups < p.heads;
    const WalkSide side_dy = {dy, dy_batch, dy_step, dy_head, 1};
    const int dots = walk_blocks((int)p.dv, (int)p.dk);
    float* last = dstate_out ? floats(plan.last) : nullptr;
    hipError_t e;

    // S forwards, and its gradient backwards with dv
    Walk s = base(p), g = base(p);
    s.dk = g.dk = (int)p.dk, s.dv = g.dv = (int)p.dv;
    s.k = side_k(p), s.v = side_v(p);
    s.first = {const_cast<float*>(p.state), p.dv, 1};
    s.last = {last, p.dv, 1};
    if ((e = cut_rows(p.type, s, p, plan.cut, mem, stream)) != hipSuccess) return e;
    g.reverse = true;
    g.q = side_k(p), g.k = side_q(p), g.v = side_dy;
    g.inner = (float)p.scale;
    g.first = {const_cast<float*>(dstate_out), p.dv, 1};
    g.last = {dstate, p.dv, 1};
    g.out = dv;
    if ((e = cut_rows(p.type, g, p, plan.back, mem, stream)) != hipSuccess) return e;
    if ((e = run(p.type, g, false, stream)) != hipSuccess) return e;

    Walk w = s;  // dq, with S turned over
    w.dk = (int)p.dv, w.dv = (int)p.dk;
    w.q = side_dy, w.k = side_v(p), w.v = side_k(p);
    w.outer = (float)p.scale;
    w.first = {s.first.p, 1, p.dv};
    w.last = {s.last.p, 1, p.dv};
    w.out = shared ? floats(plan.dq) : dq;
    w.wide = shared;
    w.e = side_q(p);
    w.dots = floats(plan.dq_dots);
    if ((e = run(p.type, w, false, stream)) != hipSuccess) return e;

    w.reverse = true;  // dk
    w.q = side_v(p), w.k = side_dy, w.v = side_q(p);
    w.inner = (float)p.scale, w.outer = 1.0f;
    w.first = {g.first.p, 1, p.dv};
    w.last = {};
    w.out = shared ? floats(plan.dk) : dk;
    w.e = side_k(p);
    w.dots = floats(plan.dk_dots);
    if ((e = run(p.type, w, false, stream)) != hipSuccess) return e;

    const uint32_t rows = (uint32_t)(p.batch * p.heads);
    const int64_t each = p.dk * p.dv;
    if (rows) {
        k_gates<<<rows, kGateThreads, 0, stream>>>(
            w, floats(plan.dq_dots), dots, floats(plan.dk_dots), dots, dstate_out, last, each,
            p.fixed ? floats(plan.gates) : dlog_decay);
        if (dstate && p.steps) k_first_decay<<<rows, 256, 0, stream>>>(w, dstate, each);
    }
    if (p.fixed && p.heads)
        k_gate_sum<<<(uint32_t)p.heads, kGateThreads, 0, stream>>>(
            floats(plan.gates), dlog_decay, p.batch * p.steps, (int)p.heads);
    const int64_t count = p.batch * p.steps * p.groups * p.dk;
    if (shared && count) {
        const uint32_t grid = (uint32_t)((count + 255) / 256);
        const auto join = [&](auto zero) {
            using T = decltype(zero);
            const int per = (int)(p.heads / p.groups);
            k_join_heads<<<grid, 256, 0, stream>>>(floats(plan.dq), (T*)dq, count, per, (int)p.dk);
            k_join_heads<<<grid, 256, 0, stream>>>(floats(plan.dk), (T*)dk, count, per, (int)p.dk);
        };
        if (p.type == LIBSCAN_F32) join(float());
        else if (p.type == LIBSCAN_F16) join(_Float16());
        else join(__bf16());
    }
    return hipGetLastError();
}

hipError_t launch_attend_step(const libscan_attend& p, float* states, int64_t n_states,
                              const int32_t* slots, void* y, hipStream_t stream) {
    const uint32_t grid = (uint32_t)(p.batch * p.heads * ((p.dv + kCols - 1) / kCols));
    if (p.type == LIBSCAN_F32)
        k_attend_step<float><<<grid, kCols, 0, stream>>>(p, states, n_states, slots, (float*)y);
    else if (p.type == LIBSCAN_F16)
        k_attend_step<_Float16><<<grid, kCols, 0, stream>>>(p, states, n_states, slots,
                                                            (_Float16*)y);
    else
        k_attend_step<__bf16><<<grid, kCols, 0, stream>>>(p, states, n_states, slots, (__bf16*)y);
    return hipGetLastError();
}

}  // namespace ls
