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

hipError_t run(int64_t type, const Walk& w, Grade grade, bool states, hipStream_t stream) {
    return type == LIBSCAN_F32   ? launch_walk<float>(w, grade, states, stream)
           : type == LIBSCAN_F16 ? launch_walk<_Float16>(w, grade, states, stream)
                                 : launch_walk<__bf16>(w, grade, states, stream);
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

// Scratch of the gradients, in bytes from its start.
struct BackPlan {
    int64_t dq_dots, dk_dots, gates, last, dq, dk, bytes;
};
BackPlan back_plan(const libscan_attend& p) {
    BackPlan r{};
    const int64_t tokens = p.batch * p.steps * p.heads;
    int64_t at = 0;
    const auto take = [&](int64_t floats) {
        const int64_t here = at;
        at += (floats * 4 + 255) / 256 * 256;
        return here;
    };
    r.dq_dots = take(tokens * walk_blocks((int)p.dv, (int)p.dk));
    r.dk_dots = take(tokens * walk_blocks((int)p.dv, (int)p.dk));
    r.gates = take(p.fixed ? tokens : 0);
    r.last = take(p.batch * p.heads * p.dk * p.dv);
    r.dq = take(p.groups < p.heads ? tokens * p.dk : 0);
    r.dk = take(p.groups < p.heads ? tokens * p.dk : 0);
    r.bytes = at;
    return r;
}

}  // namespace

size_t attend_scratch_bytes(const libscan_attend& p) { return 0; }
size_t attend_back_scratch_bytes(const libscan_attend& p) { return (size_t)back_plan(p).bytes; }

hipError_t launch_attend(const libscan_attend& p, void* y, float* state_out, void* scratch,
                         hipStream_t stream) {
    Walk w = base(p);
    w.dk = (int)p.dk, w.dv = (int)p.dv;
    w.q = side_q(p), w.k = side_k(p), w.v = side_v(p);
    w.outer = (float)p.scale;
    w.first = {const_cast<float*>(p.state), p.dv, 1};
    w.last = {state_out, p.dv, 1};
    w.out = y;
    return run(p.type, w, Grade::Narrow, false, stream);
}

hipError_t launch_attend_back(const libscan_attend& p, const void* dy, int64_t dy_batch,
                              int64_t dy_step, int64_t dy_head, const float* dstate_out, void* dq,
                              void* dk, void* dv, float* dlog_decay, float* dstate, void* scratch,
                              hipStream_t stream) {
    const BackPlan plan = back_plan(p);
    char* mem = (char*)scratch;
    const auto floats = [&](int64_t at) { return (float*)(mem + at); };
    const bool shared = p.groups < p.heads;
    const WalkSide side_dy = {dy, dy_batch, dy_step, dy_head, 1};
    const int64_t state = p.dk * p.dv;
    hipError_t e;

    Walk w = base(p);  // dq
    w.dk = (int)p.dv, w.dv = (int)p.dk;
    w.q = side_dy, w.k = side_v(p), w.v = side_k(p);
    w.outer = (float)p.scale;
    w.first = {const_cast<float*>(p.state), 1, p.dv};
    w.last = {dstate_out ? floats(plan.last) : nullptr, 1, p.dv};
    w.out = shared ? floats(plan.dq) : dq;
    w.wide = shared;
    w.e = side_q(p);
    w.dots = floats(plan.dq_dots);
    if ((e = run(p.type, w, Grade::Wide, false, stream)) != hipSuccess) return e;

    w.reverse = true;  // dk
    w.q = side_v(p), w.k = side_dy, w.v = side_q(p);
    w.inner = (float)p.scale, w.outer = 1.0f;
    w.first = {const_cast<float*>(dstate_out), 1, p.dv};
    w.last = {};
    w.out = shared ? floats(plan.dk) : dk;
    w.e = side_k(p);
    w.dots = floats(plan.dk_dots);
    if ((e = run(p.type, w, Grade::Wide, false, stream)) != hipSuccess) return e;

    w = base(p);  // dv
    w.reverse = true;
    w.dk = (int)p.dk, w.dv = (int)p.dv;
    w.q = side_k(p), w.k = side_q(p), w.v = side_dy;
    w.inner = (float)p.scale;
    w.first = {const_cast<float*>(dstate_out), p.dv, 1};
    w.last = {dstate, p.dv, 1};
    w.out = dv;
    if ((e = run(p.type, w, Grade::Narrow, false, stream)) != hipSuccess) return e;

    const uint32_t rows = (uint32_t)(p.batch * p.heads);
    if (rows) {
        k_gates<<<rows, kGateThreads, 0, stream>>>(
            w, floats(plan.dq_dots), walk_blocks((int)p.dv, (int)p.dk), floats(plan.dk_dots), walk_blocks((int)p.dv, (int)p.dk),
            dstate_out, floats(plan.last), state, p.fixed ? floats(plan.gates) : dlog_decay);
        if (dstate) k_first_decay<<<rows, 256, 0, stream>>>(w, dstate, state);
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
