// attend.hip -- linear attention with a decay for each head: the walk over a
// row's tokens (attend.hpp), the gradients made of it, and the single token.
#include "attend.hpp"
#include "launch.hpp"

namespace ls {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

// Gradients by head, batch x steps x heads x width fp32, to those of the groups: dq's
// and dk's at once.
template <class T>
__global__ void __launch_bounds__(256) k_join_heads(const float* dq_in, const float* dk_in, T* dq,
                                                    T* dk, int64_t count, int per, int width) {
    const float* in = blockIdx.y ? dk_in : dq_in;
    T* out = blockIdx.y ? dk : dq;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < count;
         i += (int64_t)gridDim.x * 256) {
        const int64_t at = i / width * per * width + i % width;
        float sum = 0.0f;
#pragma unroll 4
        for (int j = 0; j < per; ++j) sum += in[at + (int64_t)j * width];
        out[i] = from_f32<T>(sum);
    }
}

// A sum in 64 bits, over what comes behind the last place that starts it anew.
struct Run {
    double sum;
    int anew;  // there is such a place
};
__device__ __forceinline__ Run then(const Run& a, const Run& b) {
    return b.anew ? b : Run{a.sum + b.sum, a.anew};
}

// Runs over the workgroup's threads: v becomes the run over the threads before this one (no
// difference of sums: a NaN of its own or behind it is not in it); returns that of all.
constexpr int kGateThreads = 256, kGateWaves = kGateThreads / 64;
__device__ Run block_scan(Run& v, Run* s) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const Run up{__shfl_up(v.sum, m), __shfl_up(v.anew, m)};
        if (lane >= m) v = then(up, v);
    }
    if (lane == 63) s[wave] = v;
    v = {__shfl_up(v.sum, 1), __shfl_up(v.anew, 1)};
    if (lane == 0) v = {};
    __syncthreads();
    Run all{};
#pragma unroll
    for (int i = 0; i < kGateWaves; ++i) {
        if (i == wave) v = then(all, v);
        all = then(all, s[i]);
    }
    __syncthreads();
    return all;
}
__device__ double block_sum(double v, Run* s) {
    Run run{v, 0};
    return block_scan(run, s).sum;
}

// The decays' gradients: dg[t] = <G[t], e^g[t] S[t-1]> at the tokens whose states are there
// (kMark), and <dS, S> behind a row's last token; before them dg[t] = dg[t+1] + (q.dq -
// k.dk)[t].  And dS_0 = e^g[0] G[0], in place (a row without tokens keeps dS).  A token
// whose decay clears the state has a gradient of 0, and those before it have no part in the
// sums behind it, which start anew there.  A workgroup to kMark tokens of a row and head: 64
// rows of 2048 tokens, 128 x 128, 11 us for 30 MB.
struct Gates {
    const float* dq_dots;
    const float* dk_dots;
    int blocks;            // of dots
    const float* s_marks;  // S, and G
    const float* g_marks;
    const float* dstate_out;  // and the last state, where it is given
    const float* last;
    int64_t state, mark;  // elements of a state, and of one of the marks
    float* dstate;        // nullable
    float* out;
};
__device__ double inner_product(const float* a, const float* b, int64_t n, Run* s) {
    typedef f4 Vec __attribute__((aligned(4)));
    double v = 0.0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < n / 4; i += kGateThreads) {
        const f4 x = ((const Vec*)a)[i], y = ((const Vec*)b)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) v += (double)x[e] * y[e];
    }
    const int64_t i = n / 4 * 4 + threadIdx.x;
    if (i < n) v += (double)a[i] * b[i];
    return block_sum(v, s);
}
__global__ void __launch_bounds__(kGateThreads) k_gates(Walk w, Gates a) {
    constexpr int PER = kMark / kGateThreads;
    __shared__ Run s[kGateWaves];
    const int tid = threadIdx.x, marks = walk_marks(w.steps);
    const int64_t tokens = (int64_t)w.batch * w.steps * w.heads;
    const int64_t count = (int64_t)w.batch * w.heads * (marks + 1);
    for (int64_t at = blockIdx.x; at < count; at += gridDim.x) {
        const int part = (int)(at % (marks + 1));
        const int64_t bh = at / (marks + 1);
        const int h = (int)(bh % w.heads), b = (int)(bh / w.heads);
        const int len = walk_len(w, b), end = part * kMark + kMark;
        const float* g = w.g + b * w.g_batch + h;
        Run after{};
        if (end < len) {
            const float decay = g[end * w.g_step];
            const int64_t mark = (bh * marks + part) * a.mark;
            const double all = inner_product(a.g_marks + mark, a.s_marks + mark, a.mark, s);
            if (!clears(decay)) after.sum = all * exp2_fast(decay * kLog2e);
        } else if (a.dstate_out && end - kMark < len) {
            after.sum = inner_product(a.dstate_out + bh * a.state, a.last + bh * a.state, a.state, s);
        }
        const int t0 = end - 1 - tid * PER;  // thread 0 has the last tokens
        const int64_t to = ((int64_t)b * w.steps + t0) * w.heads + h;
        Run v[PER], sum{};
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            v[i] = {};
            if (t0 - i < len) {
                v[i].anew = clears(g[(t0 - i) * w.g_step]);
                if (!v[i].anew)
                    for (int k = 0; k < a.blocks; ++k)
                        v[i].sum += (double)a.dq_dots[k * tokens + to - (int64_t)i * w.heads] -
                                    a.dk_dots[k * tokens + to - (int64_t)i * w.heads];
            }
            v[i] = sum = then(sum, v[i]);
        }
        block_scan(sum, s);
        const Run before = then(after, sum);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (t0 - i < w.steps)
                a.out[to - (int64_t)i * w.heads] =
                    t0 - i < len ? (float)then(before, v[i]).sum : 0.0f;
        if (a.dstate && part == 0 && len > 0) {
            typedef f4 Vec __attribute__((aligned(4)));
            const float decay = exp2_fast(g[0] * kLog2e);
            float* state = a.dstate + bh * a.state;
#pragma unroll 8
            for (int64_t i = tid; i < a.state / 4; i += kGateThreads) ((Vec*)state)[i] *= decay;
            const int64_t i = a.state / 4 * 4 + tid;
            if (i < a.state) state[i] *= decay;
        }
    }
}

// One decay for all tokens of a head: the sum of their gradients.
__global__ void __launch_bounds__(kGateThreads) k_gate_sum(const float* in, float* out,
                                                           int64_t tokens, int heads) {
    __shared__ Run s[kGateWaves];
    double v = 0.0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < tokens; i += kGateThreads) v += in[i * heads + blockIdx.x];
    v = block_sum(v, s);
    if (threadIdx.x == 0) out[blockIdx.x] = (float)v;
}

// The states before every piece from what each adds, in place: a workgroup to 256
// elements of a row and head; piece i of element x is states[i * each + x].  A piece's
// product of decays, x 2^y (WholePiece), may be beyond fp32 where the state that it meets is 0
// or small: the state is scaled by the exponent first, which leaves 0 what it is.
struct Carry {
    float* states;
    const WholePiece* whole;
    const float* first;  // nullable
    float* last;         // nullable
};
struct Carries {
    Carry c[2];
};
// AHEAD loads on their way; the chain itself is a scaling and a multiply-add each.  16 are for the few rows
// that are cut into many pieces (52 pieces of 8 rows' 64 x 128: 15 to 8 us); where there
// are enough threads without them they cost (64 rows' 8 pieces of 128 x 128: 14 to 18).
template <int AHEAD>
__global__ void __launch_bounds__(256) k_carry(Carries all, int pieces, int64_t each) {
    const Carry& c = all.c[blockIdx.y];
    const int64_t groups = (each + 255) / 256, bh = blockIdx.x / groups;
    const int64_t x = blockIdx.x % groups * 256 + threadIdx.x;
    if (x >= each) return;
    float* at = c.states + bh * pieces * each + x;
    const WholePiece* whole = c.whole + bh * pieces;
    float run = c.first ? c.first[bh * each + x] : 0.0f;
    for (int first = 0; first < pieces; first += AHEAD) {
        float more[AHEAD];
        WholePiece decay[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (first + i < pieces) more[i] = at[(first + i) * each], decay[i] = whole[first + i];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (first + i >= pieces) break;
            at[(first + i) * each] = run;
            run = __builtin_fmaf(decay[i].factor,
                                 __builtin_amdgcn_ldexpf(run, decay[i].exponent), more[i]);
        }
    }
    if (c.last) c.last[bh * each + x] = run;
}

// ------------------------------------------------ a single token

// A workgroup to `cols` columns (a multiple of 4) of a row's head: a thread has four
// columns of every `down`-th row, and the threads of a column add up what they have of
// the output.  Bound by the state's bytes, read and written once: 64 x 32 states of 128 x
// 128 in 43 us (97 by single loads, a column to a thread).
constexpr int kStepThreads = 256;
template <class T>
__global__ void __launch_bounds__(kStepThreads)
    k_attend_step(libscan_attend p, float* states, int64_t n_states, const int32_t* slots, T* y,
                  int cols) {
    constexpr int AHEAD = 8;
    __shared__ float s_q[256], s_k[256];
    __shared__ f4 s_out[kStepThreads];
    const int dk = (int)p.dk, dv = (int)p.dv, heads = (int)p.heads;
    const int blocks = (dv + cols - 1) / cols;
    const int block = blockIdx.x % blocks, bh = blockIdx.x / blocks;
    const int h = bh % heads, b = bh / heads, tid = threadIdx.x;
    const int across = cols / 4, down = kStepThreads / across;
    const int c = block * cols + tid % across * 4, row = tid / across, count = dv - c;
    const int64_t slot = slots ? slots[b] : b;
    const bool held = slot >= 0 && slot < n_states;
    const bool on = held && row < down && count > 0;
    const int share = heads / (int)p.groups;
    float g = p.fixed ? p.log_decay[h] : p.log_decay[b * p.decay_batch + h];
    f4 v{}, o{};
    if (on) {
        Pack<T, 4> x;
        x.load((const T*)p.v + b * p.v_batch + h * p.v_head + c, count);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = to_f32(x.v[e]);
    }
    for (int r = tid; r < dk; r += kStepThreads) {
        s_q[r] = to_f32(((const T*)p.q + b * p.q_batch + (h / share) * p.q_head)[r]);
        s_k[r] = to_f32(((const T*)p.k + b * p.k_batch + (h / share) * p.k_head)[r]);
    }
    __syncthreads();
    if (on) {
        const float a = exp2_fast(g * kLog2e);
        float* s = states + ((slot * heads + h) * dk + row) * dv + c;
        const int64_t step = (int64_t)down * dv;
        for (int r = row; r < dk; r += AHEAD * down, s += AHEAD * step) {
            Pack<float, 4> x[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (r + i * down < dk) x[i].load(s + i * step, count);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (r + i * down >= dk) break;
                const float k = s_k[r + i * down], q = s_q[r + i * down];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[i].v[e] = __builtin_fmaf(k, v[e], a * x[i].v[e]);
                    o[e] = __builtin_fmaf(q, x[i].v[e], o[e]);
                }
                x[i].store(s + i * step, count);
            }
        }
    }
    // a column's threads lie `across` apart: those of a wave by shifts, if that is a power
    // of two, then what is left one by one (four columns of 64 rows: 63 LDS reads otherwise,
    // 1 of 5.5 us)
    int apart = across;
    if ((across & (across - 1)) == 0 && across <= 64) {
        for (int m = across; m < 64; m <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m);
        apart = 64;
    }
    s_out[tid] = o;
    __syncthreads();
    if (row == 0 && count > 0) {
        for (int i = tid + apart; i < across * down; i += apart) o += s_out[i];
        Pack<T, 4> out;
#pragma unroll
        for (int e = 0; e < 4; ++e) out.v[e] = from_f32<T>(held ? o[e] * (float)p.scale : 0.0f);
        out.store(y + (int64_t)bh * dv + c, count);
    }
}

// ------------------------------------------------ launches

hipError_t run(int64_t type, const Walks& w, bool states, hipStream_t stream) {
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
// v gives what each piece adds to the state.  More pieces make for more workgroups and a
// longer carry, which reads and writes every piece's state.  The times that are weighed
// up are those of 128 x 128 states in bf16, in units of 5 us: 512 workgroups (two to a CU) walk
// n chunks of 64 tokens in 2 n + 1.5 and run for their states in 0.8 n + 1.4, 256 in 1.2 n
// + 1.5 and 0.45 n + 1.3; the carry moves 4.6 TB/s; two launches take 1.  (Measured with
// scores and states in two terms; with three the walks take 3 to 15 % more.)  fp32's chunks
// take more than twice as long, in six products for three.
struct Pieces {
    int count, places;
};
// `together`: walks of one launch.
Pieces pieces(const libscan_attend& p, int together) {
    const int64_t chunk = 64, chunks = (p.steps + chunk - 1) / chunk;
    const int64_t groups = together * p.batch * p.heads * walk_blocks((int)p.dv);
    const auto time = [](int64_t count, double full, double half) {
        const int64_t left = count % 512;
        return count / 512 * full + (left > 256 ? full : left ? half : 0.0);
    };
    const double slow = p.type == LIBSCAN_F32 ? 2.2 : 1.0;
    const auto walk = [&](int64_t n, int64_t size) {
        return time(groups * n, slow * 2.0 * size + 1.5, slow * 1.2 * size + 1.5);
    };
    int64_t each = chunks;
    double best = walk(1, chunks);
    for (int64_t n = 2; n <= chunks && groups * n <= 2048; ++n) {
        const int64_t size = (chunks + n - 1) / n, count = (chunks + size - 1) / size;
        const double cost = walk(count, size) +
                            time(groups * count, slow * 0.8 * size + 1.4, slow * 0.45 * size + 1.3) +
                            together * p.batch * p.heads * count * p.dk * p.dv * 8 / 4.6e6 / 5 + 1;
        if (cost < best) best = cost, each = size;
    }
    if (each >= chunks) return {1, (int)(chunks * chunk)};
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
    Pieces n;
    int64_t states, whole;
    Cut(const libscan_attend& p, int together, Room& room) : n(pieces(p, together)) {
        const int64_t all = n.count > 1 ? p.batch * p.heads * n.count : 0;
        states = room.floats(all * p.dk * p.dv);
        whole = room.floats(all * (int64_t)(sizeof(WholePiece) / 4));
    }
};
struct FrontPlan {
    Room room;
    Cut cut;
    FrontPlan(const libscan_attend& p) : cut(p, 1, room) {}
};
struct BackPlan {
    Room room;
    Cut cut, back;  // of S, and of its gradient
    int64_t dq_dots, dk_dots, mark, s_marks, g_marks, gates, last, dq, dk;
    BackPlan(const libscan_attend& p) : cut(p, 2, room), back(p, 2, room) {
        const int64_t tokens = p.batch * p.steps * p.heads;
        const int64_t blocks = walk_blocks((int)p.dk);
        const bool shared = p.groups < p.heads;
        dq_dots = room.floats(tokens * blocks);
        dk_dots = room.floats(tokens * blocks);
        const int64_t state = p.batch * p.heads * p.dk * p.dv;
        mark = p.dk * walk_width((int)p.dv);
        s_marks = room.floats(p.batch * p.heads * walk_marks((int)p.steps) * mark);
        g_marks = room.floats(p.batch * p.heads * walk_marks((int)p.steps) * mark);
        gates = room.floats(p.fixed ? tokens : 0);
        last = room.floats(state);
        dq = room.floats(shared ? tokens * p.dk : 0);
        dk = room.floats(shared ? tokens * p.dk : 0);
    }
};

// The states before every piece of the walks, whose first and last states are their
// rows'; the walks then take them.
hipError_t cut_rows(const libscan_attend& p, Walks& walks, const Cut* const (&cuts)[2], char* mem,
                    hipStream_t stream) {
    const Pieces n = cuts[0]->n;
    for (int i = 0; i < walks.count; ++i) walks.w[i].pieces = n.count, walks.w[i].piece = n.places;
    if (n.count == 1) return hipSuccess;
    Walks states = walks;
    Carries carries{};
    for (int i = 0; i < walks.count; ++i) {
        Walk &s = states.w[i], &w = walks.w[i];
        s.first = {};
        s.last = {(float*)(mem + cuts[i]->states), p.dv, 1};
        s.whole = (WholePiece*)(mem + cuts[i]->whole);
        carries.c[i] = {s.last.p, s.whole, w.first.p, w.last.p};
        w.first = s.last;
        w.last = {};
    }
    const hipError_t e = run(p.type, states, true, stream);
    if (e != hipSuccess) return e;
    const int64_t each = p.dk * p.dv, blocks = p.batch * p.heads * ((each + 255) / 256);
    if (blocks == 0) return hipSuccess;
    const dim3 grid((uint32_t)blocks, walks.count);
    if (n.count > 8)
        k_carry<16><<<grid, 256, 0, stream>>>(carries, n.count, each);
    else
        k_carry<8><<<grid, 256, 0, stream>>>(carries, n.count, each);
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
    const FrontPlan plan(p);
    Walks walks{{w}, 1};
    const hipError_t e = cut_rows(p, walks, {&plan.cut, nullptr}, (char*)scratch, stream);
    return e != hipSuccess ? e : run(p.type, walks, false, stream);
}

hipError_t launch_attend_back(const libscan_attend& p, const void* dy, int64_t dy_batch,
                              int64_t dy_step, int64_t dy_head, const float* dstate_out, void* dq,
                              void* dk, void* dv, float* dlog_decay, float* dstate, void* scratch,
                              hipStream_t stream) {
    const BackPlan plan(p);
    char* mem = (char*)scratch;
    const auto floats = [&](int64_t at) { return (float*)(mem + at); };
    const bool shared = p.groups != p.heads;  // without heads, the groups' sums are over none
    const WalkSide side_dy = {dy, dy_batch, dy_step, dy_head, 1};
    const int dots = walk_blocks((int)p.dk);
    float* last = dstate_out ? floats(plan.last) : nullptr;
    hipError_t e;

    // S forwards, and its gradient G backwards
    Walks both{{base(p), base(p)}, 2};
    Walk &s = both.w[0], &g = both.w[1];
    s.dk = g.dk = (int)p.dk, s.dv = g.dv = (int)p.dv;
    s.k = side_k(p), s.v = side_v(p);
    s.first = {const_cast<float*>(p.state), p.dv, 1};
    s.last = {last, p.dv, 1};
    g.reverse = true;
    g.k = side_q(p), g.v = side_dy;
    g.inner = (float)p.scale;
    g.first = {const_cast<float*>(dstate_out), p.dv, 1};
    g.last = {dstate, p.dv, 1};
    if ((e = cut_rows(p, both, {&plan.cut, &plan.back}, mem, stream)) != hipSuccess) return e;

    Walks one{{g}, 1};  // dv, with G
    one.w[0].q = side_k(p);
    one.w[0].out = dv;
    if ((e = run(p.type, one, false, stream)) != hipSuccess) return e;

    Walks two{{s, g}, 2};  // dq with S and dk with G, turned over
    Walk &wq = two.w[0], &wk = two.w[1];
    wq.dk = wk.dk = (int)p.dv, wq.dv = wk.dv = (int)p.dk;
    wq.q = side_dy, wq.k = side_v(p), wq.v = side_k(p);
    wq.outer = (float)p.scale;
    wq.first = {s.first.p, 1, p.dv};
    wq.last = {s.last.p, 1, p.dv};
    wq.out = shared ? floats(plan.dq) : dq;
    wq.e = side_q(p);
    wq.dots = floats(plan.dq_dots);
    wq.marks = floats(plan.s_marks);
    wk.q = side_v(p), wk.k = side_dy, wk.v = side_q(p);
    wk.first = {g.first.p, 1, p.dv};
    wk.last = {};
    wk.out = shared ? floats(plan.dk) : dk;
    wk.e = side_k(p);
    wk.dots = floats(plan.dk_dots);
    wk.marks = floats(plan.g_marks);
    wq.wide = wk.wide = shared;
    if ((e = run(p.type, two, false, stream)) != hipSuccess) return e;

    const int64_t parts = p.steps ? p.batch * p.heads * (walk_marks((int)p.steps) + 1) : 0;
    const int64_t most = 1 << 20;  // workgroups; the rest in further turns
    if (parts) {
        const Gates a{floats(plan.dq_dots), floats(plan.dk_dots), dots, floats(plan.s_marks),
                      floats(plan.g_marks), dstate_out, last, p.dk * p.dv, plan.mark, dstate,
                      p.fixed ? floats(plan.gates) : dlog_decay};
        k_gates<<<(uint32_t)(parts < most ? parts : most), kGateThreads, 0, stream>>>(g, a);
    }
    if (p.fixed && p.heads)
        k_gate_sum<<<(uint32_t)p.heads, kGateThreads, 0, stream>>>(
            floats(plan.gates), dlog_decay, p.batch * p.steps, (int)p.heads);
    const int64_t count = p.batch * p.steps * p.groups * p.dk;
    if (shared && count) {
        const int64_t blocks = (count + 255) / 256;
        const dim3 grid((uint32_t)(blocks < most ? blocks : most), 2);
        const auto join = [&](auto zero) {
            using T = decltype(zero);
            k_join_heads<<<grid, 256, 0, stream>>>(floats(plan.dq), floats(plan.dk), (T*)dq, (T*)dk,
                                                   count, (int)(p.heads / p.groups), (int)p.dk);
        };
        if (p.type == LIBSCAN_F32) join(float());
        else if (p.type == LIBSCAN_F16) join(_Float16());
        else join(__bf16());
    }
    return hipGetLastError();
}

hipError_t launch_attend_step(const libscan_attend& p, float* states, int64_t n_states,
                              const int32_t* slots, void* y, hipStream_t stream) {
    // whole rows of the state to a workgroup, where that makes enough of them: longer runs
    // of bytes, fewer sums
    const int64_t rows = p.batch * p.heads;
    int64_t cols = (p.dv + 3) / 4 * 4;
    while (cols > 16 && rows * ((p.dv + cols - 1) / cols) < 512) cols = (cols / 2 + 3) / 4 * 4;
    const uint32_t grid = (uint32_t)(rows * ((p.dv + cols - 1) / cols));
    const auto go = [&](auto zero) {
        using T = decltype(zero);
        k_attend_step<T><<<grid, kStepThreads, 0, stream>>>(p, states, n_states, slots, (T*)y,
                                                            (int)cols);
    };
    if (p.type == LIBSCAN_F32) go(float());
    else if (p.type == LIBSCAN_F16) go(_Float16());
    else go(__bf16());
    return hipGetLastError();
}

}  // namespace ls
