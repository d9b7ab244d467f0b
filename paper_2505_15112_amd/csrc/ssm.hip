// ssm.hip -- the selective scan (prompts) and its single-token step.
//
// h[t] = a[t] h[t-1] + b[t] per channel and state index, a = exp(delta A),
// b = delta x B; y = sum over the state index of C h, plus D x, times
// silu(z).  One exponential and four multiply-adds for every step, channel and
// state, against 2 n of them to the bytes of one x: the vector units bound a
// scan (4 waves to a SIMD: 10.5 ns for the five instructions of a wave), not
// HBM.  States, sums and step sizes are fp32 whatever the type of the inputs;
// y is rounded once.  exp(delta A) is 2^(delta (A log2 e)), A scaled once.
//
// Two ways to cut a call up (lane_plan says which, from measured times):
// tiles (k_ssm_scan), one kernel that walks every row from end to end with a
// channel's states shared out over lanes, for rows that fill the chip or are
// short; and chunks (k_ssm_bc, k_ssm_ends, k_ssm_starts, k_ssm_lanes) with a
// channel to a lane, for few long rows, whose steps are the latency.
#include "launch.hpp"
#include "lm.hpp"
#include "ssm.hpp"

namespace ls {

namespace {

constexpr int kTile = 32;     // steps per tile
constexpr int kThreads = 256;

// The tiles.  A workgroup owns CH channels of one row and walks the row in tiles
// of 32 steps.  What depends on step and channel alone (softplus, delta x) is
// computed once per tile by threads that own 16 bytes of channels, and goes
// through LDS to the lanes that own (channel, state) pairs; their sums over
// the state index are shared out over the lanes of a channel, 16 steps at a
// time, and go back the same way to be gated and stored.  The states stay in
// registers for the whole row.
// WHOLE: every row has all its steps, in whole tiles, and every workgroup all its
// channels and states, so that nothing needs a check.  n = 16, with and without
// the checks: 4 x 2048 x 4096 169 and 184 us, 1 x 2048 x 4096 98 and 116; four
// lanes to a channel took a third longer on the first, for want of waves.
// Ragged 16 x 501 x 4096: 95 us.
// Lanes whose states are padding read a delta and x of 0 (column CH): an infinite one
// would make infinity times 0 of the padding's B, and NaN of the channel's sum.  PART:
// some lane's states are padding in part (n is no multiple of SPL), and are held at 0.
template <class T, int LN, int SPL, bool WHOLE, bool PART>
__global__ __launch_bounds__(kThreads) void k_ssm_scan(libscan_ssm p, T* y, float* state_out,
                                                       float* ckpt, int nb) {
    using L = SsmLanes<LN, SPL>;
    constexpr int CH = L::CH, NP = L::NP, TPR = kThreads / kTile, VW = CH / TPR, YS = CH + 4;
    constexpr int NBC = kTile * NP / kThreads;
    __shared__ float2 s_du[kTile][WHOLE ? CH : CH + 2];  // delta, delta x
    __shared__ float2 s_bc[kTile][NP];
    __shared__ float s_y[kTile][YS];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int steps = (int)p.steps, dim = (int)p.dim, n = (int)p.n;
    const SsmBlock k = ssm_block(p, nb, CH, blockIdx.x);
    const int len = WHOLE ? steps : ssm_len(p, k.b);
    const int lim = WHOLE ? CH : k.lim;
    const bool gate = p.z != nullptr;

    // loader: one step, VW channels; NBC states of B and C
    const int row = tid / TPR, lc = (tid % TPR) * VW;
    const int lcount = WHOLE ? VW : lim - lc;  // channels that exist (may be <= 0)
    const int64_t ch0 = k.c0 + lc;
    const T* px = (const T*)p.x + k.b * p.x_batch + row * p.x_step + ch0;
    const T* pdt = (const T*)p.dt + k.b * p.dt_batch + row * p.dt_step + ch0;
    const T* pz = (const T*)p.z + k.b * p.z_batch + row * p.z_step + ch0;
    const int bt = tid * NBC / NP, bn = tid * NBC % NP;
    const T* pB = (const T*)p.B + k.b * p.B_batch + k.g * p.B_group + bt * p.B_step + bn;
    const T* pC = (const T*)p.C + k.b * p.C_batch + k.g * p.C_group + bt * p.C_step + bn;
    T* py = y + ((int64_t)k.b * steps + row) * dim + ch0;
    float bias[VW], skip[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) {
        bias[i] = p.dt_bias && (WHOLE || i < lcount) ? p.dt_bias[ch0 + i] : 0.0f;
        skip[i] = p.D && (WHOLE || i < lcount) ? p.D[ch0 + i] : 0.0f;
    }

    // scanner: channel wc, states n0 .. n0 + SPL
    const int wc = wave * L::CPW + L::channel(lane), n0 = L::part(lane) * SPL;
    const int from = WHOLE || n0 < n ? wc : CH;
    if (!WHOLE && tid < kTile) s_du[tid][CH] = float2{0.0f, 0.0f};
    float a2[SPL], h[SPL];
    const int64_t sbase = ((int64_t)k.b * dim + k.c0 + wc) * n + n0;
    float* pck = ckpt + ((int64_t)k.b * ((steps + kSsmBlock - 1) / kSsmBlock) * dim + k.c0 + wc) * n +
                 n0;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        const bool in = WHOLE || (wc < lim && n0 + s < n);
        a2[s] = in ? p.A[(int64_t)(k.c0 + wc) * n + n0 + s] * kLog2e : 0.0f;
        h[s] = in && p.state ? p.state[sbase + s] : 0.0f;
    }

    Pack<T, VW> nx, ndt, nz;
    Pack<T, NBC> nB, nC;
    auto fetch = [&](int t0) {
        const bool all = WHOLE || (lim == CH && n == NP && t0 + kTile <= len);
        const int count = all ? VW : t0 + row < len ? lcount : 0;
        const int bcount = all ? NBC : t0 + bt < len ? n - bn : 0;
        nx.load(px + t0 * p.x_step, count);
        ndt.load(pdt + t0 * p.dt_step, count);
        nz.load(pz + t0 * p.z_step, gate ? count : 0);
        nB.load(pB + t0 * p.B_step, bcount);
        nC.load(pC + t0 * p.C_step, bcount);
    };

    if (len > 0) fetch(0);
    for (int t0 = 0; t0 < len; t0 += kTile) {
        const bool live = WHOLE || t0 + row < len;
        const Pack<T, VW> rx = nx, rz = nz;
        float delta[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) delta[i] = to_f32(ndt.v[i]) + bias[i];
        if (p.softplus) {
#pragma unroll
            for (int i = 0; i < VW; ++i) delta[i] = softplus(delta[i]);
        }
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            const float d = WHOLE || (live && i < lcount) ? delta[i] : 0.0f;  // then a = 1, b = 0
            s_du[row][lc + i] = float2{d, d * to_f32(rx.v[i])};
        }
#pragma unroll
        for (int i = 0; i < NBC; ++i)
            s_bc[bt][bn + i] = float2{to_f32(nB.v[i]), to_f32(nC.v[i])};
        __syncthreads();
        if (t0 + kTile < len) fetch(t0 + kTile);

#pragma unroll 1
        for (int tb = 0; tb < kTile; tb += kSsmBlock) {
            if (!WHOLE && t0 + tb >= len) break;
            if (ckpt) {
                float* pc = pck + (int64_t)((t0 + tb) / kSsmBlock) * dim * n;
#pragma unroll
                for (int s = 0; s < SPL; ++s)
                    if (WHOLE || (wc < lim && n0 + s < n)) pc[s] = h[s];
            }
            float v[kSsmBlock];
#pragma unroll
            for (int t = 0; t < kSsmBlock; ++t) {
                const float2 du = s_du[tb + t][from];
                float acc = 0.0f;
#pragma unroll
                for (int s = 0; s < SPL; ++s) {
                    const float2 bc = s_bc[tb + t][n0 + s];
                    const float a = exp2_fast(du.x * a2[s]);
                    h[s] = __builtin_fmaf(a, h[s], du.y * bc.x);
                    if (PART && s && n0 + s >= n) h[s] = 0.0f;
                    acc = __builtin_fmaf(h[s], bc.y, acc);
                }
                v[t] = acc;
            }
            L::sum_states(v, lane, [&](int t, float sum) { s_y[tb + t][wc] = sum; });
        }
        __syncthreads();
        if (WHOLE || t0 + row < steps) {
            Pack<T, VW> out;
            float v[VW];
#pragma unroll
            for (int i = 0; i < VW; ++i)
                v[i] = __builtin_fmaf(skip[i], to_f32(rx.v[i]), s_y[row][lc + i]);
            if (gate) {
#pragma unroll
                for (int i = 0; i < VW; ++i) {
                    const float z = to_f32(rz.v[i]);
                    v[i] *= z * sigmoid(z);
                }
            }
#pragma unroll
            for (int i = 0; i < VW; ++i) out.v[i] = from_f32<T>(live ? v[i] : 0.0f);
            out.store(py + (int64_t)t0 * dim, lcount);
        }
    }
    // the steps past the row's tokens that no tile above has reached
    for (int t = (len + kTile - 1) / kTile * kTile; !WHOLE && t + row < steps; t += kTile) {
        Pack<T, VW> out;
#pragma unroll
        for (int i = 0; i < VW; ++i) out.v[i] = T(0);
        out.store(py + (int64_t)t * dim, lcount);
    }
    if (state_out) {
#pragma unroll
        for (int s = 0; s < SPL; ++s)
            if (WHOLE || (wc < lim && n0 + s < n)) state_out[sbase + s] = h[s];
    }
}

// ---------------------------------------------------------------- long rows

// B and C of the whole call for k_ssm_lanes and k_ssm_ends, which read them with
// scalar loads and thus in fp32: 1 x 4096 tokens, n = 16: 5 us, launch and latency.
template <class T, int NP>
__global__ __launch_bounds__(kThreads) void k_ssm_bc(libscan_ssm p, float* bc) {
    constexpr int GP = LaneGroups<NP>::GP;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= p.batch * p.steps * p.groups * NP) return;
    const int nn = (int)(i % NP);
    const int64_t tok = i / NP, bt = tok / p.groups;
    const int g = (int)(tok % p.groups), b = (int)(bt / p.steps), t = (int)(bt % p.steps);
    const bool in = nn < p.n && t < ssm_len(p, b);
    const T* pB = (const T*)p.B + b * p.B_batch + t * p.B_step + g * p.B_group;
    const T* pC = (const T*)p.C + b * p.C_batch + t * p.C_step + g * p.C_group;
    float* out = bc + tok * 2 * NP + nn / GP * 2 * GP + nn % GP;
    out[0] = in ? to_f32(pB[nn]) : 0.0f;
    out[GP] = in ? to_f32(pC[nn]) : 0.0f;
}

// The scan with a channel to a lane and all of its states in registers: B and C
// are the same for all lanes and come by scalar loads, so that a step costs five
// vector instructions for each state (one of them the exponential) and nothing
// goes through LDS.  Rows are cut into chunks until the waves fill the chip;
// `starts` (NULL for one chunk) holds the states that the chunks start from.
// 1 x 4096 x 4096, n = 16, 64 chunks: 72 us, against 43 for those instructions
// alone.  A step issues 113 vector instructions, not those 80 (the softplus, the gate,
// types and addresses are the others), and the vector units are busy for 76 % of the
// time; the scalar loads are not what they wait for (with the loads taken out it was
// no faster).  1 x 16389 x 2048: 149 us against 86.
// PAD: n < NP, and the states past n (n > NP / 2 but for 8) are held at 0 or left out,
// four at a time: an infinite delta or x would make NaN of them, and of y.
template <class T, int NP, bool GATE, bool PAD>
__global__ __launch_bounds__(kWave * kLaneWaves) void k_ssm_lanes(libscan_ssm p, const float* bc_,
                                                                  const float* starts, T* y,
                                                                  float* state_out, float* ckpt,
                                                                  int nb, int chunk,
                                                                  uint32_t waves) {
    using Groups = LaneGroups<NP>;
    constexpr int GP = Groups::GP, NG = Groups::NG;
    if (blockIdx.x * kLaneWaves + threadIdx.x / kWave >= waves) return;
    const LaneBlock w = lane_block(p, nb, chunk, blockIdx.y);
    const int b = w.k.b, c0 = w.k.c0, ch = c0 + (int)w.lo;
    const uint32_t lo = w.lo;
    const int dim = (int)p.dim, n = (int)p.n, steps = (int)p.steps;
    const int64_t bc_step = p.groups * 2 * NP;
    ScalarPtr bc = (ScalarPtr)bc_ + (((int64_t)b * steps + w.t0) * p.groups + w.k.g) * 2 * NP;
    StepPtr<const T> px{(const T*)p.x + b * p.x_batch + w.t0 * p.x_step + c0, p.x_step};
    StepPtr<const T> pdt{(const T*)p.dt + b * p.dt_batch + w.t0 * p.dt_step + c0, p.dt_step};
    StepPtr<const T> pz{GATE ? (const T*)p.z + b * p.z_batch + w.t0 * p.z_step + c0 : nullptr,
                        p.z_step};
    StepPtr<T> py{y + ((int64_t)b * steps + w.t0) * dim + c0, dim};
    const float bias = p.dt_bias ? p.dt_bias[ch] : 0.0f, skip = p.D ? p.D[ch] : 0.0f;
    const int64_t row = (int64_t)b * dim + ch;
    float a2[NP], h[NP];
    {
        const float* from = starts ? starts + ((int64_t)w.c * p.batch * dim + row) * NP
                                   : p.state ? p.state + row * n : nullptr;
        const int have = starts || p.state ? n : 0;
        load_states<NP>(p.A + (int64_t)ch * n, n, a2);
        load_states<NP>(from, have, h);
#pragma unroll
        for (int i = 0; i < NP; ++i) a2[i] *= kLog2e;
    }

    Groups cur;
    if (w.t0 < w.end) cur.template load<2 * GP>(bc);
    auto step = [&](T x, float delta, T z) {
        const float u = delta * to_f32(x);
        float acc[2] = {skip * to_f32(x), 0.0f};
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            scalar_loads_done();
            Groups next;  // of this step, or the first of the next (one past the last is there)
            if (g + 1 == NG) bc += bc_step;
            next.template load<2 * GP>(g + 1 < NG ? bc + (g + 1) * 2 * GP : bc);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i0 = 0; i0 < GP; i0 += 4) {
                const int s0 = g * GP + i0;
                if (PAD && s0 >= NP / 2 && s0 >= n) break;
#pragma unroll
                for (int i = i0; i < i0 + 4; ++i) {
                    float& hi = h[g * GP + i];
                    hi = __builtin_fmaf(exp2_fast(delta * a2[g * GP + i]), hi, u * cur.v[i]);
                    if (PAD && (NP == 8 || s0 >= NP / 2) && g * GP + i >= n) hi = 0.0f;
                    acc[i & 1] = __builtin_fmaf(hi, cur.v[GP + i], acc[i & 1]);
                }
            }
            cur = next;
        }
        float v = acc[0] + acc[1];
        if (GATE) {
            const float zf = to_f32(z);
            v *= zf * sigmoid(zf);
        }
        py.p[lo] = from_f32<T>(v);
        py.next();
    };
    auto keep = [&](int t) {
        if (!ckpt || t % kSsmBlock) return;
        const int64_t blk = (int64_t)b * ((steps + kSsmBlock - 1) / kSsmBlock) + t / kSsmBlock;
        store_states<NP>(ckpt + (blk * dim + ch) * n, n, h);
    };

    int t = w.t0;
    T nx[kAhead], ndt[kAhead], nz[kAhead];
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            nx[i] = px.p[lo];
            ndt[i] = pdt.p[lo];
            nz[i] = GATE ? pz.p[lo] : T(0);
            px.next();
            pdt.next();
            if (GATE) pz.next();
        }
    };
    if (t + kAhead <= w.end) fetch();
    for (; t + kAhead <= w.end; t += kAhead) {
        T cx[kAhead], cz[kAhead];
        float delta[kAhead];
        step_sizes(p, ndt, bias, delta);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            cx[i] = nx[i];
            cz[i] = nz[i];
        }
        if (t + 2 * kAhead <= w.end) fetch();
        keep(t);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) step(cx[i], delta[i], cz[i]);
    }
#pragma unroll 1
    for (; t < w.end; ++t) {
        keep(t);
        const T dt[1] = {pdt.p[lo]};
        float delta[1];
        step_sizes(p, dt, bias, delta);
        step(px.p[lo], delta[0], GATE ? pz.p[lo] : T(0));
        px.next();
        pdt.next();
        if (GATE) pz.next();
    }
    const int stop = w.t0 + chunk < steps ? w.t0 + chunk : steps;
#pragma unroll 1
    for (t = w.t0 > w.len ? w.t0 : w.len; t < stop; ++t) {
        py.p[lo] = T(0);
        py.next();
    }
    if (state_out && stop == steps) store_states<NP>(state_out + row * n, n, h);
}

// What a chunk does to any state it starts from: its decay exp(A sum delta) and
// the state it ends in from zero.  1 x 4096 x 4096: 54 us; the price of the
// chunks, and with them still less than one walk over the row (tiles: 192 us
// for the call, chunks 128).
template <class T, int NP>
__global__ __launch_bounds__(kWave * kLaneWaves) void k_ssm_ends(libscan_ssm p, const float* bc_,
                                                                 float* ends, float* sums, int nb,
                                                                 int chunk, uint32_t waves) {
    using Groups = LaneGroups<NP>;
    constexpr int GP = Groups::GP, NG = Groups::NG;
    if (blockIdx.x * kLaneWaves + threadIdx.x / kWave >= waves) return;
    const LaneBlock w = lane_block(p, nb, chunk, blockIdx.y);
    const int b = w.k.b, c0 = w.k.c0, ch = c0 + (int)w.lo;
    const uint32_t lo = w.lo;
    const int dim = (int)p.dim, n = (int)p.n;
    const int64_t bc_step = p.groups * 2 * NP;
    ScalarPtr bc = (ScalarPtr)bc_ + (((int64_t)b * p.steps + w.t0) * p.groups + w.k.g) * 2 * NP;
    StepPtr<const T> px{(const T*)p.x + b * p.x_batch + w.t0 * p.x_step + c0, p.x_step};
    StepPtr<const T> pdt{(const T*)p.dt + b * p.dt_batch + w.t0 * p.dt_step + c0, p.dt_step};
    const float bias = p.dt_bias ? p.dt_bias[ch] : 0.0f;
    float a2[NP], h[NP], sum = 0.0f;
    load_states<NP>(p.A + (int64_t)ch * n, n, a2);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        a2[i] *= kLog2e;
        h[i] = 0.0f;
    }
    Groups cur;
    if (w.t0 < w.end) cur.template load<GP>(bc);
    auto step = [&](T x, float delta) {
        const float u = delta * to_f32(x);
        sum += delta;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            scalar_loads_done();
            Groups next;
            if (g + 1 == NG) bc += bc_step;
            next.template load<GP>(g + 1 < NG ? bc + (g + 1) * 2 * GP : bc);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < GP; ++i) {
                float& hi = h[g * GP + i];
                hi = __builtin_fmaf(exp2_fast(delta * a2[g * GP + i]), hi, u * cur.v[i]);
            }
            cur = next;
        }
    };
    int t = w.t0;
    T nx[kAhead], ndt[kAhead];
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            nx[i] = px.p[lo];
            ndt[i] = pdt.p[lo];
            px.next();
            pdt.next();
        }
    };
    if (t + kAhead <= w.end) fetch();
    for (; t + kAhead <= w.end; t += kAhead) {
        T cx[kAhead];
        float delta[kAhead];
        step_sizes(p, ndt, bias, delta);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) cx[i] = nx[i];
        if (t + 2 * kAhead <= w.end) fetch();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) step(cx[i], delta[i]);
    }
#pragma unroll 1
    for (; t < w.end; ++t) {
        const T dt[1] = {pdt.p[lo]};
        float delta[1];
        step_sizes(p, dt, bias, delta);
        step(px.p[lo], delta[0]);
        px.next();
        pdt.next();
    }
    const int64_t row = ((int64_t)w.c * p.batch + b) * dim + ch;
    store_states<NP>(ends + row * NP, NP, h);
    sums[row] = sum;
}

// Chains the chunks: a thread owns a (channel, state) pair and goes through the
// ends in order, 16 loads in flight.  1 x 4096 x 4096, n = 16, 64 chunks: 11 us.
// A whole chunk's decay 2^v may be beyond fp32 where h 2^v is not (of h = 0 nothing
// grows): then h 2^(v/2) 2^(v/2), with finite factors.  Only then, as it is one more
// multiplication after the other for every chunk (1 x 4096 x 2048, 128 chunks: 1.3 us).
template <int NP>
__global__ __launch_bounds__(kThreads) void k_ssm_starts(libscan_ssm p, const float* init,
                                                         float* ends, const float* sums,
                                                         int chunks, bool backward) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, rows = p.batch * p.dim;
    if (i >= rows * NP) return;
    const int64_t row = i / NP;
    const int nn = (int)(i % NP);
    const float a2 = nn < p.n ? p.A[row % p.dim * p.n + nn] * kLog2e : 0.0f;
    float h = init && nn < p.n ? init[row * p.n + nn] : 0.0f;
    constexpr int kBatch = 16;  // loads in flight together
    for (int j0 = 0; j0 < chunks; j0 += kBatch) {
        float e[kBatch], v[kBatch];
        bool beyond = false;
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const bool in = j0 + j + 1 < chunks;
            const int64_t at = (int64_t)(backward ? chunks - 1 - j0 - j : j0 + j) * rows;
            e[j] = in ? ends[at * NP + i] : 0.0f;
            v[j] = (in ? sums[at + row] : 0.0f) * a2;
            beyond |= v[j] >= 127.0f;
        }
        auto chain = [&](auto decayed) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (j0 + j < chunks) {
                    const int64_t at = (int64_t)(backward ? chunks - 1 - j0 - j : j0 + j) * rows;
                    ends[at * NP + i] = h;
                    h = decayed(v[j], e[j]);
                }
        };
        if (__any(beyond))
            chain([&](float v, float e) {
                float half = exp2_fast(0.5f * v);
                half = half > __FLT_MAX__ ? __FLT_MAX__ : half;
                return __builtin_fmaf(half, half * h, e);
            });
        else
            chain([&](float v, float e) { return __builtin_fmaf(exp2_fast(v), h, e); });
    }
}

// One token.  A quad of lanes owns a channel's states, four at a time: the
// states, read and written once, are all the traffic that counts.  128 rows of
// 5120 channels, n = 16: 20 us for 88 MB, 4.4 TB/s; one row of 2048: 4 us, launch
// and the latency of two dependent loads.
template <class T>
__global__ __launch_bounds__(kThreads) void k_ssm_step(libscan_ssm p, float* states,
                                                       int64_t n_states, const int32_t* slots,
                                                       T* y) {
    constexpr int CH = kThreads / 4;
    const int dim = (int)p.dim, n = (int)p.n;
    const int nb = (dim + CH - 1) / CH;
    const int b = blockIdx.x / nb, d = (blockIdx.x % nb) * CH + (threadIdx.x >> 2);
    const int q = threadIdx.x & 3;
    if (d >= dim) return;  // whole quads
    const int64_t slot = slots ? slots[b] : b;
    T* py = y + (int64_t)b * dim + d;
    if (slot < 0 || slot >= n_states) {
        if (q == 0) *py = T(0);
        return;
    }
    const int g = d / (dim / (int)p.groups);
    const float x = to_f32(((const T*)p.x)[b * p.x_batch + d]);
    float delta = to_f32(((const T*)p.dt)[b * p.dt_batch + d]) + (p.dt_bias ? p.dt_bias[d] : 0.0f);
    if (p.softplus) delta = softplus(delta);
    const float u = delta * x;
    const T* pB = (const T*)p.B + b * p.B_batch + g * p.B_group;
    const T* pC = (const T*)p.C + b * p.C_batch + g * p.C_group;
    const float* pA = p.A + (int64_t)d * n;
    float* ph = states + (slot * dim + d) * n;
    float acc = 0.0f;
    for (int i0 = q * 4; i0 < n; i0 += 16) {
        Pack<float, 4> h, a;
        Pack<T, 4> B, C;
        h.load(ph + i0, n - i0);
        a.load(pA + i0, n - i0);
        B.load(pB + i0, n - i0);
        C.load(pC + i0, n - i0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h.v[i] = __builtin_fmaf(exp2_fast(delta * (a.v[i] * kLog2e)), h.v[i],
                                    u * to_f32(B.v[i]));
            if (i0 + i < n) acc = __builtin_fmaf(h.v[i], to_f32(C.v[i]), acc);
        }
        h.store(ph + i0, n - i0);
    }
    acc += dpp_f<0xB1>(acc);
    acc += dpp_f<0x4E>(acc);
    if (q == 0) {
        if (p.D) acc += p.D[d] * x;
        if (p.z) {
            const float z = to_f32(((const T*)p.z)[b * p.z_batch + d]);
            acc *= z * sigmoid(z);
        }
        *py = from_f32<T>(acc);
    }
}

template <class T, int LN, int SPL>
hipError_t scan_as(const libscan_ssm& p, void* y, float* state_out, float* ckpt,
                   hipStream_t stream) {
    const int nb = ssm_blocks(p, SsmLanes<LN, SPL>::CH);
    const int64_t grid = p.batch * p.groups * nb;
    const bool whole = !p.lengths && p.steps % kTile == 0 && p.n == LN * SPL &&
                       p.dim / p.groups % SsmLanes<LN, SPL>::CH == 0;
    auto* scan = whole       ? k_ssm_scan<T, LN, SPL, true, false>
                 : p.n % SPL ? k_ssm_scan<T, LN, SPL, false, (SPL > 1)>
                             : k_ssm_scan<T, LN, SPL, false, false>;
    scan<<<dim3((unsigned)grid), kThreads, 0, stream>>>(p, (T*)y, state_out, ckpt, nb);
    return hipGetLastError();
}

// From so many channels on, eight lanes to a channel in the tiles (n <= 16) are
// enough waves for the chip, and share sums over fewer lanes; below, sixteen.
// Eight and sixteen, rows of 2048 steps: 8192 channels 135 and 118 us, 12288 168
// and 148, 16384 169 and 184; 32768 of 512 steps 75 and 89.
constexpr int64_t kTileChannels = 16384;

// How a call is cut up: `np` states to a lane and chunks of `chunk` steps.  np = 0:
// the tiles, whose workgroups share a channel's states out over lanes.
struct LanePlan {
    int np, nb, chunk, chunks;
    size_t bc, ends, sums;  // bytes of scratch
};
// The time of either way in us, as measured over 1 to 16 rows of 64 to 8192 steps and
// 70 to 4096 channels with 8 to 64 states.  The tiles walk a row at a step's
// latency, and share SIMDs beyond 4096 channels.  The chunks have four kernels and
// two chunks' steps to wait for, and then the vector units to keep busy (a call that
// fills the chip with one chunk has two of them, and is rated the same).  Other sizes
// go by the same two lines.
// E.g. n = 16, tiles against chunks: 1 x 512 x 1024 26.6 and 29.5, 1 x 1024 x 4096 51.5
// and 51.8, 1 x 2048 x 1024 96 and 44, 1 x 8192 x 512 373 and 66, 2 x 2048 x 4096 118
// and 124 us.
bool chunks_pay(const libscan_ssm& p, int np) {
    // (lanes without a channel take their time all the same)
    const int64_t channels = p.batch * p.groups * ssm_blocks(p, kWave) * kWave;
    const double over = p.batch * p.dim > 4096 ? (double)(p.batch * p.dim - 4096) : 0.0;
    const double step = 0.031 + 0.00103 * (np < 16 ? 16 : np);
    const double tiles = (double)p.steps * step * (1.0 + 6.6e-5 * over);
    const double chunks = 14.0 + 0.9 * np + 0.36e-6 * np * (double)p.steps * (double)channels;
    return chunks < tiles;
}

LanePlan lane_plan(const libscan_ssm& p) {
    LanePlan r{0, 0, 0, 0, 0, 0, 0};
    if (p.batch == 0 || p.dim == 0) return r;
    r.np = p.n <= 8 ? 8 : p.n <= 16 ? 16 : p.n <= 32 ? 32 : 64;
    if (p.steps < 64 || !chunks_pay(p, r.np)) {
        r.np = 0;
        return r;
    }
    r.nb = ssm_blocks(p, kWave);
    const int64_t waves = p.batch * p.groups * r.nb;
    int64_t chunks = (4096 + waves - 1) / waves;  // 4 waves to each of the 1024 SIMDs
    // a chunk's steps pass one after the other, but more chunks are more to chain
    const int64_t least = p.steps > 4096 ? 32 : 16;
    if (chunks > p.steps / least) chunks = p.steps / least;
    r.chunk = (int)(((p.steps + chunks - 1) / chunks + kSsmBlock - 1) / kSsmBlock * kSsmBlock);
    r.chunks = (int)((p.steps + r.chunk - 1) / r.chunk);
    r.bc = ssm_bc_bytes(p, r.np);
    if (r.chunks > 1) {
        r.ends = (size_t)r.chunks * p.batch * p.dim * r.np * 4;
        r.sums = (size_t)r.chunks * p.batch * p.dim * 4;
    }
    return r;
}

template <class T, int NP>
hipError_t lanes_as(const libscan_ssm& p, const LanePlan& l, void* y, float* state_out,
                    float* ckpt, void* scratch, hipStream_t stream) {
    float* bc = (float*)scratch;
    float* ends = bc + l.bc / 4;
    float* sums = ends + l.ends / 4;
    launch_ssm_bc(p, NP, bc, stream);
    const unsigned waves = (unsigned)(p.batch * p.groups * l.nb);
    const unsigned grid = (waves + kLaneWaves - 1) / kLaneWaves;
    if (l.chunks > 1) {
        k_ssm_ends<T, NP><<<dim3(grid, l.chunks - 1), kWave * kLaneWaves, 0, stream>>>(
            p, bc, ends, sums, l.nb, l.chunk, waves);
        launch_ssm_starts(p, NP, p.state, ends, sums, l.chunks, false, stream);
    }
    auto* scan = p.n == NP ? p.z ? k_ssm_lanes<T, NP, true, false> : k_ssm_lanes<T, NP, false, false>
                           : p.z ? k_ssm_lanes<T, NP, true, true> : k_ssm_lanes<T, NP, false, true>;
    scan<<<dim3(grid, l.chunks), kWave * kLaneWaves, 0, stream>>>(
        p, bc, l.chunks > 1 ? ends : nullptr, (T*)y, state_out, ckpt, l.nb, l.chunk,
        waves);
    return hipGetLastError();
}

template <class T>
hipError_t scan_type(const libscan_ssm& p, void* y, float* state_out, float* ckpt, void* scratch,
                     hipStream_t stream) {
    const LanePlan l = lane_plan(p);
    switch (l.np) {
        case 8: return lanes_as<T, 8>(p, l, y, state_out, ckpt, scratch, stream);
        case 16: return lanes_as<T, 16>(p, l, y, state_out, ckpt, scratch, stream);
        case 32: return lanes_as<T, 32>(p, l, y, state_out, ckpt, scratch, stream);
        case 64: return lanes_as<T, 64>(p, l, y, state_out, ckpt, scratch, stream);
        default: break;
    }
    if (p.n > 32) return scan_as<T, 16, 4>(p, y, state_out, ckpt, stream);
    if (p.n > 16) return scan_as<T, 16, 2>(p, y, state_out, ckpt, stream);
    if (p.batch * p.dim >= kTileChannels) return scan_as<T, 8, 2>(p, y, state_out, ckpt, stream);
    return scan_as<T, 16, 1>(p, y, state_out, ckpt, stream);
}

}  // namespace

size_t ssm_bc_bytes(const libscan_ssm& p, int np) {
    // one more token, which the last scalar load of a row runs into
    return (size_t)(p.batch * p.steps + 1) * p.groups * 2 * np * 4;
}

void launch_ssm_bc(const libscan_ssm& p, int np, float* bc, hipStream_t stream) {
    const dim3 grid((unsigned)((p.batch * p.steps * p.groups * np + kThreads - 1) / kThreads));
    auto with = [&](auto t) {
        using T = decltype(t);
        auto* k = np == 8    ? k_ssm_bc<T, 8>
                  : np == 16 ? k_ssm_bc<T, 16>
                  : np == 32 ? k_ssm_bc<T, 32>
                             : k_ssm_bc<T, 64>;
        k<<<grid, kThreads, 0, stream>>>(p, bc);
    };
    switch (p.type) {
        case LIBSCAN_F16: with(_Float16()); break;
        case LIBSCAN_BF16: with(__bf16()); break;
        default: with(float());
    }
}

void launch_ssm_starts(const libscan_ssm& p, int np, const float* init, float* ends,
                       const float* sums, int chunks, bool backward, hipStream_t stream) {
    const dim3 grid((unsigned)((p.batch * p.dim * np + kThreads - 1) / kThreads));
    auto* k = np == 8    ? k_ssm_starts<8>
              : np == 16 ? k_ssm_starts<16>
              : np == 32 ? k_ssm_starts<32>
                         : k_ssm_starts<64>;
    k<<<grid, kThreads, 0, stream>>>(p, init, ends, sums, chunks, backward);
}

size_t ssm_scratch_bytes(const libscan_ssm& p) {
    const LanePlan l = lane_plan(p);
    return l.bc + l.ends + l.sums;
}

hipError_t launch_ssm_scan(const libscan_ssm& p, void* y, float* state_out, float* ckpt,
                           void* scratch, hipStream_t stream) {
    if (p.batch == 0 || p.dim == 0) return hipSuccess;
    switch (p.type) {
        case LIBSCAN_F16: return scan_type<_Float16>(p, y, state_out, ckpt, scratch, stream);
        case LIBSCAN_BF16: return scan_type<__bf16>(p, y, state_out, ckpt, scratch, stream);
        default: return scan_type<float>(p, y, state_out, ckpt, scratch, stream);
    }
}

hipError_t launch_ssm_step(const libscan_ssm& p, float* states, int64_t n_states,
                           const int32_t* slots, void* y, hipStream_t stream) {
    if (p.batch == 0 || p.dim == 0) return hipSuccess;
    const int64_t grid = p.batch * ((p.dim + kThreads / 4 - 1) / (kThreads / 4));
    const dim3 g((unsigned)grid);
    switch (p.type) {
        case LIBSCAN_F16:
            k_ssm_step<<<g, kThreads, 0, stream>>>(p, states, n_states, slots, (_Float16*)y);
            break;
        case LIBSCAN_BF16:
            k_ssm_step<<<g, kThreads, 0, stream>>>(p, states, n_states, slots, (__bf16*)y);
            break;
        default:
            k_ssm_step<<<g, kThreads, 0, stream>>>(p, states, n_states, slots, (float*)y);
    }
    return hipGetLastError();
}

}  // namespace ls
