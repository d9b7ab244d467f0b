// ssm_back.hip -- gradients of the selective scan.
//
// With G[t] the gradient of h[t] and w = dy silu(z):
//   G[t] = w[t] C[t] + a[t+1] G[t+1]
//   dC[t] = sum_d w h[t]            dB[t] = sum_d G[t] delta x
//   du = sum_i G[t] B[t]            r = G[t] a[t] h[t-1]
//   ddelta = sum_i r A + du x       dA = sum_t r delta
//   dx = du delta + D w             ddt = ddelta softplus'(dt + dt_bias)
// A workgroup owns CH channels of one row and walks the row backwards in
// blocks of 16 steps (staged two at a time), from the checkpoints that the
// forward pass left: h and a of a block are formed again in registers, then the
// recurrence of G runs through them.  Sums over a channel's states go to the
// block's outputs through LDS; sums over channels (dB, dC) are reduced in the
// workgroup and added over workgroups by a second kernel, in a fixed order, so
// that the same call gives the same bits.  Everything between the inputs and the
// gradients is fp32; a gradient is rounded to its input's type once.
//
// The vector units bound it: one exponential and about 13 multiply-adds for each
// step, channel and state, and the sums over lanes.
#include "launch.hpp"
#include "lm.hpp"
#include "ssm.hpp"

namespace ls {

namespace {

constexpr int kThreads = 256;
constexpr int kT = kSsmBlock;

struct BackArgs {
    const void* dy;
    int64_t dy_batch, dy_step;
    const float* ckpt;
    const float* dstate_out;
    void *dx, *ddt, *dz;
    float* dstate;
    float2* part_bc;  // [block of the group][batch][step][group][n] of (dB, dC)
    float* part_a;    // [chunk][batch][dim][n]
    float* part_d;    // [chunk][batch][dim]
    float* part_bias; // [chunk][batch][dim]
    // steps of a chunk (blockIdx.y) of the rows; with more than one, a[t] G[t] of the
    // steps that follow its pieces, [piece][batch][dim][np], `split` pieces to a chunk
    int chunk, np, split, pieces;
    const float* starts;
};

// What a chunk gives the chunk before it from nothing behind it, and its sum of
// delta (as k_ssm_ends in ssm.hip, backwards in time, with the gate in place of
// the softplus's input).
template <class T, int NP>
__global__ __launch_bounds__(kWave * kLaneWaves) void k_ssm_back_ends(libscan_ssm p, const void* dy,
                                                                      int64_t dy_batch,
                                                                      int64_t dy_step,
                                                                      const float* bc_, float* ends,
                                                                      float* sums, int nb,
                                                                      int chunk, uint32_t waves) {
    using Groups = LaneGroups<NP>;
    constexpr int GP = Groups::GP, NG = Groups::NG;
    if (blockIdx.x * kLaneWaves + threadIdx.x / kWave >= waves) return;
    const LaneBlock w = lane_block(p, nb, chunk, blockIdx.y + 1);  // the first chunk has none before
    const int b = w.k.b, c0 = w.k.c0, ch = c0 + (int)w.lo;
    const uint32_t lo = w.lo;
    const int dim = (int)p.dim, n = (int)p.n;
    const bool gate = p.z != nullptr;
    float a2[NP], cg[NP], sum = 0.0f;
    load_states<NP>(p.A + (int64_t)ch * n, n, a2);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        a2[i] *= kLog2e;
        cg[i] = 0.0f;
    }
    if (w.t0 < w.end) {
        const int t1 = w.end - 1;
        const int64_t bc_step = p.groups * 2 * NP;
        // C follows B in every group
        ScalarPtr bc = (ScalarPtr)bc_ + (((int64_t)b * p.steps + t1) * p.groups + w.k.g) * 2 * NP + GP;
        StepPtr<const T> pdt((const T*)p.dt + b * p.dt_batch + t1 * p.dt_step + c0, -p.dt_step);
        StepPtr<const T> pdy((const T*)dy + b * dy_batch + t1 * dy_step + c0, -dy_step);
        StepPtr<const T> pz(gate ? (const T*)p.z + b * p.z_batch + t1 * p.z_step + c0 : nullptr,
                            -p.z_step);
        const float bias = p.dt_bias ? p.dt_bias[ch] : 0.0f;
        Groups cur;
        cur.template load<GP>(bc);
        T nx[kAhead], ndt[kAhead], nz[kAhead];
        auto fetch = [&](int count) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                ndt[i] = nx[i] = nz[i] = T(0);
                if (i < count) {
                    ndt[i] = pdt.p[lo];
                    nx[i] = pdy.p[lo];
                    if (gate) nz[i] = pz.p[lo];
                    pdt.next();
                    pdy.next();
                    if (gate) pz.next();
                }
            }
        };
        int left = w.end - w.t0;
        fetch(left);
        for (; left > 0; left -= kAhead) {
            float delta[kAhead], wt[kAhead];
            step_sizes(p, ndt, bias, delta);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) wt[i] = to_f32(nx[i]);
            if (gate) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const float z = to_f32(nz[i]);
                    wt[i] *= z * sigmoid(z);
                }
            }
            if (left > kAhead) fetch(left - kAhead);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (i >= left) break;
                sum += delta[i];
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    scalar_loads_done();
                    Groups next;  // of this step, or of the one before (t0 > 0: it is there)
                    if (g + 1 == NG) bc -= bc_step;
                    next.template load<GP>(g + 1 < NG ? bc + (g + 1) * 2 * GP : bc);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int j = 0; j < GP; ++j) {
                        float& c = cg[g * GP + j];
                        c = exp2_fast(delta[i] * a2[g * GP + j]) * __builtin_fmaf(wt[i], cur.v[j], c);
                    }
                    cur = next;
                }
            }
        }
    }
    const int64_t row = ((int64_t)w.c * p.batch + b) * dim + ch;
    store_states<NP>(ends + row * NP, NP, cg);
    sums[row] = sum;
}

// Keeps the loads from two LDS addresses behind the computation of v: left
// alone, the compiler loads a whole block's inputs first, into registers that
// the block's states need.
constexpr int kGroup = 4;  // steps whose inputs are loaded together
typedef const __attribute__((address_space(3))) float4* LdsIn;
typedef const __attribute__((address_space(3))) float2* LdsBc;
__device__ __forceinline__ float4 load_lds(LdsIn p) { return float4{p->x, p->y, p->z, p->w}; }
__device__ __forceinline__ float2 load_lds(LdsBc p) { return float2{p->x, p->y}; }
__device__ __forceinline__ void after(float v, LdsIn& p, LdsBc& q) {
    asm volatile("" : "+v"(p), "+v"(q) : "v"(v));
}

// WHOLE: every row has all its steps, in whole tiles, and every workgroup all its
// channels and states, so that nothing needs a check.  4 x 2048 x 4096, n = 16,
// the whole call: 541 us, with the checks 601; 16 steps staged at a time instead of
// 32 took 35 us more, four lanes to a channel (one wave to a SIMD for want of
// registers) 200 more.
// Lanes whose channel or states are padding read zeros alone (column CH of s_in, NP on
// of s_bc), so that no infinity there meets a 0 and no NaN the sums.  PART: some lane's
// states are padding in part (n is no multiple of SPL), and are held at 0.
template <class T, int LN, int SPL, bool WHOLE, bool PART>
__global__ __launch_bounds__(kThreads) void k_ssm_back(libscan_ssm p, BackArgs o, int nb) {
    using L = SsmLanes<LN, SPL>;
    constexpr int CH = L::CH, NP = L::NP, YS = CH + 4;
    // steps that are staged together, in blocks of kT; threads to a step, channels to a thread
    constexpr int TS = NP > 32 ? 16 : 32, SUB = TS / kT, TPR = kThreads / TS, VW = CH / TPR;
    constexpr int NBC = TS * NP / kThreads;
    static_assert(VW * TPR == CH && NBC * kThreads == TS * NP, "a tile is shared out evenly");
    constexpr int INS = WHOLE ? CH : CH + 1, BCS = WHOLE ? NP : NP + (SPL > 2 ? SPL : 2);
    __shared__ float4 s_in[TS][INS];  // delta, delta x, w
    __shared__ float2 s_bc[TS][BCS];
    __shared__ float s_y[TS][YS], s_du[TS][YS], s_dd[TS][YS];
    __shared__ float2 s_g[4][TS][NP + 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int steps = (int)p.steps, dim = (int)p.dim, n = (int)p.n, groups = (int)p.groups;
    const SsmBlock k = ssm_block(p, nb, CH, blockIdx.x);
    const int len = WHOLE ? steps : ssm_len(p, k.b);
    const int lim = WHOLE ? CH : k.lim;
    const int blocks = (steps + kT - 1) / kT;
    // this workgroup's steps; those of its row's tokens
    const int begin = blockIdx.y * o.chunk;
    const int stop = begin + o.chunk < steps ? begin + o.chunk : steps;
    const int end = stop < len ? stop : len;
    const int64_t crow = (int64_t)blockIdx.y * p.batch + k.b;
    const int piece = ((int)blockIdx.y + 1) * o.split;  // the first behind this chunk
    const int64_t behind = (int64_t)((piece < o.pieces ? piece : o.pieces) - 1) * p.batch + k.b;
    const bool gate = p.z != nullptr;

    const int row = tid / TPR, lc = (tid % TPR) * VW;
    const int lcount = WHOLE ? VW : lim - lc;
    const int64_t ch0 = k.c0 + lc;
    const T* px = (const T*)p.x + k.b * p.x_batch + row * p.x_step + ch0;
    const T* pdt = (const T*)p.dt + k.b * p.dt_batch + row * p.dt_step + ch0;
    const T* pz = (const T*)p.z + k.b * p.z_batch + row * p.z_step + ch0;
    const T* pdy = (const T*)o.dy + k.b * o.dy_batch + row * o.dy_step + ch0;
    const int bt = tid * NBC / NP, bn = tid * NBC % NP;
    const T* pB = (const T*)p.B + k.b * p.B_batch + k.g * p.B_group + bt * p.B_step + bn;
    const T* pC = (const T*)p.C + k.b * p.C_batch + k.g * p.C_group + bt * p.C_step + bn;
    const int64_t obase = ((int64_t)k.b * steps + row) * dim + ch0;
    float bias[VW], skip[VW], sum_d[VW], sum_bias[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) {
        bias[i] = p.dt_bias && (WHOLE || i < lcount) ? p.dt_bias[ch0 + i] : 0.0f;
        skip[i] = p.D && (WHOLE || i < lcount) ? p.D[ch0 + i] : 0.0f;
        sum_d[i] = sum_bias[i] = 0.0f;
    }

    const int wc = wave * L::CPW + L::channel(lane), n0 = L::part(lane) * SPL;
    const bool used = WHOLE || (wc < lim && n0 < n);
    if (!WHOLE && tid < TS) {
        s_in[tid][CH] = float4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < SPL; ++s) s_bc[tid][NP + s] = float2{0.0f, 0.0f};
    }
    float a2[SPL], da[SPL], cg[SPL];  // cg: a[t+1] G[t+1] of the step that follows
    const int64_t sbase = ((int64_t)k.b * dim + k.c0 + wc) * n + n0;
    const float* pck = o.ckpt + ((int64_t)k.b * blocks * dim + k.c0 + wc) * n + n0;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        const bool in = WHOLE || (wc < lim && n0 + s < n);
        a2[s] = in ? p.A[(int64_t)(k.c0 + wc) * n + n0 + s] * kLog2e : 0.0f;
        if (o.starts)
            cg[s] = in ? o.starts[(behind * dim + k.c0 + wc) * o.np + n0 + s] : 0.0f;
        else
            cg[s] = in && o.dstate_out ? o.dstate_out[sbase + s] : 0.0f;
        da[s] = 0.0f;
    }

    // the steps past the row's tokens
    const int tail = (len + TS - 1) / TS * TS;
    for (int t = tail > begin ? tail : begin; !WHOLE && t + row < stop; t += TS) {
        Pack<T, VW> zero;
#pragma unroll
        for (int i = 0; i < VW; ++i) zero.v[i] = T(0);
        const int64_t at = obase + (int64_t)t * dim;
        zero.store((T*)o.dx + at, lcount);
        zero.store((T*)o.ddt + at, lcount);
        if (gate) zero.store((T*)o.dz + at, lcount);
    }

    // What a tile reads, loaded while the tile after it is worked on.  Tiles that
    // lie inside the row, with all of their channels and states, need no checks.
    Pack<T, VW> nx, ndt, nz, ndy;
    Pack<T, NBC> nB, nC;
    float nh[SUB][SPL];
    auto fetch = [&](int t0) {
        const bool all = WHOLE || (lim == CH && n == NP && t0 + TS <= len);
        const int count = all ? VW : t0 + row < len ? lcount : 0;
        const int bcount = all ? NBC : t0 + bt < len ? n - bn : 0;
        nx.load(px + t0 * p.x_step, count);
        ndt.load(pdt + t0 * p.dt_step, count);
        nz.load(pz + t0 * p.z_step, gate ? count : 0);
        ndy.load(pdy + t0 * o.dy_step, count);
        nB.load(pB + t0 * p.B_step, bcount);
        nC.load(pC + t0 * p.C_step, bcount);
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
            const float* pc = pck + ((int64_t)t0 / kT + sub) * dim * n;
            const bool there = t0 + sub * kT < len && wc < lim;
#pragma unroll
            for (int s = 0; s < SPL; ++s)
                nh[sub][s] = all || (there && n0 + s < n) ? pc[s] : 0.0f;
        }
    };

    const int last = begin + (end - begin + TS - 1) / TS * TS - TS;  // < begin: no tokens here
    if (last >= begin) fetch(last);
    for (int t0 = last; t0 >= begin; t0 -= TS) {
        const bool live = WHOLE || t0 + row < len;
        const Pack<T, VW> rx = nx, rdt = ndt, rz = nz, rdy = ndy;
        float starts[SUB][SPL];
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int s = 0; s < SPL; ++s) starts[sub][s] = nh[sub][s];
#pragma unroll
        for (int i = 0; i < NBC; ++i)
            s_bc[bt][bn + i] = float2{to_f32(nB.v[i]), to_f32(nC.v[i])};
        float delta[VW], w[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) delta[i] = to_f32(rdt.v[i]) + bias[i];
        if (p.softplus) {
#pragma unroll
            for (int i = 0; i < VW; ++i) delta[i] = softplus(delta[i]);
        }
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            delta[i] = WHOLE || (live && i < lcount) ? delta[i] : 0.0f;  // past the end: a = 1, b = 0
            w[i] = to_f32(rdy.v[i]);
        }
        if (gate) {
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                const float z = to_f32(rz.v[i]);
                w[i] *= z * sigmoid(z);
            }
        }
#pragma unroll
        for (int i = 0; i < VW; ++i)
            s_in[row][lc + i] = float4{delta[i], delta[i] * to_f32(rx.v[i]), w[i], 0.0f};
        if (t0 > begin) fetch(t0 - TS);
        __syncthreads();

        // blocks past the row's tokens (there is one before: t0 < len) leave cg as it is
        const int top = WHOLE || t0 + TS - kT < len ? SUB - 1 : (len - 1 - t0) / kT;
#pragma unroll 1
        for (int sub = top; sub >= 0; --sub) {
            const int tb = sub * kT;
            float h[kT][SPL], a[kT][SPL], h0[SPL];
#pragma unroll
            for (int s = 0; s < SPL; ++s) h0[s] = sub ? starts[SUB - 1][s] : starts[0][s];
            LdsIn in_at = (LdsIn)&s_in[tb][WHOLE || used ? wc : CH];
            LdsBc bc_at = (LdsBc)&s_bc[tb][WHOLE || used ? n0 : NP];
            {
                float hr[SPL], v[kT];
#pragma unroll
                for (int s = 0; s < SPL; ++s) hr[s] = h0[s];
#pragma unroll
                for (int t = 0; t < kT; ++t) {
                    if (t % kGroup == 0) after(hr[0], in_at, bc_at);
                    const float4 in = load_lds(in_at + t * INS);
                    float acc = 0.0f;
#pragma unroll
                    for (int s = 0; s < SPL; ++s) {
                        const float2 bc = load_lds(bc_at + t * BCS + s);
                        a[t][s] = exp2_fast(in.x * a2[s]);
                        hr[s] = __builtin_fmaf(a[t][s], hr[s], in.y * bc.x);
                        if (PART && s && n0 + s >= n) a[t][s] = hr[s] = 0.0f;
                        h[t][s] = hr[s];
                        acc = __builtin_fmaf(hr[s], bc.y, acc);
                    }
                    v[t] = acc;
                }
                if (gate) L::sum_states(v, lane, [&](int t, float sum) { s_y[tb + t][wc] = sum; });
            }
            // A block that the row ends in has steps past it, which leave cg as it is and
            // must not multiply their delta of 0 with a state or a gradient that is infinite.
            const int left = len - t0 - tb;
            {
                float vu[kT], vd[kT];
#pragma unroll
                for (int t = kT - 1; t >= 0; --t) {
                    if (t % kGroup == kGroup - 1) after(cg[0], in_at, bc_at);
                    const float4 in = load_lds(in_at + t * INS);
                    float du = 0.0f, dd = 0.0f;
#pragma unroll
                    for (int s = 0; s < SPL; ++s) {
                        const float2 bc = load_lds(bc_at + t * BCS + s);
                        float g = __builtin_fmaf(in.z, bc.y, cg[s]);
                        if (PART && s && n0 + s >= n) g = 0.0f;
                        du = __builtin_fmaf(g, bc.x, du);
                        cg[s] = a[t][s] * g;
                        float r = cg[s] * (t ? h[t ? t - 1 : 0][s] : h0[s]);
                        if (!WHOLE && t >= left) r = 0.0f;
                        dd = __builtin_fmaf(r, a2[s], dd);
                        da[s] = __builtin_fmaf(r, in.x, da[s]);
                        a[t][s] = g * in.y;  // a and h of this step are done with: dB and dC
                        h[t][s] *= in.z;
                        // formed here and now: put off, the products hold both factors
                        asm volatile("" : "+v"(a[t][s]), "+v"(h[t][s]));
                    }
                    vu[t] = du;
                    vd[t] = dd;
                    asm volatile("" : "+v"(vu[t]), "+v"(vd[t]));
                }
                L::sum_states(vu, lane, [&](int t, float sum) { s_du[tb + t][wc] = sum; });
                L::sum_states(vd, lane, [&](int t, float sum) { s_dd[tb + t][wc] = sum; });
            }
#pragma unroll
            for (int s = 0; s < SPL; ++s) {
                float v[kT], u[kT];
#pragma unroll
                for (int t = 0; t < kT; ++t) {
                    v[t] = a[t][s];
                    u[t] = h[t][s];
                }
                L::sum_channels(v, lane,
                                [&](int t, float sum) { s_g[wave][tb + t][n0 + s].x = sum; });
                L::sum_channels(u, lane,
                                [&](int t, float sum) { s_g[wave][tb + t][n0 + s].y = sum; });
            }
        }
        __syncthreads();

        if (WHOLE || t0 + row < steps) {
            Pack<T, VW> ox, odt, oz;
            float ddt[VW];
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                const float x = to_f32(rx.v[i]), du = s_du[row][lc + i];
                const float dx = __builtin_fmaf(du, delta[i], skip[i] * w[i]);
                ox.v[i] = from_f32<T>(live ? dx : 0.0f);
                ddt[i] = __builtin_fmaf(du, x, s_dd[row][lc + i] * kLn2);
                sum_d[i] = __builtin_fmaf(w[i], x, sum_d[i]);  // both 0 past the end
            }
            if (p.softplus) {
#pragma unroll
                for (int i = 0; i < VW; ++i) ddt[i] *= sigmoid(to_f32(rdt.v[i]) + bias[i]);
            }
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                ddt[i] = WHOLE || (live && i < lcount) ? ddt[i] : 0.0f;
                odt.v[i] = from_f32<T>(ddt[i]);
                sum_bias[i] += ddt[i];
            }
            const int64_t at = obase + (int64_t)t0 * dim;
            ox.store((T*)o.dx + at, lcount);
            odt.store((T*)o.ddt + at, lcount);
            if (gate) {
#pragma unroll
                for (int i = 0; i < VW; ++i) {
                    const float z = to_f32(rz.v[i]), sig = sigmoid(z);
                    const float yv = __builtin_fmaf(skip[i], to_f32(rx.v[i]), s_y[row][lc + i]);
                    const float dz = to_f32(rdy.v[i]) * yv * sig *
                                     __builtin_fmaf(z, 1.0f - sig, 1.0f);
                    oz.v[i] = from_f32<T>(live ? dz : 0.0f);
                }
                oz.store((T*)o.dz + at, lcount);
            }
        }
#pragma unroll
        for (int i = 0; i < NBC; ++i) {
            if (WHOLE || (t0 + bt < len && bn + i < n)) {
                float2 sum = s_g[0][bt][bn + i];
#pragma unroll
                for (int wv = 1; wv < 4; ++wv) {
                    sum.x += s_g[wv][bt][bn + i].x;
                    sum.y += s_g[wv][bt][bn + i].y;
                }
                o.part_bc[((((int64_t)k.k * p.batch + k.b) * steps + t0 + bt) * groups + k.g) * n +
                          bn + i] = sum;
            }
        }
    }

#pragma unroll
    for (int s = 0; s < SPL; ++s)
        if (WHOLE || (wc < lim && n0 + s < n)) {
            if (o.dstate && begin == 0) o.dstate[sbase + s] = cg[s];
            o.part_a[(crow * dim + k.c0 + wc) * n + n0 + s] = da[s];
        }
    // dD and ddt_bias: the TS threads of each channel, in order
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VW; ++i) {
        s_y[row][lc + i] = sum_d[i];
        s_du[row][lc + i] = sum_bias[i];
    }
    __syncthreads();
    if (tid < lim) {
        float d = 0.0f, e = 0.0f;
        for (int r = 0; r < TS; ++r) {
            d += s_y[r][tid];
            e += s_du[r][tid];
        }
        o.part_d[crow * dim + k.c0 + tid] = d;
        o.part_bias[crow * dim + k.c0 + tid] = e;
    }
}

// dB and dC: the workgroups' sums of a group, added in order (eight threads to an
// output from 17 parts on).  4 x 2048 x 4096, n = 16, 128 parts: 24 us for 134 MB.
template <class T, int SLICES>
__global__ __launch_bounds__(kSumThreads) void k_ssm_sum_bc(libscan_ssm p, const float2* part,
                                                            int nb, T* dB, T* dC) {
    const int64_t per_step = p.groups * p.n, total = p.batch * p.steps * per_step;
    const int64_t i = (int64_t)blockIdx.x * kSumOuts<SLICES> + threadIdx.x % kSumOuts<SLICES>;
    const int64_t bt = i < total ? i / per_step : 0;
    const int b = (int)(bt / p.steps), t = (int)(bt % p.steps);
    const bool live = i < total && t < ssm_len(p, b);
    const float2 sum = sum_parts<SLICES>(part, live ? nb : 0, total, i);
    if (threadIdx.x < kSumOuts<SLICES> && i < total) {
        dB[i] = from_f32<T>(sum.x);
        dC[i] = from_f32<T>(sum.y);
    }
}

// The sums of dA, dD and ddt_bias over `rows` rows (or their chunks), added in order.
template <int SLICES>
__global__ __launch_bounds__(kSumThreads) void k_ssm_sum_rows(int64_t rows, int64_t dim, int64_t n,
                                                              const float* part_a,
                                                              const float* part_d,
                                                              const float* part_bias, float* dA,
                                                              float* dD, float* ddt_bias) {
    const int64_t i = (int64_t)blockIdx.x * kSumOuts<SLICES> + threadIdx.x % kSumOuts<SLICES>;
    const bool first = threadIdx.x < kSumOuts<SLICES>;
    const float a = sum_parts<SLICES>(part_a, i < dim * n ? rows : 0, dim * n, i);
    if (first && i < dim * n) dA[i] = a;
    if ((int64_t)blockIdx.x * kSumOuts<SLICES> >= dim) return;  // the whole workgroup
    const float d = sum_parts<SLICES>(part_d, i < dim ? rows : 0, dim, i);
    const float e = sum_parts<SLICES>(part_bias, i < dim ? rows : 0, dim, i);
    if (first && i < dim) {
        if (dD) dD[i] = d;
        if (ddt_bias) ddt_bias[i] = e;
    }
}

// How a call is cut up, the same for the sizes and the launch.  Eight lanes to a
// channel do the least work, if there are 16384 channels for them or the rows are
// cut into chunks: until two workgroups are there for each CU (one with n > 32;
// so many fit by their registers).  Uncut rows of 2048 steps, n = 16, with eight
// lanes and with sixteen: 8192 channels 391 and 350 us, 12288 525 and 458, 16384
// 539 and 654.  What the chunks hand on is formed by a pass over smaller pieces,
// four waves of them to a SIMD.
struct BackPlan {
    int lanes, nb, chunk, chunks, np, piece, pieces;
    size_t part_bc, part_a, part_d, bc, ends, sums;  // bytes of scratch
};

constexpr int64_t kWideLanes = 16384;

size_t align16(size_t v) { return (v + 15) / 16 * 16; }

BackPlan back_plan(const libscan_ssm& p) {
    BackPlan r{};
    const int64_t channels = p.batch * p.dim;
    r.np = p.n <= 8 ? 8 : p.n <= 16 ? 16 : p.n <= 32 ? 32 : 64;
    r.lanes = p.n <= 16 ? 8 : 16;
    r.nb = ssm_blocks(p, 256 / r.lanes);
    r.chunks = 1;
    r.chunk = (int)((p.steps + 31) / 32 * 32);
    const int64_t groups = p.batch * p.groups * r.nb, fit = p.n > 32 ? 256 : 512;
    int64_t chunks = groups > 0 ? fit / groups : 1;
    if (chunks > p.steps / 64) chunks = p.steps / 64;
    // Times in us of a 32-step tile: uncut, and with the CUs full, as measured for 1 to 16
    // rows of 128 to 8192 steps (other sizes go by the same lines).  The whole call, n =
    // 16, uncut and in chunks: 1 x 2048 x 4096 271 and 186, 2 x 2048 x 4096 350 and 345,
    // 1 x 8192 x 512 1005 and 131; n = 64, 1 x 8192 x 512: 2848 and 480.
    const double share = channels > 4096 ? 3.5e-4 * (double)(channels - 4096) : 0.0;
    const double uncut = p.n > 32   ? 12.4
                         : p.n > 16 ? 6.3
                         : channels < kWideLanes ? 4.1 + share
                                                 : 8.3;
    const double full = p.n > 32 ? 12.4 : p.n > 16 ? 9.5 : 8.3;
    const double tiles = (double)p.steps / 32;
    const int64_t waves = p.batch * p.groups * ssm_blocks(p, kWave);
    if (chunks > 1 &&
        45.0 + 0.25e-6 * r.np * (double)p.steps * (double)(waves * kWave) + tiles / chunks * full <
            tiles * uncut) {
        int64_t pieces = (4096 + waves - 1) / waves;
        if (pieces > p.steps / 32) pieces = p.steps / 32;
        r.piece = (int)(((p.steps + pieces - 1) / pieces + 31) / 32 * 32);
        const int64_t want = (p.steps + chunks - 1) / chunks;
        r.chunk = (int)((want + r.piece - 1) / r.piece * r.piece);
        r.chunks = (int)((p.steps + r.chunk - 1) / r.chunk);
        r.pieces = (int)((p.steps + r.piece - 1) / r.piece);
    }
    if (r.chunks == 1 && r.lanes == 8 && channels < kWideLanes) {
        r.lanes = 16;
        r.nb = ssm_blocks(p, 256 / r.lanes);
    }
    const size_t rows = (size_t)channels;
    r.part_bc = align16((size_t)r.nb * p.batch * p.steps * p.groups * p.n * 8);
    r.part_a = align16(r.chunks * rows * p.n * 4);
    r.part_d = align16(r.chunks * rows * 4);
    if (r.chunks > 1) {
        r.bc = align16(ssm_bc_bytes(p, r.np));
        r.ends = align16(r.pieces * rows * r.np * 4);
        r.sums = align16(r.pieces * rows * 4);
    }
    return r;
}

template <class T, int LN, int SPL>
void back_as(const libscan_ssm& p, const BackArgs& o, const BackPlan& l, hipStream_t stream) {
    const int64_t grid = p.batch * p.groups * l.nb;
    if (grid == 0) return;
    const bool whole = !p.lengths && p.steps % 32 == 0 && p.n == LN * SPL &&
                       p.dim / p.groups % SsmLanes<LN, SPL>::CH == 0;
    auto* back = whole       ? k_ssm_back<T, LN, SPL, true, false>
                 : p.n % SPL ? k_ssm_back<T, LN, SPL, false, (SPL > 1)>
                             : k_ssm_back<T, LN, SPL, false, false>;
    back<<<dim3((unsigned)grid, l.chunks), kThreads, 0, stream>>>(p, o, l.nb);
}

template <class T>
void ends_of(const libscan_ssm& p, const BackArgs& o, const BackPlan& l, const float* bc,
             float* ends, float* sums, hipStream_t stream) {
    const int nb = ssm_blocks(p, kWave);
    const unsigned waves = (unsigned)(p.batch * p.groups * nb);
    auto* k = l.np == 8    ? k_ssm_back_ends<T, 8>
              : l.np == 16 ? k_ssm_back_ends<T, 16>
              : l.np == 32 ? k_ssm_back_ends<T, 32>
                           : k_ssm_back_ends<T, 64>;
    k<<<dim3((waves + kLaneWaves - 1) / kLaneWaves, l.pieces - 1), kWave * kLaneWaves, 0, stream>>>(
        p, o.dy, o.dy_batch, o.dy_step, bc, ends, sums, nb, l.piece, waves);
}

template <class T>
hipError_t back_type(const libscan_ssm& p, BackArgs o, const BackPlan& l, char* more, float* dA,
                     T* dB, T* dC, float* dD, float* ddt_bias, hipStream_t stream) {
    if (l.chunks > 1) {
        float* bc = (float*)more;
        float* ends = (float*)(more + l.bc);
        float* sums = (float*)(more + l.bc + l.ends);
        launch_ssm_bc(p, l.np, bc, stream);
        ends_of<T>(p, o, l, bc, ends, sums, stream);
        launch_ssm_starts(p, l.np, o.dstate_out, ends, sums, l.pieces, true, stream);
        o.starts = ends;
        o.split = l.chunk / l.piece;
        o.pieces = l.pieces;
    }
    if (p.n > 32)
        back_as<T, 16, 4>(p, o, l, stream);
    else if (p.n > 16)
        back_as<T, 16, 2>(p, o, l, stream);
    else
        l.lanes == 8 ? back_as<T, 8, 2>(p, o, l, stream) : back_as<T, 16, 1>(p, o, l, stream);
    const int64_t bc = p.batch * p.steps * p.groups * p.n;
    auto grid = [](int64_t outs, int per) { return dim3((unsigned)((outs + per - 1) / per)); };
    if (bc > 0 && long_sum(l.nb))
        k_ssm_sum_bc<T, 8><<<grid(bc, kSumOuts<8>), kSumThreads, 0, stream>>>(p, o.part_bc, l.nb,
                                                                              dB, dC);
    else if (bc > 0)
        k_ssm_sum_bc<T, 1><<<grid(bc, kSumOuts<1>), kSumThreads, 0, stream>>>(p, o.part_bc, l.nb,
                                                                              dB, dC);
    const int64_t outs = p.dim * p.n, rows = p.batch * l.chunks;
    if (outs > 0 && long_sum(rows))
        k_ssm_sum_rows<8><<<grid(outs, kSumOuts<8>), kSumThreads, 0, stream>>>(
            rows, p.dim, p.n, o.part_a, o.part_d, o.part_bias, dA, dD, ddt_bias);
    else if (outs > 0)
        k_ssm_sum_rows<1><<<grid(outs, kSumOuts<1>), kSumThreads, 0, stream>>>(
            rows, p.dim, p.n, o.part_a, o.part_d, o.part_bias, dA, dD, ddt_bias);
    return hipGetLastError();
}

}  // namespace

size_t ssm_ckpt_bytes(const libscan_ssm& p) {
    return (size_t)p.batch * ((p.steps + kT - 1) / kT) * p.dim * p.n * 4;
}

size_t ssm_back_scratch_bytes(const libscan_ssm& p) {
    const BackPlan l = back_plan(p);
    return l.part_bc + l.part_a + 2 * l.part_d + l.bc + l.ends + l.sums;
}

hipError_t launch_ssm_back(const libscan_ssm& p, const void* dy, int64_t dy_batch, int64_t dy_step,
                           const float* ckpt, const float* dstate_out, void* dx, void* ddt,
                           float* dA, void* dB, void* dC, float* dD, void* dz, float* ddt_bias,
                           float* dstate, void* scratch, hipStream_t stream) {
    const BackPlan l = back_plan(p);
    char* s = (char*)scratch;
    BackArgs o{};
    o.dy = dy;
    o.dy_batch = dy_batch;
    o.dy_step = dy_step;
    o.ckpt = ckpt;
    o.dstate_out = dstate_out;
    o.dx = dx;
    o.ddt = ddt;
    o.dz = dz;
    o.dstate = dstate;
    o.part_bc = (float2*)s;
    s += l.part_bc;
    o.part_a = (float*)s;
    s += l.part_a;
    o.part_d = (float*)s;
    s += l.part_d;
    o.part_bias = (float*)s;
    s += l.part_d;
    o.chunk = l.chunk;
    o.np = l.np;
    switch (p.type) {
        case LIBSCAN_F16:
            return back_type<_Float16>(p, o, l, s, dA, (_Float16*)dB, (_Float16*)dC, dD, ddt_bias,
                                       stream);
        case LIBSCAN_BF16:
            return back_type<__bf16>(p, o, l, s, dA, (__bf16*)dB, (__bf16*)dC, dD, ddt_bias,
                                     stream);
        default:
            return back_type<float>(p, o, l, s, dA, (float*)dB, (float*)dC, dD, ddt_bias, stream);
    }
}

}  // namespace ls
