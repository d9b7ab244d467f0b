// ssm.hip -- the selective scan (prompts) and its single-token step.
//
// h[t] = a[t] h[t-1] + b[t] per channel and state index, a = exp(delta A),
// b = delta x B; y = sum over the state index of C h, plus D x, times
// silu(z).  A workgroup owns CH channels of one row and walks the row in tiles
// of 32 steps.  What depends on step and channel alone (softplus, delta x) is
// computed once per tile by threads that own 16 bytes of channels, and goes
// through LDS to the lanes that own (channel, state) pairs; their sums over
// the state index go back the same way to be gated and stored.  The states
// stay in registers for the whole row.
#include "launch.hpp"
#include "lm.hpp"
#include "ssm.hpp"

namespace ls {

namespace {

constexpr int kTile = 32;     // steps per tile
constexpr int kThreads = 256;

template <class T, int LN, int SPL>
__global__ __launch_bounds__(kThreads) void k_ssm_scan(libscan_ssm p, T* y, float* state_out,
                                                       float* ckpt, int nb) {
    using L = SsmLanes<LN, SPL>;
    constexpr int CH = L::CH, NP = L::NP, VW = CH / 8, YS = CH + 4;
    constexpr int NBC = kTile * NP / kThreads;
    __shared__ float2 s_du[kTile][CH];
    __shared__ float2 s_bc[kTile][NP];
    __shared__ float s_y[kTile][YS];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int steps = (int)p.steps, dim = (int)p.dim, n = (int)p.n;
    const SsmBlock k = ssm_block(p, nb, CH);
    const int len = ssm_len(p, k.b);

    // loader: one step, VW channels
    const int row = tid >> 3, lc = (tid & 7) * VW;
    const int lcount = k.lim - lc;  // channels of this thread that exist (may be <= 0)
    const int64_t ch0 = k.c0 + lc;
    const T* px = (const T*)p.x + k.b * p.x_batch + ch0;
    const T* pdt = (const T*)p.dt + k.b * p.dt_batch + ch0;
    const T* pz = p.z ? (const T*)p.z + k.b * p.z_batch + ch0 : nullptr;
    const T* pB = (const T*)p.B + k.b * p.B_batch + k.g * p.B_group;
    const T* pC = (const T*)p.C + k.b * p.C_batch + k.g * p.C_group;
    T* py = y + ((int64_t)k.b * steps) * dim + ch0;
    float bias[VW], skip[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) {
        bias[i] = p.dt_bias && i < lcount ? p.dt_bias[ch0 + i] : 0.0f;
        skip[i] = p.D && i < lcount ? p.D[ch0 + i] : 0.0f;
    }

    // scanner: channel wc, states n0 .. n0 + SPL
    const int wc = wave * L::CPW + L::channel(lane), n0 = L::part(lane) * SPL;
    float a2[SPL], h[SPL];
    const int64_t sbase = ((int64_t)k.b * dim + k.c0 + wc) * n + n0;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        const bool in = wc < k.lim && n0 + s < n;
        a2[s] = in ? p.A[(int64_t)(k.c0 + wc) * n + n0 + s] * kLog2e : 0.0f;
        h[s] = in && p.state ? p.state[sbase + s] : 0.0f;
    }

    Pack<T, VW> rx, rdt, rz;
    T rB[NBC], rC[NBC];
    auto fetch = [&](int t0) {
        const int t = t0 + row;
        const int count = t < len ? lcount : 0;
        rx.load(px + t * p.x_step, count);
        rdt.load(pdt + t * p.dt_step, count);
        rz.load(pz + t * p.z_step, pz ? count : 0);
#pragma unroll
        for (int i = 0; i < NBC; ++i) {
            const int e = tid + i * kThreads, tt = t0 + e / NP, nn = e % NP;
            const bool in = tt < len && nn < n;
            rB[i] = in ? pB[tt * p.B_step + nn] : T(0);
            rC[i] = in ? pC[tt * p.C_step + nn] : T(0);
        }
    };

    fetch(0);
    for (int t0 = 0; t0 < len; t0 += kTile) {
        const bool live = t0 + row < len;
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            float d = to_f32(rdt.v[i]) + bias[i];
            if (p.softplus) d = softplus(d);
            d = live && i < lcount ? d : 0.0f;  // past the end: a = 1, b = 0
            s_du[row][lc + i] = float2{d, d * to_f32(rx.v[i])};
        }
#pragma unroll
        for (int i = 0; i < NBC; ++i) {
            const int e = tid + i * kThreads;
            s_bc[e / NP][e % NP] = float2{to_f32(rB[i]), to_f32(rC[i])};
        }
        const Pack<T, VW> cx = rx, cz = rz;
        __syncthreads();
        if (t0 + kTile < len) fetch(t0 + kTile);

#pragma unroll 1
        for (int tb = 0; tb < kTile; tb += kSsmBlock) {
            if (ckpt && t0 + tb < len) {
                const int64_t blk = (int64_t)k.b * ((steps + kSsmBlock - 1) / kSsmBlock) +
                                    (t0 + tb) / kSsmBlock;
                float* pc = ckpt + (blk * dim + k.c0 + wc) * n + n0;
#pragma unroll
                for (int s = 0; s < SPL; ++s)
                    if (wc < k.lim && n0 + s < n) pc[s] = h[s];
            }
            float v[kSsmBlock];
#pragma unroll
            for (int t = 0; t < kSsmBlock; ++t) {
                const float2 du = s_du[tb + t][wc];
                float acc = 0.0f;
#pragma unroll
                for (int s = 0; s < SPL; ++s) {
                    const float2 bc = s_bc[tb + t][n0 + s];
                    const float a = exp2_fast(du.x * a2[s]);
                    h[s] = __builtin_fmaf(a, h[s], du.y * bc.x);
                    acc = __builtin_fmaf(h[s], bc.y, acc);
                }
                v[t] = acc;
            }
            L::sum_states(v, lane, [&](int t, float sum) { s_y[tb + t][wc] = sum; });
        }
        __syncthreads();
        if (t0 + row < steps) {
            Pack<T, VW> out;
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                float v = s_y[row][lc + i] + skip[i] * to_f32(cx.v[i]);
                if (pz) {
                    const float z = to_f32(cz.v[i]);
                    v *= z * sigmoid(z);
                }
                out.v[i] = from_f32<T>(live ? v : 0.0f);
            }
            out.store(py + (int64_t)(t0 + row) * dim, lcount);
        }
    }
    // the steps past the row's tokens that no tile above has reached
    for (int t = (len + kTile - 1) / kTile * kTile + row; t < steps; t += kTile) {
        Pack<T, VW> out;
#pragma unroll
        for (int i = 0; i < VW; ++i) out.v[i] = T(0);
        out.store(py + (int64_t)t * dim, lcount);
    }
    if (state_out) {
#pragma unroll
        for (int s = 0; s < SPL; ++s)
            if (wc < k.lim && n0 + s < n) state_out[sbase + s] = h[s];
    }
}

// One token.  A quad of lanes owns a channel's states, four at a time: the
// states, read and written once, are all the traffic that counts.
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
            acc = __builtin_fmaf(h.v[i], to_f32(C.v[i]), acc);
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
    k_ssm_scan<T, LN, SPL><<<dim3((unsigned)grid), kThreads, 0, stream>>>(p, (T*)y, state_out,
                                                                          ckpt, nb);
    return hipGetLastError();
}

template <class T>
hipError_t scan_type(const libscan_ssm& p, void* y, float* state_out, float* ckpt, void* scratch,
                     hipStream_t stream) {
    if (p.n > 32) return scan_as<T, 16, 4>(p, y, state_out, ckpt, stream);
    if (p.n > 16) return scan_as<T, 16, 2>(p, y, state_out, ckpt, stream);
    if (p.batch * p.dim >= 16384) return scan_as<T, 4, 4>(p, y, state_out, ckpt, stream);
    return scan_as<T, 16, 1>(p, y, state_out, ckpt, stream);
}

}  // namespace

size_t ssm_scratch_bytes(const libscan_ssm&) { return 0; }

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
