// logits.hip -- penalties, biases and grammar masks on logits, and their softmax.
//
// A workgroup owns a segment of kSeg places of one row.  How often the segment's
// tokens were seen is counted in LDS from the row's history (and the row's
// biases noted by their list places), then the logits stream through once.
// Rows longer than a segment take two kernels for probabilities: the
// segments' maxima and sums, then the same again with the row's total.
#include "launch.hpp"
#include "lm.hpp"

#include "../../include/libscan.h"

namespace ls {

namespace {

constexpr int kThreads = 512;
constexpr int kSeg = 8192;
constexpr int kV = 8;
constexpr int kPer = kSeg / (kThreads * kV);  // groups of kV places a thread owns

constexpr uint32_t kSeen = 0x80000000u;  // in a count: seen at all
constexpr uint32_t kTwice = 0x80000000u; // in a bias word: more than one entry

enum class Mode { Process, Stats, Probs, Whole };  // Whole: a row of one segment

constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ int clamp_count(const int32_t* p, int row, int64_t cols, int missing) {
    if (!p) return missing;
    const int v = p[row];
    return v < 0 ? 0 : v < cols ? v : (int)cols;
}

// LDS words of the segment: counts first, then biases, each only if used.
__device__ __forceinline__ void note_history(const libscan_logits& p, int row, int lo, int size,
                                             uint32_t* count, uint32_t* slot) {
    const int words = (count ? size : 0) + (slot ? size : 0);
    uint32_t* first = count ? count : slot;
    if (!first) return;
    for (int i = threadIdx.x; i < words; i += kThreads) first[i] = 0;
    __syncthreads();
    if (count) {
        const int n = clamp_count(p.history_len, row, p.history_cols, (int)p.history_cols);
        const int np = clamp_count(p.prompt_len, row, p.history_cols, 0);
        const int32_t* ids = p.history + row * p.history_row;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const uint32_t at = (uint32_t)ids[i] - (uint32_t)lo;
            if (at < (uint32_t)size && ids[i] >= 0) {
                if (i >= np) atomicAdd(&count[at], 1u);
                atomicOr(&count[at], kSeen);
            }
        }
    }
    if (slot) {
        const int32_t* ids = p.bias_ids + row * p.biases;
        for (int i = threadIdx.x; i < (int)p.biases; i += kThreads) {
            const uint32_t at = (uint32_t)ids[i] - (uint32_t)lo;
            if (at < (uint32_t)size && ids[i] >= 0) {
                const uint32_t old = atomicMax(&slot[at], (uint32_t)i + 1);
                if (old) atomicOr(&slot[at], kTwice);
            }
        }
    }
    __syncthreads();
}

struct RowParams {
    float rep, inv_rep, pres, freq;
};

template <class T, Mode M>
__global__ __launch_bounds__(kThreads) void k_logits(libscan_logits p, T* out, int64_t out_row,
                                                     float* probs, float2* stats, int segs) {
    extern __shared__ uint32_t s_words[];
    __shared__ float2 s_wave[kThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / segs, seg = blockIdx.x % segs;
    const int vocab = (int)p.vocab, lo = seg * kSeg;
    const int size = vocab - lo < kSeg ? vocab - lo : kSeg;
    uint32_t* count = p.history ? s_words : nullptr;
    uint32_t* slot = p.biases ? s_words + (p.history ? size : 0) : nullptr;
    note_history(p, row, lo, size, count, slot);

    const T* px = (const T*)p.logits + row * p.logits_row + lo;
    const float rep = p.repetition ? p.repetition[row] : 1.0f;
    const float pres = p.presence ? p.presence[row] : 0.0f;
    const float freq = p.frequency ? p.frequency[row] : 0.0f;
    float temp = 1.0f;
    if (M != Mode::Process && p.temperature) temp = p.temperature[row];
    const bool greedy = temp == 0.0f;
    const float inv = greedy ? 1.0f : 1.0f / temp;
    const int32_t* bits = p.allowed ? p.allowed + row * p.allowed_row : nullptr;

    float v[kPer][kV];
    float top = kNegInf;
#pragma unroll
    for (int g = 0; g < kPer; ++g) {
        const int at = (g * kThreads + tid) * kV;
        Pack<T, kV> x;
        x.load(px + at, size - at);
        // lo and at are multiples of kV, so the kV bits lie in one word
        uint32_t open = ~0u;
        if (bits && at < size) open = (uint32_t)bits[(lo + at) >> 5] >> ((lo + at) & 31);
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            float l = to_f32(x.v[i]);
            if (at + i < size) {
                if (count) {
                    const uint32_t c = count[at + i];
                    if (c) {
                        l = l > 0.0f ? l / rep : l * rep;
                        if (c & ~kSeen) l = l - (float)(c & ~kSeen) * freq - pres;
                    }
                }
                if (slot) {
                    const uint32_t s = slot[at + i];
                    if (s) {
                        const float* values = p.bias_values + row * p.biases;
                        if (!(s & kTwice)) {
                            l += values[s - 1];
                        } else {
                            const int32_t* ids = p.bias_ids + row * p.biases;
                            for (int j = 0; j < (int)p.biases; ++j)
                                if (ids[j] == lo + at + i) l += values[j];
                        }
                    }
                }
                if (!((open >> i) & 1)) l = kNegInf;
            } else {
                l = kNegInf;
            }
            v[g][i] = M == Mode::Process ? l : l == kNegInf ? l : l * inv;
            top = __builtin_fmaxf(top, v[g][i]);
        }
        if (M == Mode::Process) {
            Pack<T, kV> o;
#pragma unroll
            for (int i = 0; i < kV; ++i) o.v[i] = from_f32<T>(v[g][i]);
            o.store(out + row * out_row + lo + at, size - at);
        }
    }
    if (M == Mode::Process) return;

    // the share of a value below the maximum m
    auto share = [&](float l, float m) {
        if (l == kNegInf) return 0.0f;
        if (greedy) return l == m ? 1.0f : l != l ? l : 0.0f;
        return exp2_fast((l - m) * kLog2e);
    };
    float m, sum;
    if (M != Mode::Probs) {
#pragma unroll
        for (int o = 32; o; o >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o));
        if (lane == 0) s_wave[wave].x = top;
        __syncthreads();
        m = s_wave[0].x;
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) m = __builtin_fmaxf(m, s_wave[w].x);
        sum = 0.0f;
#pragma unroll
        for (int g = 0; g < kPer; ++g)
#pragma unroll
            for (int i = 0; i < kV; ++i) sum += share(v[g][i], m);
        sum = wave_sum(sum);
        if (lane == 0) s_wave[wave].y = sum;
        __syncthreads();
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) sum += s_wave[w].y;
        if (M == Mode::Stats) {
            if (tid == 0) stats[(int64_t)row * segs + seg] = float2{m, sum};
            return;
        }
    } else {
        const float2* st = stats + (int64_t)row * segs;
        m = kNegInf;
        for (int i = 0; i < segs; ++i) m = __builtin_fmaxf(m, st[i].x);
        sum = 0.0f;
        for (int i = 0; i < segs; ++i) sum += st[i].y == 0.0f ? 0.0f : st[i].y * share(st[i].x, m);
    }
    const float scale = 1.0f / sum;
    float* po = probs + (int64_t)row * vocab + lo;
#pragma unroll
    for (int g = 0; g < kPer; ++g) {
        const int at = (g * kThreads + tid) * kV;
        Pack<float, kV> o;
#pragma unroll
        for (int i = 0; i < kV; ++i)
            o.v[i] = v[g][i] == kNegInf ? 0.0f : share(v[g][i], m) * scale;
        o.store(po + at, size - at);
    }
}

int segments(const libscan_logits& p) { return (int)((p.vocab + kSeg - 1) / kSeg); }

unsigned lds_bytes(const libscan_logits& p) {
    const int64_t size = p.vocab < kSeg ? p.vocab : kSeg;
    return (unsigned)(((p.history ? 1 : 0) + (p.biases ? 1 : 0)) * size * 4);
}

template <class T>
hipError_t process_as(const libscan_logits& p, void* out, int64_t out_row, hipStream_t s) {
    const int segs = segments(p);
    k_logits<T, Mode::Process><<<(unsigned)(p.rows * segs), kThreads, lds_bytes(p), s>>>(
        p, (T*)out, out_row, nullptr, nullptr, segs);
    return hipGetLastError();
}

template <class T>
hipError_t probs_as(const libscan_logits& p, float* probs, void* scratch, hipStream_t s) {
    const int segs = segments(p);
    const unsigned grid = (unsigned)(p.rows * segs), lds = lds_bytes(p);
    if (segs == 1) {
        k_logits<T, Mode::Whole><<<grid, kThreads, lds, s>>>(p, nullptr, 0, probs, nullptr, 1);
    } else {
        k_logits<T, Mode::Stats><<<grid, kThreads, lds, s>>>(p, nullptr, 0, nullptr,
                                                             (float2*)scratch, segs);
        k_logits<T, Mode::Probs><<<grid, kThreads, lds, s>>>(p, nullptr, 0, probs,
                                                             (float2*)scratch, segs);
    }
    return hipGetLastError();
}

}  // namespace

bool logits_fit(const libscan_logits& p) {
    return p.rows <= INT32_MAX / ((p.vocab + kSeg - 1) / kSeg + 1);
}

size_t logits_scratch(const libscan_logits& p) {
    return segments(p) > 1 ? (size_t)p.rows * segments(p) * 8 : 0;
}

hipError_t launch_logits_process(const libscan_logits& p, void* out, int64_t out_row,
                                 hipStream_t stream) {
    if (p.rows == 0 || p.vocab == 0) return hipSuccess;
    switch (p.type) {
        case LIBSCAN_F16: return process_as<_Float16>(p, out, out_row, stream);
        case LIBSCAN_BF16: return process_as<__bf16>(p, out, out_row, stream);
        default: return process_as<float>(p, out, out_row, stream);
    }
}

hipError_t launch_logits_probs(const libscan_logits& p, float* probs, void* scratch,
                               hipStream_t stream) {
    if (p.rows == 0 || p.vocab == 0) return hipSuccess;
    switch (p.type) {
        case LIBSCAN_F16: return probs_as<_Float16>(p, probs, scratch, stream);
        case LIBSCAN_BF16: return probs_as<__bf16>(p, probs, scratch, stream);
        default: return probs_as<float>(p, probs, scratch, stream);
    }
}

}  // namespace ls
