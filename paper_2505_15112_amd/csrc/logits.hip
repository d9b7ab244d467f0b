// logits.hip -- penalties, biases and grammar masks on logits, and their softmax.
//
// A workgroup owns a segment of one row.  The tokens that the row's history and
// biases name are few beside the vocabulary, so they are dealt with one by one:
// counted in LDS, and the new logit of each left there by the one thread that
// claims it.  The segment then streams through once, taking those places from
// LDS (a bit per place tells) and all others as they are.
// Rows longer than a segment take two kernels for probabilities.  The first
// finds the segments' maxima and sums, and leaves the named tokens' logits in
// their places of the output and the bits in scratch memory; the second has
// nothing to count and only streams.  Logits are fp32 from the load to the one
// rounding of the result; shares and sums are fp32.
//
// HBM bounds large calls: 300 x 200003 fp32 with everything on, processed, 94 us
// (487 MB, 5.2 TB/s); 128 x 131072 bf16 to probabilities with 2048 seen tokens a
// row, 21 + 24 us (34 MB, then 101 MB), where the first kernel waits for its
// counting.  One row of 131072: 5.6 + 3.7 us, launch and latency.
#include "launch.hpp"
#include "lm.hpp"

#include "../../include/libscan.h"

namespace ls {

namespace {

constexpr int kV = 8;  // consecutive places of a thread
// Workgroups of so many threads, each with so many groups of kV places.  A few
// rows are cut into small segments, to have more than a handful of workgroups:
// one row of 131072 with 777 seen tokens takes 9.0 us of kernels in small segments
// and 11.0 in large ones; 64 such rows of bf16 24 and 22.
template <int THREADS, int PER>
struct Cut {
    static constexpr int kThreads = THREADS, kPer = PER, kSeg = THREADS * PER * kV;
};
using Large = Cut<512, 2>;
using Small = Cut<256, 1>;

enum class Mode { Process, Stats, Probs, Whole };  // Whole: a row of one segment

constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ int clamp_count(const int32_t* p, int row, int64_t cols, int missing) {
    if (!p) return missing;
    const int v = p[row];
    return v < 0 ? 0 : v < cols ? v : (int)cols;
}

// A segment's notes.  word: the count of a seen token, later its new logit;
// bits: named (word holds a logit), biased (by some entry), twice (by several);
// repeats: whether there is a place of the last kind.
template <class C>
struct Notes {
    uint32_t word[C::kSeg];
    uint32_t named[C::kSeg / 32], biased[C::kSeg / 32], twice[C::kSeg / 32];
    uint32_t repeats, unused[3];
};

// The first ids of this thread's share (i = thread, thread + kThreads, ...), which
// set out before anything else and are gone through more than once.
constexpr int kHold = 4;
struct Held {
    int id[kHold];
    template <class C>
    __device__ __forceinline__ void load(const int32_t* ids, int64_t n) {
#pragma unroll
        for (int j = 0; j < kHold; ++j) {
            const int i = threadIdx.x + j * C::kThreads;
            id[j] = i < n ? ids[i] : -1;
        }
    }
};

// Calls f(i, ids[i]) for this thread's share of i < n.
template <class C, class F>
__device__ __forceinline__ void each_id(const int32_t* ids, int n, const Held& held, F f) {
#pragma unroll
    for (int j = 0; j < kHold; ++j) {
        const int i = threadIdx.x + j * C::kThreads;
        if (i < n) f(i, held.id[j]);
    }
#pragma unroll 1
    for (int i0 = threadIdx.x + kHold * C::kThreads; i0 < n; i0 += kHold * C::kThreads) {
        Held more;
        more.load<C>(ids + (i0 - threadIdx.x), n - (i0 - threadIdx.x));
#pragma unroll
        for (int j = 0; j < kHold; ++j)
            if (i0 + j * C::kThreads < n) f(i0 + j * C::kThreads, more.id[j]);
    }
}

// Adds the biases of the places that several entries name, in the list's order: every
// wave goes through the list, 64 entries at a time, and adds those of its own places.
// The time grows with the list's length, whatever repeats: 16384 entries for a row of
// 131072 with each id twice 82 us a call (33 without repeats, 670 if all are one id).
template <class C>
__device__ __forceinline__ void add_repeats(const int32_t* ids, const float* values, int n, int lo,
                                            int size, Notes<C>& s) {
    constexpr int kWaves = C::kThreads / 64, kBatch = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += 64 * kBatch) {
        int id[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int i = i0 + j * 64 + lane;
            id[j] = i < n ? ids[i] : -1;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint32_t at = id[j] >= 0 ? (uint32_t)id[j] - (uint32_t)lo : ~0u;
            const bool mine = at < (uint32_t)size && (int)(at >> 5) % kWaves == wave &&
                              (s.twice[at >> 5] >> (at & 31) & 1);
            uint64_t todo = __ballot(mine);
            if (!todo) continue;
            const float v = mine ? values[i0 + j * 64 + lane] : 0.0f;
            while (todo) {
                const uint32_t place = __builtin_amdgcn_readlane(at, __builtin_ctzll(todo));
                uint64_t same = __ballot(mine && at == place);
                todo &= ~same;
                float l = as_f32(s.word[place]);
                for (; same; same &= same - 1)
                    l += as_f32(__builtin_amdgcn_readlane(as_u32(v), __builtin_ctzll(same)));
                s.word[place] = as_u32(l);
            }
        }
    }
}

// Fills s with the new logits of the places lo .. lo + size that the row's
// history or biases name.
template <class C, class T>
__device__ __forceinline__ void note_named(const libscan_logits& p, const T* px, int row, int lo,
                                           int size, const Held& first_ids, const Held& first_biases,
                                           Notes<C>& s) {
    uint4* all = reinterpret_cast<uint4*>(&s);
    for (int i = threadIdx.x; i < (int)(sizeof(s) / 16); i += C::kThreads)
        all[i] = uint4{0, 0, 0, 0};
    const int n = p.history ? clamp_count(p.history_len, row, p.history_cols, (int)p.history_cols)
                            : 0;
    const int made = clamp_count(p.prompt_len, row, p.history_cols, 0);
    const int32_t* ids = p.history + row * p.history_row;
    const int32_t* bias_ids = p.bias_ids + row * p.biases;
    const float* bias_values = p.bias_values + row * p.biases;
    auto place = [&](int id) { return id >= 0 ? (uint32_t)id - (uint32_t)lo : ~0u; };
    __syncthreads();
    each_id<C>(ids, n, first_ids, [&](int i, int id) {
        const uint32_t at = place(id);
        if (at < (uint32_t)size && i >= made) atomicAdd(&s.word[at], 1u);
    });
    each_id<C>(bias_ids, (int)p.biases, first_biases, [&](int, int id) {
        const uint32_t at = place(id), bit = 1u << (at & 31);
        if (at < (uint32_t)size && (atomicOr(&s.biased[at >> 5], bit) & bit)) {
            atomicOr(&s.twice[at >> 5], bit);
            s.repeats = 1;
        }
    });
    __syncthreads();
    const bool repeats = s.repeats;
    if (n > 0) {
        const float rep = p.repetition ? p.repetition[row] : 1.0f;
        // l / rep, rounded once, as the product with the reciprocal in 64 bits: it is off by
        // at most 2^-52 of the quotient, and a normal quotient of 24-bit numbers at least 2^-49
        // of itself from where the rounding to 24 bits turns.  (19 rows of 3185 places
        // with 7381 tokens: a division for each token 14.7 us, this 13.4, a product with the
        // rounded reciprocal, which rounds twice, 12.7.)
        const double inv_rep = 1.0 / (double)rep;
        const float pres = p.presence ? p.presence[row] : 0.0f;
        const float freq = p.frequency ? p.frequency[row] : 0.0f;
        each_id<C>(ids, n, first_ids, [&](int, int id) {
            const uint32_t at = place(id), bit = 1u << (at & 31);
            if (at < (uint32_t)size && !(atomicOr(&s.named[at >> 5], bit) & bit)) {
                const uint32_t c = s.word[at];
                float l = to_f32(px[at]);
                l = l > 0.0f ? (float)((double)l * inv_rep) : l * rep;
                if (c) l = l - (float)c * freq - pres;
                s.word[at] = as_u32(l);
            }
        });
        if (p.biases) __syncthreads();
    }
    each_id<C>(bias_ids, (int)p.biases, first_biases, [&](int i, int id) {
        const uint32_t at = place(id), bit = 1u << (at & 31);
        if (at >= (uint32_t)size) return;
        if (repeats && (s.twice[at >> 5] & bit)) {  // one of them puts the logit there, without a bias
            if (!(atomicOr(&s.named[at >> 5], bit) & bit)) s.word[at] = as_u32(to_f32(px[at]));
            return;
        }
        const float l = s.named[at >> 5] & bit ? as_f32(s.word[at]) : to_f32(px[at]);
        s.word[at] = as_u32(l + bias_values[i]);
        atomicOr(&s.named[at >> 5], bit);
    });
    __syncthreads();
    if (repeats) {
        add_repeats<C>(bias_ids, bias_values, (int)p.biases, lo, size, s);
        __syncthreads();
    }
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v = __builtin_fmaxf(v, __shfl_xor(v, o));
    return v;
}

// NAMED: the rows have a history or biases.
template <class T, Mode M, class C, bool NAMED>
__global__ __launch_bounds__(C::kThreads) void k_logits(libscan_logits p, T* out, int64_t out_row,
                                                        float* probs, float2* stats,
                                                        uint32_t* named_bits, int segs) {
    constexpr int kWaves = C::kThreads / 64, kPer = C::kPer, kWords = C::kSeg / 32;
    constexpr bool kNote = NAMED && M != Mode::Probs;
    __shared__ __align__(16) char s_mem[kNote ? sizeof(Notes<C>) : 16];
    __shared__ float2 s_wave[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / segs, seg = blockIdx.x % segs;
    const int vocab = (int)p.vocab, lo = seg * C::kSeg;
    const int size = vocab - lo < C::kSeg ? vocab - lo : C::kSeg;
    Notes<C>& notes = *reinterpret_cast<Notes<C>*>(s_mem);

    // everything that is read from memory sets out before anything is waited for
    Held first_ids, first_biases;
    if (kNote) {
        first_ids.load<C>(p.history + row * p.history_row, p.history ? p.history_cols : 0);
        first_biases.load<C>(p.bias_ids + row * p.biases, p.biases);
    }
    const T* px = (const T*)p.logits + row * p.logits_row + lo;
    const int32_t* bits = p.allowed ? p.allowed + row * p.allowed_row : nullptr;
    Pack<T, kV> x[kPer];
    uint32_t named[kPer];
    uint32_t open[kPer];  // lo and a thread's places are multiples of kV: one word has their bits
#pragma unroll
    for (int g = 0; g < kPer; ++g) {
        const int at = (g * C::kThreads + tid) * kV;
        x[g].load(px + at, size - at);
        open[g] = ~0u;
        if (bits && at < size) open[g] = (uint32_t)bits[(lo + at) >> 5] >> ((lo + at) & 31);
        named[g] = 0;
        if (NAMED && M == Mode::Probs)
            named[g] = named_bits[((int64_t)row * segs + seg) * kWords + (at >> 5)];
        if (size - at < kV) open[g] &= at < size ? (1u << (size - at)) - 1 : 0u;
    }
    const float2* row_stats = M == Mode::Probs ? stats + (int64_t)row * segs : nullptr;
    float2 st{kNegInf, 0.0f};
    if (M == Mode::Probs && lane < segs) st = row_stats[lane];
    float temp = 1.0f;
    if (M != Mode::Process && p.temperature) temp = p.temperature[row];

    float* po = M == Mode::Process ? nullptr : probs + (int64_t)row * vocab + lo;
    if (kNote) {
        note_named<C>(p, px, row, lo, size, first_ids, first_biases, notes);
        if (M == Mode::Stats && tid < kWords)
            named_bits[((int64_t)row * segs + seg) * kWords + tid] = notes.named[tid];
    }

    // Shares are e^((l - m) / temperature) for the row's largest logit m: the
    // difference first, as a logit times 1 / temperature may overflow (rows masked
    // by the type's lowest value).  A negative temperature turns the logits over;
    // -0.0, whose slope is -infinity, is not one.
    const float scale = __builtin_fabsf(kLog2e / temp);
    const bool greedy = scale == -kNegInf, flip = temp < 0.0f, odd = greedy || scale == 0.0f;
    const bool masked = bits != nullptr || size < C::kSeg;
    float v[kPer][kV];
    float top = kNegInf;
#pragma unroll
    for (int g = 0; g < kPer; ++g) {
        const int at = (g * C::kThreads + tid) * kV;
#pragma unroll
        for (int i = 0; i < kV; ++i) v[g][i] = to_f32(x[g].v[i]);
        if (NAMED) {
            if (kNote) named[g] = notes.named[at >> 5];
            named[g] = named[g] >> (at & 31) & ((1u << kV) - 1);
            if (named[g]) {
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    if (!(named[g] >> i & 1)) continue;
                    v[g][i] = kNote ? as_f32(notes.word[at + i]) : po[at + i];
                    if (M == Mode::Stats) po[at + i] = v[g][i];
                }
            }
        }
        if (M != Mode::Process && flip) {
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (v[g][i] != kNegInf) v[g][i] = -v[g][i];
        }
        if (masked) {
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (!(open[g] >> i & 1)) v[g][i] = kNegInf;
        }
        if (M == Mode::Process) {
            Pack<T, kV> o;
#pragma unroll
            for (int i = 0; i < kV; ++i) o.v[i] = from_f32<T>(v[g][i]);
            o.store(out + row * out_row + lo + at, size - at);
        } else {
#pragma unroll
            for (int i = 0; i < kV; ++i) top = __builtin_fmaxf(top, v[g][i]);
        }
    }
    if (M == Mode::Process) return;

    // the share of a value below the maximum m (a row of -infinity alone: 0)
    auto share = [&](float l, float m) {
        if (odd) {
            if (greedy) return l == m ? 1.0f : l != l ? l : 0.0f;
            if (l == kNegInf) return 0.0f;
        }
        return exp2_fast((l - m) * scale);
    };
    auto base = [](float m) { return m == kNegInf ? 0.0f : m; };
    float m, sum;
    if (M != Mode::Probs) {
        top = wave_max(top);
        if (lane == 0) s_wave[wave].x = top;
        __syncthreads();
        top = s_wave[0].x;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = __builtin_fmaxf(top, s_wave[w].x);
        m = base(top);
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
        for (int w = 0; w < kWaves; ++w) sum += s_wave[w].y;
        if (M == Mode::Stats) {
            if (tid == 0) stats[(int64_t)row * segs + seg] = float2{top, sum};
            return;
        }
    } else {
        // the segments' maxima and sums, one to a lane (the first 64 loaded above)
        m = st.x;
        for (int i = lane + 64; i < segs; i += 64) m = __builtin_fmaxf(m, row_stats[i].x);
        m = base(wave_max(m));
        sum = st.y == 0.0f ? 0.0f : st.y * share(base(st.x), m);
        for (int i = lane + 64; i < segs; i += 64) {
            const float2 o = row_stats[i];
            sum += o.y == 0.0f ? 0.0f : o.y * share(base(o.x), m);
        }
        sum = wave_sum(sum);
    }
    const float one = sum == 0.0f ? 0.0f : 1.0f / sum;
    const bool spoilt = !(one >= 0.0f);  // NaN or +infinity in the row: 0 at -infinity even so
#pragma unroll
    for (int g = 0; g < kPer; ++g) {
        const int at = (g * C::kThreads + tid) * kV;
        Pack<float, kV> o;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            o.v[i] = share(v[g][i], m) * one;
            if (spoilt && v[g][i] == kNegInf) o.v[i] = 0.0f;
        }
        o.store(po + at, size - at);
    }
}

template <class C>
int64_t segments(const libscan_logits& p) {
    return (p.vocab + C::kSeg - 1) / C::kSeg;
}

// Small segments where the large ones would leave CUs without work; for
// probabilities only if the row takes two kernels anyway.
bool small(const libscan_logits& p, bool probs) {
    return p.rows * segments<Large>(p) < 256 && !(probs && p.vocab <= Large::kSeg);
}

template <class T, class C, bool NAMED>
hipError_t process_as(const libscan_logits& p, void* out, int64_t out_row, hipStream_t s) {
    const int segs = (int)segments<C>(p);
    k_logits<T, Mode::Process, C, NAMED><<<(unsigned)(p.rows * segs), C::kThreads, 0, s>>>(
        p, (T*)out, out_row, nullptr, nullptr, nullptr, segs);
    return hipGetLastError();
}

template <class T, class C, bool NAMED>
hipError_t probs_as(const libscan_logits& p, float* probs, void* scratch, hipStream_t s) {
    const int segs = (int)segments<C>(p);
    const unsigned grid = (unsigned)(p.rows * segs), n = C::kThreads;
    float2* stats = (float2*)scratch;
    uint32_t* bits = (uint32_t*)(stats + p.rows * segs);
    if (segs == 1) {
        k_logits<T, Mode::Whole, C, NAMED><<<grid, n, 0, s>>>(p, nullptr, 0, probs, nullptr, nullptr,
                                                                 1);
    } else {
        k_logits<T, Mode::Stats, C, NAMED><<<grid, n, 0, s>>>(p, nullptr, 0, probs, stats, bits,
                                                                 segs);
        k_logits<T, Mode::Probs, C, NAMED><<<grid, n, 0, s>>>(p, nullptr, 0, probs, stats, bits,
                                                                 segs);
    }
    return hipGetLastError();
}

// f(element, cut, named) for the call's kernels
template <class F>
hipError_t by_kind(const libscan_logits& p, bool probs, F f) {
    auto named = [&](auto t, auto cut) {
        return p.history || p.biases ? f(t, cut, std::true_type()) : f(t, cut, std::false_type());
    };
    auto cut = [&](auto t) { return small(p, probs) ? named(t, Small()) : named(t, Large()); };
    switch (p.type) {
        case LIBSCAN_F16: return cut(_Float16());
        case LIBSCAN_BF16: return cut(__bf16());
        default: return cut(float());
    }
}

}  // namespace

bool logits_fit(const libscan_logits& p) {
    return p.rows <= (INT32_MAX / 512) / (segments<Large>(p) + 1);
}

size_t logits_scratch(const libscan_logits& p) {
    const int64_t segs = small(p, true) ? segments<Small>(p) : segments<Large>(p);
    if (segs == 1) return 0;
    const int64_t bits = !p.history && !p.biases ? 0 : small(p, true) ? Small::kSeg / 8 : Large::kSeg / 8;
    return (size_t)p.rows * segs * (8 + bits);
}

hipError_t launch_logits_process(const libscan_logits& p, void* out, int64_t out_row,
                                 hipStream_t stream) {
    if (p.rows == 0 || p.vocab == 0) return hipSuccess;
    return by_kind(p, false, [&](auto t, auto cut, auto named) {
        return process_as<decltype(t), decltype(cut), decltype(named)::value>(p, out, out_row,
                                                                              stream);
    });
}

hipError_t launch_logits_probs(const libscan_logits& p, float* probs, void* scratch,
                               hipStream_t stream) {
    if (p.rows == 0 || p.vocab == 0) return hipSuccess;
    return by_kind(p, true, [&](auto t, auto cut, auto named) {
        return probs_as<decltype(t), decltype(cut), decltype(named)::value>(p, probs, scratch,
                                                                            stream);
    });
}

}  // namespace ls
