// attend_walk.hpp -- the walk of linear attention (attend.hpp) on the matrix cores.
//
// A workgroup takes a row's head in chunks of kChunk tokens.  With c the running sum of
// the decays' logarithms inside the chunk and S the state before it,
//   o[i] = e^c[i] q[i] S + sum over j <= i of (q[i] . k[j]) e^(c[i] - c[j]) v[j],
//   S' = e^c[last] S + sum over j of k[j] (e^(c[last] - c[j]) v[j])^T:
// four matrix products.  S stays in fp32 accumulators; its fragments are what the
// next product takes.  The logarithms are added up in 64 bits: their sums over a
// chunk are far larger than the differences that count.
//
// Terms.  All products are bfloat16 matrix instructions with fp32 sums.  An operand
// of more bits is split into terms of 8 bits each, all but the last by truncation
// (what is left is exact, and nothing overflows): fp16 inputs into two and fp32
// inputs into three, which hold them exactly.  Term i of one operand meets term j of
// the other where i + j < 3.  bfloat16's exponents are fp32's, so neither scores nor
// states overflow or lose their small values, as they would in fp16.  Scores and states are
// three terms whatever the type of the outputs, whose last rounding is the only one to
// fewer bits than fp32's.  (Two terms, 2^-17 off, take 96 to 99 % of the time, 85 % where one
// chain of chunks is all, but leave bfloat16 outputs 1.3e-4 of their 2-norm off those of
// 32-bit products, by last roundings that went the other way; three leave 4e-5.)
#pragma once

#include <type_traits>

#include "attend.hpp"

namespace ls {
namespace walk {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));

template <class T>
inline constexpr int kTerms = 3;
template <>
inline constexpr int kTerms<_Float16> = 2;
template <>
inline constexpr int kTerms<__bf16> = 1;

// N (even) values to TERMS terms, each packed in pairs.
template <int TERMS, int N>
__device__ __forceinline__ void split(const float (&in)[N], unsigned (&out)[TERMS][N / 2]) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        float a = in[i], b = in[i + 1];
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            if (t == TERMS - 1) {
                typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
                const bf2 r{(__bf16)a, (__bf16)b};
                out[t][i / 2] = __builtin_bit_cast(unsigned, r);
            } else {
                const unsigned ha = as_u32(a) & 0xffff0000u, hb = as_u32(b) & 0xffff0000u;
                out[t][i / 2] = __builtin_amdgcn_perm(hb, ha, 0x07060302u);
                a -= as_f32(ha);
                b -= as_f32(hb);
            }
        }
    }
}

template <int TERMS>
struct Frag {
    bf8 t[TERMS];
    __device__ __forceinline__ void from(const float (&v)[8]) {
        unsigned u[TERMS][4];
        split<TERMS, 8>(v, u);
#pragma unroll
        for (int i = 0; i < TERMS; ++i)
            t[i] = __builtin_bit_cast(bf8, u4{u[i][0], u[i][1], u[i][2], u[i][3]});
    }
    __device__ __forceinline__ float value(int e) const {
        float v = (float)t[TERMS - 1][e];
#pragma unroll
        for (int i = TERMS - 2; i >= 0; --i) v += (float)t[i][e];
        return v;
    }
};

// c += a b.  Lane l has row (a) or column (b) l % 16 at the eight places from 8 (l /
// 16) of the 32 summed over, and of the result column l % 16, rows from 4 (l / 16).
constexpr int kTerms32 = 3;  // of an fp32 value
template <int NA, int NB>
__device__ __forceinline__ void mma(f4& c, const Frag<NA>& a, const Frag<NB>& b) {
#pragma unroll
    for (int s = kTerms32 - 1; s >= 0; --s)  // small parts first
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (i + j == s)
                    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.t[i], b.t[j], c, 0, 0, 0);
}

// A tile of ROWS x WIDTH elements in LDS, by terms.  PAD elements behind a row spread
// the lanes of an access over the banks: 16 bytes each of 16 rows (along), or 8 bytes each
// of 8 rows, 16 apart (down).
template <int TERMS, int ROWS, int WIDTH, int PAD>
struct Tile {
    static constexpr int ROW = WIDTH + PAD;
    alignas(16) __bf16 v[TERMS][ROWS][ROW];

    // Eight elements along a row.
    __device__ __forceinline__ Frag<TERMS> along(int row, int col) const {
        Frag<TERMS> f;
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
            f.t[t] = *reinterpret_cast<const bf8*>(&v[t][row][col]);
        return f;
    }
    // The values of four elements along a row.
    __device__ __forceinline__ f4 four(int row, int col) const {
        f4 sum{};
#pragma unroll
        for (int t = TERMS - 1; t >= 0; --t) {
            typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
            const bf4 x = *reinterpret_cast<const bf4*>(&v[t][row][col]);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += (float)x[e];
        }
        return sum;
    }
    // Eight elements down a column, rows row + 8 (l / 16) and on, of 16 columns: `col` is
    // where this lane's four (those of all lanes l % 4) lie, and lane l gets
    // element l % 4 of the four that lane (l % 16) / 4 names.
    __device__ __forceinline__ Frag<TERMS> down(int row, int col, int lane) const {
        Frag<TERMS> f;
        const int r = row + 8 * (lane / 16) + lane % 16 / 4;
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            typedef __attribute__((address_space(3))) s4* Lds;
            const s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(&v[t][r][col]));
            const s4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(&v[t][r + 4][col]));
            f.t[t] = __builtin_bit_cast(bf8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return f;
    }
};

// The chunks of one operand on their way from global memory to LDS: vectors of 16 bytes in
// registers, the addresses of the first ones moving on from chunk to chunk.
template <class T, int ROWS, int WIDTH, int THREADS>
struct Fetch {
    static constexpr int V = 16 / sizeof(T), PER_ROW = WIDTH / V, ALL = ROWS * PER_ROW;
    static constexpr int N = (ALL + THREADS - 1) / THREADS, BETWEEN = THREADS / PER_ROW;
    typedef typename Pack<T, V>::Vec Vec;
    Vec r[N];
    const T* at;      // this thread's first vector of the next chunk
    int64_t forward;  // elements to the next place
    int width;

    // p: the operand's row at place `base`, and elements to the next place.
    __device__ __forceinline__ void init(const T* p, int64_t step, int elements) {
        forward = step;
        width = elements;
        at = p + threadIdx.x / PER_ROW * step + threadIdx.x % PER_ROW * V;
    }
    // The next chunk, whose places from `skip` to `rows` have tokens; 0 elsewhere.
    __device__ __forceinline__ void load(int skip, int rows) {
        const bool mine = ALL % THREADS == 0 || threadIdx.x < ALL;
        if (skip <= 0 && rows >= ROWS && width >= WIDTH) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (mine) r[i] = *reinterpret_cast<const Vec*>(at + i * BETWEEN * forward);
        } else {
            const int col = threadIdx.x % PER_ROW * V, row = threadIdx.x / PER_ROW;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                Vec v{};
                const int place = row + i * BETWEEN;
                if (mine && place >= skip && place < rows && col < width) {
                    const T* from = at + i * BETWEEN * forward;
                    if (col + V <= width) {
                        v = *reinterpret_cast<const Vec*>(from);
                    } else {
#pragma unroll
                        for (int e = 0; e < V - 1; ++e)
                            if (col + e < width) v[e] = from[e];
                    }
                }
                r[i] = v;
            }
        }
        at += ROWS * forward;
    }
    template <class S>
    __device__ __forceinline__ void store(S& s) const {
        constexpr int TERMS = kTerms<T>;
        if (ALL % THREADS != 0 && threadIdx.x >= ALL) return;
        const int col = threadIdx.x % PER_ROW * V, row = threadIdx.x / PER_ROW;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (TERMS == 1) {
                *reinterpret_cast<u4*>(&s.v[0][row + i * BETWEEN][col]) =
                    __builtin_bit_cast(u4, r[i]);
            } else {
                float f[V];
                unsigned u[TERMS][V / 2];
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = to_f32(r[i][e]);
                split<TERMS, V>(f, u);
#pragma unroll
                for (int t = 0; t < TERMS; ++t) {
                    __bf16* to = &s.v[t][row + i * BETWEEN][col];
                    if constexpr (V == 8)
                        *reinterpret_cast<u4*>(to) = u4{u[t][0], u[t][1], u[t][2], u[t][3]};
                    else
                        *reinterpret_cast<u2*>(to) = u2{u[t][0], u[t][1]};
                }
            }
        }
    }
};

__device__ __forceinline__ double lane_value(double c, int lane) {
    const auto b = __builtin_bit_cast(u2, c);
    return __builtin_bit_cast(double, u2{(unsigned)__builtin_amdgcn_readlane(b[0], lane),
                                         (unsigned)__builtin_amdgcn_readlane(b[1], lane)});
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double add_from(double c) {
    const auto b = __builtin_bit_cast(u2, c);
    u2 m;
    m[0] = __builtin_amdgcn_update_dpp(0, b[0], CTRL, ROWS, 0xf, false);
    m[1] = __builtin_amdgcn_update_dpp(0, b[1], CTRL, ROWS, 0xf, false);
    return c + __builtin_bit_cast(double, m);
}

// Running sums of the chunk's decays over the lanes of a wave, in powers of two.  A
// decay past +-1024 is one of 0 or infinity either way; infinities would turn the
// differences of sums to NaN.
__device__ __forceinline__ double running_sum(float g) {
    double c = (double)g * 1.4426950408889634;
    c = c < -1024.0 ? -1024.0 : c > 1024.0 ? 1024.0 : c;  // a NaN stays
    // rows of 16 lanes by shifts of 1, 2, 4 and 8, then the rows before
    c = add_from<0x111, 0xf>(c);
    c = add_from<0x112, 0xf>(c);
    c = add_from<0x114, 0xf>(c);
    c = add_from<0x118, 0xf>(c);
    c = add_from<0x142, 0xa>(c);
    return add_from<0x143, 0xc>(c);
}

// A running sum's part in 256ths.  Such parts fit fp32 (a chunk's sums stay below 2^16),
// and so do their differences, which makes that of two sums exact to the rest's 2^-33.
__device__ __forceinline__ float high_part(double c) {
    return (float)(__builtin_rint(c * 256.0) * (1.0 / 256.0));
}

// DK: the width of q and k rounded up, WAVES of 16 columns of v each.  OUT: with outputs; else the
// pieces' states alone.  DOTS: with the sums of the outputs times e.  What a token gives
// its own output, whatever the decays are, is not in these: dq's and dk's sums differ by what
// other tokens give, of which rapid decays leave little.  So it is added to the outputs last,
// in fp32.
//
// A walk of 4 x 2048 tokens and 16 heads of 128 x 128, bf16, in eight pieces takes 51 us for
// 168 MB, 32 at the rate of a copy: the vector units are busy 51 % of the time (a third of
// their work is splitting the state into terms and scaling it), LDS 34 %, the matrix units
// 26 %, and waves wait for barriers and LDS half of theirs.
template <class T, int DK, int WAVES_, bool OUT, bool DOTS>
struct Kernel {
    static constexpr int WAVES = WAVES_, COLS = 16 * WAVES, THREADS = 64 * WAVES;
    static constexpr int TERMS = kTerms<T>, TP = kTerms32;
    static constexpr bool WITH_DOTS = DOTS;
    static constexpr int CH = kChunk, PAIRS = DK / 32;
    struct Shared {
        Tile<TERMS, CH, DK, DK == 64 ? 16 : 24> k;
        Tile<TERMS, CH, COLS, 8> v;
        Tile<TERMS, OUT ? CH : 1, DK, 8> q;
        Tile<TP, OUT ? CH : 1, CH, 8> p;  // the scores
        float2 c[CH];            // the running sums in two parts, see high_part
        float in[CH], left[CH];  // e^c outer; e^(c[last] - c) inner
        float own[DOTS ? CH : 1];  // the scores of tokens with themselves
        float whole;

        // A wave's part of a token's dot product, in the padding of k's row.
        __device__ __forceinline__ float& dot(int wave, int token) {
            static_assert(WAVES <= 8, "eight floats");
            return reinterpret_cast<float*>(&k.v[0][token][DK])[wave];
        }
    };

    // Scores of 16 x 16 tokens, of the three such tiles on and below the diagonal the one
    // of this wave: lane l gets those of token l % 16 with four others, next to each other
    // in a row.
    static __device__ __forceinline__ void scores(Shared& s, float factor, int wave, int lane) {
        if (wave >= 3) return;
        const int g = lane / 16, n = lane % 16, row = wave > 0, col = wave > 1;
        f4 acc{};
#pragma unroll
        for (int p = 0; p < PAIRS; ++p)
            mma(acc, s.k.along(16 * col + n, 32 * p + 8 * g),
                     s.q.along(16 * row + n, 32 * p + 8 * g));
        const int i = 16 * row + n, j = 16 * col + 4 * g;
        const float2 ci = s.c[i];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 cj = s.c[j + e];
            const float d = exp2_fast((ci.x - cj.x) + (ci.y - cj.y)) * factor;
            v[e] = j + e <= i ? acc[e] * d : 0.0f;
            if (DOTS && j + e == i) {
                s.own[i] = v[e];
                v[e] = 0.0f;
            }
        }
        unsigned u[TP][2];
        split<TP, 4>(v, u);
#pragma unroll
        for (int t = 0; t < TP; ++t)
            *reinterpret_cast<u2*>(&s.p.v[t][i][j]) = u2{u[t][0], u[t][1]};
    }

    // o += the scores times v where v has an infinity or a NaN: such an element
    // counts for its own token and later ones alone (0 times it is not 0).
    static __device__ __forceinline__ void careful(const Shared& s, f4 (&o)[2],
                                                   const Frag<TERMS>& v, int wave, int lane) {
        const int g = lane / 16, n = lane % 16;
        Frag<TERMS> clean;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool fine = __builtin_isfinite(v.value(e));
#pragma unroll
            for (int t = 0; t < TERMS; ++t) clean.t[t][e] = fine ? v.t[t][e] : (__bf16)0.0f;
        }
#pragma unroll
        for (int row = 0; row < 2; ++row) {
            mma(o[row], clean, s.p.along(16 * row + n, 8 * g));
            for (int j = 0; j < 16 * row + n + !DOTS; ++j) {
                float p = 0.0f;
#pragma unroll
                for (int t = TP - 1; t >= 0; --t) p += (float)s.p.v[t][16 * row + n][j];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float value = 0.0f;
#pragma unroll
                    for (int t = TERMS - 1; t >= 0; --t)
                        value += (float)s.v.v[t][j][wave * 16 + 4 * g + e];
                    if (!__builtin_isfinite(value)) o[row][e] += p * value;
                }
            }
        }
    }

    // Element (r, c) of a state, from its address and strides: the lane's eight rows of
    // each of PAIRS are 32 p + 8 g + 0..7, its column 16 wave + n.
    typedef f4 State[PAIRS][2];
    static __device__ __forceinline__ void load_state(State& state, const float* p, const Walk& w,
                                                      const WalkState& at, int c, int g) {
        p += c * at.col + 8 * g * at.row;
        if (w.dk == DK && at.row == 1) {
            typedef f4 Vec __attribute__((aligned(4)));
#pragma unroll
            for (int x = 0; x < PAIRS; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    state[x][y] = *reinterpret_cast<const Vec*>(p + 32 * x + 4 * y);
            return;
        }
#pragma unroll
        for (int x = 0; x < PAIRS; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (32 * x + 8 * g + e < w.dk)
                    state[x][e / 4][e % 4] = p[(32 * x + e) * at.row];
    }
    static __device__ __forceinline__ void store_state(const State& state, float* p, const Walk& w,
                                                       const WalkState& at, int c, int g) {
        p += c * at.col + 8 * g * at.row;
#pragma unroll
        for (int x = 0; x < PAIRS; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (32 * x + 8 * g + e < w.dk)
                    p[(32 * x + e) * at.row] = state[x][e / 4][e % 4];
    }

    static __device__ __forceinline__ void run(const Walk& w, Shared& s) {
        const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, g = lane / 16, n = lane % 16;
        const int blocks = (w.dv + COLS - 1) / COLS;
        int at = blockIdx.x;
        const int block = at % blocks;
        at /= blocks;
        const int h = at % w.heads;
        at /= w.heads;
        const int piece = at % w.pieces, b = at / w.pieces, bh = b * w.heads + h;
        const int len = walk_len(w, b), skip = walk_skip(w, len), c0 = block * COLS;
        const int start = piece * w.piece, end = start + w.piece;
        const int live = len + skip < end ? len + skip : end;  // where the piece's tokens end
        const int64_t number = (int64_t)bh * w.pieces + piece;
        const int column = c0 + wave * 16 + n;  // of the state

        // The first place's token, and the way from token to token.
        const int way = w.reverse ? -1 : 1, first = walk_token(w, start, len);
        const auto side = [&](const WalkSide& x, int t) {
            return (const T*)x.p + b * x.batch + (h / x.share) * x.head + t * x.step;
        };
        Fetch<T, CH, DK, THREADS> fq, fk;
        Fetch<T, CH, COLS, THREADS> fv;
        float decay = 0.0f;
        const auto fetch = [&](int base) {
            fk.load(skip - base, live - base);
            fv.load(skip - base, live - base);
            if constexpr (OUT) fq.load(skip - base, live - base);
            if (wave == 0)
                decay = lane < CH && base + lane < live ? walk_decay(w, b, h, base + lane, len) : 0.0f;
        };
        State state;
#pragma unroll
        for (int x = 0; x < PAIRS; ++x) state[x][0] = state[x][1] = f4{};
        if (start < live) {
            fk.init(side(w.k, first), way * w.k.step, w.dk);
            fv.init(side(w.v, first) + c0, way * w.v.step, w.dv - c0);
            if constexpr (OUT) fq.init(side(w.q, first), way * w.q.step, w.dk);
            fetch(start);
        }
        if (OUT && w.first.p && column < w.dv)
            load_state(state, w.first.p + number * w.dk * w.dv, w, w.first, column, g);

        if constexpr (OUT) {
            // what lies behind the row's end, and the scores' tiles above the diagonal
            const int cols = w.dv - c0 < COLS ? w.dv - c0 : COLS;
            for (int i = (len > start ? len : start) + wave; i < end && i < w.steps; i += WAVES) {
                const int64_t o = (((int64_t)b * w.steps + i) * w.heads + h) * w.dv + c0;
                for (int c = lane; c < cols; c += 64) {
                    if (w.wide)
                        ((float*)w.out)[o + c] = 0.0f;
                    else
                        ((T*)w.out)[o + c] = T(0);
                }
            }
            for (int i = tid; i < TP * CH * s.p.ROW; i += THREADS)
                (&s.p.v[0][0][0])[i] = (__bf16)0.0f;
        }

        const auto put_dots = [&](int base) {
            if (tid >= CH || base + tid < skip || base + tid >= live) return;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) sum += s.dot(i, tid);
            const int t = walk_token(w, base + tid, len);
            w.dots[(((int64_t)block * w.batch + b) * w.steps + t) * w.heads + h] = sum;
        };

        // The lane's outputs: 4 columns of token n of every tile of 16.
        const int c = c0 + wave * 16 + 4 * g, count = w.dv - c;
        const int row_step = way * w.heads * w.dv;  // at most 2^24
        int64_t to = (((int64_t)b * w.steps + first) * w.heads + h) * w.dv + c0;
        // the lane's place by itself is a register less; with dots, where scalar registers
        // are short, added to the rest
        int lane_to = c - c0 + n * row_step;
        if constexpr (DOTS) to += lane_to, lane_to = 0;
        const T* pe = nullptr;
        if constexpr (DOTS) pe = side(w.e, first) + c + n * way * w.e.step;

        double total = 0.0;
        for (int base = start; base < live; base += CH) {
            if constexpr (DOTS) {
                // tokens in front of the chunk, or up to its end in reverse
                const int before = w.reverse ? len + skip - base : base;
                if (before % kMark == 0 && before > 0 && before < len && column < w.dv) {
                    const int64_t mark = (int64_t)bh * walk_marks(w.steps) + before / kMark - 1;
                    float* p = w.marks + (mark * w.dv + column) * DK + 8 * g;
#pragma unroll
                    for (int x = 0; x < PAIRS; ++x)
#pragma unroll
                        for (int y = 0; y < 2; ++y)
                            *reinterpret_cast<f4*>(p + 32 * x + 4 * y) = state[x][y];
                }
            }
            __syncthreads();  // the last chunk's tiles are read
            if (DOTS && base > start) put_dots(base - CH);
            fk.store(s.k);
            fv.store(s.v);
            if constexpr (OUT) fq.store(s.q);
            if (wave == 0) {
                const double sum = running_sum(decay), last = lane_value(sum, CH - 1);
                if (lane < CH) {
                    const float high = high_part(sum);
                    s.c[lane] = float2{high, (float)(sum - high)};
                    s.in[lane] = exp2_fast((float)sum) * w.outer;
                    s.left[lane] = exp2_fast((float)(last - sum)) * w.inner;
                }
                // a cleared state stays so, however much the piece's other decays grow
                total += __any(clears(decay)) ? -1e30 : last;
                if (lane == 0) s.whole = exp2_fast((float)last);
            }
            __syncthreads();
            if (base + CH < live) fetch(base + CH);

            const Frag<TERMS> v = s.v.down(0, wave * 16 + 4 * (lane % 4), lane);

            if constexpr (OUT) {
                scores(s, w.inner * w.outer, wave, lane);
                f4 o[2]{};
#pragma unroll
                for (int p = 0; p < PAIRS; ++p) {
                    const f4 lo = state[p][0], hi = state[p][1];
                    const float r[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    Frag<TP> f;
                    f.from(r);
#pragma unroll
                    for (int row = 0; row < 2; ++row)
                        mma(o[row], f, s.q.along(16 * row + n, 32 * p + 8 * g));
                }
#pragma unroll
                for (int row = 0; row < 2; ++row) o[row] *= s.in[16 * row + n];
                // 0 times a finite v adds up to 0
                const f4 zero =
                    __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.t[0], bf8{}, f4{}, 0, 0, 0);
                const bool fine =
                    __all(zero[0] == 0.0f && zero[1] == 0.0f && zero[2] == 0.0f && zero[3] == 0.0f);
                __syncthreads();  // the scores are written
                if (fine) {
#pragma unroll
                    for (int row = 0; row < 2; ++row)
                        mma(o[row], v, s.p.along(16 * row + n, 8 * g));
                } else {
                    careful(s, o, v, wave, lane);
                }
#pragma unroll
                for (int row = 0; row < 2; ++row) {
                    float dot = 0.0f;
                    const int here = lane_to + 16 * row * row_step;
                    const int place = base + 16 * row + n;
                    if (place >= skip && place < live && count > 0) {
                        if constexpr (DOTS) {
                            Pack<T, 4> e;
                            e.load(pe + 16 * row * way * w.e.step, count);
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                if (y < count) dot = __builtin_fmaf(o[row][y], to_f32(e.v[y]), dot);
                            const float own = s.own[16 * row + n];
                            const f4 x = s.v.four(16 * row + n, wave * 16 + 4 * g);
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                o[row][y] = __builtin_fmaf(own, x[y], o[row][y]);
                        }
                        if (w.wide) {
                            Pack<float, 4> r;
#pragma unroll
                            for (int y = 0; y < 4; ++y) r.v[y] = o[row][y];
                            r.store((float*)w.out + to + here, count);
                        } else {
                            Pack<T, 4> r;
#pragma unroll
                            for (int y = 0; y < 4; ++y) r.v[y] = from_f32<T>(o[row][y]);
                            r.store((T*)w.out + to + here, count);
                        }
                    }
                    if constexpr (DOTS) {
                        dot += __shfl_xor(dot, 16);
                        dot += __shfl_xor(dot, 32);
                        if (g == 0) s.dot(wave, 16 * row + n) = dot;
                    }
                }
                to += CH * row_step;
                if constexpr (DOTS) pe += CH * way * w.e.step;
            }

            // the state behind the chunk
            const float whole = s.whole;
#pragma unroll
            for (int p = 0; p < PAIRS; ++p) state[p][0] *= whole, state[p][1] *= whole;
            Frag<TP> vw;
            float r[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = v.value(e) * s.left[8 * g + e];
            vw.from(r);
#pragma unroll
            for (int p = 0; p < PAIRS; ++p)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    mma(state[p][y], s.k.down(0, 32 * p + 8 * (lane % 4) + 4 * y, lane), vw);
        }
        if (DOTS && live > start) {
            __syncthreads();
            put_dots(start + (live - start - 1) / CH * CH);
        }
        if (w.last.p && (!OUT || w.pieces == 1) && column < w.dv)
            store_state(state, w.last.p + number * w.dk * w.dv, w, w.last, column, g);
        if (!OUT && block == 0 && tid == 0) {
            // no product of 2^8192 leaves a state in fp32; a NaN goes into the factor
            const double down = __builtin_floor(total), most = 8192.0;
            w.whole[number] = {exp2_fast((float)(total - down)),
                               (int)__builtin_fmax(__builtin_fmin(down, most), -most)};
        }
    }
};

// Where two workgroups of eight waves fit a CU they hide each other's latencies between
// barriers; that takes no more than 128 registers, which bf16 with keys of up to 128
// channels makes do with, and fp16 with up to 64 (not with dots).
template <class K>
constexpr int kPerSimd =
    K::PAIRS * K::TERMS <= 4 && !(K::TERMS == 2 && K::WITH_DOTS) ? K::WAVES / 2 : 2;

// One walk, or two of the same sizes, one after the other in the grid.
template <class K>
__global__ void __launch_bounds__(K::THREADS, kPerSimd<K>) k_walk(Walks walks) {
    __shared__ typename K::Shared s;
    K::run(walks.w[blockIdx.y], s);
}

template <class T, int DK, int WAVES>
hipError_t launch(const Walks& walks, bool states, hipStream_t stream) {
    const Walk& w = walks.w[0];
    constexpr int COLS = 16 * WAVES, THREADS = 64 * WAVES;
    const int64_t blocks = (int64_t)w.batch * w.heads * w.pieces * ((w.dv + COLS - 1) / COLS);
    if (blocks == 0) return hipSuccess;
    const dim3 grid((uint32_t)blocks, walks.count);
    if (states)
        k_walk<Kernel<T, DK, WAVES, false, false>><<<grid, THREADS, 0, stream>>>(walks);
    else if (!w.dots)
        k_walk<Kernel<T, DK, WAVES, true, false>><<<grid, THREADS, 0, stream>>>(walks);
    else
        k_walk<Kernel<T, DK, WAVES, true, true>><<<grid, THREADS, 0, stream>>>(walks);
    return hipGetLastError();
}

}  // namespace walk

template <class T>
hipError_t launch_walk(const Walks& walks, bool states, hipStream_t stream) {
    const Walk& w = walks.w[0];
    const bool wide = walk_columns(w.dv) == 128;
    const auto by_width = [&](auto dk) {
        return wide ? walk::launch<T, dk.value, 8>(walks, states, stream)
                    : walk::launch<T, dk.value, 4>(walks, states, stream);
    };
    const int width = walk_width(w.dk);
    if (width == 256) return by_width(std::integral_constant<int, 256>());
    if (width == 128) return by_width(std::integral_constant<int, 128>());
    return by_width(std::integral_constant<int, 64>());
}

}  // namespace ls
