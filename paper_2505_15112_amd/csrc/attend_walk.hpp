// attend_walk.hpp -- the walk of linear attention (attend.hpp) on the matrix cores.
//
// A workgroup takes a row's head in chunks of CH tokens.  With c the running sum of
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
// the other where i + j < LIM.  bfloat16's exponents are fp32's, so neither scores nor
// states overflow or lose their small values, as they would in fp16.
#pragma once

#include <type_traits>

#include "attend.hpp"

namespace ls {
namespace walk {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
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
        float v = 0.0f;
#pragma unroll
        for (int i = TERMS - 1; i >= 0; --i) v += (float)t[i][e];
        return v;
    }
};

// c += a b.  Lane l has row (a) or column (b) l % 16 at the eight places from 8 (l /
// 16) of the 32 summed over, and of the result column l % 16, rows from 4 (l / 16).
template <int LIM, int NA, int NB>
__device__ __forceinline__ void mma(f4& c, const Frag<NA>& a, const Frag<NB>& b) {
#pragma unroll
    for (int s = LIM - 1; s >= 0; --s)  // small parts first
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (i + j == s)
                    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.t[i], b.t[j], c, 0, 0, 0);
}

// A tile of ROWS x WIDTH elements in LDS, by terms.
template <int TERMS, int ROWS, int WIDTH>
struct Tile {
    static constexpr int ROW = WIDTH + 8;  // rows of 16 lanes fall on different banks
    __bf16 v[TERMS][ROWS][ROW];

    // Eight elements along a row.
    __device__ __forceinline__ Frag<TERMS> along(int row, int col) const {
        Frag<TERMS> f;
#pragma unroll
        for (int t = 0; t < TERMS; ++t)
            f.t[t] = *reinterpret_cast<const bf8*>(&v[t][row][col]);
        return f;
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

// A tile on its way from global memory: vectors of 16 bytes in registers.
template <class T, int ROWS, int WIDTH, int THREADS>
struct Fetch {
    static constexpr int V = 16 / sizeof(T), PER_ROW = WIDTH / V, ALL = ROWS * PER_ROW;
    static constexpr int N = (ALL + THREADS - 1) / THREADS;
    Pack<T, V> r[N];

    // Rows at places `base` and on, those below `live`, of which `width` elements exist.
    __device__ __forceinline__ void load(const Walk& w, const T* p, int64_t step, int width,
                                         int base, int live, int len) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = threadIdx.x + i * THREADS, col = at % PER_ROW * V;
            if (ALL % THREADS != 0 && at >= ALL) break;
            const int place = base + at / PER_ROW;
            const int count = place < live ? width - col : 0;
            r[i].load(p + walk_token(w, place < live ? place : base, len) * step +
                          (col < width ? col : 0),
                      count);
        }
    }
    __device__ __forceinline__ void store(Tile<kTerms<T>, ROWS, WIDTH>& s) const {
        constexpr int TERMS = kTerms<T>;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = threadIdx.x + i * THREADS, col = at % PER_ROW * V, row = at / PER_ROW;
            if (ALL % THREADS != 0 && at >= ALL) break;
            if constexpr (TERMS == 1) {
                *reinterpret_cast<u4*>(&s.v[0][row][col]) = __builtin_bit_cast(u4, r[i].v);
            } else {
                float f[V];
                unsigned u[TERMS][V / 2];
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = to_f32(r[i].v[e]);
                split<TERMS, V>(f, u);
#pragma unroll
                for (int t = 0; t < TERMS; ++t) {
                    if constexpr (V == 8)
                        *reinterpret_cast<u4*>(&s.v[t][row][col]) =
                            u4{u[t][0], u[t][1], u[t][2], u[t][3]};
                    else
                        *reinterpret_cast<u2*>(&s.v[t][row][col]) = u2{u[t][0], u[t][1]};
                }
            }
        }
    }
};

// Running sums of the chunk's decays over the lanes of a wave, in powers of two.  A
// decay past +-1024 is one of 0 or infinity either way; infinities would turn the
// differences of sums to NaN.
__device__ __forceinline__ double running_sum(float g, int lane) {
    double c = (double)g * 1.4426950408889634;
    c = c < -1024.0 ? -1024.0 : c > 1024.0 ? 1024.0 : c;  // a NaN stays
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const double up = __shfl_up(c, m);
        if (lane >= m) c += up;
    }
    return c;
}

// TP terms of scores and states, LIM for the products that make outputs, DK the
// width of q and k rounded up, WAVES of 16 columns of v each, CH tokens to a chunk.
// OUT: with outputs; else the pieces' states alone.
template <class T, int TP, int LIM, int DK, int WAVES, int CH, bool OUT>
struct Kernel {
    static constexpr int TERMS = kTerms<T>, COLS = 16 * WAVES, THREADS = 64 * WAVES;
    static constexpr int STEPS = CH / 32, TILES = CH / 16, PAIRS = DK / 32;
    static constexpr int DIAGONALS = TILES * (TILES + 1) / 2;
    struct Shared {
        Tile<TERMS, CH, DK> k;
        Tile<TERMS, CH, COLS> v;
        Tile<TERMS, OUT ? CH : 1, DK> q;
        Tile<TP, OUT ? CH : 1, CH> p;
        double c[CH];
        float in[CH], left[CH];  // e^c outer; e^(c[last] - c) inner
        float whole;
        float dots[WAVES][CH];
    };

    // Scores of the tiles on and below the diagonal, shared out over the waves: lane l
    // gets those of token l % 16 with four others, next to each other in a row.
    static __device__ __forceinline__ void scores(Shared& s, float factor, int wave, int lane) {
        const int g = lane / 16, n = lane % 16;
#pragma unroll
        for (int x = 0; x < (DIAGONALS + WAVES - 1) / WAVES; ++x) {
            const int at = x * WAVES + wave;
            if (at >= DIAGONALS) break;
            // the tile's place in the lower triangle
            const int row = at < 1 ? 0 : at < 3 ? 1 : at < 6 ? 2 : 3, col = at - row * (row + 1) / 2;
            f4 acc{};
#pragma unroll
            for (int p = 0; p < PAIRS; ++p)
                mma<LIM>(acc, s.k.along(16 * col + n, 32 * p + 8 * g),
                         s.q.along(16 * row + n, 32 * p + 8 * g));
            const int i = 16 * row + n, j = 16 * col + 4 * g;
            const double ci = s.c[i];
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float d = exp2_fast((float)(ci - s.c[j + e])) * factor;
                v[e] = j + e <= i ? acc[e] * d : 0.0f;
            }
            unsigned u[TP][2];
            split<TP, 4>(v, u);
#pragma unroll
            for (int t = 0; t < TP; ++t)
                *reinterpret_cast<u2*>(&s.p.v[t][i][j]) = u2{u[t][0], u[t][1]};
        }
    }

    // o += the scores times v where v has an infinity or a NaN: such an element
    // counts for its own token and later ones alone (0 times it is not 0).
    static __device__ __forceinline__ void careful(const Shared& s, f4 (&o)[TILES],
                                                   const Frag<TERMS> (&v)[STEPS], int wave,
                                                   int lane) {
        const int g = lane / 16, n = lane % 16;
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
            Frag<TERMS> clean;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool fine = __builtin_isfinite(v[step].value(e));
#pragma unroll
                for (int t = 0; t < TERMS; ++t)
                    clean.t[t][e] = fine ? v[step].t[t][e] : (__bf16)0.0f;
            }
#pragma unroll
            for (int row = 0; row < TILES; ++row)
                if (32 * step <= 16 * row)
                    mma<LIM>(o[row], clean, s.p.along(16 * row + n, 32 * step + 8 * g));
        }
#pragma unroll
        for (int row = 0; row < TILES; ++row)
            for (int j = 0; j <= 16 * row + n; ++j) {
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

    static __device__ __forceinline__ void run(const Walk& w, Shared& s) {
        const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, g = lane / 16, n = lane % 16;
        const int blocks = (w.dv + COLS - 1) / COLS;
        int at = blockIdx.x;
        const int block = at % blocks;
        at /= blocks;
        const int h = at % w.heads;
        at /= w.heads;
        const int piece = at % w.pieces, b = at / w.pieces, bh = b * w.heads + h;
        const int len = walk_len(w, b), c0 = block * COLS;
        const int start = piece * w.piece;
        const int end = start + w.piece < w.steps ? start + w.piece : w.steps;
        const int live = len < end ? len : end;  // places of this piece that have tokens
        const int64_t number = (int64_t)bh * w.pieces + piece;

        const auto side = [&](const WalkSide& x) {
            return (const T*)x.p + b * x.batch + (h / x.share) * x.head;
        };
        const T *pq = side(w.q), *pk = side(w.k), *pv = side(w.v) + c0;

        if constexpr (OUT) {
            // places without a token, and the scores' tiles above the diagonal
            const int cols = w.dv - c0 < COLS ? w.dv - c0 : COLS;
            for (int i = (live > start ? live : start) + wave; i < end; i += WAVES) {
                const int64_t o = (((int64_t)b * w.steps + i) * w.heads + h) * w.dv + c0;
                for (int c = lane; c < cols; c += 64) {
                    if (w.wide)
                        ((float*)w.out)[o + c] = 0.0f;
                    else
                        ((T*)w.out)[o + c] = T(0);
                }
            }
            for (int i = tid; i < TP * CH * (CH + 8); i += THREADS)
                (&s.p.v[0][0][0])[i] = (__bf16)0.0f;
        }

        // The state: column c0 + 16 wave + n, rows 32 p + 8 g + 4 y + e.
        f4 state[PAIRS][2];
        const auto each = [&](auto f) {
            const int c = c0 + wave * 16 + n;
            if (c >= w.dv) return;
#pragma unroll
            for (int p = 0; p < PAIRS; ++p)
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int r = 32 * p + 8 * g + 4 * y + e;
                        if (r < w.dk) f(r, c, p, y, e);
                    }
        };
#pragma unroll
        for (int p = 0; p < PAIRS; ++p) state[p][0] = state[p][1] = f4{};
        if (OUT && w.first.p) {
            const float* from = w.first.p + number * w.dk * w.dv;
            each([&](int r, int c, int p, int y, int e) {
                state[p][y][e] = from[r * w.first.row + c * w.first.col];
            });
        }

        Fetch<T, CH, DK, THREADS> fq, fk;
        Fetch<T, CH, COLS, THREADS> fv;
        float decay;
        const auto fetch = [&](int base) {
            fk.load(w, pk, w.k.step, w.dk, base, live, len);
            fv.load(w, pv, w.v.step, w.dv - c0, base, live, len);
            if constexpr (OUT) fq.load(w, pq, w.q.step, w.dk, base, live, len);
            if (wave == 0)
                decay = lane < CH && base + lane < live ? walk_decay(w, b, h, base + lane, len) : 0.0f;
        };
        const auto put_dots = [&](int base) {
            if (tid >= CH || base + tid >= live) return;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) sum += s.dots[i][tid];
            const int t = walk_token(w, base + tid, len);
            w.dots[(((int64_t)block * w.batch + b) * w.steps + t) * w.heads + h] = sum;
        };

        double total = 0.0;
        if (start < live) fetch(start);
        for (int base = start; base < live; base += CH) {
            __syncthreads();  // the last chunk's tiles are read
            if (OUT && w.dots && base > start) put_dots(base - CH);
            fk.store(s.k);
            fv.store(s.v);
            if constexpr (OUT) fq.store(s.q);
            if (wave == 0) {
                const double c = running_sum(decay, lane), last = __shfl(c, CH - 1);
                if (lane < CH) {
                    s.c[lane] = c;
                    s.in[lane] = exp2_fast((float)c) * w.outer;
                    s.left[lane] = exp2_fast((float)(last - c)) * w.inner;
                }
                total += last;
                if (lane == 0) s.whole = exp2_fast((float)last);
            }
            __syncthreads();
            if (base + CH < live) fetch(base + CH);

            Frag<TERMS> v[STEPS];
#pragma unroll
            for (int step = 0; step < STEPS; ++step)
                v[step] = s.v.down(32 * step, wave * 16 + 4 * (lane % 4), lane);

            if constexpr (OUT) {
                scores(s, w.inner * w.outer, wave, lane);
                f4 o[TILES];
#pragma unroll
                for (int row = 0; row < TILES; ++row) o[row] = f4{};
#pragma unroll
                for (int p = 0; p < PAIRS; ++p) {
                    const f4 lo = state[p][0], hi = state[p][1];
                    const float r[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    Frag<TP> f;
                    f.from(r);
#pragma unroll
                    for (int row = 0; row < TILES; ++row)
                        mma<LIM>(o[row], f, s.q.along(16 * row + n, 32 * p + 8 * g));
                }
#pragma unroll
                for (int row = 0; row < TILES; ++row) o[row] *= s.in[16 * row + n];
                // 0 times a finite v adds up to 0
                f4 zero{};
#pragma unroll
                for (int step = 0; step < STEPS; ++step)
                    zero = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[step].t[0], bf8{}, zero, 0, 0, 0);
                const bool fine =
                    __all(zero[0] == 0.0f && zero[1] == 0.0f && zero[2] == 0.0f && zero[3] == 0.0f);
                __syncthreads();  // the scores are written
                if (fine) {
#pragma unroll
                    for (int row = 0; row < TILES; ++row)
#pragma unroll
                        for (int step = 0; step < STEPS; ++step)
                            if (32 * step <= 16 * row)
                                mma<LIM>(o[row], v[step],
                                         s.p.along(16 * row + n, 32 * step + 8 * g));
                } else {
                    careful(s, o, v, wave, lane);
                }
#pragma unroll
                for (int row = 0; row < TILES; ++row) {
                    const int place = base + 16 * row + n, c = c0 + wave * 16 + 4 * g;
                    float dot = 0.0f;
                    if (place < live && c < w.dv) {
                        const int t = walk_token(w, place, len), count = w.dv - c;
                        const int64_t to = (((int64_t)b * w.steps + t) * w.heads + h) * w.dv + c;
                        if (w.dots) {
                            Pack<T, 4> e;
                            e.load(side(w.e) + t * w.e.step + c, count);
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                if (y < count) dot = __builtin_fmaf(o[row][y], to_f32(e.v[y]), dot);
                        }
                        if (w.wide) {
                            Pack<float, 4> r;
#pragma unroll
                            for (int y = 0; y < 4; ++y) r.v[y] = o[row][y];
                            r.store((float*)w.out + to, count);
                        } else {
                            Pack<T, 4> r;
#pragma unroll
                            for (int y = 0; y < 4; ++y) r.v[y] = from_f32<T>(o[row][y]);
                            r.store((T*)w.out + to, count);
                        }
                    }
                    if (w.dots) {
                        dot += __shfl_xor(dot, 16);
                        dot += __shfl_xor(dot, 32);
                        if (g == 0) s.dots[wave][16 * row + n] = dot;
                    }
                }
            }

            // the state behind the chunk
            const float whole = s.whole;
            Frag<3> vw[STEPS];
#pragma unroll
            for (int step = 0; step < STEPS; ++step) {
                float r[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) r[e] = v[step].value(e) * s.left[32 * step + 8 * g + e];
                vw[step].from(r);
            }
#pragma unroll
            for (int p = 0; p < PAIRS; ++p)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    state[p][y] *= whole;
#pragma unroll
                    for (int step = 0; step < STEPS; ++step)
                        mma<3>(state[p][y],
                               s.k.down(32 * step, 32 * p + 8 * (lane % 4) + 4 * y, lane),
                               vw[step]);
                }
        }
        if (OUT && w.dots && live > start) {
            __syncthreads();
            put_dots(start + (live - start - 1) / CH * CH);
        }
        if (w.last.p && (!OUT || w.pieces == 1)) {
            float* to = w.last.p + number * w.dk * w.dv;
            each([&](int r, int c, int p, int y, int e) {
                to[r * w.last.row + c * w.last.col] = state[p][y][e];
            });
        }
        if (!OUT && block == 0 && tid == 0) w.whole[number] = exp2_fast((float)total);
    }
};

template <class T, int TP, int LIM, int DK, int WAVES, int CH, bool OUT>
__global__ void __launch_bounds__(64 * WAVES, 2) k_walk(Walk w) {
    using K = Kernel<T, TP, LIM, DK, WAVES, CH, OUT>;
    __shared__ typename K::Shared s;
    K::run(w, s);
}

template <class T, int DK, int WAVES, int CH>
hipError_t launch(const Walk& w, Grade grade, bool states, hipStream_t stream) {
    constexpr int COLS = 16 * WAVES, THREADS = 64 * WAVES, NARROW = kTerms<T> == 3 ? 3 : 2;
    const int64_t grid = (int64_t)w.batch * w.heads * w.pieces * ((w.dv + COLS - 1) / COLS);
    if (grid == 0) return hipSuccess;
    if (states)
        k_walk<T, 1, 3, DK, WAVES, CH, false><<<(uint32_t)grid, THREADS, 0, stream>>>(w);
    else if (grade == Grade::Narrow)
        k_walk<T, NARROW, NARROW, DK, WAVES, CH, true><<<(uint32_t)grid, THREADS, 0, stream>>>(w);
    else
        k_walk<T, 3, 3, DK, WAVES, CH, true><<<(uint32_t)grid, THREADS, 0, stream>>>(w);
    return hipGetLastError();
}

}  // namespace walk

template <class T>
hipError_t launch_walk(const Walk& w, Grade grade, bool states, hipStream_t stream) {
    constexpr int CH = walk::kTerms<T> == 1 ? 64 : 32;
    const bool wide = walk_columns(w.dk, w.dv) == 128;
    const auto by_width = [&](auto dk) {
        return wide ? walk::launch<T, dk.value, 8, CH>(w, grade, states, stream)
                    : walk::launch<T, dk.value, 4, CH>(w, grade, states, stream);
    };
    if (w.dk > 128) return by_width(std::integral_constant<int, 256>());
    if (w.dk > 64) return by_width(std::integral_constant<int, 128>());
    return by_width(std::integral_constant<int, 64>());
}

}  // namespace ls
