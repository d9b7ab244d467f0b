// attend.hpp -- linear attention as one operator used four times.
//
// With D[i,j] = e^(g[j+1] + .. + g[i]) for j <= i, the output is
//   o[i] = sum over j <= i of D[i,j] (q[i] . k[j]) v[j],
// which a state S[i] = e^g[i] S[i-1] + k[i] v[i]^T carries: o[i] = q[i] S[i].
// Its gradients are the same sum with the operands in other places: dq = (do,
// v, k); and backwards in time, where step j decays by the next token's g,
// dk = (v, do, q) and dv = (k, q, do).  A Walk is one of them.
#pragma once

#include "../../include/libscan.h"
#include "lm.hpp"

namespace ls {

// An operand of batch x steps x some heads x width: head h of the walk reads
// head h / share of it.
struct WalkSide {
    const void* p;
    int64_t batch, step, head;
    int share;
};

// States, dk x dv each: element (r, c) of number i at p[i * dk * dv + r * row + c * col].
struct WalkState {
    float* p;
    int64_t row, col;
};

// The product of a piece's decays, factor * 2^exponent with a factor of 1 to 2: over
// hundreds of tokens it may be beyond fp32 both ways.
struct WholePiece {
    float factor;
    int exponent;
};

// Tokens of a chunk: as many as one matrix instruction sums over.  64 make the states'
// part of the work half as large, but leave room for one workgroup on a CU, not two (4 x
// 2048 x 16 x 128 x 128, bf16, with scores and states in two terms: 50 us a walk against 45).
constexpr int kChunk = 32;

// A walk with dots leaves its states at the tokens whose numbers are multiples of kMark, S
// before and G at each, for the decays' gradients: their sums then run over kMark tokens.
// 512: 128 KB for S and G of 128 x 128, beside 900 KB of a head's operands and gradients
// (4 x 2048 x 16 x 128, bf16: 1 us of the walks' 118 against marks every 4096).
constexpr int kMark = 512;
__host__ __device__ constexpr int walk_marks(int steps) { return steps > 0 ? (steps - 1) / kMark : 0; }

struct Walk {
    int batch, steps, heads, dk, dv;
    bool reverse;
    WalkSide q, k, v;  // q and k of width dk, v of dv
    const float* g;    // log decays, [batch, step, head]
    int64_t g_batch, g_step;
    float inner, outer;  // factors of k v^T, and of the output
    const int32_t* lengths;
    // Every row's places are cut into `pieces` of `piece` (a multiple of kChunk), a workgroup
    // to each (and to a block of columns of v).
    int pieces, piece;
    // The states that the rows (pieces == 1: one for each row and head) or their pieces
    // (one for each row, head and piece) begin with, nullable; and the last ones: the
    // row's, if pieces == 1, or in a run for the states alone what each piece adds.
    WalkState first, last;
    WholePiece* whole;  // in such a run, for each row, head and piece: the product of its decays
    // Output: batch x steps x heads x dv, dense; fp32 where `wide`.  With `dots`
    // (batch x steps x heads for each block of columns), the sums of the output
    // times e, before it is rounded and without the part that is the token's own.
    void* out;
    bool wide;
    WalkSide e;
    float* dots;
    float* marks;  // with dots: walk_marks(steps) of each row and head, dv x walk_width(dk) each
};

// A logarithm past -1024 to base 2 is one of 0: what decays by it is gone.
__device__ __forceinline__ bool clears(float g) { return g < -709.79f; }

__device__ __forceinline__ int walk_len(const Walk& w, int b) {
    if (!w.lengths) return w.steps;
    const int n = w.lengths[b];
    return n < 0 ? 0 : n < w.steps ? n : w.steps;
}

// In reverse a row's first places may have no tokens, so that chunks lie at the same
// tokens both ways.
__device__ __forceinline__ int walk_skip(const Walk& w, int len) {
    return w.reverse ? (kChunk - len % kChunk) % kChunk : 0;
}
// The token at a place of the walk, and that place's decay.
__device__ __forceinline__ int walk_token(const Walk& w, int place, int len) {
    return w.reverse ? len + walk_skip(w, len) - 1 - place : place;
}
__device__ __forceinline__ float walk_decay(const Walk& w, int b, int h, int place, int len) {
    const int t = walk_token(w, place, len) + w.reverse;
    return t >= len ? 0.0f : w.g[b * w.g_batch + t * w.g_step + h];
}

// The width that q and k have in a workgroup, filled up by zeros, and the columns of v.
inline int walk_width(int dk) { return dk > 128 ? 256 : dk > 64 ? 128 : 64; }
inline int walk_columns(int dv) { return dv > 64 ? 128 : 64; }
inline int walk_blocks(int dv) {
    const int columns = walk_columns(dv);
    return (dv + columns - 1) / columns;
}

// Walks of one launch: of the same sizes, and both with dots or without.
struct Walks {
    Walk w[2];
    int count;
};

// One instance for each element type (attend_f32.hip and so on).  `states`: what each
// piece adds to the state and no outputs.
template <class T>
hipError_t launch_walk(const Walks& walks, bool states, hipStream_t stream);
extern template hipError_t launch_walk<float>(const Walks&, bool, hipStream_t);
extern template hipError_t launch_walk<_Float16>(const Walks&, bool, hipStream_t);
extern template hipError_t launch_walk<__bf16>(const Walks&, bool, hipStream_t);

}  // namespace ls
