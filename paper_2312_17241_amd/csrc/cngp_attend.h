// Linear attention with a decay for each head: what its translation units share.
#pragma once
#include <algorithm>

#include "cngp_launch.h"

namespace cngp {

constexpr int kChunk = 64;               // rows that are worked on together: pairs inside a chunk as products, everything before through the state
constexpr int kChunkShift = 6;
constexpr int kAnchorChunks = 16;        // chunks between two places where the decays' gradient starts from states again
constexpr int kAnchorShift = 10;         // ... in rows: 2^10 = kAnchorChunks * kChunk
constexpr int kAttendDim = 128;          // most columns of a head

// One walk over the rows of sequences with a state [kdim, vdim] per head, in the order of time or against it:
//     out_t = pair_scale * sum over rows s up to t of exp(F_t - F_s) (q_t . k_s) v_s  (inside a chunk)   +   far_scale * exp(F_t) q_t . state
//     state <- exp(F_end) state + state_scale * sum over s of exp(F_end - F_s) k_s v_s
// F: sum of the log decays from the chunk's start, the row's own included (forward: the state decays before it takes a row in) or not
// (reverse: it decays after).  The forward pass is one walk; its three gradients are walks with the parts exchanged.
struct WalkArgs {
    const void  *q, *k, *v;              // [N, heads / div, kdim], same, [N, heads / div, vdim]
    void        *out;                    // [N, heads, vdim] of the storage type, or of fp32
    const float *decay;                  // [N, heads] or [heads]
    const int32_t *offsets;              // or NULL: rows_each rows
    const float *first;                  // states before the first row, or NULL: zeros
    float       *final;                  // ... behind the last one, or NULL
    float       *anchors;                // states at every kAnchorChunks-th chunk's start but a sequence's first, as they lie in registers (entries
                                         // outside kdim, vdim are anything); or NULL
    const void  *x;                      // rows [N, heads / x_div, vdim] to take products of the outputs with, or NULL
    float       *dot_near, *dot_far;     // [heads, N]: x_t . the part of out_t inside the chunk, and the rest
    float       *total;                  // [segments, heads]: log2 of a segment's decay, or NULL
    int64_t      N;
    int32_t      S, rows_each, heads, q_div, k_div, v_div, x_div, kdim, vdim;
    int32_t      seg_rows;               // 0: sequences whole; else segments have this many rows (a multiple of kChunk), counted from a sequence's start
    int32_t      piece0;                 // first of this launch
    int32_t      segments;               // whole sequences: S
    int32_t      first_i, first_j, final_i, final_j;   // strides of the states' two dimensions
    float        pair_scale, far_scale, state_scale;
    int32_t      reverse, row_decay, out_f32;
    int32_t      own;                    // the row's own part stays out of dot_near (and of the sums inside the chunk: it is added to the output)
    int32_t      whole;                  // every array's 16-byte pieces (out, x: four values) lie whole and aligned in its rows
};

// Rows [begin, end) of sequence s.
struct Span { int32_t begin, end; };
__host__ __device__ inline Span span_of(const int32_t *offsets, const int32_t s, const int64_t N, const int32_t rows_each) {
    if (!offsets) return {s * rows_each, s * rows_each + rows_each};
    const int32_t lo = offsets[s], hi = offsets[s + 1], n = (int32_t)N;
    Span p;
    p.begin = lo < 0 ? 0 : lo > n ? n : lo;
    p.end = hi < p.begin ? p.begin : hi > n ? n : hi;
    return p;
}

// Numbers of pieces of `each` rows, sequence after sequence: those of sequence s start at piece begin / each + s, which leaves room for all of them
// whatever the lengths (a sequence of n rows has at most (begin + n) / each - begin / each + 1, rounded down each).
__host__ __device__ inline int32_t piece_base(const int32_t begin, const int32_t s, const int32_t each) { return (int32_t)((uint32_t)begin / (uint32_t)each) + s; }
inline int64_t pieces(const int64_t N, const int64_t S, const int64_t each) { return N / each + S; }

// Sequence of a piece: the last whose pieces start at or before it.
__device__ inline int32_t sequence_of(const int32_t *offsets, const int32_t piece, const int64_t N, const int32_t S, const int32_t rows_each, const int32_t each) {
    int32_t lo = 0, hi = S - 1;
    while (lo < hi) {
        const int32_t mid = lo + (hi - lo + 1) / 2;
        if (piece_base(span_of(offsets, mid, N, rows_each).begin, mid, each) <= piece) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Where the state at the start of chunk `number` (a multiple of kAnchorChunks, not 0) of a sequence is kept: slots 1 .. N / (rows between two).
__host__ __device__ inline int32_t anchor_slot(const int32_t begin, const int32_t number) { return (begin >> kAnchorShift) + number / kAnchorChunks; }

// Launches a walk (states_only: no outputs).  Defined for each storage type in a translation unit of its own.
int attend_walk_f16(const WalkArgs &a, bool states_only, hipStream_t s);
int attend_walk_f32(const WalkArgs &a, bool states_only, hipStream_t s);

__host__ __device__ inline int tiles_of(int dim) { return dim <= 32 ? 1 : dim <= 64 ? 2 : 4; }
inline size_t anchor_floats(int kdim, int vdim) { return (size_t)tiles_of(kdim) * tiles_of(vdim) * 1024; }

// Row and column of the state that entry e of an anchor is: 32 columns of v after each other, in each the tiles of 32 rows, 16 registers of 64 lanes.
__device__ inline int anchor_row(const int e, const int kdim) {
    const int r = e >> 6 & 15, kt = (e >> 10) % tiles_of(kdim);
    return 32 * kt + 8 * (r >> 2) + 4 * (e >> 5 & 1) + (r & 3);
}
__device__ inline int anchor_column(const int e, const int kdim) { return 32 * ((e >> 10) / tiles_of(kdim)) + (e & 31); }

}  // namespace cngp
