// Linear attention with a decay for each head: what its translation units share.
#pragma once
#include <algorithm>

#include "cngp_launch.h"

namespace cngp {

constexpr int kChunk = 64;               // rows that are worked on together: pairs inside a chunk as products, everything before through the state
constexpr int kChunkShift = 6;
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
    float       *anchors;                // states at the chunks' starts but a sequence's first, as they lie in registers: a forward walk leaves them there, a
                                         // reverse one takes products of its states with them; or NULL
    const float *met;                    // (with anchors, first_i 1) states as `first` of whole sequences, for the product behind a sequence's last row of the walk; or NULL
    double      *products;               // (with anchors) <state, anchor>, a part from each wavefront: reverse [chunk_number, heads, waves], forward (met alone) [S, heads, waves]
    const void  *x;                      // rows [N, heads / x_div, vdim] to take products of the outputs with, or NULL
    float       *dot;                    // [heads, N]: x_t . out_t, the row's own part left out
    float       *total;                  // [segments, heads]: log2 of a segment's decay, or NULL
    int64_t      N;
    int32_t      S, rows_each, heads, q_div, k_div, v_div, x_div, kdim, vdim;
    int32_t      seg_rows;               // 0: sequences whole; else segments have this many rows (a multiple of kChunk), counted from a sequence's start
    int32_t      piece0;                 // first of this launch
    int32_t      segments;               // whole sequences: S
    int32_t      first_i, first_j, final_i, final_j;   // strides of the states' two dimensions
    float        pair_scale, far_scale, state_scale;
    int32_t      reverse, row_decay, out_f32;
    int32_t      own;                    // the row's own part stays out of the sums inside the chunk (it is added to the output); anchors and x want that
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

// ... of kChunk rows: 64 bits, for their number may be that of 2^31 sequences and more.
__host__ __device__ inline int64_t chunk_number(const int32_t begin, const int32_t s, const int32_t number) { return (int64_t)(begin >> kChunkShift) + s + number; }

// Sequence of a piece: the last whose pieces start at or before it.
__device__ inline int32_t sequence_of(const int32_t *offsets, const int64_t piece, const int64_t N, const int32_t S, const int32_t rows_each, const int32_t each) {
    int32_t lo = 0, hi = S - 1;
    while (lo < hi) {
        const int32_t mid = lo + (hi - lo + 1) / 2;
        if ((int64_t)((uint32_t)span_of(offsets, mid, N, rows_each).begin / (uint32_t)each) + mid <= piece) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Where the state at the start of chunk `number` (not 0) of a sequence is kept: slots 1 .. N / kChunk.
__host__ __device__ inline int32_t anchor_slot(const int32_t begin, const int32_t number) { return (begin >> kChunkShift) + number; }

// Launches a walk (states_only: no outputs).  Defined for each storage type in a translation unit of its own.
int attend_walk_f16(const WalkArgs &a, bool states_only, hipStream_t s);
int attend_walk_f32(const WalkArgs &a, bool states_only, hipStream_t s);

constexpr int tiles_of(int dim) { return dim <= 32 ? 1 : dim <= 64 ? 2 : 4; }
// Values of an anchor: for each 32 columns of v and 32 rows four pieces of 64 lanes' four registers.
inline size_t anchor_floats(int kdim, int vdim) { return (size_t)tiles_of(kdim) * tiles_of(vdim) * 1024; }
// Wavefronts of a workgroup: one for each 32 columns of v, by two where k has more than 32 (each keeps one half of the state's rows, and takes one half
// of the chunk's rows for the outputs).
constexpr int walk_waves(int kdim, int vdim) { return tiles_of(vdim) * (kdim > 32 ? 2 : 1); }

}  // namespace cngp
