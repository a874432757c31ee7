// Gated linear recurrence h_t = a_t h_{t-1} + v_t over the rows of sequences, and its gradient.
//
//     dh_t = dy_t + a_{t+1} dh_{t+1} (+ dlast at the last row)      dx = dh, or (1 - a) dh with mixed inputs
//     da_t = dh_t (h_{t-1} [- x_t])     log gates: times a_t        dh0 = a_0 dh_0
#pragma once
#include <algorithm>
#include <cstdint>

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "cngp_launch.h"

namespace cngp {

constexpr int kRecurBlock = 256;
constexpr int kRowsEach = 8;             // rows of a tile per lane
constexpr int kRowsNarrow = 4;           // ... where a lane holds all channels
constexpr int kNarrowBlock = 64;         // rows of up to four channels, each whole in a lane: a wavefront by itself

constexpr int kWideBlock = 512;          // workgroups that walk whole long sequences

__device__ __forceinline__ float load(const float *p, const int64_t i) { return p[i]; }
__device__ __forceinline__ float load(const __half *p, const int64_t i) { return __half2float(p[i]); }
__device__ __forceinline__ void store(float *p, const int64_t i, const float v) { p[i] = v; }
__device__ __forceinline__ void store(__half *p, const int64_t i, const float v) { p[i] = __float2half_rn(v); }

// V neighbouring values at once, on whatever boundary they start: global memory takes that, the compiler makes one access of it.
template <typename T, int N>
struct Run { T e[N]; };
template <typename T, int V>
__device__ __forceinline__ void load_vec(float (&out)[V], const T *p) {
    Run<T, V> t;
    __builtin_memcpy(&t, p, sizeof t);
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = load(t.e, v);
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(T *p, const float (&in)[V]) {
    Run<T, V> t;
#pragma unroll
    for (int v = 0; v < V; ++v) store(t.e, v, in[v]);
    __builtin_memcpy(p, &t, sizeof t);
}

// The gate of a row and how much of the input it lets in.  1 - exp(g) cancels for small g: there it is -g times the series of
// (exp(g) - 1) / g to the ninth term (0.5^9 / 10! = 5e-10 below one), and exp(g) is one minus that, to the last bit.
template <bool LOG, bool MIX>
__device__ __forceinline__ void gate_of(const float g, float &a, float &in) {
    a = LOG ? expf(g) : g;
    in = 1.0f - a;
    if (LOG && MIX) {
        float s = fmaf(g, 1.0f / 362880.0f, 1.0f / 40320.0f);
        s = fmaf(s, g, 1.0f / 5040.0f);
        s = fmaf(s, g, 1.0f / 720.0f);
        s = fmaf(s, g, 1.0f / 120.0f);
        s = fmaf(s, g, 1.0f / 24.0f);
        s = fmaf(s, g, 1.0f / 6.0f);
        s = fmaf(s, g, 0.5f);
        s = fmaf(s, g, 1.0f);
        const bool small = fabsf(g) < 0.5f;
        in = small ? -g * s : in;
        a = small ? 1.0f - in : a;
    }
}

using pos = int32_t;                     // rows and sequences: at most kMostRows of each, so that the end of a tile behind the last is one too
constexpr int64_t kMostRows = 0x7fff0000;

struct RecurArgs {
    const void    *gate, *x;
    const int32_t *offsets;
    const float   *h0, *dlast;
    const void    *y, *dy;               // backward; y_f32: y is the workspace's fp32 copy
    void          *out_y, *dgate, *dx;
    float         *last, *dh0;
    float         *slope;                // backward of a gate that several channel tiles share: their sums, fp32 [tiles][N]
    pos            N, S, rows_each;
    int32_t        C, G;
    uint32_t       flags;
    int32_t        y_f32;
};

struct Order {
    const int32_t *offsets;
    pos        N, S, rows_each;
    bool           back;                 // taken from the last row to the first
    __device__ __forceinline__ pos at(const pos q) const {       // ps(q), 0 <= q <= S
        if (!offsets) return q * rows_each;
        pos o = offsets[back ? S - q : q];
        o = o < 0 ? 0 : o > N ? N : o;
        return back ? N - o : o;
    }
    __device__ __forceinline__ pos sequence(const pos q) const { return back ? S - 1 - q : q; }
    // First q with ps(q) >= p, for two p at once (S + 1 if there is none); a wavefront calls this together, 64 probes at a time.
    __device__ void first_from(const pos pa, const pos pb, pos &qa, pos &qb) const {
        if (!offsets) {
            qa = (pa + rows_each - 1) / rows_each;
            qb = (pb + rows_each - 1) / rows_each;
            qa = qa < S + 1 ? qa : S + 1;
            qb = qb < S + 1 ? qb : S + 1;
            return;
        }
        const pos lane = threadIdx.x & 63;
        pos lo[2] = {0, 0}, hi[2] = {S + 1, S + 1};         // the answers lie in [lo, hi]
        const pos want[2] = {pa, pb};
        while (lo[0] < hi[0] || lo[1] < hi[1]) {
            bool    less[2];
            pos step[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                step[i] = (hi[i] - lo[i] + 63) / 64;
                const pos probe = lo[i] + lane * step[i];
                less[i] = probe < hi[i] && at(probe < S ? probe : S) < want[i];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint64_t before = __ballot(less[i]);
                if (!before) { hi[i] = lo[i]; continue; }
                const pos last = lo[i] + (63 - __clzll(before)) * step[i];      // the last probe that lies before p
                lo[i] = last + 1;
                hi[i] = last + step[i] < hi[i] ? last + step[i] : hi[i];
            }
        }
        qa = lo[0];
        qb = lo[1];
    }
};

// Windows of rows: workgroup (k, channel tile) of a launch takes the sequences that start in [k R, (k + 1) R) -- or exactly those
// rows, where a long sequence is cut: then the state at k R comes from `carry`.
struct Cut {
    pos      R;
    uint32_t K;
    float   *piece_a, *piece_b, *carry;  // [K][C]
    int32_t *piece_cut;                  // [K]
    int      exact;
};

// How a call is cut.  CL lanes side by side hold V channels each: as many as there are channels, at most 32 (a row of a tile is then a
// 128-byte line of fp32).
struct RecurPlan {
    int      CL, V, block, tiles;        // channel tiles
    int64_t  R;                          // rows per window
    uint32_t K;                          // windows
    bool     exact;                      // long sequences are cut at the windows' edges
};

// Where the parts of a workspace lie.
struct RecurSpace { size_t y, slope, piece_a, piece_b, carry, piece_cut, state, bytes; };
// One direction's launches (cngp_recur_fwd.hip, cngp_recur_bwd.hip: the instances of the kernels are many, they are compiled side by side).
template <bool BWD>
int recur_launch(const cngp_recur_config *c, RecurArgs a, const RecurPlan &p, const RecurSpace &sp, char *ws, hipStream_t s);

int recur_copy(const float *from, float *to, int64_t n, hipStream_t s);      // zeros without `from`
int recur_carry(const Cut &cut, int C, hipStream_t s);                       // the state that reaches each window

}  // namespace cngp
