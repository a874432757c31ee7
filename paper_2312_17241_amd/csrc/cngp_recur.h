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

// A state in 32 bits as its rounding to fp16, which the caller keeps, and sixteen bits beside it: the lower half of |h| + 2^-15 in fp32.
// Values with that lower half lie 2^16 steps of fp32 apart and the fp16 value is at most 2^12 steps away (below 2^-14, where steps of fp16
// are 2^-24: of the 2^-38 that the sum's are), so the nearest one is meant, also where the fp16 value is a step off.  h comes back with two
// roundings of fp32, or to 2^-39.  Where fp16 has infinity or no number, the sixteen bits are the upper half of h.
struct LowHalf { uint16_t bits; };
constexpr float kLowOffset = 0x1p-15f, kHalfOverflow = 65520.0f;      // what rounds to infinity in fp16
__host__ __device__ __forceinline__ uint16_t low_half(const float h) {
    const float m = fabsf(h);
    return m < kHalfOverflow ? (uint16_t)__builtin_bit_cast(uint32_t, m + kLowOffset) : (uint16_t)(__builtin_bit_cast(uint32_t, h) >> 16);
}
__host__ __device__ __forceinline__ float with_low_half(const float rounded, const uint16_t low) {
    const float    m = fabsf(rounded);
    const uint32_t near = __builtin_bit_cast(uint32_t, m + kLowOffset), z = near + (uint32_t)(int32_t)(int16_t)(uint16_t)(low - (uint16_t)near);
    return m < kHalfOverflow ? copysignf(__builtin_bit_cast(float, z) - kLowOffset, rounded) : __builtin_bit_cast(float, (uint32_t)low << 16);
}
__device__ __forceinline__ void store(LowHalf *p, const int64_t i, const float v) { p[i].bits = low_half(v); }

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
    const void    *y, *dy;               // backward; states: where those before the rows come from
    void          *out_y, *dgate, *dx;
    float         *last, *dh0;
    float         *slope;                // backward of a gate that several channel tiles share: their sums, fp32 [tiles][N]
    pos            N, S, rows_each;
    int32_t        C, G;
    uint32_t       flags;
    int32_t        states;               // STATES_*
};

// Where the backward pass has the states from, and what a forward launch writes as states: the caller's array y, in its type; the workspace,
// in fp32; y in fp16 and the low halves in dx, until the gradients take their place.
enum { STATES_Y = 0, STATES_F32, STATES_LOW };

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
    // Sequences of equal length: first q with ps(q) >= p (S + 1 if there is none) and its ps(q) (ps(S) then), 0 <= p <= N.
    __host__ __device__ void equal_from(const pos p, pos &q, pos &v) const {
        q = p / rows_each + (p % rows_each != 0);             // no sum: p + rows_each may pass 2^31
        q = q < S + 1 ? q : S + 1;
        v = (q < S ? q : S) * rows_each;
    }
    // The same for any sequences and two p at once; a wavefront calls this together, 64 probes at
    // a time.  The first ones lie around where sequences of equal length would have it: with lengths drawn at random that leaves a few
    // entries, and fewer dependent loads than from the ends (16.7 M rows of three channels in sequences of about 1023: 129 us and 121 so).
    __device__ void first_from(const pos pa, const pos pb, pos &qa, pos &qb, pos &va, pos &vb) const {
        if (!offsets) {
            equal_from(pa, qa, va);
            equal_from(pb, qb, vb);
            return;
        }
        const pos lane = threadIdx.x & 63, want[2] = {pa, pb}, end = at(S);
        pos       lo[2] = {0, 0}, hi[2] = {S + 1, S + 1}, val[2] = {end, end};         // the answers lie in [lo, hi], val = ps(hi)
        const int spread = min(1 + (int)(sqrtf((float)S) * 0.0625f), 1024);
        bool      guess = true;
        while (lo[0] < hi[0] || lo[1] < hi[1]) {
            pos probe[2], here[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const pos step = (hi[i] - lo[i] + 63) / 64;
                probe[i] = lo[i] + lane * step;
                if (guess) {
                    const pos middle = (pos)fminf((float)want[i] * ((float)S / (float)N), (float)(S > 128 ? S - 128 : 0));
                    probe[i] = max((pos)(middle + (lane - 32) * spread), (pos)0);
                }
                probe[i] = min(probe[i], hi[i] - 1);           // a range that is done: read, not used
                here[i] = at(min(max(probe[i], (pos)0), S));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (lo[i] >= hi[i]) continue;
                const uint64_t before = __ballot(here[i] < want[i]);
                const int      n = before ? 64 - __clzll(before) : 0;      // probes up to the last that lies before p
                if (n < 64) {                                  // the next one does not
                    hi[i] = __builtin_amdgcn_readlane(probe[i], n);
                    val[i] = __builtin_amdgcn_readlane(here[i], n);
                }
                if (n > 0) lo[i] = __builtin_amdgcn_readlane(probe[i], n - 1) + 1;
            }
            guess = false;
        }
        qa = hi[0];
        qb = hi[1];
        va = val[0];
        vb = val[1];
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
