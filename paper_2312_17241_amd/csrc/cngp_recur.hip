// Gated linear recurrence h_t = a_t h_{t-1} + v_t over the rows of sequences, and its gradient.
//
//     dh_t = dy_t + a_{t+1} dh_{t+1} (+ dlast at the last row)      dx = dh, or (1 - a) dh with mixed inputs
//     da_t = dh_t (h_{t-1} [- x_t])     log gates: times a_t        dh0 = a_0 dh_0
#include <algorithm>
#include <cstdint>

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "cngp_launch.h"

namespace {

using namespace cngp;

constexpr int kRecurBlock = 256;

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct RecurArgs {
    const void    *gate, *x;
    const int32_t *offsets;
    const float   *h0, *dlast;
    const void    *y, *dy;               // backward; y_f32: y is the workspace's fp32 copy
    void          *out_y, *dgate, *dx;
    float         *last, *dh0;
    float         *slope;                // backward of a gate that several channel tiles share: their sums, fp32 [tiles][N]
    int64_t        N, S, rows_each;
    int32_t        C, G;
    uint32_t       flags;
    int32_t        y_f32;
};

__device__ __forceinline__ float load(const float *p, const int64_t i) { return p[i]; }
__device__ __forceinline__ float load(const __half *p, const int64_t i) { return __half2float(p[i]); }
__device__ __forceinline__ void store(float *p, const int64_t i, const float v) { p[i] = v; }
__device__ __forceinline__ void store(__half *p, const int64_t i, const float v) { p[i] = __float2half_rn(v); }

// The gate of a row and how much of the input it lets in.
template <bool MIX>
__device__ __forceinline__ void gate_of(const bool log_gate, const float g, float &a, float &in) {
    in = !MIX ? 1.0f : log_gate ? -expm1f(g) : 1.0f - g;
    a = log_gate ? expf(g) : g;
}

// ---------------------------------------------------------------- the scan
// A row is the map h -> a h + v, and maps compose: rows (A, B) then (a, v) give (a A, a B + v).  So a sequence need not be walked
// row after row: a workgroup takes a tile of RL * RB rows by CL * V channels, every lane composes the maps of its RB consecutive
// rows, the lanes of the same channels join theirs (shuffles inside a wavefront, LDS between the four), and with the state that
// then reaches its first row each lane walks its rows once more and writes.  The loads of a tile are all in flight at once, every
// input is read once, every output written once.
// The backward runs the same scan the other way: with u = a_{t+1} dh_{t+1} what arrives from later rows, dh = dy + u and what goes
// on is a dh = a u + a dy.
// Sequences are not handled one by one: the rows of all of them lie one behind the other, and the first row of a sequence takes
// its map from h0 (or dlast) and forgets what came before -- a flag that travels with the map, not a factor of zero, so that
// nothing that is not finite crosses over.
// Positions: p counts rows in the order they are taken, p = row or N - 1 - row; ps(q) is where the q-th sequence in that order starts.

constexpr int kFlagRows = 2048;          // rows whose first / last marks are in LDS at a time; a multiple of every tile

struct Order {
    const int32_t *offsets;
    int64_t        N, S, rows_each;
    bool           back;                 // taken from the last row to the first
    __device__ __forceinline__ int64_t at(const int64_t q) const {       // ps(q), 0 <= q <= S
        if (!offsets) return q * rows_each;
        int64_t o = offsets[back ? S - q : q];
        o = o < 0 ? 0 : o > N ? N : o;
        return back ? N - o : o;
    }
    __device__ __forceinline__ int64_t sequence(const int64_t q) const { return back ? S - 1 - q : q; }
    // First q with ps(q) >= p, for two p at once (S + 1 if there is none); a wavefront calls this together, 64 probes at a time.
    __device__ void first_from(const int64_t pa, const int64_t pb, int64_t &qa, int64_t &qb) const {
        if (!offsets) {
            qa = (pa + rows_each - 1) / rows_each;
            qb = (pb + rows_each - 1) / rows_each;
            qa = qa < S + 1 ? qa : S + 1;
            qb = qb < S + 1 ? qb : S + 1;
            return;
        }
        const int64_t lane = threadIdx.x & 63;
        int64_t lo[2] = {0, 0}, hi[2] = {S + 1, S + 1};         // the answers lie in [lo, hi]
        const int64_t want[2] = {pa, pb};
        while (lo[0] < hi[0] || lo[1] < hi[1]) {
            bool    less[2];
            int64_t step[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                step[i] = (hi[i] - lo[i] + 63) / 64;
                const int64_t probe = lo[i] + lane * step[i];
                less[i] = probe < hi[i] && at(probe < S ? probe : S) < want[i];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint64_t before = __ballot(less[i]);
                if (!before) { hi[i] = lo[i]; continue; }
                const int64_t last = lo[i] + (63 - __clzll(before)) * step[i];      // the last probe that lies before p
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
    int64_t  R;
    uint32_t K;
    float   *piece_a, *piece_b, *carry;  // [K][C]
    int32_t *piece_cut;                  // [K]
    int      exact;
};

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

// Where a tile's rows lie.  Row j of a lane is memory row low + mine + j, or low + mine - j taken backwards; `low` is the same for
// the whole workgroup, so a load is a scalar base and a 32-bit lane offset.
struct Place {
    int64_t  low;
    uint32_t mine;                       // rows
    int      dir;                        // 1 or -1
};

// RB rows of V values each, `width` values to a row of the array.  `shift`: the rows one further in the order taken.
// Not a whole tile: rows outside [p0, p1) are read as the nearest row inside.
template <typename T, int RB, int V>
__device__ __forceinline__ void load_rows(float (&out)[RB][V], const void *array, const Place &at, const int width, const int c, const bool whole,
                                          const int64_t pr, const int64_t p0, const int64_t p1)
{
    const uint32_t mine = at.mine * (uint32_t)width + (uint32_t)c;
    const T       *base = (const T *)array + at.low * width;
    if (whole) {
#pragma unroll
        for (int j = 0; j < RB; ++j) load_vec<T, V>(out[j], base + (int64_t)(at.dir * j) * width + mine);
    } else {
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            const int64_t p = pr + j < p0 ? p0 : pr + j < p1 ? pr + j : p1 - 1;
            load_vec<T, V>(out[j], base + (int64_t)mine + at.dir * (p - pr) * width);
        }
    }
}

// A lane that holds all V values of its rows (CL = 1) reads its RB rows as one run of RB * V neighbouring values, 16 bytes at a time and
// turns them round when the rows are taken backwards.
template <typename T, int RB, int V>
__device__ __forceinline__ void load_run(float (&out)[RB][V], const T *lowest, const bool back)
{
    Run<T, RB * V> raw;
    __builtin_memcpy(&raw, lowest, sizeof raw);
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float f = load(&raw.e[j * V + v], 0), b = load(&raw.e[(RB - 1 - j) * V + v], 0);
            out[j][v] = back ? b : f;
        }
}
template <typename T, int RB, int V>
__device__ __forceinline__ void store_run(T *lowest, const float (&in)[RB][V], const bool back)
{
    Run<T, RB * V> raw;
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) store(&raw.e[j * V + v], 0, back ? in[RB - 1 - j][v] : in[j][v]);
    __builtin_memcpy(lowest, &raw, sizeof raw);
}

// As load_rows for such a lane: its run if that lies inside the array, else row by row.  Rows outside [p0, p1) hold anything.
template <typename T, int RB, int V>
__device__ __forceinline__ void load_narrow(float (&out)[RB][V], const void *array, const Place &at, const bool whole, const int64_t N,
                                            const int64_t pr, const int64_t p0, const int64_t p1)
{
    const int64_t lowest = at.low + (int64_t)at.mine - (at.dir < 0 ? RB - 1 : 0);
    if (whole || (lowest >= 0 && lowest + RB <= N)) {
        load_run<T, RB, V>(out, (const T *)array + lowest * V, at.dir < 0);
    } else {
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            const int64_t p = pr + j < p0 ? p0 : pr + j < p1 ? pr + j : p1 - 1;
            load_vec<T, V>(out[j], (const T *)array + (at.low + (int64_t)at.mine + at.dir * (p - pr)) * V);
        }
    }
}

// PIECE: only the composed map of the rows that the next window continues, for `carry`; else the outputs.
// CL lanes side by side hold V channels each of a row, RB rows each.
template <typename Io, typename Gate, int BLOCK, int CL, int V, int RB, bool SHARED, bool MIX, bool BWD, bool PIECE>
__global__ __launch_bounds__(BLOCK) void recur_scan_kernel(const RecurArgs a, const Cut cut)
{
    constexpr int RL = BLOCK / CL, TR = RL * RB, W = BLOCK / 64, GV = SHARED ? 1 : V;
    constexpr bool NARROW = CL == 1;                           // a lane holds all channels
    static_assert(kFlagRows % TR == 0 && 32 % RB == 0, "a tile's marks lie in one block of them, a lane's in one word");
    __shared__ uint32_t bits_first[PIECE ? 1 : kFlagRows / 32], bits_last[PIECE ? 1 : kFlagRows / 32];
    __shared__ int32_t  mark_first[PIECE ? 1 : kFlagRows], mark_last[PIECE ? 1 : kFlagRows];     // sequence (in order taken), where the bit is set
    __shared__ float    tot_a[2][W][CL * GV], tot_b[2][W][CL * V];
    __shared__ int      tot_cut[2][W];
    __shared__ int      q_next;
    const int      t = threadIdx.x, lane = t & 63, w = t >> 6, cl = t % CL, rl = t / CL;
    const uint32_t k = blockIdx.x % cut.K, tile_c = blockIdx.x / cut.K;
    const int      c_here = (int)tile_c * (CL * V) + cl * V;
    const bool     c_ok = c_here < a.C;                        // V divides C
    const int      c = c_ok ? c_here : a.C - V;                // lanes without a channel read the last ones and write nothing
    const int      gc = SHARED ? 0 : c, gw = SHARED ? 1 : a.C;
    const bool     log_gate = a.flags & CNGP_RECUR_LOG_GATE;
    const Order    o{a.offsets, a.N, a.S, a.rows_each, ((a.flags & CNGP_RECUR_REVERSE) != 0) != BWD};
    const float   *before = BWD ? a.dlast : a.h0;              // what a sequence starts from, in the order taken
    const int      dir = o.back ? -1 : 1;

    // the window's sequences [qa, qb) and rows [p0, p1)
    const int64_t edge0 = (int64_t)k * cut.R, edge1 = edge0 + cut.R;
    const bool    final_window = k + 1 == cut.K;
    int64_t qa, qb, p0, p1;
    o.first_from(edge0, edge1, qa, qb);
    if (k == 0) qa = 0;
    if (final_window || qb > a.S) qb = a.S;
    if (cut.exact) {
        const int64_t lo = o.at(0), hi = o.at(a.S);
        p0 = edge0 < lo ? lo : edge0;
        p1 = edge1 < hi && !final_window ? edge1 : hi;
    } else {
        p0 = qa <= a.S ? o.at(qa) : 0;
        p1 = qa <= a.S ? o.at(qb) : 0;
    }

    float carry_a[GV], carry_b[V];
#pragma unroll
    for (int v = 0; v < GV; ++v) carry_a[v] = 1.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) carry_b[v] = 0.0f;
    if (PIECE) {
        // only a sequence that goes on in the next window counts: the one that starts last in here, or none does and it is all rows
        const int64_t q = qb - 1;
        const bool    goes_on = !final_window && p1 > p0 && q >= 0 && o.at(q + 1) > p1;
        const int64_t begin = goes_on ? o.at(q) : p1;
        const bool    starts = !goes_on || begin >= p0;
        if (t == 0 && tile_c == 0) cut.piece_cut[k] = starts;
        if (!goes_on) return;                                  // the next window's first row starts a sequence
        if (starts) {
            p0 = begin;
            if (before) load_vec<float, V>(carry_b, before + o.sequence(q) * a.C + c);
        }
    } else if (cut.exact && k > 0) {
        load_vec<float, V>(carry_b, cut.carry + (int64_t)k * a.C + c);
    }

    int64_t q_at = PIECE ? 0 : qa > 0 ? qa - 1 : 0;            // no sequence before this one reaches p0
    int64_t flags_from = p0;
    int     buf = 0;
    for (int64_t pt = p0; pt < p1 || (!PIECE && pt == p0); pt += TR) {
        if (!PIECE && (pt - p0) % kFlagRows == 0) {
            // marks of the rows [flags_from, flags_to): first and last rows of sequences; sequences without rows pass their state on here
            flags_from = pt;
            const int64_t flags_to = p1 - pt < kFlagRows ? p1 : pt + kFlagRows;
            const bool    at_end = flags_to == p1;
            for (int i = t; i < kFlagRows / 32; i += BLOCK) { bits_first[i] = 0; bits_last[i] = 0; }
            if (t == 0) q_next = (int)q_at;
            __syncthreads();
            int furthest = (int)q_at;
            for (int64_t q = q_at + t; q < qb; q += BLOCK) {
                const int64_t f = o.at(q), l = o.at(q + 1);
                if (f > flags_to || (f == flags_to && !at_end)) break;
                if (f < l) {
                    if (f < flags_to) furthest = (int)q;
                    if (f >= flags_from && f < flags_to) {
                        const int i = (int)(f - flags_from);
                        mark_first[i] = (int32_t)q;
                        atomicOr(&bits_first[i >> 5], 1u << (i & 31));
                    }
                    if (l > flags_from && l <= flags_to) {
                        const int i = (int)(l - 1 - flags_from);
                        mark_last[i] = (int32_t)q;
                        atomicOr(&bits_last[i >> 5], 1u << (i & 31));
                    }
                } else if (f >= flags_from && q >= qa) {
                    float        *to = BWD ? a.dh0 : a.last;
                    const int64_t i = o.sequence(q) * a.C;
                    for (int j = (int)tile_c * (CL * V); to && j < ((int)tile_c + 1) * (CL * V) && j < a.C; ++j) to[i + j] = before ? before[i + j] : 0.0f;
                }
            }
            if (furthest > (int)q_at) atomicMax(&q_next, furthest);
            __syncthreads();
            q_at = q_next;
        }
        if (pt >= p1) break;

        const int64_t pr = pt + rl * RB;                       // this lane's first row, in the order taken
        const bool    whole = pt + TR <= p1;
        const Place   at{o.back ? a.N - TR - pt : pt, (uint32_t)(o.back ? TR - 1 - rl * RB : rl * RB), dir};
        uint32_t first = 0, last = 0, live = (1u << RB) - 1u;
        if (!whole) live = pr >= p1 ? 0u : pr + RB <= p1 ? live : (1u << (uint32_t)(p1 - pr)) - 1u;
        if (!PIECE) {
            const uint32_t i = (uint32_t)(pr - flags_from);
            first = (bits_first[i >> 5] >> (i & 31)) & live;
            last = (bits_last[i >> 5] >> (i & 31)) & live;
        }

        // gates and what comes in: x, or dy
        float g[RB][GV], in[RB][V], share[MIX ? RB : 1][GV], left[BWD && !PIECE ? RB : 1][V];
        if constexpr (NARROW) load_narrow<Gate, RB, GV>(g, a.gate, at, whole, a.N, pr, p0, p1);
        else load_rows<Gate, RB, GV>(g, a.gate, at, gw, gc, whole, pr, p0, p1);
        if (!BWD || a.dy) {
            if constexpr (NARROW) load_narrow<Io, RB, V>(in, BWD ? a.dy : a.x, at, whole, a.N, pr, p0, p1);
            else load_rows<Io, RB, V>(in, BWD ? a.dy : a.x, at, a.C, c, whole, pr, p0, p1);
        } else {
#pragma unroll
            for (int j = 0; j < RB; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) in[j][v] = 0.0f;
        }
        if constexpr (BWD && !PIECE) {
            // the state before the row is that of the next row in the order taken (of the next window's first, at the end of this one)
            const int64_t end = p1 + 1 <= a.N ? p1 + 1 : p1;
            const Place   next{at.low + dir, at.mine, dir};
            const bool    all = pt + TR + 1 <= end;
            if constexpr (NARROW) {
                if (a.y_f32) load_narrow<float, RB, V>(left, a.y, next, all, a.N, pr + 1, p0, end);
                else load_narrow<Io, RB, V>(left, a.y, next, all, a.N, pr + 1, p0, end);
            } else {
                if (a.y_f32) load_rows<float, RB, V>(left, a.y, next, a.C, c, all, pr + 1, p0, end);
                else load_rows<Io, RB, V>(left, a.y, next, a.C, c, all, pr + 1, p0, end);
            }
            if (__any(last != 0)) {
                float h[RB][V];
#pragma unroll
                for (int j = 0; j < RB; ++j) {
#pragma unroll
                    for (int v = 0; v < V; ++v) h[j][v] = 0.0f;
                    if (a.h0) {
                        const int64_t q = (last >> j) & 1u ? mark_last[(uint32_t)(pr - flags_from) + j] : 0;
                        load_vec<float, V>(h[j], a.h0 + o.sequence(q) * a.C + c);
                    }
                }
#pragma unroll
                for (int j = 0; j < RB; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) left[j][v] = (last >> j) & 1u ? h[j][v] : left[j][v];
            }
            if (MIX) {
                float x[RB][V];
                if constexpr (NARROW) load_narrow<Io, RB, V>(x, a.x, at, whole, a.N, pr, p0, p1);
                else load_rows<Io, RB, V>(x, a.x, at, a.C, c, whole, pr, p0, p1);
#pragma unroll
                for (int j = 0; j < RB; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) left[j][v] -= x[j][v];
            }
        }
#pragma unroll
        for (int j = 0; j < RB; ++j) {
#pragma unroll
            for (int v = 0; v < GV; ++v) {
                float in_share;
                gate_of<MIX>(log_gate, g[j][v], g[j][v], in_share);
                if (MIX) share[MIX ? j : 0][v] = in_share;
            }
            if (MIX && !BWD) {
#pragma unroll
                for (int v = 0; v < V; ++v) in[j][v] *= share[MIX ? j : 0][SHARED ? 0 : v];
            }
        }
        if (!whole) {                                          // rows that are not there change nothing
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                const bool there = (live >> j) & 1u;
#pragma unroll
                for (int v = 0; v < GV; ++v) g[j][v] = there ? g[j][v] : 1.0f;
#pragma unroll
                for (int v = 0; v < V; ++v) in[j][v] = there ? in[j][v] : 0.0f;
            }
        }
        if (!PIECE && before && __any(first != 0)) {
            float h[RB][V];
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                const int64_t q = (first >> j) & 1u ? mark_first[(uint32_t)(pr - flags_from) + j] : 0;
                load_vec<float, V>(h[j], before + o.sequence(q) * a.C + c);
            }
#pragma unroll
            for (int j = 0; j < RB; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float with = BWD ? in[j][v] + h[j][v] : fmaf(g[j][SHARED ? 0 : v], h[j][v], in[j][v]);
                    in[j][v] = (first >> j) & 1u ? with : in[j][v];
                }
        }

        // this lane's rows as one map, then those of the lanes before it: a lane takes in what lies before it until a sequence starts
        float A[GV], B[V];
        const uint64_t starts = PIECE ? 0 : __ballot(first != 0);
        const uint64_t upto = starts & (~0ull >> (63 - (lane | (CL - 1))));
        const int      since = upto ? (63 - __clzll(upto)) / CL : -1, mine = lane / CL;     // last lane of rows, up to this one, with a start
#pragma unroll
        for (int v = 0; v < GV; ++v) A[v] = 1.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) B[v] = 0.0f;
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            const bool f = (first >> j) & 1u;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float gj = g[j][SHARED ? 0 : v];
                B[v] = BWD ? gj * ((f ? 0.0f : B[v]) + in[j][v]) : (f ? in[j][v] : fmaf(gj, B[v], in[j][v]));
            }
#pragma unroll
            for (int v = 0; v < GV; ++v) A[v] *= g[j][v];
        }
#pragma unroll
        for (int d = 1; d < 64 / CL; d <<= 1) {
            float Al[GV], Bl[V];
#pragma unroll
            for (int v = 0; v < GV; ++v) Al[v] = __shfl_up(A[v], d * CL, 64);
#pragma unroll
            for (int v = 0; v < V; ++v) Bl[v] = __shfl_up(B[v], d * CL, 64);
            const bool joins = mine >= d && since <= mine - d;
#pragma unroll
            for (int v = 0; v < V; ++v) B[v] = joins ? fmaf(A[SHARED ? 0 : v], Bl[v], B[v]) : B[v];
#pragma unroll
            for (int v = 0; v < GV; ++v) A[v] = joins ? A[v] * Al[v] : A[v];
        }
        if (lane >= 64 - CL) {
#pragma unroll
            for (int v = 0; v < GV; ++v) tot_a[buf][w][cl * GV + v] = A[v];
#pragma unroll
            for (int v = 0; v < V; ++v) tot_b[buf][w][cl * V + v] = B[v];
            if (lane == 63) tot_cut[buf][w] = starts != 0;
        }
        __syncthreads();
        float h[V];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int forget = tot_cut[buf][i];
            float     Ai[GV];
#pragma unroll
            for (int v = 0; v < GV; ++v) Ai[v] = tot_a[buf][i][cl * GV + v];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (i == w) h[v] = carry_b[v];
                const float Bi = tot_b[buf][i][cl * V + v];
                carry_b[v] = forget ? Bi : fmaf(Ai[SHARED ? 0 : v], carry_b[v], Bi);
            }
            if (PIECE) {
#pragma unroll
                for (int v = 0; v < GV; ++v) carry_a[v] *= Ai[v];
            }
        }
        buf ^= 1;
        if (PIECE) continue;
        {
            const bool forget = (starts & ((1ull << (mine * CL)) - 1ull)) != 0;
            float      Ae[GV];
#pragma unroll
            for (int v = 0; v < GV; ++v) Ae[v] = __shfl_up(A[v], CL, 64);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float Be = __shfl_up(B[v], CL, 64);
                if (lane >= CL) h[v] = forget ? Be : fmaf(Ae[SHARED ? 0 : v], h[v], Be);
            }
        }

        // the rows once more, now with the state that reaches them
        const uint32_t put = c_ok ? live : 0u;
        const int64_t  row0 = at.low + (int64_t)at.mine;
        float          slope[BWD ? RB : 1][GV];
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            const bool f = (first >> j) & 1u;
            float      sum = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float gj = g[j][SHARED ? 0 : v];
                if constexpr (!BWD) {
                    h[v] = f ? in[j][v] : fmaf(gj, h[v], in[j][v]);
                    in[j][v] = h[v];                           // now the output
                } else {
                    const float dh = (f ? 0.0f : h[v]) + in[j][v];
                    const float da = dh * left[j][v];
                    in[j][v] = MIX ? share[MIX ? j : 0][SHARED ? 0 : v] * dh : dh;
                    if (!SHARED) slope[j][SHARED ? 0 : v] = log_gate ? da * gj : da;
                    else sum += c_ok ? da : 0.0f;
                    h[v] = gj * dh;
                }
            }
            if constexpr (BWD && SHARED) {
#pragma unroll
                for (int d = 1; d < CL; d <<= 1) sum += __shfl_xor(sum, d, 64);
                slope[j][0] = log_gate ? sum * g[j][0] : sum;
            }
            if ((last >> j) & 1u) {
                float        *to = BWD ? a.dh0 : a.last;
                const int64_t q = mark_last[(uint32_t)(pr - flags_from) + j];
                if (c_ok && to) store_vec<float, V>(to + o.sequence(q) * a.C + c, h);
            }
        }
        if constexpr (NARROW) {
            const int64_t lowest = row0 - (o.back ? RB - 1 : 0);
            if (live == (1u << RB) - 1u) {
                if constexpr (BWD) {
                    store_run<Io, RB, V>((Io *)a.dx + lowest * V, in, o.back);
                    store_run<Gate, RB, GV>((Gate *)a.dgate + lowest * GV, slope, o.back);
                } else if (a.out_y) {
                    if (a.y_f32) store_run<float, RB, V>((float *)a.out_y + lowest * V, in, o.back);
                    else store_run<Io, RB, V>((Io *)a.out_y + lowest * V, in, o.back);
                }
            } else if (live) {
#pragma unroll
                for (int j = 0; j < RB; ++j) {
                    if (!((live >> j) & 1u)) continue;
                    const int64_t r = row0 + dir * j;
                    if constexpr (BWD) {
                        store_vec<Io, V>((Io *)a.dx + r * V, in[j]);
                        store_vec<Gate, GV>((Gate *)a.dgate + r * GV, slope[j]);
                    } else if (a.out_y) {
                        if (a.y_f32) store_vec<float, V>((float *)a.out_y + r * V, in[j]);
                        else store_vec<Io, V>((Io *)a.out_y + r * V, in[j]);
                    }
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                const int64_t r = row0 + dir * j;
                const bool    ok = (put >> j) & 1u;
                if constexpr (!BWD) {
                    if (!a.out_y || !ok) continue;
                    if (a.y_f32) store_vec<float, V>((float *)a.out_y + r * a.C + c, in[j]);
                    else store_vec<Io, V>((Io *)a.out_y + r * a.C + c, in[j]);
                } else {
                    if (ok) store_vec<Io, V>((Io *)a.dx + r * a.C + c, in[j]);
                    if constexpr (!SHARED) {
                        if (ok) store_vec<Gate, V>((Gate *)a.dgate + r * a.C + c, slope[j]);
                    } else if (cl == 0 && ((live >> j) & 1u)) {
                        if (a.slope) a.slope[(int64_t)tile_c * a.N + r] = slope[j][0];
                        else store((Gate *)a.dgate, r, slope[j][0]);
                    }
                }
            }
        }
        if ((pt + TR - p0) % kFlagRows == 0) __syncthreads();  // the marks are written anew
    }
    if (PIECE && rl == 0 && c_ok) {
        float A[V];
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = carry_a[SHARED ? 0 : v];
        store_vec<float, V>(cut.piece_a + (int64_t)k * a.C + c, A);
        store_vec<float, V>(cut.piece_b + (int64_t)k * a.C + c, carry_b);
    }
}

// The state that reaches each window, from the windows' maps: 16 channels to a workgroup, 64 lanes with up to 16 windows each, held in
// registers between composing them and walking them with the state.
constexpr int kCarryChannels = 16, kCarryLanes = 64, kCarryEach = 16, kMostWindows = kCarryLanes * kCarryEach;
__global__ __launch_bounds__(kCarryChannels * kCarryLanes) void recur_carry_kernel(const Cut cut, const int C)
{
    __shared__ float sum_a[kCarryLanes][kCarryChannels], sum_b[kCarryLanes][kCarryChannels];
    __shared__ int   sum_cut[kCarryLanes];
    const int      cl = threadIdx.x % kCarryChannels, rl = threadIdx.x / kCarryChannels;
    const int      c_here = (int)blockIdx.x * kCarryChannels + cl, c = c_here < C ? c_here : C - 1;
    const uint32_t per = (cut.K + kCarryLanes - 1) / kCarryLanes, k0 = rl * per;
    float a[kCarryEach], b[kCarryEach];
    int   f[kCarryEach];
#pragma unroll
    for (int i = 0; i < kCarryEach; ++i) {
        const uint32_t k = k0 + i;
        const bool     there = (uint32_t)i < per && k < cut.K;
        const size_t   at = (size_t)(there ? k : 0) * C + c;
        f[i] = there ? cut.piece_cut[there ? k : 0] : 0;
        a[i] = there ? cut.piece_a[at] : 1.0f;
        b[i] = there ? cut.piece_b[at] : 0.0f;
    }
    float A = 1.0f, B = 0.0f;
    int   gone = 0;
#pragma unroll
    for (int i = 0; i < kCarryEach; ++i) {
        B = f[i] ? b[i] : fmaf(a[i], B, b[i]);
        A *= a[i];
        gone |= f[i];
    }
    sum_a[rl][cl] = A;
    sum_b[rl][cl] = B;
    if (cl == 0) sum_cut[rl] = gone;
    __syncthreads();
    float h = 0.0f;
#pragma unroll 8
    for (int i = 0; i < kCarryLanes; ++i) {
        const float next = sum_cut[i] ? sum_b[i][cl] : fmaf(sum_a[i][cl], h, sum_b[i][cl]);
        h = i < rl ? next : h;
    }
#pragma unroll
    for (int i = 0; i < kCarryEach; ++i) {
        const uint32_t k = k0 + i;
        if ((uint32_t)i < per && k < cut.K && c_here < C) cut.carry[(size_t)k * C + c] = h;
        h = f[i] ? b[i] : fmaf(a[i], h, b[i]);
    }
}

__global__ __launch_bounds__(kRecurBlock) void recur_copy_kernel(const float *__restrict__ from, float *__restrict__ to, const int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * kRecurBlock + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.0f;
}

// dgate of a gate that all channels share, from the sums of the channel tiles.
template <typename Gate>
__global__ __launch_bounds__(kRecurBlock) void recur_slope_kernel(const RecurArgs a, const int tiles)
{
    const int64_t r = (int64_t)blockIdx.x * kRecurBlock + threadIdx.x;
    const Order   o{a.offsets, a.N, a.S, a.rows_each, false};
    if (r >= a.N || r < o.at(0) || r >= o.at(a.S)) return;
    float sum = 0.0f;
    for (int i = 0; i < tiles; ++i) sum += a.slope[(int64_t)i * a.N + r];
    store((Gate *)a.dgate, r, sum);
}

int check(const cngp_recur_config *c, int64_t N, int64_t S, bool ragged) {
    if (!c) return CNGP_ERR_NULL;
    if (c->channels < 1 || c->channels > 65536) return CNGP_ERR_INVALID;
    if (c->gate_channels != 1 && c->gate_channels != c->channels) return CNGP_ERR_INVALID;
    if (c->io_dtype != CNGP_F32 && c->io_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->gate_dtype != CNGP_F32 && c->gate_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->longest < 0) return CNGP_ERR_INVALID;
    if (c->flags & ~(uint32_t)(CNGP_RECUR_REVERSE | CNGP_RECUR_LOG_GATE | CNGP_RECUR_MIX)) return CNGP_ERR_INVALID;
    if (N < 0 || N > 0x7fffffffLL || S < 0 || S > 0x7ffffffeLL) return CNGP_ERR_INVALID;
    if (!ragged && (S == 0 ? N != 0 : N % S != 0)) return CNGP_ERR_INVALID;
    return CNGP_OK;
}

RecurArgs args_of(const cngp_recur_config *c, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t S, const float *h0) {
    RecurArgs a{};
    a.gate = gate; a.x = x; a.offsets = offsets; a.h0 = h0;
    a.N = N; a.S = S; a.rows_each = S ? N / S : 0;
    a.C = c->channels; a.G = c->gate_channels; a.flags = c->flags;
    return a;
}

// How a call is cut.  CL lanes side by side hold V channels each: as many as there are channels, at most 32 (a row of a tile is then a
// 128-byte line of fp32).
struct RecurPlan {
    int      CL, V, block, tiles;        // channel tiles
    int64_t  R;                          // rows per window
    uint32_t K;                          // windows
    bool     exact;                      // long sequences are cut at the windows' edges
};

constexpr int     kRowsEach = 8, kRowsNarrow = 4;     // rows of a tile per lane; where a lane holds all channels
constexpr int     kWideBlock = 512;
constexpr int64_t kEnoughGroups = 2048;               // workgroups that fill the chip's 256 CUs with eight each

RecurPlan plan_of(const cngp_recur_config *c, int64_t N, int64_t S, bool ragged) {
    RecurPlan p{};
    const int C = c->channels;
    p.CL = C <= 4 ? 1 : C <= 16 ? 16 : 32;
    p.V = C <= 4 ? C : C > 32 && C % 2 == 0 ? 2 : 1;
    p.block = kRecurBlock;
    p.tiles = (C + p.CL * p.V - 1) / (p.CL * p.V);
    const int64_t tile_rows = kRecurBlock / p.CL * (p.CL == 1 ? kRowsNarrow : kRowsEach);
    const int64_t mean = S ? (N + S - 1) / S : 0;
    const int64_t longest = !ragged ? mean : c->longest ? std::min<int64_t>(c->longest, N) : 4 * mean;
    // windows that give every CU eight workgroups, of whole tiles
    int64_t R = (N * p.tiles + kEnoughGroups - 1) / kEnoughGroups;
    R = std::max<int64_t>((R + tile_rows - 1) / tile_rows * tile_rows, tile_rows);
    // sequences that are no longer than a few windows stay whole: one launch, every input read once.  Longer ones are cut
    p.exact = longest > 4 * R;
    if (p.exact && p.V == 2 && !ragged && S * ((C + 31) / 32) >= 192) {
        // enough sequences by channels to give most CUs one of 32 channels, walked by eight wavefronts: whole after all
        p.CL = 16;
        p.block = kWideBlock;
        p.tiles = (C + 31) / 32;
        p.exact = false;
        R = mean;
    }
    if (p.exact) R = std::max(R, ((N + kMostWindows - 1) / kMostWindows + tile_rows - 1) / tile_rows * tile_rows);
    else if (!ragged) R = std::max<int64_t>((R + mean / 2) / std::max<int64_t>(mean, 1), 1) * mean;
    else if (2 * mean < R) R -= 2 * mean;      // a window's last sequence reaches over its edge: that still fits its tiles
    p.R = std::max<int64_t>(R, 1);
    p.K = (uint32_t)std::max<int64_t>((N + p.R - 1) / p.R, 1);
    return p;
}

// Where the parts of a workspace lie.
struct RecurSpace { size_t y, slope, piece_a, piece_b, carry, piece_cut, state, bytes; };
RecurSpace space_of(const cngp_recur_config *c, const RecurPlan &p, int64_t N, int64_t S, uint32_t call) {
    RecurSpace s{};
    size_t at = 0;
    auto take = [&](bool wanted, size_t bytes) { const size_t o = at; if (wanted) at += align256(bytes); return o; };
    const size_t C = (size_t)c->channels;
    const bool   bwd = call & CNGP_RECUR_CALL_BWD;
    s.y = take(bwd && (call & CNGP_RECUR_CALL_NO_Y), (size_t)N * C * 4);
    s.slope = take(bwd && c->gate_channels == 1 && p.tiles > 1, (size_t)N * (size_t)p.tiles * 4);
    s.piece_a = take(p.exact, p.K * C * 4);
    s.piece_b = take(p.exact, p.K * C * 4);
    s.carry = take(p.exact, p.K * C * 4);
    s.piece_cut = take(p.exact, p.K * 4);
    s.state = take(p.exact, (size_t)S * C * 4);
    s.bytes = at;
    return s;
}

template <typename Io, typename Gate, int BLOCK, int CL, int V, bool SHARED, bool MIX, bool BWD>
int launch_scan(const RecurArgs &a, const RecurPlan &p, const Cut &cut, hipStream_t s) {
    constexpr int  RB = CL == 1 ? kRowsNarrow : kRowsEach;
    const unsigned groups = cut.K * (unsigned)p.tiles;
    if constexpr (BLOCK == kRecurBlock) {
        if (cut.exact) {
            {
                LaunchTimer t(s, BWD ? K_RECUR_BWD : K_RECUR_FWD);
                recur_scan_kernel<Io, Gate, BLOCK, CL, V, RB, SHARED, MIX, BWD, true><<<groups, BLOCK, 0, s>>>(a, cut);
                if (int rc = launch_status("recur_scan_kernel (pieces)")) return rc;
            }
            LaunchTimer t(s, K_RECUR_CARRY);
            recur_carry_kernel<<<(unsigned)((a.C + kCarryChannels - 1) / kCarryChannels), kCarryChannels * kCarryLanes, 0, s>>>(cut, a.C);
            if (int rc = launch_status("recur_carry_kernel")) return rc;
        }
    }
    LaunchTimer t(s, BWD ? K_RECUR_BWD : K_RECUR_FWD);
    recur_scan_kernel<Io, Gate, BLOCK, CL, V, RB, SHARED, MIX, BWD, false><<<groups, BLOCK, 0, s>>>(a, cut);
    return launch_status("recur_scan_kernel");
}

template <typename Io, typename Gate, bool MIX, bool BWD>
int launch_lanes(const RecurArgs &a, const RecurPlan &p, const Cut &cut, hipStream_t s) {
    const bool shared = a.G == 1;
#define CNGP_RECUR(BLOCK, CL, V) \
    return shared ? launch_scan<Io, Gate, BLOCK, CL, V, true, MIX, BWD>(a, p, cut, s) : launch_scan<Io, Gate, BLOCK, CL, V, false, MIX, BWD>(a, p, cut, s)
    if (p.CL == 1) {
        if (a.C == 1) return launch_scan<Io, Gate, kRecurBlock, 1, 1, true, MIX, BWD>(a, p, cut, s);
        if (a.C == 2) CNGP_RECUR(kRecurBlock, 1, 2);
        if (a.C == 3) CNGP_RECUR(kRecurBlock, 1, 3);
        CNGP_RECUR(kRecurBlock, 1, 4);
    }
    if (p.block == kWideBlock) {
        CNGP_RECUR(kWideBlock, 16, 2);
    }
    if (p.CL == 16) CNGP_RECUR(kRecurBlock, 16, 1);
    if (p.V == 1) CNGP_RECUR(kRecurBlock, 32, 1);
    CNGP_RECUR(kRecurBlock, 32, 2);
#undef CNGP_RECUR
}

template <typename Io, typename Gate, bool BWD>
int launch_inputs(const RecurArgs &a, const RecurPlan &p, const Cut &cut, hipStream_t s) {
    return a.flags & CNGP_RECUR_MIX ? launch_lanes<Io, Gate, true, BWD>(a, p, cut, s) : launch_lanes<Io, Gate, false, BWD>(a, p, cut, s);
}

// One direction's launches.  state_in / state_out: what a sequence starts from and where it ends up; where they are one array and
// sequences are cut, the workgroup that ends a sequence is not the one that starts it, so the start is taken from a copy.
template <bool BWD>
int launch(const cngp_recur_config *c, RecurArgs a, const RecurPlan &p, const RecurSpace &sp, char *ws, hipStream_t s) {
    if ((int64_t)p.K * p.tiles > 0x7fffffffLL) return CNGP_ERR_UNSUPPORTED;
    Cut cut{p.R, p.K, (float *)(ws + sp.piece_a), (float *)(ws + sp.piece_b), (float *)(ws + sp.carry), (int32_t *)(ws + sp.piece_cut), p.exact};
    const float *&in = BWD ? a.dlast : a.h0;
    float        *out = BWD ? a.dh0 : a.last;
    if (p.exact && in && in == out) {
        float        *copy = (float *)(ws + sp.state);
        const int64_t n = a.S * a.C;
        LaunchTimer t(s, K_RECUR_CARRY);
        recur_copy_kernel<<<(unsigned)((n + kRecurBlock - 1) / kRecurBlock), kRecurBlock, 0, s>>>(in, copy, n);
        if (int rc = launch_status("recur_copy_kernel")) return rc;
        in = copy;
    }
    const bool io16 = c->io_dtype == CNGP_F16, g16 = c->gate_dtype == CNGP_F16;
    return io16 ? (g16 ? launch_inputs<__half, __half, BWD>(a, p, cut, s) : launch_inputs<__half, float, BWD>(a, p, cut, s))
                : (g16 ? launch_inputs<float, __half, BWD>(a, p, cut, s) : launch_inputs<float, float, BWD>(a, p, cut, s));
}

int pass_states(const float *in, float *out, int64_t n, hipStream_t s) {      // no rows at all
    if (!out || in == out || n == 0) return CNGP_OK;
    LaunchTimer t(s, K_RECUR_CARRY);
    recur_copy_kernel<<<(unsigned)((n + kRecurBlock - 1) / kRecurBlock), kRecurBlock, 0, s>>>(in, out, n);
    return launch_status("recur_copy_kernel");
}

}  // namespace

extern "C" {

size_t cngp_recur_workspace_bytes(const cngp_recur_config *cfg, int64_t N, int64_t sequences, uint32_t call) {
    if (check(cfg, N, sequences, call & CNGP_RECUR_CALL_RAGGED)) return 0;
    return space_of(cfg, plan_of(cfg, N, sequences, call & CNGP_RECUR_CALL_RAGGED), N, sequences, call).bytes;
}

int cngp_recur_fwd(const cngp_recur_config *cfg, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t sequences,
                   const float *h0, void *y, float *last, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N, sequences, offsets != nullptr)) return rc;
    if (sequences == 0) return CNGP_OK;
    if (N && (!gate || !x || (!last && !y))) return CNGP_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    if (N == 0) return pass_states(h0, last, sequences * cfg->channels, s);
    const RecurPlan  p = plan_of(cfg, N, sequences, offsets != nullptr);
    const RecurSpace sp = space_of(cfg, p, N, sequences, offsets ? CNGP_RECUR_CALL_RAGGED : 0);
    if (sp.bytes && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < sp.bytes)) return CNGP_ERR_WORKSPACE;
    RecurArgs a = args_of(cfg, gate, x, N, offsets, sequences, h0);
    a.out_y = y; a.last = last;
    return launch<false>(cfg, a, p, sp, (char *)workspace, s);
}

int cngp_recur_bwd(const cngp_recur_config *cfg, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t sequences,
                   const float *h0, const void *y, const void *dy, const float *dlast, void *dgate, void *dx, float *dh0,
                   void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N, sequences, offsets != nullptr)) return rc;
    if (sequences == 0) return CNGP_OK;
    if (N && (!gate || !x || !dgate || !dx || (!dy && !dlast))) return CNGP_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    if (N == 0) return pass_states(dlast, dh0, sequences * cfg->channels, s);
    const RecurPlan  p = plan_of(cfg, N, sequences, offsets != nullptr);
    const uint32_t   call = CNGP_RECUR_CALL_BWD | (offsets ? CNGP_RECUR_CALL_RAGGED : 0) | (y ? 0 : CNGP_RECUR_CALL_NO_Y);
    const RecurSpace sp = space_of(cfg, p, N, sequences, call);
    char            *ws = (char *)workspace;
    if (sp.bytes && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < sp.bytes)) return CNGP_ERR_WORKSPACE;
    RecurArgs a = args_of(cfg, gate, x, N, offsets, sequences, h0);
    a.y = y;
    if (!y) {
        a.out_y = ws + sp.y;
        a.y_f32 = 1;
        if (int rc = launch<false>(cfg, a, p, sp, ws, s)) return rc;
        a.y = a.out_y;
    }
    a.dy = dy; a.dlast = dlast; a.dgate = dgate; a.dx = dx; a.dh0 = dh0;
    const bool sums = cfg->gate_channels == 1 && p.tiles > 1;
    a.slope = sums ? (float *)(ws + sp.slope) : nullptr;
    if (int rc = launch<true>(cfg, a, p, sp, ws, s)) return rc;
    if (!sums) return CNGP_OK;
    LaunchTimer t(s, K_RECUR_BWD);
    const unsigned blocks = (unsigned)((N + kRecurBlock - 1) / kRecurBlock);
    if (cfg->gate_dtype == CNGP_F16) recur_slope_kernel<__half><<<blocks, kRecurBlock, 0, s>>>(a, p.tiles);
    else recur_slope_kernel<float><<<blocks, kRecurBlock, 0, s>>>(a, p.tiles);
    return launch_status("recur_slope_kernel");
}

}  // extern "C"
