// The scan of the gated linear recurrence: kernels for wide rows and for rows of up to four channels, and their launches.
#pragma once
#include <type_traits>

#include "cngp_recur.h"

namespace {

using namespace cngp;

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

// A window's sequences [qa, qb) and rows [p0, p1), in the order taken.
struct Window {
    pos qa, qb, p0, p1;
    __device__ __forceinline__ bool find(const RecurArgs &a, const Cut &cut, const Order &o, const uint32_t k) {
        const pos     edge0 = (pos)k * cut.R, edge1 = k + 1 == cut.K ? a.N : edge0 + cut.R;
        const bool    final_window = k + 1 == cut.K;
        pos from, to;
        o.first_from(edge0, edge1, qa, qb, from, to);
        if (k == 0 && qa > 0) { qa = 0; from = o.at(0); }
        if (final_window || qb > a.S) { qb = a.S; to = o.at(a.S); }
        if (cut.exact) {
            const pos lo = o.at(0), hi = o.at(a.S);
            p0 = edge0 < lo ? lo : edge0;
            p1 = edge1 < hi && !final_window ? edge1 : hi;
            return true;
        }
        p0 = from;
        p1 = to;
        return qa < qb;                                        // else no sequence starts in here
    }
    // The rows whose map the next window needs: those of the sequence that goes on in it.  False: none does, or it starts there.
    // q: that sequence if it starts in here, else -1.
    __device__ __forceinline__ bool piece(const RecurArgs &a, const Cut &cut, const Order &o, const uint32_t k, const bool writes, pos &q) {
        q = qb - 1;
        const bool    goes_on = k + 1 != cut.K && p1 > p0 && q >= 0 && o.at(q + 1) > p1;
        const pos begin = goes_on ? o.at(q) : p1;
        const bool    starts = !goes_on || begin >= p0;
        if (writes) cut.piece_cut[k] = starts;
        if (!goes_on) return false;
        if (starts) p0 = begin;
        else q = -1;
        return true;
    }
};

// Where a tile's rows lie.  Row j of a lane is memory row low + mine + j, or low + mine - j taken backwards; `low` is the same for
// the whole workgroup, so a load is a scalar base and a 32-bit lane offset.
struct Place {
    pos  low;
    uint32_t mine;                       // rows
    int      dir;                        // 1 or -1
};

// A lane's first row in an array of `width` values to a row; the next one lies dir * width further.
template <typename T>
__device__ __forceinline__ T *row_at(T *array, const Place &at, const int width, const int c) {
    return array + (int64_t)at.low * width + (at.mine * (uint32_t)width + (uint32_t)c);
}
template <typename T>
__device__ __forceinline__ const T *row_at(const void *array, const Place &at, const int width, const int c) {
    return row_at<const T>((const T *)array, at, width, c);
}

// RB rows of V values each as they lie in memory, so that a tile's loads can be under way while another is worked on.
// A lane that holds all values of its rows (NARROW) reads them as one run, 16 bytes at a time, in the order of the memory.
template <typename T, int RB, int V, bool NARROW>
struct Rows {
    Run<T, RB * V> raw;

    // `width` values to a row of the array, this lane's from c on.  Not a whole tile: rows outside [p0, p1) hold those of the nearest row
    // inside, or, in a run that lies inside the N rows of the array, whatever is there.  pr: the lane's first row, in the order taken.
    __device__ __forceinline__ void load_from(const void *array, const Place &at, const int width, const int c, const bool whole, const pos N,
                                              const pos pr, const pos p0, const pos p1) {
        if constexpr (NARROW) {
            const pos lowest = at.low + (pos)at.mine - (at.dir < 0 ? RB - 1 : 0);
            if (whole || (lowest >= 0 && lowest + RB <= N)) {
                __builtin_memcpy(&raw, (const T *)array + (int64_t)lowest * V, sizeof raw);
            } else {
#pragma unroll
                for (int j = 0; j < RB; ++j) {                 // row j of the run
                    const pos p = pr + (at.dir < 0 ? RB - 1 - j : j), q = p < p0 ? p0 : p < p1 ? p : p1 - 1;
                    __builtin_memcpy(&raw.e[j * V], (const T *)array + (int64_t)(at.low + (pos)at.mine + at.dir * (q - pr)) * V, sizeof(T) * V);
                }
            }
        } else {
            const T *row = row_at<T>(array, at, width, c);
            if (whole) {
                const int64_t step = (int64_t)at.dir * width;
#pragma unroll
                for (int j = 0; j < RB; ++j, row += step) __builtin_memcpy(&raw.e[j * V], row, sizeof(T) * V);
            } else {
#pragma unroll
                for (int j = 0; j < RB; ++j) {
                    const pos p = pr + j < p0 ? p0 : pr + j < p1 ? pr + j : p1 - 1;
                    __builtin_memcpy(&raw.e[j * V], row + (int64_t)(at.dir * (p - pr)) * width, sizeof(T) * V);
                }
            }
        }
    }
    __device__ __forceinline__ float get(const int j, const int v, const bool back) const {
        if constexpr (!NARROW) return load(raw.e, j * V + v);
        const float f = load(raw.e, j * V + v), b = load(raw.e, (RB - 1 - j) * V + v);      // both, then one: values, not an index
        return back ? b : f;
    }
};

template <typename T, int RB, int V>
__device__ __forceinline__ void store_run(T *lowest, const float (&in)[RB][V], const bool back) {
    Run<T, RB * V> raw;
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) store(raw.e, j * V + v, back ? in[RB - 1 - j][v] : in[j][v]);
    __builtin_memcpy(lowest, &raw, sizeof raw);
}

// The gates of a lane's rows.  The two forms are two loops: chosen value by value, the compiler computes both.
template <int RB, int GV, bool MIX, typename R>
__device__ __forceinline__ void gates_of(const bool log_gate, const R &raw, const bool back, float (&g)[RB][GV], float (&share)[MIX ? RB : 1][GV]) {
    float in;
    if (log_gate) {
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int v = 0; v < GV; ++v) {
                gate_of<true, MIX>(raw.get(j, v, back), g[j][v], in);
                if (MIX) share[MIX ? j : 0][v] = in;
            }
    } else {
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int v = 0; v < GV; ++v) {
                gate_of<false, MIX>(raw.get(j, v, back), g[j][v], in);
                if (MIX) share[MIX ? j : 0][v] = in;
            }
    }
}

// PIECE: only the composed map of the rows that the next window continues, for `carry`; else the outputs.
// CL lanes side by side hold V channels each of a row, RB rows each.  Y: type of the states, written forward and read backward; LowHalf:
// the low halves alone, written to and read from dx, whose rows the workgroup that read them overwrites: those of a tile after the barrier
// that follows their loads, the first of the next tile's with that tile.
// Bound by memory: 8 sequences of 4096 rows of 1024 in fp16, forward 62 us for 201 MB (rows in pieces of 64 bytes, so that 256 workgroups walk
// whole sequences), the low halves right behind it 47, backward 106 us for 403 MB.
template <typename Io, typename Gate, typename Y, int BLOCK, int CL, int V, int RB, bool SHARED, bool MIX, bool BWD, bool PIECE>
__global__ __launch_bounds__(BLOCK) void recur_scan_kernel(const RecurArgs a, const Cut cut)
{
    constexpr int  RL = BLOCK / CL, TR = RL * RB, W = BLOCK / 64, GV = SHARED ? 1 : V;
    constexpr bool LOW = std::is_same_v<Y, LowHalf>;
    constexpr int  kFlagRows = 2048;                           // rows whose first / last marks are in LDS at a time
    static_assert(kFlagRows % TR == 0 && 32 % RB == 0, "a tile's marks lie in one block of them, a lane's in one word");
    __shared__ uint32_t bits_first[PIECE ? 1 : kFlagRows / 32], bits_last[PIECE ? 1 : kFlagRows / 32];
    __shared__ int32_t  mark_first[PIECE ? 1 : kFlagRows], mark_last[PIECE ? 1 : kFlagRows];     // sequence, where the bit is set
    __shared__ float    tot_a[2][W][CL * GV], tot_b[2][W][CL * V];
    __shared__ int      tot_cut[2][W];
    __shared__ int      q_next;
    const int      t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), cl = t % CL, rl = t / CL;
    const uint32_t k = blockIdx.x % cut.K, tile_c = blockIdx.x / cut.K;
    const int      c_here = (int)tile_c * (CL * V) + cl * V;
    const bool     c_ok = c_here < a.C;                        // V divides C
    const int      c = c_ok ? c_here : a.C - V;                // lanes without a channel read the last ones and write nothing
    const int      gc = SHARED ? 0 : c, gw = SHARED ? 1 : a.C;
    const bool     log_gate = a.flags & CNGP_RECUR_LOG_GATE;
    const Order    o{a.offsets, a.N, a.S, a.rows_each, ((a.flags & CNGP_RECUR_REVERSE) != 0) != BWD};
    const float   *before = BWD ? a.dlast : a.h0;              // what a sequence starts from, in the order taken
    const int      dir = o.back ? -1 : 1;

    Window win;
    if (!win.find(a, cut, o, k)) return;
    float carry_a[GV], carry_b[V];
#pragma unroll
    for (int v = 0; v < GV; ++v) carry_a[v] = 1.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) carry_b[v] = 0.0f;
    if (PIECE) {
        pos q;
        if (!win.piece(a, cut, o, k, t == 0 && tile_c == 0, q)) return;
        if (q >= 0 && before) load_vec<float, V>(carry_b, before + (int64_t)o.sequence(q) * a.C + c);
    } else if (cut.exact && k > 0) {
        load_vec<float, V>(carry_b, cut.carry + (int64_t)k * a.C + c);
    }
    const pos qa = win.qa, qb = win.qb, p0 = win.p0, p1 = win.p1;

    // a tile's loads: gates, what comes in (x, or dy), backward the states before the rows and, with mixed inputs, x
    struct Tile {
        Rows<Gate, RB, GV, false> g;
        Rows<Io, RB, V, false>    in;
        Rows<LowHalf, (BWD && LOW && !PIECE ? RB : 1), V, false>                      low;
        Rows<std::conditional_t<LOW, Io, Y>, (BWD && !PIECE ? RB : 1), V, false>     left;
        Rows<Io, (BWD && MIX && !PIECE ? RB : 1), V, false> x;
    };
    const auto place = [&](const pos pt) {
        return Place{o.back ? a.N - TR - pt : pt, (uint32_t)(o.back ? TR - 1 - rl * RB : rl * RB), dir};
    };
    const auto fetch = [&](Tile &f, const pos pt) {
        const pos pr = pt + rl * RB;
        const bool    whole = pt + TR <= p1;
        const Place   at = place(pt);
        // the row behind the window is another workgroup's, and its state not used: these windows hold whole sequences
        if constexpr (BWD && LOW && !PIECE)
            f.low.load_from(a.dx, Place{at.low + dir, at.mine, dir}, a.C, c, pt + TR + 1 <= p1, a.N, pr + 1, p0, p1);
        f.g.load_from(a.gate, at, gw, gc, whole, a.N, pr, p0, p1);
        if (!BWD || a.dy) f.in.load_from(BWD ? a.dy : a.x, at, a.C, c, whole, a.N, pr, p0, p1);
        if constexpr (BWD && !PIECE) {
            // the state before the row is that of the next row in the order taken (of the next window's first, at the end of this one)
            const pos end = p1 + 1 <= a.N ? p1 + 1 : p1;
            f.left.load_from(a.y, Place{at.low + dir, at.mine, dir}, a.C, c, pt + TR + 1 <= end, a.N, pr + 1, p0, end);
            if constexpr (MIX) f.x.load_from(a.x, at, a.C, c, whole, a.N, pr, p0, p1);
        }
    };

    pos q_at = PIECE ? 0 : qa > 0 ? qa - 1 : 0;            // no sequence before this one reaches p0
    pos flags_from = p0;
    int     buf = 0;
    Tile    now, next;
    if (p0 < p1) fetch(now, p0);
    for (int64_t pt = p0; pt < p1 || (!PIECE && pt == p0); pt += TR) {
        if (!PIECE && (pt - p0) % kFlagRows == 0) {
            // marks of the rows [flags_from, flags_to): first and last rows of sequences; sequences without rows pass their state on here
            flags_from = pt;
            const pos flags_to = p1 - pt < kFlagRows ? p1 : pt + kFlagRows;
            const bool    at_end = flags_to == p1;
            for (int i = t; i < kFlagRows / 32; i += BLOCK) { bits_first[i] = 0; bits_last[i] = 0; }
            if (t == 0) q_next = (int)q_at;
            __syncthreads();
            int furthest = (int)q_at;
            for (int64_t q = q_at + t; q < qb; q += BLOCK) {
                const pos f = o.at(q), l = o.at(q + 1);
                if (f > flags_to || (f == flags_to && !at_end)) break;
                if (f < l) {
                    if (f < flags_to) furthest = (int)q;
                    if (f >= flags_from && f < flags_to) {
                        const int i = (int)(f - flags_from);
                        mark_first[i] = (int32_t)o.sequence(q);
                        atomicOr(&bits_first[i >> 5], 1u << (i & 31));
                    }
                    if (l > flags_from && l <= flags_to) {
                        const int i = (int)(l - 1 - flags_from);
                        mark_last[i] = (int32_t)o.sequence(q);
                        atomicOr(&bits_last[i >> 5], 1u << (i & 31));
                    }
                } else if (f >= flags_from && q >= qa) {
                    float        *to = BWD ? a.dh0 : a.last;
                    const int64_t i = (int64_t)o.sequence(q) * a.C;
                    for (int j = (int)tile_c * (CL * V); to && j < ((int)tile_c + 1) * (CL * V) && j < a.C; ++j) to[i + j] = before ? before[i + j] : 0.0f;
                }
            }
            if (furthest > (int)q_at) atomicMax(&q_next, furthest);
            __syncthreads();
            q_at = q_next;
        }
        if (pt >= p1) break;

        const pos pr = pt + rl * RB;                       // this lane's first row, in the order taken
        const bool    whole = pt + TR <= p1;
        const Place   at = place(pt);
        uint32_t      first = 0, last = 0, live = (1u << RB) - 1u, mark0 = 0;
        if (!whole) live = pr >= p1 ? 0u : pr + RB <= p1 ? live : (1u << (uint32_t)(p1 - pr)) - 1u;
        if (!PIECE) {
            mark0 = (uint32_t)(pr - flags_from);
            first = (bits_first[mark0 >> 5] >> (mark0 & 31)) & live;
            last = (bits_last[mark0 >> 5] >> (mark0 & 31)) & live;
        }
        if (pt + TR < p1) fetch(next, pt + TR);                // under way while this tile is worked on
        // what the sequences that start in here start from; backward, what those that end in here started from
        float      h_first[PIECE ? 1 : RB][V], h_last[BWD && !PIECE ? RB : 1][V];
        const bool starts_here = !PIECE && __any(first != 0), ends_here = !PIECE && __any(last != 0);
        if constexpr (!PIECE) {
            if (starts_here && before) {
#pragma unroll
                for (int j = 0; j < RB; ++j)
                    if ((first >> j) & 1u) load_vec<float, V>(h_first[j], before + (uint64_t)(uint32_t)mark_first[mark0 + j] * (uint32_t)a.C + c);
            }
        }
        if constexpr (BWD && !PIECE) {
            if (ends_here && a.h0) {
#pragma unroll
                for (int j = 0; j < RB; ++j)
                    if ((last >> j) & 1u) load_vec<float, V>(h_last[j], a.h0 + (uint64_t)(uint32_t)mark_last[mark0 + j] * (uint32_t)a.C + c);
            }
        }

        float g[RB][GV], in[RB][V], share[MIX ? RB : 1][GV];
        gates_of<RB, GV, MIX>(log_gate, now.g, o.back, g, share);
#pragma unroll
        for (int j = 0; j < RB; ++j) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                in[j][v] = !BWD || a.dy ? now.in.get(j, v, o.back) : 0.0f;
                if (MIX && !BWD) in[j][v] *= share[MIX ? j : 0][SHARED ? 0 : v];
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
        if constexpr (!PIECE) {
            if (starts_here && before) {
#pragma unroll
                for (int j = 0; j < RB; ++j)
                    if ((first >> j) & 1u) {
#pragma unroll
                        for (int v = 0; v < V; ++v) in[j][v] = BWD ? in[j][v] + h_first[j][v] : fmaf(g[j][SHARED ? 0 : v], h_first[j][v], in[j][v]);
                    }
            }
        }

        // this lane's rows as one map, then those of the lanes before it: a lane takes in what lies before it until a sequence starts
        float          A[GV], B[V];
        const uint64_t starts = PIECE ? 0 : __ballot(first != 0);
        const uint64_t upto = starts & (~0ull >> (63 - (lane | (CL - 1))));
        const int      since = upto ? (63 - __clzll(upto)) / CL : -1, mine = lane / CL;     // last lane of rows, up to this one, with a start
#pragma unroll
        for (int v = 0; v < GV; ++v) A[v] = 1.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) B[v] = 0.0f;
        const auto compose = [&](auto with_starts) {
#pragma unroll
            for (int j = 0; j < RB; ++j) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float gj = g[j][SHARED ? 0 : v], from = with_starts && ((first >> j) & 1u) ? 0.0f : B[v];
                    B[v] = BWD ? gj * (from + in[j][v]) : fmaf(gj, from, in[j][v]);
                }
#pragma unroll
                for (int v = 0; v < GV; ++v) A[v] *= g[j][v];
            }
        };
        if (starts_here) compose(std::true_type());            // two loops, not one of selects
        else compose(std::false_type());
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
        float h[V];
        if (lane >= 64 - CL) {
#pragma unroll
            for (int v = 0; v < GV; ++v) tot_a[buf][w][cl * GV + v] = A[v];
#pragma unroll
            for (int v = 0; v < V; ++v) tot_b[buf][w][cl * V + v] = B[v];
            if (lane == 63) tot_cut[buf][w] = starts != 0;
        }
        __syncthreads();
        int forgets[W], any_forgets = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) { forgets[i] = tot_cut[buf][i]; any_forgets |= forgets[i]; }
        const auto fold = [&](auto with_starts) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                float Ai[GV], Bi[V];
#pragma unroll
                for (int v = 0; v < GV; ++v) Ai[v] = tot_a[buf][i][cl * GV + v];
#pragma unroll
                for (int v = 0; v < V; ++v) Bi[v] = tot_b[buf][i][cl * V + v];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    h[v] = i == w ? carry_b[v] : h[v];
                    const float next_b = fmaf(Ai[SHARED ? 0 : v], carry_b[v], Bi[v]);
                    carry_b[v] = with_starts && forgets[i] ? Bi[v] : next_b;
                }
                if (PIECE) {
#pragma unroll
                    for (int v = 0; v < GV; ++v) carry_a[v] *= Ai[v];
                }
            }
        };
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = 0.0f;
        if (!PIECE && __builtin_amdgcn_readfirstlane(any_forgets)) fold(std::true_type());
        else fold(std::false_type());
        buf ^= 1;
        if constexpr (PIECE) {
            now = next;
            continue;
        }
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
        float slope[BWD ? RB : 1][GV];
        const auto walk = [&](auto with_edges) {
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                float sum = 0.0f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float gj = g[j][SHARED ? 0 : v], from = with_edges && ((first >> j) & 1u) ? 0.0f : h[v];
                    if constexpr (!BWD) {
                        h[v] = fmaf(gj, from, in[j][v]);
                        in[j][v] = h[v];                       // now the output
                    } else if constexpr (!PIECE) {
                        float left = now.left.get(j, v, o.back);
                        if constexpr (LOW) left = with_low_half(left, now.low.raw.e[j * V + v].bits);
                        if (with_edges && ((last >> j) & 1u)) left = a.h0 ? h_last[j][v] : 0.0f;
                        if constexpr (MIX) left -= now.x.get(j, v, o.back);
                        const float dh = from + in[j][v], da = dh * left;
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
                if (with_edges && ((last >> j) & 1u)) {
                    float *to = BWD ? a.dh0 : a.last;
                    if (c_ok && to) store_vec<float, V>(to + (uint64_t)(uint32_t)mark_last[mark0 + j] * (uint32_t)a.C + c, h);
                }
            }
        };
        if (starts_here || ends_here) walk(std::true_type());
        else walk(std::false_type());
        const int64_t step = (int64_t)dir * a.C;
        if (c_ok && (BWD || a.out_y)) {
            const auto put = [&](const int j, Io *dx, Gate *dg, Y *y) {
                if constexpr (!BWD) {
                    store_vec<Y, V>(y + step * j, in[j]);
                } else {
                    store_vec<Io, V>(dx + step * j, in[j]);
                    if constexpr (!SHARED) store_vec<Gate, V>(dg + step * j, slope[j]);
                }
            };
            Io   *dx = BWD ? row_at<Io>((Io *)a.dx, at, a.C, c) : nullptr;
            Gate *dg = BWD && !SHARED ? row_at<Gate>((Gate *)a.dgate, at, a.C, c) : nullptr;
            Y    *y = BWD ? nullptr : row_at<Y>((Y *)a.out_y, at, a.C, c);
            if (whole) {
#pragma unroll
                for (int j = 0; j < RB; ++j) put(j, dx, dg, y);
            } else {
#pragma unroll
                for (int j = 0; j < RB; ++j)
                    if ((live >> j) & 1u) put(j, dx, dg, y);
            }
        }
        if constexpr (BWD && SHARED) {
            if (cl == 0) {
                float *sl = a.slope ? row_at<float>(a.slope + (int64_t)tile_c * a.N, at, 1, 0) : nullptr;
                Gate  *dg = row_at<Gate>((Gate *)a.dgate, at, 1, 0);
#pragma unroll
                for (int j = 0; j < RB; ++j)
                    if ((live >> j) & 1u) {
                        if (sl) sl[dir * j] = slope[j][0];
                        else store(dg + dir * j, 0, slope[j][0]);
                    }
            }
        }
        now = next;
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

// The value of another lane of the wavefront by the lane permutations that instructions have (no trip through LDS): that of the lane CTRL names,
// 0 where there is none.
constexpr int kLaneBefore = 0x138, kRowEndBefore = 0x142, kLane31 = 0x143;       // lane - 1; lane 15 of the sixteen before; lane 31 for the upper half
constexpr int lane_less(const int d) { return 0x110 + d; }                        // lane - d, inside the sixteen
template <int CTRL>
__device__ __forceinline__ float lane_value(const float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float last_lane_value(const float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
// One step of the scan over a wavefront's maps: `ok` where the map of the lane CTRL names lies right before what this lane's covers.
template <int CTRL, int GV, int V>
__device__ __forceinline__ void take_in(float (&A)[GV], float (&B)[V], const bool ok) {
    float Al[GV], Bl[V];
#pragma unroll
    for (int v = 0; v < GV; ++v) Al[v] = lane_value<CTRL>(A[v]);
#pragma unroll
    for (int v = 0; v < V; ++v) Bl[v] = lane_value<CTRL>(B[v]);
#pragma unroll
    for (int v = 0; v < V; ++v) B[v] = ok ? fmaf(A[GV == 1 ? 0 : v], Bl[v], B[v]) : B[v];
#pragma unroll
    for (int v = 0; v < GV; ++v) A[v] = ok ? A[v] * Al[v] : A[v];
}

// Rows of up to four channels: a lane holds RB whole rows, a workgroup is one wavefront, so nothing is joined through LDS and no barrier
// waits.  What bounds such rows is not their bytes but the chain of loads: where the sequences start, what they start from, the rows.
// All three are loaded a tile ahead; the start states of a tile's first 64 sequences go through LDS to the lanes whose rows start them.
// Lanes join by the instructions' lane permutations: with shuffles through LDS 4096 rays forward and backward took 32.2 us, so 29.2.  A frame of
// 1920 x 1080 rays with 16.6 M samples takes 98 us for 323 MB: 510 vector instructions to a tile of 256 rows keep the vector ALU busy for half
// of it, and wavefronts wait for loads 70 % of their time.
template <typename Io, typename Gate, typename Y, int V, bool SHARED, bool MIX, bool BWD, bool PIECE>
__device__ __forceinline__ void narrow_rows(const RecurArgs &a, const Cut &cut, const Order &o, Window win, const uint32_t k)
{
    constexpr int RB = kRowsNarrow, TR = 64 * RB, GV = SHARED ? 1 : V;
    __shared__ __align__(16) uint32_t mark_first[PIECE ? 4 : TR], mark_last[PIECE ? 4 : TR];     // sequence (in order taken) + 1, or 0
    __shared__ float from_s[PIECE ? 1 : 64 * V], left_s[BWD && !PIECE ? 64 * V : 1];
    const int      lane = threadIdx.x;
    const bool     log_gate = a.flags & CNGP_RECUR_LOG_GATE;
    const float   *before = BWD ? a.dlast : a.h0;              // what a sequence starts from, in the order taken
    const int      dir = o.back ? -1 : 1;

    float carry_a[GV], carry_b[V];
#pragma unroll
    for (int v = 0; v < GV; ++v) carry_a[v] = 1.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) carry_b[v] = 0.0f;
    if (PIECE) {
        pos q;
        if (!win.piece(a, cut, o, k, lane == 0, q)) return;
        if (q >= 0 && before) load_vec<float, V>(carry_b, before + (int64_t)o.sequence(q) * V);
    } else if (cut.exact && k > 0) {
        load_vec<float, V>(carry_b, cut.carry + (int64_t)k * V);
    }
    const pos qa = win.qa, qb = win.qb, p0 = win.p0, p1 = win.p1;

    struct Tile {
        Rows<Gate, RB, GV, true> g;
        Rows<Io, RB, V, true>    in;
        Rows<Y, (BWD && !PIECE ? RB : 1), V, true>         left;
        Rows<Io, (BWD && MIX && !PIECE ? RB : 1), V, true> x;
        pos first, behind;                                 // rows of sequence q + lane
        float   from[V], ends[BWD ? V : 1];                    // its state to start from; backward, the one it started from
    };
    const auto place = [&](const pos pt) {
        return Place{o.back ? a.N - TR - pt : pt, (uint32_t)(o.back ? TR - 1 - lane * RB : lane * RB), dir};
    };
    const auto fetch_sequences = [&](Tile &f, const pos q) {
        const pos s = q + lane < qb ? q + lane : qb - 1 > 0 ? qb - 1 : 0;
        f.first = o.at(s);
        f.behind = o.at(s + 1);
        if (before) load_vec<float, V>(f.from, before + (int64_t)o.sequence(s) * V);
        if (BWD && a.h0) load_vec<float, BWD ? V : 1>(f.ends, a.h0 + (int64_t)o.sequence(s) * V);
    };
    const auto fetch_rows = [&](Tile &f, const pos pt) {
        const pos pr = pt + lane * RB;
        const bool    whole = pt + TR <= p1;
        const Place   at = place(pt);
        f.g.load_from(a.gate, at, GV, 0, whole, a.N, pr, p0, p1);
        if (!BWD || a.dy) f.in.load_from(BWD ? a.dy : a.x, at, V, 0, whole, a.N, pr, p0, p1);
        if constexpr (BWD && !PIECE) {
            const pos end = p1 + 1 <= a.N ? p1 + 1 : p1;
            f.left.load_from(a.y, Place{at.low + dir, at.mine, dir}, V, 0, pt + TR + 1 <= end, a.N, pr + 1, p0, end);
            if constexpr (MIX) f.x.load_from(a.x, at, V, 0, whole, a.N, pr, p0, p1);
        }
    };

    pos q_at = qa > 0 ? qa - 1 : 0;                        // no sequence before this one reaches p0
    Tile    now, next;
    if (!PIECE) fetch_sequences(now, q_at);
    if (p0 < p1) fetch_rows(now, p0);
    for (int64_t pt = p0; pt < p1 || (!PIECE && pt == p0); pt += TR) {
        const pos to = p1 - pt < TR ? p1 : pt + TR, q0 = q_at;
        const bool    whole = pt + TR <= p1;
        if (!PIECE) {
#pragma unroll
            for (int i = 0; i < RB; i += 4) {
                *reinterpret_cast<uint4 *>(mark_first + lane * RB + i) = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4 *>(mark_last + lane * RB + i) = make_uint4(0, 0, 0, 0);
            }
            __syncthreads();
            for (int64_t q = q0;;) {
                const pos f = now.first, l = now.behind;
                const bool    here = q + lane < qb && (f < to || (f == to && to == p1));
                if (here && f < l) {
                    if (f >= pt && f < to) mark_first[(int)(f - pt)] = (uint32_t)(q + lane) + 1u;
                    if (l > pt && l <= to) mark_last[(int)(l - 1 - pt)] = (uint32_t)(q + lane) + 1u;
                    if (q == q0) {
#pragma unroll
                        for (int v = 0; v < V; ++v) from_s[lane * V + v] = before ? now.from[v] : 0.0f;
                        if constexpr (BWD) {
#pragma unroll
                            for (int v = 0; v < V; ++v) left_s[lane * V + v] = a.h0 ? now.ends[v] : 0.0f;
                        }
                    }
                } else if (here && f >= pt && q + lane >= qa) {        // no rows: the state passes on
                    float *pass = BWD ? a.dh0 : a.last;
                    float  h[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) h[v] = before ? now.from[v] : 0.0f;
                    if (pass) store_vec<float, V>(pass + (int64_t)o.sequence(q + lane) * V, h);
                }
                const uint64_t inside = __ballot(here && f < to), all = __ballot(here);
                if (inside) q_at = q + (63 - __clzll(inside));
                if (all != ~0ull) break;
                q += 64;                                       // more than 64 sequences touch the tile: these are not loaded ahead
                fetch_sequences(now, q);
            }
            __syncthreads();
        }
        if (pt + TR < p1) {
            if (!PIECE) fetch_sequences(next, q_at);
            fetch_rows(next, pt + TR);
        }
        if (pt >= p1) break;

        const pos pr = pt + lane * RB;
        const Place   at = place(pt);
        uint32_t      first[RB], last[RB], live = (1u << RB) - 1u;
        if (!whole) live = pr >= p1 ? 0u : pr + RB <= p1 ? live : (1u << (uint32_t)(p1 - pr)) - 1u;
        bool any_first = false;
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            first[j] = PIECE ? 0u : mark_first[lane * RB + j];
            last[j] = PIECE ? 0u : mark_last[lane * RB + j];
            any_first |= first[j] != 0;
        }

        float g[RB][GV], in[RB][V], share[MIX ? RB : 1][GV];
        gates_of<RB, GV, MIX>(log_gate, now.g, o.back, g, share);
#pragma unroll
        for (int j = 0; j < RB; ++j) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                in[j][v] = !BWD || a.dy ? now.in.get(j, v, o.back) : 0.0f;
                if (MIX && !BWD) in[j][v] *= share[MIX ? j : 0][SHARED ? 0 : v];
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
        // the state of sequence q + 1 == mark out of LDS, or of the array if the tile has more than 64
        const auto state = [&](float (&h)[V], const float *table, const float *array, const uint32_t mark) {
            const uint32_t i = mark - 1u - (uint32_t)q0;
            if (i < 64u) {
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = table[i * V + v];
            } else if (array) {
                load_vec<float, V>(h, array + (int64_t)o.sequence((pos)mark - 1) * V);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = 0.0f;
            }
        };
        if (!PIECE && before) {
#pragma unroll
            for (int j = 0; j < RB; ++j)
                if (first[j]) {
                    float h[V];
                    state(h, from_s, before, first[j]);
#pragma unroll
                    for (int v = 0; v < V; ++v) in[j][v] = BWD ? in[j][v] + h[v] : fmaf(g[j][SHARED ? 0 : v], h[v], in[j][v]);
                }
        }

        float          A[GV], B[V];
        const uint64_t starts = PIECE ? 0 : __ballot(any_first);
        const uint64_t upto = starts & (~0ull >> (63 - lane));
        const int      since = upto ? 63 - __clzll(upto) : -1;  // last lane, up to this one, with a start
#pragma unroll
        for (int v = 0; v < GV; ++v) A[v] = 1.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) B[v] = 0.0f;
#pragma unroll
        for (int j = 0; j < RB; ++j) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float gj = g[j][SHARED ? 0 : v], b = first[j] ? 0.0f : B[v];
                B[v] = BWD ? gj * (b + in[j][v]) : fmaf(gj, b, in[j][v]);
            }
#pragma unroll
            for (int v = 0; v < GV; ++v) A[v] *= g[j][v];
        }
        // sixteen lanes, then the sixteen before, then the lower half; a lane may take in `room` lanes, back to one where a sequence starts
        const int room = lane - (since > 0 ? since : 0), inside = min(room, lane & 15);
        take_in<lane_less(1), GV, V>(A, B, inside >= 1);
        take_in<lane_less(2), GV, V>(A, B, inside >= 2);
        take_in<lane_less(4), GV, V>(A, B, inside >= 4);
        take_in<lane_less(8), GV, V>(A, B, inside >= 8);
        take_in<kRowEndBefore, GV, V>(A, B, (lane & 16) && room > (lane & 15));
        take_in<kLane31, GV, V>(A, B, (lane & 32) && room > (lane & 31));
        float h[V];
        const bool cut_before = (starts & ((1ull << lane) - 1ull)) != 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float Ae = lane_value<kLaneBefore>(A[SHARED ? 0 : v]), Be = lane_value<kLaneBefore>(B[v]);
            const float At = last_lane_value(A[SHARED ? 0 : v]), Bt = last_lane_value(B[v]);
            h[v] = lane == 0 ? carry_b[v] : cut_before ? Be : fmaf(Ae, carry_b[v], Be);
            carry_b[v] = starts ? Bt : fmaf(At, carry_b[v], Bt);
        }
        if constexpr (PIECE) {
#pragma unroll
            for (int v = 0; v < GV; ++v) carry_a[v] *= last_lane_value(A[v]);
            now = next;
            continue;
        }

        float slope[BWD ? RB : 1][GV];
#pragma unroll
        for (int j = 0; j < RB; ++j) {
            float sum = 0.0f, left[V];
            if constexpr (BWD && !PIECE) {
#pragma unroll
                for (int v = 0; v < V; ++v) left[v] = now.left.get(j, v, o.back);
                if (last[j]) state(left, left_s, a.h0, last[j]);
                if constexpr (MIX) {
#pragma unroll
                    for (int v = 0; v < V; ++v) left[v] -= now.x.get(j, v, o.back);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float gj = g[j][SHARED ? 0 : v], b = first[j] ? 0.0f : h[v];
                if constexpr (!BWD) {
                    h[v] = fmaf(gj, b, in[j][v]);
                    in[j][v] = h[v];                           // now the output
                } else {
                    const float dh = b + in[j][v], da = dh * left[v];
                    in[j][v] = MIX ? share[MIX ? j : 0][SHARED ? 0 : v] * dh : dh;
                    if (!SHARED) slope[j][SHARED ? 0 : v] = log_gate ? da * gj : da;
                    else sum += da;
                    h[v] = gj * dh;
                }
            }
            if constexpr (BWD && SHARED) slope[j][0] = log_gate ? sum * g[j][0] : sum;
            if (last[j]) {
                float *pass = BWD ? a.dh0 : a.last;
                if (pass) store_vec<float, V>(pass + (int64_t)o.sequence((pos)last[j] - 1) * V, h);
            }
        }
        const pos low_row = at.low + (pos)at.mine, lowest = low_row - (o.back ? RB - 1 : 0);
        if (live == (1u << RB) - 1u) {
            if constexpr (BWD) {
                store_run<Io, RB, V>((Io *)a.dx + (int64_t)lowest * V, in, o.back);
                store_run<Gate, RB, GV>((Gate *)a.dgate + (int64_t)lowest * GV, slope, o.back);
            } else if (a.out_y) {
                store_run<Y, RB, V>((Y *)a.out_y + (int64_t)lowest * V, in, o.back);
            }
        } else if (live) {
#pragma unroll
            for (int j = 0; j < RB; ++j) {
                if (!((live >> j) & 1u)) continue;
                const pos r = low_row + dir * j;
                if constexpr (BWD) {
                    store_vec<Io, V>((Io *)a.dx + (int64_t)r * V, in[j]);
                    store_vec<Gate, GV>((Gate *)a.dgate + (int64_t)r * GV, slope[j]);
                } else if (a.out_y) {
                    store_vec<Y, V>((Y *)a.out_y + (int64_t)r * V, in[j]);
                }
            }
        }
        now = next;
    }
    if (PIECE && lane == 0) {
        float A[V];
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = carry_a[SHARED ? 0 : v];
        store_vec<float, V>(cut.piece_a + (int64_t)k * V, A);
        store_vec<float, V>(cut.piece_b + (int64_t)k * V, carry_b);
    }
}

template <typename Io, typename Gate, typename Y, int V, bool SHARED, bool MIX, bool BWD, bool PIECE>
__global__ __launch_bounds__(64) void recur_narrow_kernel(const RecurArgs a, const Cut cut)
{
    const Order o{a.offsets, a.N, a.S, a.rows_each, ((a.flags & CNGP_RECUR_REVERSE) != 0) != BWD};
    Window      win;
    if (win.find(a, cut, o, blockIdx.x)) narrow_rows<Io, Gate, Y, V, SHARED, MIX, BWD, PIECE>(a, cut, o, win, blockIdx.x);
}

// Backward without kept states, whole sequences: a wavefront computes the states of its own rows, then takes them back.  The states go through
// the workspace and are still in its caches.  Forward and backward of 4096 rays with 2^18 samples: 32.2 us when it came, with a launch
// of its own for the states 34.9.
template <typename Io, typename Gate, int V, bool SHARED, bool MIX>
__global__ __launch_bounds__(64) void recur_narrow_again_kernel(const RecurArgs a, const Cut cut)
{
    const bool  reverse = (a.flags & CNGP_RECUR_REVERSE) != 0;
    const Order o{a.offsets, a.N, a.S, a.rows_each, !reverse}, forward{a.offsets, a.N, a.S, a.rows_each, reverse};
    Window      win;
    if (!win.find(a, cut, o, blockIdx.x)) return;
    narrow_rows<Io, Gate, float, V, SHARED, MIX, false, false>(a, cut, forward, Window{a.S - win.qb, a.S - win.qa, a.N - win.p1, a.N - win.p0}, blockIdx.x);
    __syncthreads();                                           // the states are written
    narrow_rows<Io, Gate, float, V, SHARED, MIX, true, false>(a, cut, o, win, blockIdx.x);
}

template <typename Io, typename Gate, typename Y, int BLOCK, int CL, int V, int RB, bool SHARED, bool MIX, bool BWD>
int launch_scan(const RecurArgs &a, const RecurPlan &p, const Cut &cut, hipStream_t s) {
    const unsigned groups = cut.K * (unsigned)p.tiles;
    if constexpr (BLOCK != kWideBlock) {
        if (cut.exact) {
            {
                LaunchTimer t(s, BWD ? K_RECUR_BWD : K_RECUR_FWD);
                recur_scan_kernel<Io, Gate, Io, BLOCK, CL, V, RB, SHARED, MIX, BWD, true><<<groups, BLOCK, 0, s>>>(a, cut);
                if (int rc = launch_status("recur_scan_kernel (pieces)")) return rc;
            }
            if (int rc = recur_carry(cut, a.C, s)) return rc;
        }
    }
    LaunchTimer t(s, BWD ? K_RECUR_BWD : K_RECUR_FWD);
    recur_scan_kernel<Io, Gate, Y, BLOCK, CL, V, RB, SHARED, MIX, BWD, false><<<groups, BLOCK, 0, s>>>(a, cut);
    return launch_status("recur_scan_kernel");
}

template <typename Io, typename Gate, typename Y, int V, bool SHARED, bool MIX, bool BWD>
int launch_narrow(const RecurArgs &a, const Cut &cut, hipStream_t s) {
    if (cut.exact) {
        {
            LaunchTimer t(s, BWD ? K_RECUR_BWD : K_RECUR_FWD);
            recur_narrow_kernel<Io, Gate, Io, V, SHARED, MIX, BWD, true><<<cut.K, kNarrowBlock, 0, s>>>(a, cut);
            if (int rc = launch_status("recur_narrow_kernel (pieces)")) return rc;
        }
        if (int rc = recur_carry(cut, a.C, s)) return rc;
    }
    LaunchTimer t(s, BWD ? K_RECUR_BWD : K_RECUR_FWD);
    if constexpr (BWD && sizeof(Y) == sizeof(float)) {
        if (a.out_y) {
            recur_narrow_again_kernel<Io, Gate, V, SHARED, MIX><<<cut.K, kNarrowBlock, 0, s>>>(a, cut);
            return launch_status("recur_narrow_again_kernel");
        }
    }
    recur_narrow_kernel<Io, Gate, Y, V, SHARED, MIX, BWD, false><<<cut.K, kNarrowBlock, 0, s>>>(a, cut);
    return launch_status("recur_narrow_kernel");
}

template <typename Io, typename Gate, typename Y, bool MIX, bool BWD>
int launch_lanes(const RecurArgs &a, const RecurPlan &p, const Cut &cut, hipStream_t s) {
    const bool shared = a.G == 1;
    constexpr bool low = std::is_same_v<Y, LowHalf>;           // rows of more than four channels (states_of)
#define CNGP_RECUR(BLOCK, CL, V, RB)                                                      \
    return shared ? launch_scan<Io, Gate, Y, BLOCK, CL, V, RB, true, MIX, BWD>(a, p, cut, s) \
                  : launch_scan<Io, Gate, Y, BLOCK, CL, V, RB, false, MIX, BWD>(a, p, cut, s)
    if constexpr (!low) if (p.CL == 1) {
#define CNGP_NARROW(V) return shared ? launch_narrow<Io, Gate, Y, V, true, MIX, BWD>(a, cut, s) : launch_narrow<Io, Gate, Y, V, false, MIX, BWD>(a, cut, s)
        if (a.C == 1) return launch_narrow<Io, Gate, Y, 1, true, MIX, BWD>(a, cut, s);
        if (a.C == 2) CNGP_NARROW(2);
        if (a.C == 3) CNGP_NARROW(3);
        CNGP_NARROW(4);
#undef CNGP_NARROW
    }
    if (p.block == kWideBlock) CNGP_RECUR(kWideBlock, 16, 2, (BWD ? 1 : 2) * kRowsEach);
    if (p.CL == 8) CNGP_RECUR(kRecurBlock, 8, 1, kRowsEach);
    if (p.CL == 16) CNGP_RECUR(kRecurBlock, 16, 1, kRowsEach);
    if (p.V == 1) CNGP_RECUR(kRecurBlock, 32, 1, kRowsEach);
    CNGP_RECUR(kRecurBlock, 32, 2, kRowsEach);
#undef CNGP_RECUR
}

template <typename Io, typename Gate, bool BWD>
int launch_inputs(const RecurArgs &a, const RecurPlan &p, const Cut &cut, hipStream_t s) {
    const bool mix = a.flags & CNGP_RECUR_MIX;
    const auto launch = [&](auto y) {
        using Y = decltype(y);
        return mix ? launch_lanes<Io, Gate, Y, true, BWD>(a, p, cut, s) : launch_lanes<Io, Gate, Y, false, BWD>(a, p, cut, s);
    };
    if constexpr (sizeof(Io) != sizeof(float)) {
        if constexpr (sizeof(Gate) != sizeof(float))
            if (a.states == STATES_LOW) return launch(LowHalf{});
        if constexpr (!BWD)
            if (a.states == STATES_Y) return launch(Io{});     // the backward pass never has states in fp16
    }
    return launch(float{});
}

}  // namespace

// One direction's launches.  state_in / state_out: what a sequence starts from and where it ends up; where they are one array and
// sequences are cut, the workgroup that ends a sequence is not the one that starts it, so the start is taken from a copy.
template <bool BWD>
int cngp::recur_launch(const cngp_recur_config *c, RecurArgs a, const RecurPlan &p, const RecurSpace &sp, char *ws, hipStream_t s) {
    if ((int64_t)p.K * p.tiles > 0x7fffffffLL) return CNGP_ERR_UNSUPPORTED;
    Cut cut{(pos)p.R, p.K, (float *)(ws + sp.piece_a), (float *)(ws + sp.piece_b), (float *)(ws + sp.carry), (int32_t *)(ws + sp.piece_cut), p.exact};
    const float *&in = BWD ? a.dlast : a.h0;
    float        *out = BWD ? a.dh0 : a.last;
    if (p.exact && in && in == out) {
        float        *copy = (float *)(ws + sp.state);
        if (int rc = recur_copy(in, copy, (int64_t)a.S * a.C, s)) return rc;
        in = copy;
    }
    const bool io16 = c->io_dtype == CNGP_F16, g16 = c->gate_dtype == CNGP_F16;
    return io16 ? (g16 ? launch_inputs<__half, __half, BWD>(a, p, cut, s) : launch_inputs<__half, float, BWD>(a, p, cut, s))
                : (g16 ? launch_inputs<float, __half, BWD>(a, p, cut, s) : launch_inputs<float, float, BWD>(a, p, cut, s));
}

