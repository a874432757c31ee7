// Lookup of codes with scaling, and its gradient by sorted ids.
//
//     y[n] = base[n] + scale * table[ids[n]]          grad[r] += scale * sum over n with ids[n] == r of dy[n]
//
// The gradient needs, per row of the table, the points that chose it.  Float atomics would give sums whose order, hence bits, change
// from call to call, and frequent ids would queue at one address; so the ids are sorted (stable, with their positions), and the rows
// of dy that belong to one id are added up in the order of the points.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "cngp_launch.h"
#include "cngp_radix.h"

namespace {

using namespace cngp;

constexpr int kEmbBlock = 256;

__device__ __forceinline__ float load(const float *p, const int64_t i) { return p[i]; }
__device__ __forceinline__ float load(const __half *p, const int64_t i) { return __half2float(p[i]); }
__device__ __forceinline__ void store(float *p, const int64_t i, const float v) { p[i] = v; }
__device__ __forceinline__ void store(__half *p, const int64_t i, const float v) { p[i] = __float2half_rn(v); }

// The row an id names, or `rows` for padding.
template <typename Id>
__device__ __forceinline__ uint32_t row_of(const Id id, const int64_t rows) {
    return id >= 0 && (int64_t)id < rows ? (uint32_t)id : (uint32_t)rows;
}

// V neighbouring values at once, on whatever boundary they start: global memory takes that, the compiler makes one access of it.
template <typename T, int N>
struct Run { T e[N]; };
template <typename T, int V>
__device__ __forceinline__ void load_run(float (&out)[V], const T *p) {
    Run<T, V> r;
    __builtin_memcpy(&r, p, sizeof r);
#pragma unroll
    for (int v = 0; v < V; ++v) out[v] = load(r.e, v);
}
template <typename T, int V>
__device__ __forceinline__ void store_run(T *p, const float (&in)[V]) {
    Run<T, V> r;
#pragma unroll
    for (int v = 0; v < V; ++v) store(r.e, v, in[v]);
    __builtin_memcpy(p, &r, sizeof r);
}

// Where V does not divide the width (EVEN false), a row's last lane takes its last V columns and leaves the first `skip` of them, which
// another lane has, as they are.  Kernels of their own: with `skip` the lookup of 10^6 rows of 64 took 97 us in place of 85.
template <typename T, int V>
__device__ __forceinline__ void store_own(T *p, const float (&in)[V], const int skip) {
    if (skip == 0) {
        store_run<T, V>(p, in);
    } else {
#pragma unroll
        for (int v = 1; v < V; ++v)
            if (v >= skip) store(p, v, in[v]);
    }
}

// ---------------------------------------------------------------- lookup
// A workgroup takes `rows_each` points, a lane V neighbouring columns of a point at a time, kEmbAhead of them in flight: the id and the
// row it names are two loads one behind the other.  per_row = dim / V, rounded up; i / per_row as a multiplication.
// 10^6 of 2^20 rows of 64 fp32: 85 us for 516 MB, memory.
constexpr int kEmbAhead = 4;
template <typename Id, typename Table, typename Io, int V, bool EVEN>
__global__ __launch_bounds__(kEmbBlock) void embed_fwd_kernel(const Id *__restrict__ ids, const Table *__restrict__ table, const Io *base, Io *y,
                                                              const int64_t N, const int64_t rows, const int dim, const uint32_t per_row,
                                                              const uint32_t inverse, const uint32_t rows_each, const float scale)
{
    const int64_t  n0 = (int64_t)blockIdx.x * rows_each;
    const uint32_t mine = N - n0 < (int64_t)rows_each ? (uint32_t)(N - n0) : rows_each, items = mine * per_row;
    for (uint32_t i0 = threadIdx.x; i0 < items; i0 += kEmbBlock * kEmbAhead) {
        uint32_t n[kEmbAhead], c[kEmbAhead], r[kEmbAhead];
        int      skip[kEmbAhead];
        float    row[kEmbAhead][V], b[kEmbAhead][V];
#pragma unroll
        for (int u = 0; u < kEmbAhead; ++u) {
            const uint32_t i = i0 + u * kEmbBlock < items ? i0 + u * kEmbBlock : i0;
            n[u] = per_row == 1 ? i : mine == 1 ? 0u : __umulhi(i, inverse);
            c[u] = (i - n[u] * per_row) * V;
            skip[u] = !EVEN && c[u] + V > (uint32_t)dim ? (int)(c[u] + V) - dim : 0;
            c[u] -= (uint32_t)skip[u];
            r[u] = row_of(ids[n0 + n[u]], rows);
        }
#pragma unroll
        for (int u = 0; u < kEmbAhead; ++u) {
            load_run<Table, V>(row[u], table + (int64_t)(r[u] < (uint32_t)rows ? r[u] : 0u) * dim + c[u]);
            if (base) load_run<Io, V>(b[u], base + (n0 + n[u]) * dim + c[u]);
        }
#pragma unroll
        for (int u = 0; u < kEmbAhead; ++u) {
            if (u && i0 + u * kEmbBlock >= items) break;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float start = base ? b[u][v] : 0.0f;
                b[u][v] = r[u] < (uint32_t)rows ? fmaf(scale, row[u][v], start) : start;
            }
            store_own<Io, V>(y + (n0 + n[u]) * dim + c[u], b[u], skip[u]);
        }
    }
}

// Values [lo, hi) of the gradient cleared by a workgroup.  Where ids are sorted, the first kernel of the sort does it beside its own work, which
// is latency (16381 ids and 50000 rows of 1024: 27 us of clearing hide the sort's 14).
template <int BLOCK>
__device__ __forceinline__ void clear_values(float *__restrict__ grad, const int64_t lo, const int64_t hi) {
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t i = lo + (int64_t)threadIdx.x * 4; i < hi; i += BLOCK * 4) {
        if (i + 4 <= hi) store_run<float, 4>(grad + i, zero);
        else for (int64_t j = i; j < hi; ++j) grad[j] = 0.0f;
    }
}

__global__ __launch_bounds__(kEmbBlock) void embed_clear_kernel(float *__restrict__ grad, const int64_t n, const int64_t each)
{
    const int64_t lo = (int64_t)blockIdx.x * each;
    clear_values<kEmbBlock>(grad, lo, lo + each < n ? lo + each : n);
}

// ---------------------------------------------------------------- sort of the ids
template <typename Id, int ROUNDS, bool PREFIX>
__global__ __launch_bounds__(kTileBlock) void embed_keys_kernel(const Id *__restrict__ ids, uint32_t *__restrict__ keys, const int64_t N, const int64_t rows,
                                                                uint32_t *__restrict__ counts, const int64_t tiles, float *__restrict__ grad,
                                                                const int64_t values)
{
    __shared__ uint32_t hist[kTileWaves * kDigits];
    if (grad) {
        const int64_t each = ((values + tiles - 1) / tiles + 3) / 4 * 4, lo = each * blockIdx.x;
        clear_values<kTileBlock>(grad, lo, lo + each < values ? lo + each : values);
    }
    const int     t = threadIdx.x, w = t >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * (kTileBlock * ROUNDS);
    for (int i = t; i < kTileWaves * kDigits; i += kTileBlock) hist[i] = 0;
    __syncthreads();
    uint32_t key[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t n = n0 + (int64_t)r * kTileBlock + t;
        key[r] = n < N ? row_of(ids[n], rows) : 0u;
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t n = n0 + (int64_t)r * kTileBlock + t;
        if (n < N) {
            keys[n] = key[r];
            atomicAdd(&hist[w * kDigits + (key[r] & (kDigits - 1))], 1u);
        }
    }
    __syncthreads();
    flush_tile_histogram<PREFIX>(hist, counts, tiles, blockIdx.x, t);
}

// Up to 16384 ids are sorted in one launch (the passes above are three launches each, of which a short batch fills a few workgroups).
// Workgroup g owns an equal share of the keys: it reads all ids, keeps its own in their order, counts the smaller ones -- that is where its
// share starts -- and sorts its share in LDS.  Nothing waits for another workgroup; ids that crowd in one share cost that one time.
// The sort is stable, eight bits at a time: a wavefront ranks its strip 64 elements at a time, lanes with equal digits find each other
// by ballots; per digit the wavefronts' counts become their places.
constexpr int kSmallBlock = 1024, kSmallWaves = kSmallBlock / 64, kSmallBits = 8, kSmallDigits = 1 << kSmallBits, kSmallRounds = 16,
              kSmallMost = kSmallBlock * kSmallRounds;
template <typename Id>
__global__ __launch_bounds__(kSmallBlock) void embed_sort_small_kernel(const Id *__restrict__ ids, uint32_t *__restrict__ keys, int32_t *__restrict__ from,
                                                                       const int N, const int64_t rows, const uint32_t share, float *__restrict__ grad,
                                                                       const int dim)
{
    extern __shared__ __align__(16) uint32_t small_lds[];      // counts [waves][digits], then keys and points of the share, N each
    uint32_t *wave_count = small_lds, *stage_key = small_lds + kSmallWaves * kSmallDigits, *stage_from = stage_key + kSmallMost;
    __shared__ uint32_t sums[kSmallDigits / 64], wave_mine[kSmallRounds][kSmallWaves], wave_less[kSmallWaves];
    const int      t = threadIdx.x, w = t >> 6, lane = t & 63;
    const uint64_t below = lane ? (~0ull >> (64 - lane)) : 0ull;
    const uint32_t key_lo = blockIdx.x * share, key_hi = key_lo + share;
    const int      rounds = (N + kSmallBlock - 1) / kSmallBlock;
    if (grad) clear_values<kSmallBlock>(grad, (int64_t)key_lo * dim, (key_hi < rows ? (int64_t)key_hi : rows) * dim);

    // the ids of the share, in their order: round r, wavefront w, lane
    uint32_t key[kSmallRounds], less = 0;
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
        const int n = r * kSmallBlock + t;
        key[r] = r < rounds && n < N ? row_of(ids[n], rows) : 0xffffffffu;
    }
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
        if (r < rounds) {
            const uint64_t mine = __ballot(key[r] >= key_lo && key[r] < key_hi);
            less += (uint32_t)__popcll(__ballot(key[r] < key_lo));
            if (lane == 0) wave_mine[r][w] = (uint32_t)__popcll(mine);
        }
    }
    if (lane == 0) wave_less[w] = less;
    __syncthreads();
    uint32_t base = 0;                                         // where the share starts among the sorted ids
#pragma unroll
    for (int k = 0; k < kSmallWaves; ++k) base += wave_less[k];
    // counts of (round, wavefront) -> places, by the first four wavefronts
    if (t < kSmallRounds * kSmallWaves) {
        const uint32_t c = t < rounds * kSmallWaves ? (&wave_mine[0][0])[t] : 0u;
        uint32_t       sum;
        const uint32_t before = wave_exclusive_scan(c, &sum);
        if (lane == 0) sums[w] = sum;
        (&wave_mine[0][0])[t] = before;
    }
    __syncthreads();
    const uint32_t s0 = sums[0], s1 = s0 + sums[1], s2 = s1 + sums[2], total = s2 + sums[3];
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
        const bool     in = key[r] >= key_lo && key[r] < key_hi;
        const uint64_t mine = __ballot(in);
        const int      part = (r * kSmallWaves + w) >> 6;
        if (in) {
            const uint32_t to = wave_mine[r][w] + (part == 0 ? 0u : part == 1 ? s0 : part == 2 ? s1 : s2) + (uint32_t)__popcll(mine & below);
            stage_key[to] = key[r] - key_lo;
            stage_from[to] = (uint32_t)(r * kSmallBlock + t);
        }
    }
    __syncthreads();

    const int strips = (int)((total + kSmallBlock - 1) / kSmallBlock), n0 = w * strips * 64 + lane;      // rounds of a wavefront's strip
    uint32_t at[kSmallRounds], slot[kSmallRounds];
    for (int shift = 0; shift < 32 && ((share - 1) >> shift); shift += kSmallBits) {
#pragma unroll
        for (int r = 0; r < kSmallRounds; ++r) {
            const uint32_t n = (uint32_t)(n0 + r * 64);
            const bool     there = r < strips && n < total;
            key[r] = there ? stage_key[n] : 0xffffffffu;
            at[r] = there ? stage_from[n] : 0u;
        }
        for (int i = t; i < kSmallWaves * kSmallDigits; i += kSmallBlock) wave_count[i] = 0;
        __syncthreads();
        uint32_t *mine = wave_count + w * kSmallDigits;
#pragma unroll
        for (int r = 0; r < kSmallRounds; ++r) {
            if (r < strips) {
                const bool     valid = (uint32_t)(n0 + r * 64) < total;
                const uint32_t digit = (key[r] >> shift) & (kSmallDigits - 1);
                uint64_t       peers = __ballot(valid);
    #pragma unroll
                for (int b = 0; b < kSmallBits; ++b) {
                    const bool     bit = (digit >> b) & 1u;
                    const uint64_t has = __ballot(bit);
                    peers &= bit ? has : ~has;
                }
                if (valid) {
                    const uint32_t seen = mine[digit];
                    slot[r] = seen + (uint32_t)__popcll(peers & below);
                    if ((peers & below) == 0) mine[digit] = seen + (uint32_t)__popcll(peers);
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        __syncthreads();
        uint32_t count = 0, before = 0, sum = 0;
        if (t < kSmallDigits) {
#pragma unroll
            for (int k = 0; k < kSmallWaves; ++k) {
                const uint32_t c = wave_count[k * kSmallDigits + t];
                wave_count[k * kSmallDigits + t] = count;
                count += c;
            }
            before = wave_exclusive_scan(count, &sum);
            if (lane == 0) sums[w] = sum;
        }
        __syncthreads();
        if (t < kSmallDigits) {
            for (int k = 0; k < w; ++k) before += sums[k];
#pragma unroll
            for (int k = 0; k < kSmallWaves; ++k) wave_count[k * kSmallDigits + t] += before;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSmallRounds; ++r) {
            if (r < strips && (uint32_t)(n0 + r * 64) < total) {
                const uint32_t to = mine[(key[r] >> shift) & (kSmallDigits - 1)] + slot[r];
                stage_key[to] = key[r];
                stage_from[to] = at[r];
            }
        }
        __syncthreads();
    }
    for (uint32_t i = t; i < total; i += kSmallBlock) {
        keys[base + i] = stage_key[i] + key_lo;
        from[base + i] = (int32_t)stage_from[i];
    }
}

// ---------------------------------------------------------------- sums of the rows of an id
// The sorted positions are cut into pieces of `piece` positions, a wavefront each; its lanes are row lanes of LPR lanes that hold V
// columns each, and a row lane walks piece / (64 / LPR) positions, kSumAhead rows in flight.  An id whose positions lie inside a piece
// is summed and written there.  One that reaches over a piece's edges leaves a partial sum at each piece it touches -- `tail` where it
// starts, `head` where it came from before -- and embed_join_kernel adds those up: always in the order of the positions.
// 10^6 ids of 2^20 rows of 64 fp32: 108 us for 429 MB, memory (rows are gathered in 256-byte pieces).
constexpr int kSumAhead = 8;

struct SumArgs {
    const uint32_t *keys;
    const int32_t  *from;
    const void     *dy;
    float          *grad, *head, *tail;  // head, tail: [pieces][dim]
    int64_t         N, rows;
    uint32_t        piece, pieces;
    int             dim, accumulate;
    float           scale;
};

template <int V>
__device__ __forceinline__ void put_row(const SumArgs &a, const uint32_t key, const int c, const int skip, float (&sum)[V]) {
    float *to = a.grad + (int64_t)key * a.dim + c;
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] *= a.scale;
    if (a.accumulate) {
        float old[V];
        load_run<float, V>(old, to);
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += old[v];
    }
    store_own<float, V>(to, sum, skip);
}

template <typename Io, int V, int LPR, bool EVEN>
__global__ __launch_bounds__(kEmbBlock) void embed_sums_kernel(const SumArgs a)
{
    constexpr int  RL = 64 / LPR;                              // row lanes of a wavefront
    const int      lane = threadIdx.x & 63, cl = lane % LPR, rl = lane / LPR;
    const uint32_t piece = blockIdx.x * (kEmbBlock / 64) + (threadIdx.x >> 6);
    if (piece >= a.pieces) return;
    const int      c_first = ((int)blockIdx.y * LPR + cl) * V;
    const bool     c_ok = c_first < a.dim;
    const int      skip = !EVEN && c_ok && c_first + V > a.dim ? c_first + V - a.dim : 0, c = c_ok ? c_first - skip : 0;
    const uint32_t each = a.piece / RL;
    const int64_t  w0 = (int64_t)piece * a.piece, w1 = w0 + a.piece < a.N ? w0 + a.piece : a.N;
    const int64_t  p0 = w0 + (int64_t)rl * each < w1 ? w0 + (int64_t)rl * each : w1, p1 = p0 + each < w1 ? p0 + each : w1;

    // this row lane's first run (which may have begun before it) in `first`, its last one (which may go on) in `sum`
    float    sum[V], first[V];
    uint32_t key = 0, key0 = 0;
    bool     one_run = true;
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = first[v] = 0.0f;
    for (int64_t p = p0; p < p1; p += kSumAhead) {
        uint32_t k[kSumAhead];
        int32_t  n[kSumAhead];
        float    row[kSumAhead][V];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) {
            const int64_t at = p + u < p1 ? p + u : p1 - 1;
            k[u] = a.keys[at];
            n[u] = a.from[at];
        }
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) load_run<Io, V>(row[u], (const Io *)a.dy + (int64_t)n[u] * a.dim + c);
        if (p == p0) key = key0 = k[0];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) {
            if (p + u >= p1) break;
            if (k[u] != key) {                                 // a run ends
                if (one_run) {
#pragma unroll
                    for (int v = 0; v < V; ++v) first[v] = sum[v];
                } else if (c_ok) {
                    put_row<V>(a, key, c, skip, sum);                // began and ended in here: no padding, a larger key follows
                }
                one_run = false;
                key = k[u];
#pragma unroll
                for (int v = 0; v < V; ++v) sum[v] = 0.0f;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += row[u][v];
        }
    }
    // what reaches a row lane from those before it: a lane that is one run that came and goes on passes it on with its own sum added
    const bool     some = p0 < p1;
    const uint32_t none = 0xffffffffu;
    const uint32_t came = some && p0 > 0 ? a.keys[p0 - 1] : none, follows = some && p1 < a.N ? a.keys[p1] : none;
    const bool     from_before = some && came == key0, goes_on = some && follows == key;
    const bool     through = one_run && from_before && goes_on;
    float          reach[V], open[V];                          // open: the sum that leaves this row lane
    bool           chain = through;                            // whether `open` still misses what reaches the lanes it spans
#pragma unroll
    for (int v = 0; v < V; ++v) open[v] = goes_on ? sum[v] : 0.0f;
#pragma unroll
    for (int d = 1; d < RL; d <<= 1) {
        const bool lc = __shfl_up((int)chain, d * LPR, 64) != 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float l = __shfl_up(open[v], d * LPR, 64);
            if (rl >= d && chain) open[v] += l;
        }
        if (rl >= d) chain = chain && lc;
    }
    bool reach_chain = false;                                  // what reaches has itself come from before the piece
    if (RL > 1) reach_chain = __shfl_up((int)chain, LPR, 64) != 0;
#pragma unroll
    for (int v = 0; v < V; ++v) reach[v] = RL > 1 ? __shfl_up(open[v], LPR, 64) : 0.0f;
    if (rl == 0) {
        reach_chain = true;
#pragma unroll
        for (int v = 0; v < V; ++v) reach[v] = 0.0f;
    }
    if (!some || !c_ok) return;
    const bool last_lane = p1 == w1;
    if (!one_run || !goes_on) {                                // the first run ends in here
        float total[V];
#pragma unroll
        for (int v = 0; v < V; ++v) total[v] = (from_before ? reach[v] : 0.0f) + (one_run ? sum[v] : first[v]);
        if (from_before && reach_chain) {
            store_own<float, V>(a.head + (int64_t)piece * a.dim + c, total, skip);
        } else if (key0 < (uint32_t)a.rows) {
            put_row<V>(a, key0, c, skip, total);
        }
    }
    if (!one_run && !goes_on && key < (uint32_t)a.rows) put_row<V>(a, key, c, skip, sum);
    if (goes_on && last_lane) {                                // the last run leaves the piece
        float *to = through && reach_chain ? a.head : a.tail;  // one that also came from before it is all head
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = through ? reach[v] + sum[v] : sum[v];
        store_own<float, V>(to + (int64_t)piece * a.dim + c, sum, skip);
    }
}

// First position of the sorted keys that is not below `key`, from `lo` on; a wavefront together, 64 probes at a time.
__device__ __forceinline__ int64_t first_at(const uint32_t *__restrict__ keys, int64_t lo, const int64_t N, const uint32_t key) {
    int64_t       hi = N;
    const int64_t lane = threadIdx.x & 63;
    while (lo < hi) {
        const int64_t  step = (hi - lo + 63) / 64, probe = lo + lane * step;
        const uint64_t less = __ballot(probe < hi && keys[probe < hi ? probe : hi - 1] < key);
        if (!less) { hi = lo; break; }
        const int64_t last = lo + (63 - __clzll(less)) * step;
        lo = last + 1;
        hi = last + step < hi ? last + step : hi;
    }
    return lo;
}

// Ids that reach over pieces: the workgroup of the piece in which one starts adds its tail and the heads of the pieces up to its end,
// its wavefronts every fourth step of them.  16381 ids of 50000 rows of 1024, few of them frequent: 5.6 us.
template <int V, int LPR, bool EVEN>
__global__ __launch_bounds__(kEmbBlock) void embed_join_kernel(const SumArgs a)
{
    constexpr int  RL = 64 / LPR, W = kEmbBlock / 64, AHEAD = V == 8 ? 4 : 8;
    __shared__ float part[W][64 * V];
    const int      lane = threadIdx.x & 63, w = threadIdx.x >> 6, cl = lane % LPR, rl = lane / LPR;
    const uint32_t piece = blockIdx.x;
    const int64_t  w0 = (int64_t)piece * a.piece, w1 = w0 + a.piece;       // not the last piece: all its positions are there
    const uint32_t key = a.keys[w1 - 1], follows = a.keys[w1], came = w0 > 0 ? a.keys[w0 - 1] : 0xffffffffu;
    if (follows != key || key >= (uint32_t)a.rows || came == key) return;  // none starts here and goes on
    const uint32_t end = (uint32_t)((first_at(a.keys, w1, a.N, key + 1u) - 1) / a.piece);               // the piece it ends in
    const int      c_first = ((int)blockIdx.y * LPR + cl) * V;
    const bool     c_ok = c_first < a.dim;
    const int      skip = !EVEN && c_ok && c_first + V > a.dim ? c_first + V - a.dim : 0, c = c_ok ? c_first - skip : 0;
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.0f;
    if (w == 0 && rl == 0) load_run<float, V>(sum, a.tail + (int64_t)piece * a.dim + c);
    for (uint32_t q = piece + 1 + (uint32_t)w * RL * AHEAD + rl; q <= end; q += W * RL * AHEAD) {
        float h[AHEAD][V];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load_run<float, V>(h[u], a.head + (int64_t)(q + u * RL <= end ? q + u * RL : q) * a.dim + c);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += u == 0 || q + u * RL <= end ? h[u][v] : 0.0f;
    }
#pragma unroll
    for (int d = LPR; d < 64; d <<= 1)
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += __shfl_xor(sum[v], d, 64);
#pragma unroll
    for (int v = 0; v < V; ++v) part[w][v * 64 + lane] = sum[v];
    __syncthreads();
    if (w != 0 || rl != 0 || !c_ok) return;
#pragma unroll
    for (int i = 1; i < W; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] += part[i][v * 64 + lane];
    put_row<V>(a, key, c, skip, sum);
}

int check(const cngp_embed_config *c, int64_t N) {
    if (!c) return CNGP_ERR_NULL;
    if (c->rows < 1 || c->rows > 0x7ffffffeLL || c->dim < 1 || c->dim > 65536) return CNGP_ERR_INVALID;
    if (c->table_dtype != CNGP_F32 && c->table_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->io_dtype != CNGP_F32 && c->io_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->id_dtype != CNGP_I32 && c->id_dtype != CNGP_I64) return CNGP_ERR_INVALID;
    if (!std::isfinite(c->scale) || (c->flags & ~(uint32_t)CNGP_ZERO_GRADS)) return CNGP_ERR_INVALID;
    if (N < 0 || N > 0x7fffffffLL) return CNGP_ERR_INVALID;
    return CNGP_OK;
}

// Columns of a lane: 16 bytes of the array that is gathered, or what fits the width.
int columns_of(int dim, int most) {
    int v = most;
    while (v > dim) v >>= 1;
    return v;
}

// Lanes to a row of the gradient, `columns` values each.
int lanes_of(int dim, int columns) {
    const int n = (dim + columns - 1) / columns;
    return n <= 1 ? 1 : n <= 4 ? 4 : n <= 16 ? 16 : 64;
}

// Positions of a piece: eight per row lane (what is in flight), or as many as leave kSumWaves wavefronts over pieces and column tiles; up to 64
// to a row lane where that is all of them, which then need not be joined.  More wavefronts leave an id of many points more partial sums to
// join.  2048, 4096 and 8192 of them, lookup and gradient: 79620 points of one row of 113 68, 97 and 162 us, 16381 of 50000 rows of 1024 71, 75
// and 75, 10^6 of 2^20 rows of 64 284, 285 and 292; 1024 of them 55, 72 and 301.
constexpr int64_t kSumWaves = 2048;
uint32_t piece_of(const cngp_embed_config *c, int64_t N) {
    const int     columns = columns_of(c->dim, c->io_dtype == CNGP_F16 ? 8 : 4), lpr = lanes_of(c->dim, columns), rl = 64 / lpr;
    const int64_t tiles = ((c->dim + columns - 1) / columns + lpr - 1) / lpr, each = (N * tiles / rl + kSumWaves - 1) / kSumWaves;
    return (uint32_t)((N <= 64 * rl ? std::max<int64_t>((N + rl - 1) / rl, 1) : std::max<int64_t>(each, kSumAhead)) * rl);
}

// Elements per lane of the sort's tiles: sixteen once those fill the chip, four for shorter batches.
int rounds_of(int64_t N) { return N >= (int64_t)512 * kTile ? kRounds : 4; }

struct EmbedSpace { size_t keys_a, keys_b, from_a, from_b, counts, totals, head, tail, bytes; };
EmbedSpace space_of(const cngp_embed_config *c, int64_t N) {
    EmbedSpace s{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
    if (!N) return s;
    const size_t col = (size_t)N * 4, piece = piece_of(c, N), pieces = ((size_t)N + piece - 1) / piece;
    s.keys_a = take(col);
    s.from_a = take(col);
    if (N > kSmallMost) {
        s.keys_b = take(col);
        s.from_b = take(col);
        s.counts = take((size_t)kDigits * (size_t)((N + kTileBlock * rounds_of(N) - 1) / (kTileBlock * rounds_of(N))) * 4);
        s.totals = take((size_t)kDigits * 4);
    }
    s.head = take(pieces * (size_t)c->dim * 4);
    s.tail = take(pieces * (size_t)c->dim * 4);
    s.bytes = at;
    return s;
}

// Shares of the keys 0 .. rows: a workgroup for every 64 ids or 64 KB of table to clear, at most one per CU (each reads all ids; a share of 256
// keys is one pass).
template <typename Id>
int sort_small(const void *ids, uint32_t *keys, int32_t *from, int64_t N, int64_t rows, int dim, float *clear, hipStream_t s) {
    constexpr size_t lds = (size_t)(kSmallWaves * kSmallDigits + 2 * kSmallMost) * 4;
    if (hipError_t e = hipFuncSetAttribute((const void *)embed_sort_small_kernel<Id>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds))
        return record_hip_failure(e, "hipFuncSetAttribute(MaxDynamicSharedMemorySize)");
    const int64_t wanted = std::max<int64_t>((N + 63) / 64, clear ? rows * dim / 16384 : 0);
    const int64_t groups = std::min<int64_t>(std::max<int64_t>(wanted, 1), 256), share = (rows + 1 + groups - 1) / groups;
    embed_sort_small_kernel<Id><<<(unsigned)((rows + 1 + share - 1) / share), kSmallBlock, lds, s>>>((const Id *)ids, keys, from, (int)N, rows, (uint32_t)share,
                                                                                                    clear, dim);
    return launch_status("embed_sort_small_kernel");
}

template <typename Id, int ROUNDS, bool PREFIX>
int sort_passes(const void *ids, int64_t N, int64_t rows, int dim, float *clear, uint32_t *(&keys)[2], int32_t *(&from)[2], uint32_t *counts, uint32_t *totals,
                int *at, hipStream_t s) {
    constexpr int  TILE = kTileBlock * ROUNDS;
    const unsigned tiles = (unsigned)((N + TILE - 1) / TILE);
    embed_keys_kernel<Id, ROUNDS, PREFIX><<<tiles, kTileBlock, 0, s>>>((const Id *)ids, keys[0], N, rows, counts, tiles, clear, rows * dim);
    if (int rc = launch_status("embed_keys_kernel")) return rc;
    for (int shift = 0; shift < 32 && ((uint64_t)rows >> shift); shift += kDigitBits, *at ^= 1) {
        if (shift) {
            digit_count_kernel<ROUNDS, PREFIX><<<tiles, kTileBlock, 0, s>>>(keys[*at], N, shift, counts, tiles);
            if (int rc = launch_status("digit_count_kernel")) return rc;
        }
        if (!PREFIX) {
            digit_row_scan_kernel<<<kDigits, kScanBlock, 0, s>>>(counts, tiles, totals);
            if (int rc = launch_status("digit_row_scan_kernel")) return rc;
        }
        digit_scatter_kernel<ROUNDS, PREFIX><<<tiles, kTileBlock, 0, s>>>(keys[*at], shift ? from[*at] : nullptr, N, shift, counts, tiles, totals, keys[*at ^ 1],
                                                                          from[*at ^ 1]);
        if (int rc = launch_status("digit_scatter_kernel")) return rc;
    }
    return CNGP_OK;
}

int clear_table(float *grad, int64_t n, hipStream_t s) {
    const int64_t each = std::max<int64_t>((n + 8191) / 8192 / 4 * 4 + 4, kEmbBlock * 4);
    LaunchTimer   t(s, K_ZERO);
    embed_clear_kernel<<<(unsigned)((n + each - 1) / each), kEmbBlock, 0, s>>>(grad, n, each);
    return launch_status("embed_clear_kernel");
}

// Sorted keys and the points they came from (and `clear`, if given, set to zero), in keys[0] and from[0] or, after an odd number of passes, [1]: *at says which.
template <typename Id>
int sort_ids(const void *ids, int64_t N, int64_t rows, int dim, float *clear, uint32_t *(&keys)[2], int32_t *(&from)[2], uint32_t *counts, uint32_t *totals, int *at, hipStream_t s) {
    LaunchTimer t(s, K_EMBED_SORT);
    *at = 0;
    if (N <= kSmallMost) return sort_small<Id>(ids, keys[0], from[0], N, rows, dim, clear, s);
    if (N <= (int64_t)kPrefixTiles * kTileBlock * 4) return sort_passes<Id, 4, true>(ids, N, rows, dim, clear, keys, from, counts, totals, at, s);
    // a longer sort fills the chip by itself: cleared beside its first kernel, 2^20 rows of 64 took 299 us in place of 289
    if (clear)
        if (int rc = clear_table(clear, rows * dim, s)) return rc;
    return rounds_of(N) == kRounds ? sort_passes<Id, kRounds, false>(ids, N, rows, dim, nullptr, keys, from, counts, totals, at, s)
                                   : sort_passes<Id, 4, false>(ids, N, rows, dim, nullptr, keys, from, counts, totals, at, s);
}

template <typename Io, int V, int LPR, bool EVEN>
int sum_pieces(const SumArgs &a, hipStream_t s) {
    const unsigned columns = (unsigned)(((a.dim + V - 1) / V + LPR - 1) / LPR), groups = (a.pieces + kEmbBlock / 64 - 1) / (kEmbBlock / 64);
    LaunchTimer t(s, K_EMBED_SUMS);
    embed_sums_kernel<Io, V, LPR, EVEN><<<dim3(groups, columns), kEmbBlock, 0, s>>>(a);
    if (int rc = launch_status("embed_sums_kernel")) return rc;
    if (a.pieces < 2) return CNGP_OK;
    embed_join_kernel<V, LPR, EVEN><<<dim3(a.pieces - 1, columns), kEmbBlock, 0, s>>>(a);
    return launch_status("embed_join_kernel");
}
template <typename Io, int V, int LPR>
int sum_rows(const SumArgs &a, hipStream_t s) {
    if constexpr (V > 1)
        if (a.dim % V) return sum_pieces<Io, V, LPR, false>(a, s);
    return sum_pieces<Io, V, LPR, true>(a, s);
}
template <typename Io, int V>
int sum_columns(const SumArgs &a, hipStream_t s) {
    switch (lanes_of(a.dim, V)) {
    case 1:  return sum_rows<Io, V, 1>(a, s);
    case 4:  return sum_rows<Io, V, 4>(a, s);
    case 16: return sum_rows<Io, V, 16>(a, s);
    default: return sum_rows<Io, V, 64>(a, s);
    }
}

template <typename Id, typename Table, typename Io, int V>
int look_up(const cngp_embed_config *c, const void *ids, int64_t N, const void *table, const void *base, void *y, hipStream_t s) {
    const uint32_t per_row = (uint32_t)((c->dim + V - 1) / V), rows_each = std::max(1u, (uint32_t)(kEmbBlock * kEmbAhead) / per_row);
    // the smallest multiplier that divides every i below rows_each * per_row <= 1024 exactly (one point, or one value to a point, need none)
    const uint32_t inverse = (uint32_t)((0x100000000ull + per_row - 1) / per_row);      // not used for per_row = 1
    LaunchTimer t(s, K_EMBED_FWD);
    const auto launch = [&](auto kernel) {
        const int64_t most = kMostGroups256 * rows_each;       // points of a launch: more than there are, but for 2^24 rows and more of at least 513 vectors
        for (int64_t n = 0; n < N; n += most) {
            const int64_t here = std::min(most, N - n), at = n * c->dim;
            kernel<<<(unsigned)((here + rows_each - 1) / rows_each), kEmbBlock, 0, s>>>((const Id *)ids + n, (const Table *)table, base ? (const Io *)base + at : nullptr,
                                                                                      (Io *)y + at, here, c->rows, c->dim, per_row, inverse, rows_each, c->scale);
            if (int rc = launch_status("embed_fwd_kernel")) return rc;
        }
        return (int)CNGP_OK;
    };
    return c->dim % V == 0 ? launch(embed_fwd_kernel<Id, Table, Io, V, true>) : launch(embed_fwd_kernel<Id, Table, Io, V, V == 1>);
}
template <typename Id, typename Table, typename Io>
int look_up_columns(const cngp_embed_config *c, const void *ids, int64_t N, const void *table, const void *base, void *y, hipStream_t s) {
    switch (columns_of(c->dim, 16 / (int)std::max(sizeof(Table), sizeof(Io)))) {
    case 8:  return look_up<Id, Table, Io, 8>(c, ids, N, table, base, y, s);
    case 4:  return look_up<Id, Table, Io, 4>(c, ids, N, table, base, y, s);
    case 2:  return look_up<Id, Table, Io, 2>(c, ids, N, table, base, y, s);
    default: return look_up<Id, Table, Io, 1>(c, ids, N, table, base, y, s);
    }
}
template <typename Id>
int look_up_types(const cngp_embed_config *c, const void *ids, int64_t N, const void *table, const void *base, void *y, hipStream_t s) {
    if (c->table_dtype == CNGP_F16)
        return c->io_dtype == CNGP_F16 ? look_up_columns<Id, __half, __half>(c, ids, N, table, base, y, s)
                                       : look_up_columns<Id, __half, float>(c, ids, N, table, base, y, s);
    return c->io_dtype == CNGP_F16 ? look_up_columns<Id, float, __half>(c, ids, N, table, base, y, s)
                                   : look_up_columns<Id, float, float>(c, ids, N, table, base, y, s);
}

}  // namespace

extern "C" {

size_t cngp_embed_workspace_bytes(const cngp_embed_config *cfg, int64_t N) {
    return check(cfg, N) ? 0 : space_of(cfg, N).bytes;
}

int cngp_embed_fwd(const cngp_embed_config *cfg, const void *ids, int64_t N, const void *table, const void *base, void *y, void *stream) {
    if (int rc = check(cfg, N)) return rc;
    if (N == 0) return CNGP_OK;
    if (!ids || !table || !y) return CNGP_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    return cfg->id_dtype == CNGP_I64 ? look_up_types<int64_t>(cfg, ids, N, table, base, y, s) : look_up_types<int32_t>(cfg, ids, N, table, base, y, s);
}

int cngp_embed_bwd(const cngp_embed_config *cfg, const void *ids, int64_t N, const void *dy, float *grad_table,
                   void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N)) return rc;
    if (!grad_table) return CNGP_ERR_NULL;
    const int accumulate = (cfg->flags & CNGP_ZERO_GRADS) ? 0 : 1;
    if (N && (!ids || !dy)) return CNGP_ERR_NULL;
    const EmbedSpace sp = space_of(cfg, N);
    if (sp.bytes && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < sp.bytes)) return CNGP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    float *clear = accumulate ? nullptr : grad_table;
    if (N == 0) return clear ? clear_table(clear, cfg->rows * cfg->dim, s) : CNGP_OK;
    char     *ws = (char *)workspace;
    uint32_t *keys[2] = {(uint32_t *)(ws + sp.keys_a), (uint32_t *)(ws + sp.keys_b)};
    int32_t  *from[2] = {(int32_t *)(ws + sp.from_a), (int32_t *)(ws + sp.from_b)};
    uint32_t *counts = (uint32_t *)(ws + sp.counts), *totals = (uint32_t *)(ws + sp.totals);
    int       at = 0;
    if (int rc = cfg->id_dtype == CNGP_I64 ? sort_ids<int64_t>(ids, N, cfg->rows, cfg->dim, clear, keys, from, counts, totals, &at, s)
                                           : sort_ids<int32_t>(ids, N, cfg->rows, cfg->dim, clear, keys, from, counts, totals, &at, s))
        return rc;
    SumArgs a{};
    a.keys = keys[at]; a.from = from[at]; a.dy = dy; a.grad = grad_table;
    a.head = (float *)(ws + sp.head); a.tail = (float *)(ws + sp.tail);
    a.N = N; a.rows = cfg->rows; a.dim = cfg->dim; a.accumulate = accumulate; a.scale = cfg->scale;
    a.piece = piece_of(cfg, N);
    a.pieces = (uint32_t)((N + a.piece - 1) / a.piece);
    const bool half = cfg->io_dtype == CNGP_F16;
    switch (columns_of(cfg->dim, half ? 8 : 4)) {
    case 8:  return sum_columns<__half, 8>(a, s);
    case 4:  return half ? sum_columns<__half, 4>(a, s) : sum_columns<float, 4>(a, s);
    case 2:  return half ? sum_columns<__half, 2>(a, s) : sum_columns<float, 2>(a, s);
    default: return half ? sum_columns<__half, 1>(a, s) : sum_columns<float, 1>(a, s);
    }
}

}  // extern "C"
