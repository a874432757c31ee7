// Linear attention with a decay for each head: entry points, how a call is cut, the kernels beside the walk (cngp_attend_walk.h).
#include <cmath>

#include "cngp_attend.h"

using namespace cngp;

namespace {

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
constexpr int64_t kMostRows = 0x7fffffffll - 65536;
constexpr int     kBlock = 256;

struct StepArgs {
    const void  *q, *k, *v;
    const float *decay, *h0;
    void        *y;
    float       *last;
    int32_t      S, heads, group, kdim, vdim;
    float        scale;
    int32_t      row_decay;
};

// One row to each sequence: a workgroup per sequence and head goes over its state once (read, decayed, the row added, written, multiplied
// with the query), neighbouring lanes neighbouring columns of VEC values, bound by those reads and writes (512 states of 64 x 64, 17 MB: 6.2 us).
template <typename T, int BLOCK, int VEC>
__global__ __launch_bounds__(BLOCK) void attend_step_kernel(const StepArgs a)
{
    __shared__ float qk[2][kAttendDim];
    __shared__ float sums[BLOCK * VEC];
    int units = 1;                                          // lanes side by side: a power of two that holds the columns
    while (units * VEC < a.vdim) units *= 2;
    const int c = (int)threadIdx.x % units * VEC, r0 = (int)threadIdx.x / units, rows = BLOCK / units;
    const bool there = c < a.vdim;
    for (int64_t item = blockIdx.x; item < (int64_t)a.S * a.heads; item += gridDim.x) {
        const int     h = (int)(item % a.heads), kv = h / a.group, kvs = a.heads / a.group;
        const int64_t s = item / a.heads;
        for (int i = threadIdx.x; i < a.kdim; i += BLOCK) {
            qk[0][i] = (float)((const T *)a.q)[item * a.kdim + i] * a.scale;
            qk[1][i] = (float)((const T *)a.k)[(s * kvs + kv) * a.kdim + i];
        }
        const float g = a.row_decay ? a.decay[item] : a.decay[h], e = expf(g);
        float v[VEC], y[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            v[i] = there ? (float)((const T *)a.v)[(s * kvs + kv) * a.vdim + c + i] : 0.0f;
            y[i] = 0.0f;
        }
        __syncthreads();
        const size_t at = (size_t)item * a.kdim * a.vdim + c;
        if (there)
            for (int r = r0; r < a.kdim; r += rows) {
                float S[VEC];
                const size_t p = at + (size_t)r * a.vdim;
                if (a.h0) __builtin_memcpy(S, a.h0 + p, sizeof S);
                else
#pragma unroll
                    for (int i = 0; i < VEC; ++i) S[i] = 0.0f;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    S[i] = fmaf(e, S[i], qk[1][r] * v[i]);
                    y[i] = fmaf(qk[0][r], S[i], y[i]);
                }
                if (a.last) __builtin_memcpy(a.last + p, S, sizeof S);
            }
#pragma unroll
        for (int i = 0; i < VEC; ++i) sums[threadIdx.x * VEC + i] = y[i];
        __syncthreads();
        if (a.y)
            for (int j = threadIdx.x; j < a.vdim; j += BLOCK) {
                float t = 0.0f;
                for (int r = 0; r < rows; ++r) t += sums[(r * units + j / VEC) * VEC + j % VEC];
                ((T *)a.y)[item * a.vdim + j] = (T)t;
            }
        __syncthreads();
    }
}

// States before each segment from the segments' own parts: a thread per state entry goes through a sequence's segments.  Bound by that chain and its reads and
// writes (65 segments of 128 states of 128 x 128: 32 us).
struct CarryArgs {
    float       *states;                 // [segments, heads, size]: a segment's own part, then the state before it
    const float *total;                  // [segments, heads]
    const int32_t *offsets;
    const float *first;
    float       *final;
    int64_t      N;
    int32_t      S, rows_each, heads, seg_rows, size, reverse;
};
__global__ __launch_bounds__(kBlock) void attend_carry_kernel(const CarryArgs a)
{
    const int64_t all = (int64_t)a.S * a.heads * a.size;
    for (int64_t own = blockIdx.x * (int64_t)kBlock + threadIdx.x; own < all; own += (int64_t)gridDim.x * kBlock) {
        const int     e = (int)(own % a.size), h = (int)(own / a.size % a.heads);
        const int32_t s = (int32_t)(own / a.size / a.heads);
        const Span    span = span_of(a.offsets, s, a.N, a.rows_each);
        const int32_t n = (int32_t)(((uint32_t)(span.end - span.begin) + (uint32_t)a.seg_rows - 1) / (uint32_t)a.seg_rows), base = piece_base(span.begin, s, a.seg_rows);
        float state = a.first ? a.first[own] : 0.0f;
        // eight segments' parts are under way at a time: one after the other they would be a chain of memory latencies
        for (int32_t i0 = 0; i0 < n; i0 += 8) {
            float part[8], keep[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int32_t i = i0 + u < n ? i0 + u : n - 1;
                const int64_t at = (int64_t)(base + (a.reverse ? n - 1 - i : i)) * a.heads + h;
                part[u] = a.states[(size_t)at * a.size + e];
                keep[u] = a.total[at];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int32_t i = i0 + u;
                if (i >= n) break;
                const int64_t at = (int64_t)(base + (a.reverse ? n - 1 - i : i)) * a.heads + h;
                a.states[(size_t)at * a.size + e] = state;
                state = fmaf(__builtin_amdgcn_exp2f(keep[u]), state, part[u]);
            }
        }
        if (a.final) a.final[own] = state;
    }
}

// Gradient of the log decays.  That of row t is what reaches over it, g_t = <state before it, its gradient there>, and from one row to the next
//     g_{t+1} = g_t + k_t . dk_t - q_t . dq_t        (a row's product with itself, which both hold, left out of both)
// with g known at the chunks' ends: <state, gradient of the state> there, by the walk of dk from states that the walk of dq left (0 before a sequence without a first state
// and behind one whose last is not used).  Sums of roundings between two such places lead from one to the other but for a rest, which is taken off evenly on the way:
// summed up over a sequence, roundings weigh as many times as there are rows from the next such place.  (Sixteen heads with memories of 16 rows over 4096, their decays'
// gradients off by 4 to 5e-6 from places 1024 rows apart and one side, by 3 to 4e-7 so.)  A wavefront per chunk, a lane per row, some heads one after the other:
// bound by the search for its sequence and chains of loads (2^18 rows of 4096 sequences, 4 heads: 27 us).
constexpr int kDecayChunks = 16;                         // of a workgroup
struct DecayArgs {
    const float   *q_dot, *k_dot;                        // [heads, N]
    const double  *starts, *ends;                        // [chunk_number, heads, waves], [S, heads, waves]: parts of the products of states; ends NULL: zeros
    const int32_t *offsets;
    float         *ddecay;                               // [N, heads], or NULL
    double        *parts;                                // [workgroups, heads], or NULL
    int64_t        N, chunks;
    int32_t        S, rows_each, heads, heads_each, waves, has_first;
};
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}
__device__ __forceinline__ double upto(double v, const int lane) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}
__global__ __launch_bounds__(64 * kDecayChunks) void attend_decay_kernel(const DecayArgs a)
{
    __shared__ double sums[kDecayChunks];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h_first = (int)blockIdx.y * a.heads_each, h_end = h_first + a.heads_each < a.heads ? h_first + a.heads_each : a.heads;
    for (int64_t block = blockIdx.x; block * kDecayChunks < a.chunks; block += gridDim.x) {
        const int64_t chunk = block * kDecayChunks + wave;
        int32_t seq = 0, n = 0;
        int64_t begin = 0;
        bool    first = false, last = false;
        if (chunk < a.chunks) {
            seq = sequence_of(a.offsets, chunk, a.N, a.S, a.rows_each, kChunk);
            const Span    span = span_of(a.offsets, seq, a.N, a.rows_each);
            const int64_t number = chunk - chunk_number(span.begin, seq, 0);      // (below 0: rows before the first sequence)
            begin = span.begin + number * kChunk;
            if (number >= 0 && begin < span.end) n = span.end - begin < kChunk ? (int32_t)(span.end - begin) : kChunk;
            first = number == 0;
            last = begin + kChunk >= span.end;
        }
        for (int h = h_first; h < h_end; ++h) {
            double sum = 0.0;
            if (n) {
                auto joined = [&](const double *p) {
                    double t = 0.0;
                    for (int w = 0; w < a.waves; ++w) t += p[w];
                    return t;
                };
                const size_t at = ((size_t)chunk * a.heads + h) * a.waves, row = (size_t)h * a.N + (size_t)begin + lane;
                const double from = first && !a.has_first ? 0.0 : joined(a.starts + at);
                const double to = !last ? joined(a.starts + at + (size_t)a.heads * a.waves) : a.ends ? joined(a.ends + ((size_t)seq * a.heads + h) * a.waves) : 0.0;
                const double step = lane < n ? (double)a.k_dot[row] - (double)a.q_dot[row] : 0.0, up = upto(step, lane), all = __shfl(up, 63, 64);
                const double g = from + (up - step) + (to - from - all) * ((double)lane / (double)n);
                if (a.ddecay && lane < n) a.ddecay[(size_t)(begin + lane) * a.heads + h] = (float)g;
                sum = lane < n ? g : 0.0;
            }
            if (a.parts) {
                sum = wave_sum(sum);
                if (lane == 0) sums[wave] = sum;
                __syncthreads();
                if (threadIdx.x == 0) {
                    double t = 0.0;
                    for (int w = 0; w < kDecayChunks; ++w) t += sums[w];
                    a.parts[(size_t)block * a.heads + h] = t;
                }
                __syncthreads();
            }
        }
    }
}
__global__ __launch_bounds__(kBlock) void attend_decay_sum_kernel(const double *__restrict__ parts, float *__restrict__ ddecay, const int64_t pieces, const int heads)
{
    __shared__ double sums[kBlock / 64];
    const int h = blockIdx.x;
    double t = 0.0;
    for (int64_t p = threadIdx.x; p < pieces; p += kBlock) t += parts[p * heads + h];
    t = wave_sum(t);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x == 0) ddecay[h] = (float)(sums[0] + sums[1] + sums[2] + sums[3]);
}

// Gradients of keys or values that several heads share: the heads' parts added up in their order.  Rows of no sequence are left alone.  Bound by its
// reads (2^18 rows, 4 parts of 16 fp32: 15 us; with a division per value 26); lanes go over VEC neighbouring values of a row, 2^shift of them, and the
// rest of a workgroup over rows.
template <typename T, int VEC>
__global__ __launch_bounds__(kBlock) void attend_group_kernel(const float *__restrict__ part, T *__restrict__ out, const int32_t *offsets, const int32_t S, const int64_t N,
                                                              const int kv, const int group, const int dim, const int shift)
{
    const int64_t first = offsets ? span_of(offsets, 0, N, 0).begin : 0, end = offsets ? span_of(offsets, S - 1, N, 0).end : N;
    const int at = (int)(blockIdx.y << shift | (threadIdx.x & ((1u << shift) - 1))) * VEC, head = at / dim, e = at % dim, rows = kBlock >> shift;
    if (at >= kv * dim) return;
    for (int64_t row = first + (int64_t)blockIdx.x * rows + (threadIdx.x >> shift); row < end; row += (int64_t)gridDim.x * rows) {
        const float *p = part + (row * kv + head) * (int64_t)group * dim + e;
        float t[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) t[i] = 0.0f;
#pragma unroll 4
        for (int g = 0; g < group; ++g) {
            float x[VEC];
            __builtin_memcpy(x, __builtin_assume_aligned(p + (int64_t)g * dim, 4 * VEC), sizeof x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) t[i] += x[i];
        }
        T y[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = (T)t[i];
        __builtin_memcpy(__builtin_assume_aligned(out + row * kv * (int64_t)dim + at, sizeof y), y, sizeof y);
    }
}

int check(const cngp_attend_config *c, int64_t N, int64_t S, bool ragged) {
    if (!c) return CNGP_ERR_NULL;
    if (c->heads < 1 || c->heads > 4096 || c->kv_heads < 1 || c->heads % c->kv_heads) return CNGP_ERR_INVALID;
    if (c->key_dim < 1 || c->key_dim > kAttendDim || c->value_dim < 1 || c->value_dim > kAttendDim) return CNGP_ERR_INVALID;
    if (c->io_dtype != CNGP_F32 && c->io_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->longest < 0 || !std::isfinite(c->scale)) return CNGP_ERR_INVALID;
    if (c->flags & ~(uint32_t)CNGP_ATTEND_ROW_DECAY) return CNGP_ERR_INVALID;
    if (N < 0 || N > kMostRows || S < 0 || S > kMostRows) return CNGP_ERR_INVALID;
    if (!ragged && (S == 0 ? N != 0 : N % S != 0)) return CNGP_ERR_INVALID;
    return CNGP_OK;
}

// How a call is cut: sequences whole, a workgroup per sequence and head, or in segments of seg_rows rows where that leaves most of the chip
// without work; then a walk without outputs gives the segments' parts first.
struct Plan {
    int     seg_rows;
    int64_t segments;
};
// Workgroups of all segments together: four for each of 256 CUs, whole turns of the card whatever a CU has room for, as nearly as that can be
// had (a last segment is half a one in the mean).  Rows in powers of two left a fifth turn of a few (2^15 rows, 16 heads of 128 x 128: 312 against 338 us;
// 512 or 2048 workgroups: 356 and 367).  Twice as many of fp16 heads of at most 32 columns, whose workgroups are a wavefront or two (backward, 2 of
// 2^16 rows, 8 heads of 32: 247 against 295 us; in fp32, which keeps twice as much in registers, 2^18 rows, 4 heads of 16: 716 against 662).
constexpr int64_t kItems = 1024, kLeastSegment = 256;
int64_t longest_of(const cngp_attend_config *c, int64_t N, int64_t S, bool ragged) {
    const int64_t mean = S ? (N + S - 1) / S : 0;
    return !ragged ? mean : c->longest ? std::min<int64_t>(c->longest, N) : std::min<int64_t>(4 * mean, N);
}
Plan plan_of(const cngp_attend_config *c, int64_t N, int64_t S, bool ragged) {
    const int64_t longest = longest_of(c, N, S, ragged);
    const int64_t all = kItems * (c->io_dtype == CNGP_F16 && std::max(c->key_dim, c->value_dim) <= 32 ? 2 : 1);
    const int64_t items = std::max<int64_t>(all - (S + 1) / 2 * c->heads, all * 3 / 4), least = (N * c->heads + items - 1) / items;
    const int64_t R = std::max<int64_t>((least + kChunk - 1) / kChunk * kChunk, kLeastSegment);
    if (longest <= 4 * R) return {0, S};
    return {(int)R, pieces(N, S, R)};
}

struct Space {
    size_t states, total, dot_q, dot_k, anchors, starts, ends, parts, part_k, part_v, bytes;
};
inline int64_t chunks_of(int64_t N, int64_t S) { return pieces(N, S, kChunk); }
inline int64_t decay_parts(int64_t N, int64_t S) { return (chunks_of(N, S) + kDecayChunks - 1) / kDecayChunks; }
Space space_of(const cngp_attend_config *c, const Plan &p, int64_t N, int64_t S, uint32_t call) {
    Space sp{};
    size_t at = 0;
    auto take = [&](bool wanted, size_t bytes) { const size_t o = at; if (wanted) at += align256(bytes); return o; };
    const bool   bwd = call & CNGP_ATTEND_CALL_BWD, decays = bwd && !(call & CNGP_ATTEND_CALL_NO_DDECAY), cut = p.seg_rows != 0, shared = c->heads != c->kv_heads;
    const size_t H = (size_t)c->heads, size = (size_t)c->key_dim * c->value_dim, rows = (size_t)N, waves = (size_t)walk_waves(c->value_dim, c->key_dim);
    sp.states = take(cut, (size_t)p.segments * H * size * 4);
    sp.total = take(cut, (size_t)p.segments * H * 4);
    sp.dot_q = take(decays, rows * H * 4);
    sp.dot_k = take(decays, rows * H * 4);
    sp.anchors = take(decays, (rows / kChunk + 1) * H * anchor_floats(c->value_dim, c->key_dim) * 4);
    sp.starts = take(decays, (size_t)chunks_of(N, S) * H * waves * 8);
    sp.ends = take(decays, (size_t)S * H * waves * 8);
    sp.parts = take(decays && !(c->flags & CNGP_ATTEND_ROW_DECAY), (size_t)decay_parts(N, S) * H * 8);
    sp.part_k = take(bwd && shared, rows * H * (size_t)c->key_dim * 4);
    sp.part_v = take(bwd && shared, rows * H * (size_t)c->value_dim * 4);
    sp.bytes = at;
    return sp;
}

bool whole_rows(const void *p, int dim, int io, size_t bytes) {
    return ((uintptr_t)p & (bytes - 1)) == 0 && (size_t)dim * (io == CNGP_F16 ? 2 : 4) % bytes == 0;
}

struct Call {
    const cngp_attend_config *c;
    const float *decay;
    int64_t N, S;
    const int32_t *offsets;
    Plan p;
    Space sp;
    char *ws;
    hipStream_t s;

    WalkArgs base(const void *q, const void *k, const void *v, int q_div, int k_div, int v_div, int kdim, int vdim, bool reverse) const {
        WalkArgs a{};
        a.q = q; a.k = k; a.v = v; a.decay = decay; a.offsets = offsets;
        a.N = N; a.S = (int32_t)S; a.rows_each = (int32_t)(S ? N / S : 0);
        a.heads = c->heads; a.q_div = q_div; a.k_div = k_div; a.v_div = v_div; a.x_div = 1;
        a.kdim = kdim; a.vdim = vdim;
        a.seg_rows = p.seg_rows; a.segments = (int32_t)p.segments;
        a.first_i = a.final_i = vdim; a.first_j = a.final_j = 1;
        a.pair_scale = a.far_scale = a.state_scale = 1.0f;
        a.reverse = reverse; a.row_decay = (c->flags & CNGP_ATTEND_ROW_DECAY) != 0;
        a.whole = whole_rows(q, kdim, c->io_dtype, 16) && whole_rows(k, kdim, c->io_dtype, 16) && whole_rows(v, vdim, c->io_dtype, 16);
        return a;
    }
    void output(WalkArgs &a, void *out, bool f32) const {
        a.out = out;
        a.out_f32 = f32 || c->io_dtype == CNGP_F32;
        a.whole = a.whole && a.vdim % 4 == 0 && ((uintptr_t)out & (a.out_f32 ? 15u : 7u)) == 0;
    }
    // for the decays' gradient: states left or met with on the way, and at the end
    void meet(WalkArgs &a, const float *met, size_t products) const {
        a.anchors = (float *)(ws + sp.anchors);
        a.met = met;
        a.products = (double *)(ws + products);
        a.whole = a.whole && ((uintptr_t)met & 15u) == 0;
    }
    int walk(const WalkArgs &a, bool states_only) const {
        return c->io_dtype == CNGP_F16 ? attend_walk_f16(a, states_only, s) : attend_walk_f32(a, states_only, s);
    }
    // cut sequences: the states before each segment into the workspace, the last ones into `final`
    int carry(WalkArgs a, const float *first, float *final) const {
        a.first = nullptr;
        a.final = (float *)(ws + sp.states);
        a.total = (float *)(ws + sp.total);
        if (int rc = walk(a, true)) return rc;
        CarryArgs k{};
        k.states = a.final; k.total = a.total; k.offsets = offsets; k.first = first; k.final = final;
        k.N = N; k.S = (int32_t)S; k.rows_each = a.rows_each; k.heads = c->heads; k.seg_rows = p.seg_rows;
        k.size = a.kdim * a.vdim; k.reverse = a.reverse;
        LaunchTimer t(s, K_ATTEND_STATES);
        attend_carry_kernel<<<(unsigned)std::min<int64_t>((S * c->heads * k.size + kBlock - 1) / kBlock, 1 << 20), kBlock, 0, s>>>(k);
        return launch_status("attend_carry_kernel");
    }
};

template <typename T>
int step(const StepArgs &a, hipStream_t s) {
    const int64_t items = (int64_t)a.S * a.heads;
    const unsigned blocks = (unsigned)std::min<int64_t>(items, kMostGroups256);
    const bool vec = a.vdim % 4 == 0 && ((uintptr_t)a.h0 & 15u) == 0 && ((uintptr_t)a.last & 15u) == 0;
    const bool small = a.kdim * a.vdim <= 1024 && (vec || a.vdim <= 64);
    LaunchTimer t(s, K_ATTEND_STEP);
    if (vec) {
        if (small) attend_step_kernel<T, 64, 4><<<blocks, 64, 0, s>>>(a);
        else attend_step_kernel<T, 256, 4><<<blocks, 256, 0, s>>>(a);
    } else {
        if (small) attend_step_kernel<T, 64, 1><<<blocks, 64, 0, s>>>(a);
        else attend_step_kernel<T, 256, 1><<<blocks, 256, 0, s>>>(a);
    }
    return launch_status("attend_step_kernel");
}

int decay_sum(const double *parts, float *ddecay, int64_t pieces, int heads, hipStream_t s) {
    LaunchTimer t(s, K_ATTEND_DECAY);
    attend_decay_sum_kernel<<<(unsigned)heads, kBlock, 0, s>>>(parts, ddecay, pieces, heads);
    return launch_status("attend_decay_sum_kernel");
}

template <typename T, int VEC>
int group_sum(const float *part, void *out, const int32_t *offsets, int64_t S, int64_t N, int kv, int group, int dim, hipStream_t s) {
    const int units = (kv * dim + VEC - 1) / VEC;
    int shift = 0;
    while (shift < 8 && 1 << shift < units) ++shift;
    const int64_t rows = kBlock >> shift;
    LaunchTimer t(s, K_ATTEND_DECAY);
    attend_group_kernel<T, VEC><<<dim3((unsigned)std::min<int64_t>((N + rows - 1) / rows, 1 << 13), (unsigned)((units + (1 << shift) - 1) >> shift)), kBlock, 0, s>>>(
        part, (T *)out, offsets, (int32_t)S, N, kv, group, dim, shift);
    return launch_status("attend_group_kernel");
}

bool lent(const Space &sp, const void *ws, size_t bytes) { return !sp.bytes || (ws && ((uintptr_t)ws & 255u) == 0 && bytes >= sp.bytes); }

}  // namespace

extern "C" {

size_t cngp_attend_workspace_bytes(const cngp_attend_config *cfg, int64_t N, int64_t sequences, uint32_t call) {
    if (check(cfg, N, sequences, call & CNGP_ATTEND_CALL_RAGGED) || sequences == 0) return 0;
    return space_of(cfg, plan_of(cfg, N, sequences, call & CNGP_ATTEND_CALL_RAGGED), N, sequences, call).bytes;
}

int cngp_attend_fwd(const cngp_attend_config *cfg, const void *q, const void *k, const void *v, const float *decay, int64_t N, const int32_t *offsets,
                    int64_t sequences, const float *h0, void *y, float *last, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N, sequences, offsets != nullptr)) return rc;
    if (sequences == 0) return CNGP_OK;
    if (N && (!k || !v || !decay || (y && !q) || (!last && !y))) return CNGP_ERR_NULL;
    if (N == 0 && !last) return CNGP_OK;
    hipStream_t s = (hipStream_t)stream;
    const bool ragged = offsets != nullptr;
    if (!ragged && N == sequences) {
        StepArgs a{q ? q : k, k, v, decay, h0, y, last, (int32_t)sequences, cfg->heads, cfg->heads / cfg->kv_heads, cfg->key_dim, cfg->value_dim, cfg->scale,
                   (cfg->flags & CNGP_ATTEND_ROW_DECAY) != 0};
        if (!q && cfg->heads != cfg->kv_heads) return CNGP_ERR_NULL;
        return cfg->io_dtype == CNGP_F16 ? step<_Float16>(a, s) : step<float>(a, s);
    }
    Call call{cfg, decay, N, sequences, offsets, plan_of(cfg, N, sequences, ragged), {}, (char *)workspace, s};
    call.sp = space_of(cfg, call.p, N, sequences, ragged ? CNGP_ATTEND_CALL_RAGGED : 0);
    if (!lent(call.sp, workspace, workspace_bytes)) return CNGP_ERR_WORKSPACE;
    const int group = cfg->heads / cfg->kv_heads;
    WalkArgs a = call.base(q, k, v, 1, group, group, cfg->key_dim, cfg->value_dim, false);
    a.pair_scale = a.far_scale = cfg->scale;
    a.first = h0;
    a.final = last;
    if (call.p.seg_rows) {
        if (int rc = call.carry(a, h0, last)) return rc;
        if (!y) return CNGP_OK;
        a.first = (const float *)(call.ws + call.sp.states);
        a.final = nullptr;
    }
    if (!y) return call.walk(a, true);
    call.output(a, y, false);
    return call.walk(a, false);
}

int cngp_attend_bwd(const cngp_attend_config *cfg, const void *q, const void *k, const void *v, const float *decay, int64_t N, const int32_t *offsets,
                    int64_t sequences, const float *h0, const void *dy, const float *dlast, void *dq, void *dk, void *dv, float *ddecay, float *dh0,
                    void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N, sequences, offsets != nullptr)) return rc;
    const bool rows = cfg->flags & CNGP_ATTEND_ROW_DECAY;
    if (sequences == 0) return ddecay && !rows ? decay_sum(nullptr, ddecay, 0, cfg->heads, (hipStream_t)stream) : CNGP_OK;
    if (dh0 && dh0 == dlast) return CNGP_ERR_INVALID;
    if (N && (!q || !k || !v || !decay || !dq || !dk || !dv || (!dy && !dlast))) return CNGP_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    const bool ragged = offsets != nullptr;
    Call call{cfg, decay, N, sequences, offsets, plan_of(cfg, N, sequences, ragged), {}, (char *)workspace, s};
    call.sp = space_of(cfg, call.p, N, sequences, CNGP_ATTEND_CALL_BWD | (ragged ? CNGP_ATTEND_CALL_RAGGED : 0) | (ddecay ? 0 : CNGP_ATTEND_CALL_NO_DDECAY));
    if (!lent(call.sp, workspace, workspace_bytes)) return CNGP_ERR_WORKSPACE;
    char *ws = call.ws;
    const Space &sp = call.sp;
    const int   group = cfg->heads / cfg->kv_heads, K = cfg->key_dim, V = cfg->value_dim;
    const bool  cut = call.p.seg_rows != 0, shared = group > 1;
    float      *states = (float *)(ws + sp.states);

    // dq_t = scale (sum of e (dy_t . v_s) k_s + e state dy_t): a forward walk over the transposed state
    WalkArgs a = call.base(dy, v, k, 1, group, group, V, K, false);
    a.pair_scale = a.far_scale = cfg->scale;
    if (cut) {
        WalkArgs m = call.base(q, k, v, 1, group, group, K, V, false);
        if (int rc = call.carry(m, h0, nullptr)) return rc;
        a.first = states;
    } else a.first = h0;
    a.first_i = 1; a.first_j = V;
    a.own = 1;
    call.output(a, dq, false);
    if (ddecay) {
        a.x = q; a.x_div = 1; a.whole = a.whole && whole_rows(q, K, cfg->io_dtype, cfg->io_dtype == CNGP_F16 ? 8 : 16);
        a.dot = (float *)(ws + sp.dot_q);
        call.meet(a, dlast, sp.ends);
    }
    if (N)
        if (int rc = call.walk(a, false)) return rc;

    // dv_s = sum of scale e (k_s . q_t) dy_t + e k_s . (gradient of the state behind it): against time, with the gradient of the state
    a = call.base(k, q, dy, group, 1, 1, K, V, true);
    a.pair_scale = a.state_scale = cfg->scale;
    a.first = dlast; a.final = dh0;
    if (cut) {
        if (int rc = call.carry(a, dlast, dh0)) return rc;
        a.first = states; a.final = nullptr;
    }
    if (N == 0) {                                        // the gradient of the state passes through
        if (dh0)
            if (int rc = call.walk(a, true)) return rc;
        return ddecay && !rows ? decay_sum(nullptr, ddecay, 0, cfg->heads, s) : CNGP_OK;
    }
    call.output(a, shared ? (void *)(ws + sp.part_v) : dv, shared);
    if (int rc = call.walk(a, false)) return rc;

    // dk_s = sum of scale e (v_s . dy_t) q_t + e (gradient of the state behind it) v_s
    a = call.base(v, dy, q, group, 1, 1, V, K, true);
    a.pair_scale = a.state_scale = cfg->scale;
    a.first = cut ? states : dlast;
    a.first_i = 1; a.first_j = V;
    a.own = 1;
    call.output(a, shared ? (void *)(ws + sp.part_k) : dk, shared);
    if (ddecay) {
        a.x = k; a.x_div = group; a.whole = a.whole && whole_rows(k, K, cfg->io_dtype, cfg->io_dtype == CNGP_F16 ? 8 : 16);
        a.dot = (float *)(ws + sp.dot_k);
        call.meet(a, h0, sp.starts);
    }
    if (int rc = call.walk(a, false)) return rc;

    if (shared)
        for (int which = 0; which < 2; ++which) {
            const int    dim = which ? V : K;
            const float *part = (const float *)(ws + (which ? sp.part_v : sp.part_k));
            void        *out = which ? dv : dk;
            const bool   f16 = cfg->io_dtype == CNGP_F16, vec = dim % 4 == 0 && ((uintptr_t)out & (f16 ? 7u : 15u)) == 0;
            const auto   sum = f16 ? vec ? group_sum<_Float16, 4> : group_sum<_Float16, 1> : vec ? group_sum<float, 4> : group_sum<float, 1>;
            if (int rc = sum(part, out, offsets, sequences, N, cfg->kv_heads, group, dim, s)) return rc;
        }
    if (!ddecay) return CNGP_OK;
    DecayArgs d{};
    d.q_dot = (const float *)(ws + sp.dot_q); d.k_dot = (const float *)(ws + sp.dot_k);
    d.starts = (const double *)(ws + sp.starts); d.ends = dlast ? (const double *)(ws + sp.ends) : nullptr;
    d.offsets = offsets; d.has_first = h0 != nullptr;
    d.ddecay = rows ? ddecay : nullptr;
    d.parts = rows ? nullptr : (double *)(ws + sp.parts);
    d.N = N; d.chunks = chunks_of(N, sequences);
    d.S = (int32_t)sequences; d.rows_each = (int32_t)(N / sequences); d.heads = cfg->heads;
    d.waves = walk_waves(V, K);
    // heads one after the other by wavefronts that have found their chunk's sequence, but few where there are few chunks: eight wavefronts to a SIMD
    const int64_t groups = decay_parts(N, sequences), split = std::min<int64_t>(cfg->heads, std::max<int64_t>(1, 512 / groups));
    d.heads_each = (int32_t)((cfg->heads + split - 1) / split);
    {
        LaunchTimer t(s, K_ATTEND_DECAY);
        attend_decay_kernel<<<dim3((unsigned)std::min<int64_t>(groups, 0x3fffff), (unsigned)((cfg->heads + d.heads_each - 1) / d.heads_each)), 64 * kDecayChunks, 0, s>>>(d);
        if (int rc = launch_status("attend_decay_kernel")) return rc;
    }
    if (rows) return CNGP_OK;
    return decay_sum(d.parts, ddecay, groups, cfg->heads, s);
}

}  // extern "C"
