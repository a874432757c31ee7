// The walk of the linear attention (WalkArgs in cngp_attend.h): a workgroup per sequence (or segment) and head goes over its chunks with the
// state in registers.  Everything dense runs on the matrix cores, 32 x 32 x 16 products with fp32 sums:
//     scores of the pairs of rows       P^T = K Q^T                       (three of the four tiles: a row sees those up to it)
//     outputs inside the chunk          O^T += V^T P^T,  far ones  O^T += S^T Q^T
//     state                             S = e^F S + K^T (V e^(F - F_s))
// A wavefront owns 32 columns of v: of the state, the accumulators themselves (lane = column of v, registers = columns of k), which are at
// the same time the operand of S^T Q^T once they are rounded; the contraction's order is a permutation, the same for Q's reads.  Outputs
// are formed transposed, a row of the chunk per lane, so that decays and products with another row are per lane too.
// fp16 storage: q, k, v are exact operands; what is computed (scores, state, decayed v) would lose half of the result's accuracy if it
// were rounded once, so it is split in two fp16 numbers (22 bits) and takes two products.  fp32 storage: fp32 products.
#pragma once
#include "cngp_attend.h"
#include "cngp_matrix.h"

namespace cngp {
namespace attend {

using namespace mat;

// Power of two that brings the largest finite of a wavefront's values to 2^13 .. 2^14, as an exponent (0 if all are 0).
__device__ __forceinline__ int lift_of(float most) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
    const int e = (int)((__float_as_uint(most) >> 23) & 255u) - 127;
    const int lift = 13 - e;
    return most > 0.0f ? (lift > 120 ? 120 : lift < -120 ? -120 : lift) : 0;
}
__device__ __forceinline__ float most_of(const float most, const float v) {
    const float a = fabsf(v);
    return a <= 3.402823466e38f ? fmaxf(most, a) : most;
}
__device__ __forceinline__ float power_of_two(const int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// Registers of a thread's part of a tile [64, 32 TILES] on its way into LDS.
template <typename T, int TILES, int WAVES>
struct Staged {
    static constexpr int vec = Types<T>::vec, per_row = TILES * 32 / vec, each = kChunk * per_row / (WAVES * 64);
    uint4 r[each];

    // Rows lo + t dir of an array with `stride` values between rows, `dim` of them from `base` on; rows from `count` and columns from dim on are 0.
    __device__ __forceinline__ void load(const T *base, const int64_t row0, const int dir, const int count, const int64_t stride, const int dim, const bool whole) {
#pragma unroll
        for (int i = 0; i < each; ++i) {
            const int at = (int)threadIdx.x + i * WAVES * 64, t = at / per_row, c = at % per_row * vec;
            r[i] = make_uint4(0, 0, 0, 0);
            if (t < count && c < dim) {
                const T *p = base + (row0 + (int64_t)t * dir) * stride + c;
                if (whole) r[i] = *reinterpret_cast<const uint4 *>(p);
                else {
                    T e[vec];
#pragma unroll
                    for (int j = 0; j < vec; ++j) e[j] = c + j < dim ? p[j] : (T)0.0f;
                    __builtin_memcpy(&r[i], e, 16);
                }
            }
        }
    }
    __device__ __forceinline__ void store(T *tile) const {
#pragma unroll
        for (int i = 0; i < each; ++i) {
            const int at = (int)threadIdx.x + i * WAVES * 64, t = at / per_row, c = at % per_row * vec;
            *reinterpret_cast<uint4 *>(tile + t * (TILES * 32 + Types<T>::pad) + c) = r[i];
        }
    }
};

template <typename T, int KT, int VT, bool OUT>
struct Lds {
    static constexpr int kstride = 32 * KT + Types<T>::pad, vstride = 32 * VT + Types<T>::pad, pstride = 32 + Types<T>::pad;
    static constexpr int waves = KT > VT ? KT : VT;
    double F[kChunk];                                       // log2 of the decay from the chunk's start
    float  far[kChunk], keep[kChunk];                       // what a row takes from the state, and gives to it
    double total;
    int    lift[4];                                         // of each score tile
    float  dots[OUT ? 2 * waves : 1][kChunk];
    alignas(16) T k[kChunk * kstride];
    alignas(16) T v[kChunk * vstride];
    alignas(16) T q[OUT ? kChunk * kstride : 8];
    alignas(16) T p[OUT ? (sizeof(T) == 2 ? 2 : 1) * 3 * 32 * pstride : 8];
};

template <typename T, int KT, int VT, bool OUT>
__global__ __launch_bounds__(64 * (KT > VT ? KT : VT)) void attend_walk_kernel(const WalkArgs a)
{
    using L = Lds<T, KT, VT, OUT>;
    constexpr int  WAVES = L::waves;
    constexpr bool kSplit = sizeof(T) == 2;
    extern __shared__ __align__(16) char lds_raw[];
    L &lds = *reinterpret_cast<L *>(lds_raw);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    const bool owns = wave < VT;

    for (int64_t item = blockIdx.x; item < (int64_t)a.segments * a.heads; item += gridDim.x) {
        const int h = (int)(item % a.heads);
        const int64_t piece = item / a.heads;
        const int32_t seq = a.seg_rows ? sequence_of(a.offsets, piece, a.N, a.S, a.rows_each, a.seg_rows) : (int32_t)piece;
        const Span    span = span_of(a.offsets, seq, a.N, a.rows_each);
        int64_t begin = span.begin, end = span.end;
        int64_t chunk0 = 0;                                 // the first chunk's number in its sequence
        if (a.seg_rows) {
            const int64_t i = piece - piece_base(a.offsets, seq, a.N, a.rows_each, a.seg_rows);
            begin += i * a.seg_rows;
            if (begin >= end) continue;
            end = begin + a.seg_rows < end ? begin + a.seg_rows : end;
            chunk0 = i * (a.seg_rows / kChunk);
        }
        const int64_t chunks = (end - begin + kChunk - 1) / kChunk;
        const int64_t state_at = piece * a.heads + h;       // whole sequences: piece == sequence
        const size_t  state_size = (size_t)a.kdim * a.vdim;
        const int64_t qs = (int64_t)(a.heads / a.q_div) * a.kdim, ks = (int64_t)(a.heads / a.k_div) * a.kdim, vs = (int64_t)(a.heads / a.v_div) * a.vdim;
        const T *q = (const T *)a.q + (size_t)(h / a.q_div) * a.kdim, *k = (const T *)a.k + (size_t)(h / a.k_div) * a.kdim,
                *v = (const T *)a.v + (size_t)(h / a.v_div) * a.vdim;

        acc_t S[KT];
        const int j = 32 * wave + col;                      // this lane's column of v
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = 32 * kt + 8 * (r >> 2) + 4 * half + (r & 3);
                S[kt][r] = a.first && owns && i < a.kdim && j < a.vdim ? a.first[state_at * state_size + (size_t)i * a.first_i + (size_t)j * a.first_j] : 0.0f;
            }

        Staged<T, KT, WAVES> rq, rk;
        Staged<T, VT, WAVES> rv;
        float  rdecay = 0.0f;
        double whole = 0.0;
        // chunk c of the walk: its first row (reverse: its last), how many
        auto place = [&](const int64_t c, int64_t &row0, int &count) {
            const int64_t at = begin + (a.reverse ? chunks - 1 - c : c) * kChunk;
            count = (int)(end - at < kChunk ? end - at : kChunk);
            row0 = a.reverse ? at + count - 1 : at;
        };
        const int dir = a.reverse ? -1 : 1;
        auto fetch = [&](const int64_t c) {
            int64_t row0;
            int     count;
            place(c, row0, count);
            if (OUT) rq.load(q, row0, dir, a.q ? count : 0, qs, a.kdim, a.vec_q);
            rk.load(k, row0, dir, a.k ? count : 0, ks, a.kdim, a.vec_k);
            rv.load(v, row0, dir, a.v ? count : 0, vs, a.vdim, a.vec_v);
            if (wave == 0) rdecay = lane < count ? a.row_decay ? a.decay[(row0 + (int64_t)lane * dir) * a.heads + h] : a.decay[h] : 0.0f;
        };
        if (chunks > 0) fetch(0);
        // the state at the start of a chunk (of this number in its sequence), as it lies in the registers
        auto anchor = [&](const int64_t number) {
            if (number == 0 || number % kAnchorChunks) return;
            float *to = a.anchors + (size_t)(anchor_slot(span.begin, number) * a.heads + h) * (KT * VT * 1024) + wave * KT * 1024 + lane;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) to[(kt * 16 + r) * 64] = S[kt][r];
        };

        for (int64_t c = 0; c < chunks; ++c) {
            int64_t row0;
            int     count;
            place(c, row0, count);
            if (OUT) rq.store(lds.q);
            rk.store(lds.k);
            rv.store(lds.v);
            if (wave == 0) {
                // below -110 a decay is 0 in fp32 however it is joined; bounded, sums of them stay exact enough to be subtracted
                double g = (double)(rdecay < -110.0f ? -110.0f : rdecay) * 1.4426950408889634;
                double f = g;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const double o = __shfl_up(f, d, 64);
                    if (lane >= d) f += o;
                }
                const double all = __shfl(f, 63, 64);
                if (a.reverse) {
                    f = __shfl_up(f, 1, 64);
                    if (lane == 0) f = 0.0;
                }
                lds.F[lane] = f;
                lds.far[lane] = __builtin_amdgcn_exp2f((float)f) * a.far_scale;
                lds.keep[lane] = __builtin_amdgcn_exp2f((float)(all - f)) * a.state_scale;
                if (lane == 0) lds.total = all;
            }
            __syncthreads();
            if (c + 1 < chunks) fetch(c + 1);
            const double all = lds.total;
            whole += all;

            acc_t far[2];
            if (OUT) {
                // scores: tile (0, 0), (1, 0), (1, 1) of (rows, rows they look at)
                for (int tile = wave; tile < 3; tile += WAVES) {
                    const int tt = tile > 0, ss = tile > 1;
                    acc_t p = zero();
#pragma unroll
                    for (int s = 0; s < 2 * KT; ++s)
                        p = mfma(read8(lds.k + (32 * ss + col) * L::kstride + 16 * s + 8 * half), read8(lds.q + (32 * tt + col) * L::kstride + 16 * s + 8 * half), p);
                    const int    t = 32 * tt + col;
                    const double Ft = lds.F[t];
                    float most = 0.0f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int s = 32 * ss + 8 * (r >> 2) + 4 * half + (r & 3);
                        const float w = __builtin_amdgcn_exp2f((float)(Ft - lds.F[s])) * a.pair_scale;
                        p[r] = s <= t ? p[r] * w : 0.0f;
                        most = most_of(most, p[r]);
                    }
                    T *to = lds.p + (tile * 32 + col) * L::pstride + 4 * half;
                    if constexpr (kSplit) {
                        const int   lift = lift_of(most);
                        const float up = power_of_two(lift);
                        if (lane == 0) lds.lift[tile] = lift;
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            half4_t hi, lo;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float y = p[4 * g + e] * up;
                                hi[e] = (_Float16)y;
                                lo[e] = (_Float16)((y - (float)hi[e]) * kLow);
                            }
                            *reinterpret_cast<half4_t *>(to + 8 * g) = hi;
                            *reinterpret_cast<half4_t *>(to + 3 * 32 * L::pstride + 8 * g) = lo;
                        }
                    } else {
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            float4_t w;
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[e] = p[4 * g + e];
                            *reinterpret_cast<float4_t *>(to + 8 * g) = w;
                        }
                    }
                }
                // what the rows take from the state
                if (owns) {
                    acc_t low[2];
                    far[0] = far[1] = low[0] = low[1] = zero();
                    int lift = 0;
                    if constexpr (kSplit) {
                        float most = 0.0f;
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                            for (int r = 0; r < 16; ++r) most = most_of(most, S[kt][r]);
                        lift = lift_of(most);
                    }
                    const float up = power_of_two(lift);
#pragma unroll
                    for (int s = 0; s < 2 * KT; ++s) {
                        float x[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = S[s >> 1][8 * (s & 1) + i];
                        frag_t<T> hi, lo;
                        if constexpr (kSplit) split(x, up, hi, lo);
                        else
#pragma unroll
                            for (int i = 0; i < 8; ++i) hi[i] = x[i];
#pragma unroll
                        for (int tt = 0; tt < 2; ++tt) {
                            const frag_t<T> b = read4_4(lds.q + (32 * tt + col) * L::kstride + 16 * s + 4 * half);
                            far[tt] = mfma(hi, b, far[tt]);
                            if constexpr (kSplit) low[tt] = mfma(lo, b, low[tt]);
                        }
                    }
                    const float down = power_of_two(-lift);
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt) {
                        const float f = lds.far[32 * tt + col];
#pragma unroll
                        for (int r = 0; r < 16; ++r) far[tt][r] = (kSplit ? fmaf(low[tt][r], 1.0f / kLow, far[tt][r]) * down : far[tt][r]) * f;
                    }
                }
            }
            // the state behind the chunk
            if (owns) {
                if (a.anchors && !a.reverse) anchor(chunk0 + c);
                float    x[4][8];
                int      lift = 0;
                float    most = 0.0f;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const frag_t<T> b = read_column(lds.v, L::vstride, 16 * s, 32 * wave, lane);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[s][i] = (float)b[i] * lds.keep[16 * s + 8 * half + i];
                        if constexpr (kSplit) most = most_of(most, x[s][i]);
                    }
                }
                if constexpr (kSplit) {
                    lift = lift_of(most);
                    lift = lift > 60 ? 60 : lift;
                }
                const float tot = __builtin_amdgcn_exp2f((float)all) * power_of_two(lift), up = power_of_two(lift), down = power_of_two(-lift);
                acc_t low[KT];
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    low[kt] = zero();
#pragma unroll
                    for (int r = 0; r < 16; ++r) S[kt][r] *= tot;
                }
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    frag_t<T> hi, lo;
                    if constexpr (kSplit) split(x[s], up, hi, lo);
                    else
#pragma unroll
                        for (int i = 0; i < 8; ++i) hi[i] = x[s][i];
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) {
                        const frag_t<T> w = read_column(lds.k, L::kstride, 16 * s, 32 * kt, lane);
                        S[kt] = mfma(w, hi, S[kt]);
                        if constexpr (kSplit) low[kt] = mfma(w, lo, low[kt]);
                    }
                }
                if constexpr (kSplit)
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) S[kt][r] = fmaf(low[kt][r], 1.0f / kLow, S[kt][r]) * down;
                if (a.anchors && a.reverse) anchor(chunk0 + chunks - 1 - c);
            }
            if (OUT) {
                __syncthreads();                            // the scores are there
                if (owns) {
                    acc_t near[2];
                    near[0] = near[1] = zero();
#pragma unroll
                    for (int tile = 0; tile < 3; ++tile) {
                        const int tt = tile > 0, ss = tile > 1;
                        acc_t hi = zero(), lo = zero();
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const frag_t<T> w = read_column(lds.v, L::vstride, 32 * ss + 16 * s, 32 * wave, lane);
                            const T *p = lds.p + (tile * 32 + col) * L::pstride + 16 * s + 8 * half;
                            hi = mfma(w, read8(p), hi);
                            if constexpr (kSplit) lo = mfma(w, read8(p + 3 * 32 * L::pstride), lo);
                        }
                        const float down = kSplit ? power_of_two(-lds.lift[tile]) : 1.0f;
#pragma unroll
                        for (int r = 0; r < 16; ++r) near[tt][r] += kSplit ? fmaf(lo[r], 1.0f / kLow, hi[r]) * down : hi[r];
                    }
                    const int64_t os = (int64_t)a.heads * a.vdim, xs = (int64_t)(a.heads / a.x_div) * a.vdim;
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt) {
                        const int t = 32 * tt + col;
                        const bool there = t < count;
                        const int64_t row = row0 + (int64_t)(there ? t : 0) * dir;
                        float dn = 0.0f, df = 0.0f;
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const int j0 = 32 * wave + 8 * g + 4 * half;
                            float o[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[e] = near[tt][4 * g + e] + far[tt][4 * g + e];
                            if (a.x && there) {
                                const T *x = (const T *)a.x + (size_t)(h / a.x_div) * a.vdim + row * xs + j0;
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float xe = j0 + e < a.vdim ? (float)x[e] : 0.0f;
                                    dn = j0 + e < a.vdim ? fmaf(near[tt][4 * g + e], xe, dn) : dn;
                                    df = j0 + e < a.vdim ? fmaf(far[tt][4 * g + e], xe, df) : df;
                                }
                            }
                            if (there && j0 < a.vdim) {
                                const size_t at = (size_t)(row * os) + (size_t)h * a.vdim + j0;
                                if (a.out_f32 || !kSplit) {
                                    float *to = (float *)a.out + at;
                                    if (a.vec_out) *reinterpret_cast<float4_t *>(to) = float4_t{o[0], o[1], o[2], o[3]};
                                    else
                                        for (int e = 0; e < 4; ++e)
                                            if (j0 + e < a.vdim) to[e] = o[e];
                                } else {
                                    _Float16 *to = (_Float16 *)a.out + at;
                                    if (a.vec_out) *reinterpret_cast<half4_t *>(to) = half4_t{(_Float16)o[0], (_Float16)o[1], (_Float16)o[2], (_Float16)o[3]};
                                    else
                                        for (int e = 0; e < 4; ++e)
                                            if (j0 + e < a.vdim) to[e] = (_Float16)o[e];
                                }
                            }
                        }
                        if (a.x) {
                            dn += __shfl_xor(dn, 32, 64);
                            df += __shfl_xor(df, 32, 64);
                            if (half == 0) {
                                lds.dots[2 * wave][t] = dn;
                                lds.dots[2 * wave + 1][t] = df;
                            }
                        }
                    }
                }
                if (a.x) {
                    __syncthreads();
                    if (threadIdx.x < kChunk && (int)threadIdx.x < count) {
                        float dn = 0.0f, df = 0.0f;
#pragma unroll
                        for (int w = 0; w < VT; ++w) {
                            dn += lds.dots[2 * w][threadIdx.x];
                            df += lds.dots[2 * w + 1][threadIdx.x];
                        }
                        const size_t at = (size_t)h * a.N + (size_t)(row0 + (int64_t)threadIdx.x * dir);
                        a.dot_near[at] = dn;
                        a.dot_far[at] = df;
                    }
                }
            }
            __syncthreads();                                // the tiles may be written again
        }
        if (a.total && threadIdx.x == 0) a.total[state_at] = (float)whole;
        if (a.final && owns && j < a.vdim)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int i = 32 * kt + 8 * (r >> 2) + 4 * half + (r & 3);
                    if (i < a.kdim) a.final[state_at * state_size + (size_t)i * a.final_i + (size_t)j * a.final_j] = S[kt][r];
                }
    }
}

template <typename T, int KT, int VT, bool OUT>
int launch(const WalkArgs &a, hipStream_t s) {
    using L = Lds<T, KT, VT, OUT>;
    if (sizeof(L) > 64 * 1024)
        if (hipError_t e = hipFuncSetAttribute((const void *)attend_walk_kernel<T, KT, VT, OUT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(L)))
            return record_hip_failure(e, "hipFuncSetAttribute(MaxDynamicSharedMemorySize)");
    const int64_t items = (int64_t)a.segments * a.heads;
    LaunchTimer t(s, OUT ? K_ATTEND_WALK : K_ATTEND_STATES);
    attend_walk_kernel<T, KT, VT, OUT><<<(unsigned)std::min<int64_t>(items, kMostGroups256), 64 * L::waves, sizeof(L), s>>>(a);
    return launch_status("attend_walk_kernel");
}

template <typename T, bool OUT>
int launch_tiles(const WalkArgs &a, hipStream_t s) {
    switch (tiles_of(a.kdim) * 8 + tiles_of(a.vdim)) {
        case 8 + 1: return launch<T, 1, 1, OUT>(a, s);
        case 8 + 2: return launch<T, 1, 2, OUT>(a, s);
        case 8 + 4: return launch<T, 1, 4, OUT>(a, s);
        case 16 + 1: return launch<T, 2, 1, OUT>(a, s);
        case 16 + 2: return launch<T, 2, 2, OUT>(a, s);
        case 16 + 4: return launch<T, 2, 4, OUT>(a, s);
        case 32 + 1: return launch<T, 4, 1, OUT>(a, s);
        case 32 + 2: return launch<T, 4, 2, OUT>(a, s);
        default: return launch<T, 4, 4, OUT>(a, s);
    }
}

}  // namespace attend
}  // namespace cngp
