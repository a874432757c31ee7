// The walk of the linear attention (WalkArgs in cngp_attend.h): a workgroup per sequence (or segment) and head goes over its chunks with the
// state in registers.  Everything dense runs on the matrix cores, 32 x 32 x 16 products of fp16 operands with fp32 sums:
//     scores of the pairs of rows       P^T = K Q^T                       (three of the four tiles: a row sees those up to it)
//     outputs inside the chunk          O^T += V^T P^T,  far ones  O^T += S^T Q^T
//     state                             S = e^F S + K^T (V e^(F - F_s))
// A wavefront owns 32 columns of v: of the state, the accumulators themselves (lane = column of v, registers = columns of k), which are at
// the same time the operand of S^T Q^T once they are rounded; the contraction's order is a permutation, the same for Q's reads.  Outputs
// are formed transposed, a row of the chunk per lane, so that decays and products with another row are per lane too.  Scores pass from the
// wavefronts that form them through LDS, or stay in registers where one wavefront does everything (the same permutation again).
// Precision: rounding what is computed (scores, state, decayed v) to fp16 would cost half of the result's accuracy.  It is split in two fp16
// numbers (22 bits) after a power of two has brought its largest value to 2^13, and takes two products.  fp16 storage: q, k, v are
// exact operands.  fp32 storage: they are split as well, each row by a power of two of its own, and products take three (the fp32 products of
// the matrix cores have a sixteenth of the rate: 4096 rays of 64 samples, 4 heads of 16, a walk 526 us, so 104).
// Bound by the chain inside a chunk: two barriers or three, between them vector instructions (38 % of the cycles), LDS (28) and matrix instructions (17)
// that one or two workgroups to a CU do not lay over each other.  2^15 rows, 16 heads of 128 x 128, fp16: 250 us (233 to 264), 1.4 TB/s.
#pragma once
#include "cngp_attend.h"
#include "cngp_matrix.h"

namespace cngp {
namespace attend {

using namespace mat;

// The same for the whole wavefront, and known to be: addresses formed from it are scalar.  (Rows are numbers below 2^31.)
__device__ __forceinline__ Span scalar(const Span s) { return {__builtin_amdgcn_readfirstlane(s.begin), __builtin_amdgcn_readfirstlane(s.end)}; }

// A tile [64, W] of an array on its way into LDS: rows t of a chunk, `stride` values apart, `dim` of them (the rest and rows from `count` on are
// 0).  Reverse walks take rows from the last to the first.  Where 16-byte pieces lie whole in the rows they are fetched into registers a chunk
// ahead; else values are read one by one on the way.  Addresses are a scalar base and one 32-bit offset per lane.
template <typename T, int W, int LDS_STRIDE, int WAVES, bool WHOLE>
struct Staged {
    static constexpr int per_row = W / 8, dealt = WAVES * 64 / per_row, rows = dealt < kChunk ? dealt : kChunk, each = kChunk / rows, words = sizeof(T) / 2;
    static_assert(rows * each == kChunk, "a tile is dealt out evenly");
    words_t  r[each][words];
    uint32_t offset;                     // bytes from the lowest row of a whole chunk
    int      row;

    __device__ __forceinline__ void begin(const int stride, const bool reverse) {
        row = (int)threadIdx.x / per_row;
        offset = (uint32_t)((reverse ? kChunk - 1 - row : row) * stride + (int)threadIdx.x % per_row * 8) * (uint32_t)sizeof(T);
    }
    // low: the row where a whole chunk would begin in memory
    __device__ __forceinline__ void load(const T *low, const bool reverse, const int count, const int stride, const int dim) {
        const int column = (int)threadIdx.x % per_row * 8;
        if constexpr (!WHOLE) return;
#pragma unroll
        for (int i = 0; i < each; ++i) {
            const char *p = (const char *)(low + (int64_t)(reverse ? -i * rows : i * rows) * stride);
#pragma unroll
            for (int w = 0; w < words; ++w) {
                r[i][w] = words_t{0, 0, 0, 0};
                if (column + (int)(16 / sizeof(T)) * w < dim && row + i * rows < count) r[i][w] = *reinterpret_cast<const words_t *>(p + 16 * w + offset);
            }
        }
    }
    // hi, lo: the parts of the tile; lift: of each row (fp32 only)
    __device__ __forceinline__ void put(_Float16 *hi, _Float16 *lo, short *lift, const int t, const words_t (&v)[words]) const {
        if (dealt > kChunk && t >= kChunk) return;
        const int at = t * LDS_STRIDE + (int)threadIdx.x % per_row * 8;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<words_t *>(hi + at) = v[0];
        } else {
            float x[8];
            __builtin_memcpy(x, &v, sizeof x);
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
            const int up = lift_of_lanes<per_row>(most);
            half8_t   h, l;
            split(x, power_of_two(up), h, l);
            *reinterpret_cast<half8_t *>(hi + at) = h;
            *reinterpret_cast<half8_t *>(lo + at) = l;
            if (threadIdx.x % per_row == 0) lift[t] = (short)up;
        }
    }
    __device__ __forceinline__ void store(_Float16 *hi, _Float16 *lo, short *lift, const T *low, const bool reverse, const int count, const int stride, const int dim) const {
        if constexpr (WHOLE) {
#pragma unroll
            for (int i = 0; i < each; ++i) put(hi, lo, lift, row + i * rows, r[i]);
            return;
        }
        const int column = (int)threadIdx.x % per_row * 8;
#pragma unroll 1
        for (int i = 0; i < each; ++i) {
            const int t = row + i * rows;
            T x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (T)0.0f;
            if (t < count) {
                const T *p = low + (int64_t)(reverse ? kChunk - 1 - t : t) * stride;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int c = column + e < dim ? column + e : dim - 1;
                    x[e] = column + e < dim ? p[c] : (T)0.0f;
                }
            }
            words_t v[words];
            __builtin_memcpy(&v, x, sizeof x);
            put(hi, lo, lift, t, v);
        }
    }
};

// (walk_waves.)  One wavefront on a SIMD waits most of the time, so what it does in a row is kept short.
constexpr int walk_halves(int KW) { return walk_waves(KW, 1); }
constexpr int walk_threads(int KW, int VW) { return 64 * walk_waves(KW, VW); }
// Wavefronts of a SIMD that registers are left for.
constexpr int walk_per_simd(size_t value, int KW) { return value == 2 || KW < 128 ? 2 : 1; }

// What a walk is for: states alone; outputs; outputs with a row's own part kept apart and what the decays' gradient takes of them (in a walk of its own: it
// costs registers, with which the plain one took 316 us for a prompt in place of 306).
enum Mode { STATES, OUTPUTS, GRADIENTS };

// KW, VW: columns of k and v in a tile: 16, 32, 64 or 128.  Sums of 32 rows or columns where 16 are kept read what lies behind a row in LDS;
// the rows and columns of the state that come of it are used by nothing.
// Banks: the scores read 16 bytes of sixteen rows, so rows have an odd number of 16-byte pieces; a transposing read takes 64 bytes of four neighbouring
// rows, for which rows of 128 values are 64 bytes beyond a multiple of 256 (v, read by that alone) or five pieces (k) (128 x 128: 338 against 344 us a
// prompt; of 64 values it gained nothing).
template <typename T, int KW, int VW, Mode MODE>
struct Lds {
    static constexpr bool OUT = MODE != STATES, kDots = MODE == GRADIENTS;
    static constexpr int kstride = KW + (KW == 128 ? 40 : KW == 16 ? 0 : 8), vstride = VW + (VW == 128 ? 32 : VW == 16 ? 0 : 8);     // see above
    static constexpr int parts = sizeof(T) / 2, pstride = 32 + 8, KT = (KW + 31) / 32, VT = (VW + 31) / 32;
    static constexpr int halves = walk_halves(KW), waves = VT * halves;
    static constexpr bool scores = OUT && waves > 1;        // pass through LDS
    static constexpr int decays = waves > 1 ? 2 : 1;        // this chunk's, and the next one's where another wavefront makes them ready
    union {
        double F[kChunk];                                   // log2 of the decay from the chunk's start
        struct { float from[kChunk], to[kChunk]; };         // ... or, of mild chunks, the decay between two rows as a product, to[t] * from[s]
    } between[decays];
    float  far[decays][kChunk], keep[decays][kChunk];       // what a row takes from the state, and gives to it
    double total[decays];
    int    mild[decays];
    int    lift[4];                                         // of each score tile
    float  own[scores && kDots ? kChunk : 1];               // a row's score with itself, where it is kept apart
    short  up_q[parts == 2 ? kChunk : 1], up_k[parts == 2 ? kChunk : 1], up_v[parts == 2 ? kChunk : 1];     // lifts of the rows
    static constexpr bool folds = parts == 2 && waves == 1; // ... which go into the decays once a chunk, where no barrier is needed for that (rays: 474 against 509 us)
    float  down[folds ? kChunk : 1];                        // 2^-(lifts of k and v)
    float  dots[kDots && VT > 1 ? VT : 1][kDots && VT > 1 ? kChunk : 1];
    union {
        struct {
            alignas(16) _Float16 k[parts][kChunk * kstride];
            alignas(16) _Float16 q[parts][OUT ? kChunk * kstride : 8];
        };
        float far_half[OUT && halves == 2 ? waves : 1][16][64];     // when both tiles have been used: far outputs of the other half's rows
    };
    alignas(16) _Float16 v[parts][kChunk * vstride];
    alignas(16) _Float16 p[2][scores ? 3 * 32 * pstride : 8];
};

// A chunk's decays are mild where none is more than 2^kMild away from the middle row's: two factors in place of an exponential per pair
// of rows then, and the later row's outside the sums.  (A tile of scores spans 2^(2 kMild) by that, of the 2^28 that its high parts hold.)
constexpr double kMild = 6.0;

// Sum over the lanes 0 .. own: moves inside rows of 16 lanes, then broadcasts of the rows' last ones.
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(const double v) {
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)w, CTRL, ROWS, 0xF, ROWS == 0xF);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(w >> 32), CTRL, ROWS, 0xF, ROWS == 0xF);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double sum_upto(double v) {
    v += moved<0x111, 0xF>(v);
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);
    v += moved<0x143, 0xC>(v);
    return v;
}

template <typename T, int KW, int VW, Mode MODE, bool WHOLE>
__global__ __launch_bounds__(walk_threads(KW, VW), walk_per_simd(sizeof(T), KW)) void attend_walk_kernel(const WalkArgs a)
{
    using L = Lds<T, KW, VW, MODE>;
    constexpr bool OUT = L::OUT, kDots = L::kDots;
    constexpr int  WAVES = L::waves, VT = L::VT, KT = L::KT, HALVES = L::halves, KP = KT / HALVES;
    constexpr int  KS = KW / 16 / HALVES;                   // steps of 16 columns of k that a wavefront keeps
    constexpr int  KR = KW < 32 ? 8 : 16, VR = VW < 32 ? 8 : 16;      // registers of a tile's sums that hold rows of the state, and of the outputs
    constexpr bool kLow = sizeof(T) == 4;                   // the inputs have low parts too
    extern __shared__ __align__(16) char lds_raw[];
    L &lds = *reinterpret_cast<L *>(lds_raw);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int vt = wave % VT, kh = wave / VT;               // this wavefront's columns of v; its half of the columns of k, and of the chunk's rows
    // Workgroups go to the eight XCDs in turn, each with an L2 of its own: neighbouring heads, which share keys or lines of memory, to the same one.
    const uint32_t each = gridDim.x >> 3, rest = gridDim.x & 7, xcd = blockIdx.x & 7, item = xcd * each + (xcd < rest ? xcd : rest) + (blockIdx.x >> 3);
    const int h = (int)(item % (uint32_t)a.heads);
    const int qs = a.heads / a.q_div * a.kdim, ks = a.heads / a.k_div * a.kdim, vs = a.heads / a.v_div * a.vdim;
    const T *q = (const T *)a.q + h / a.q_div * a.kdim, *k = (const T *)a.k + h / a.k_div * a.kdim, *v = (const T *)a.v + h / a.v_div * a.vdim;
    const int j = 32 * vt + col;                            // this lane's column of v
    const bool mine_v = j < a.vdim;

    const int32_t piece = a.piece0 + (int32_t)(item / (uint32_t)a.heads);
    const int32_t seq = __builtin_amdgcn_readfirstlane(a.seg_rows ? sequence_of(a.offsets, piece, a.N, a.S, a.rows_each, a.seg_rows) : piece);
    const Span    span = scalar(span_of(a.offsets, seq, a.N, a.rows_each));
    int begin = span.begin, end = span.end;
    int chunk0 = 0;                                         // the first chunk's number in its sequence
    if (a.seg_rows) {
        const int i = piece - piece_base(span.begin, seq, a.seg_rows);
        if (i < 0 || (int64_t)begin + (int64_t)i * a.seg_rows >= end) return;      // (i < 0: rows before the first sequence)
        begin += i * a.seg_rows;
        end = end - begin > a.seg_rows ? begin + a.seg_rows : end;
        chunk0 = i * (a.seg_rows >> kChunkShift);
    }
    const int chunks = (end - begin + kChunk - 1) >> kChunkShift;
    const int64_t state_at = (int64_t)piece * a.heads + h;  // whole sequences: piece == sequence
    const size_t  state_bytes = (size_t)(a.kdim * a.vdim) * 4;
    const bool    reverse = a.reverse;
    const int     dir = reverse ? -1 : 1;

    // chunk c of the walk: its first row (reverse: its last), how many, and the row where a whole chunk of these would begin in memory
    auto place = [&](const int c, int &row0, int &count, int &low) {
        const int at = begin + (reverse ? chunks - 1 - c : c) * kChunk;
        count = end - at < kChunk ? end - at : kChunk;
        row0 = reverse ? at + count - 1 : at;
        low = reverse ? row0 - (kChunk - 1) : row0;
    };
    Staged<T, KW, L::kstride, WAVES, WHOLE> rq, rk;
    Staged<T, VW, L::vstride, WAVES, WHOLE> rv;
    if (OUT) rq.begin(qs, reverse);
    rk.begin(ks, reverse);
    rv.begin(vs, reverse);
    auto fetch = [&](const int c) {
        int row0, low, count;
        place(c, row0, count, low);
        if (OUT) rq.load(q + (int64_t)low * qs, reverse, a.q ? count : 0, qs, a.kdim);
        rk.load(k + (int64_t)low * ks, reverse, a.k ? count : 0, ks, a.kdim);
        rv.load(v + (int64_t)low * vs, reverse, a.v ? count : 0, vs, a.vdim);
    };
    // the decays of chunk c, by the last wavefront (which has the least to do with the scores), a chunk ahead; their loads another chunk ahead
    float  rdecay = 0.0f;
    double whole = 0.0;
    auto fetch_decays = [&](const int c) {
        int row0, low, count;
        place(c, row0, count, low);
        if (wave == WAVES - 1) rdecay = lane < count ? a.row_decay ? a.decay[(int64_t)(row0 + lane * dir) * a.heads + h] : a.decay[h] : 0.0f;
    };
    auto decays = [&](const int c) {
        if (wave != WAVES - 1) return;
        // below -110 a decay is 0 in fp32 however it is joined; bounded, sums of them stay exact enough to be subtracted
        const double g = (double)(rdecay < -110.0f ? -110.0f : rdecay) * 1.4426950408889634, f = sum_upto(g);
        if (c + 1 < chunks) fetch_decays(c + 1);
        const double all = __shfl(f, 63, 64), mine = reverse ? f - g : f;
        const int at = c % L::decays;
        lds.far[at][lane] = __builtin_amdgcn_exp2f((float)mine) * a.far_scale;
        lds.keep[at][lane] = __builtin_amdgcn_exp2f((float)(all - mine)) * a.state_scale;
        const double middle = __shfl(mine, 31, 64);
        const bool   mild = __all(fabs(mine - middle) <= kMild);
        if (mild) {
            lds.between[at].to[lane] = __builtin_amdgcn_exp2f((float)(mine - middle));
            lds.between[at].from[lane] = __builtin_amdgcn_exp2f((float)(middle - mine));
        } else lds.between[at].F[lane] = mine;
        if (lane == 0) {
            lds.total[at] = all;
            lds.mild[at] = mild;
        }
    };
    constexpr bool kAhead = WAVES > 1;                      // a chunk's rows are fetched while the one before is worked on (short rows: registers that
                                                            // another wavefront has more of, 740 against 725 us a pass of 4096 rays)
    if (chunks > 0) {
        fetch_decays(0);
        if (kAhead) fetch(0);
    }

    acc_t S[KP];
    {
        const char *from = a.first ? (const char *)a.first + state_at * state_bytes : nullptr;
        uint32_t  at = (uint32_t)((32 * KP * kh + 4 * half) * a.first_i + j * a.first_j) * 4;
        const int left = a.kdim - 32 * KP * kh - 4 * half;
#pragma unroll
        for (int kt = 0; kt < KP; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                S[kt][r] = 0.0f;
                if (from && mine_v && 32 * kt + 8 * (r >> 2) + (r & 3) < left) S[kt][r] = *reinterpret_cast<const float *>(from + at);
                at += (uint32_t)(r % 4 == 3 ? 5 : 1) * (uint32_t)a.first_i * 4;
            }
    }
    int up = 0;                          // the state is kept times 2^up, the scale of what is added to it
    // the state at the start of chunk `number` of its sequence, as it lies in the registers (rows behind kdim in a piece of four are 0)
    auto anchor_of = [&](const int number) -> float * {
        return a.anchors + ((size_t)anchor_slot(span.begin, number) * a.heads + h) * (KT * VT * 1024) + (vt * KT + kh * KP) * 1024 + 4 * lane;
    };
    auto leave_anchor = [&](const int number) {
        if (number == 0) return;
        float *to = anchor_of(number);
        const float f = power_of_two(-up);
        const int   left = anew(a.kdim - 32 * KP * kh - 4 * half);
#pragma unroll
        for (int kt = 0; kt < KP; ++kt)
#pragma unroll
            for (int g = 0; g < KR / 4; ++g)
                if (mine_v && 32 * kt + 8 * g < left)
                    *reinterpret_cast<float4_t *>(to + (kt * 4 + g) * 256) = float4_t{S[kt][4 * g] * f, S[kt][4 * g + 1] * f, S[kt][4 * g + 2] * f, S[kt][4 * g + 3] * f};
    };
    // this wavefront's part of the state's product with another one (an anchor, or a state of whole sequences): four at a time in fp32, these in 64 bits
    auto meet = [&](const bool an_anchor, const int number, double *to) {
        const float   *from = an_anchor ? anchor_of(number) : a.met + (size_t)seq * a.kdim * a.vdim * a.heads + (size_t)h * a.kdim * a.vdim;
        const float    f = power_of_two(-up);
        const int      left = anew(a.kdim - 32 * KP * kh - 4 * half);
        const float   *mine = an_anchor ? from : from + anew(32 * KP * kh + 4 * half + j * a.first_j);      // (such a walk's states have rows side by side)
        double sum = 0.0;
        apart();
        float4_t o[KP][KR / 4];
#pragma unroll
        for (int kt = 0; kt < KP; ++kt)
#pragma unroll
            for (int g = 0; g < KR / 4; ++g) {
                const int i = 32 * kt + 8 * g;
                o[kt][g] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
                if (!mine_v || i >= left) continue;
                if (an_anchor) o[kt][g] = *reinterpret_cast<const float4_t *>(mine + (kt * 4 + g) * 256);
                else if (WHOLE) o[kt][g] = *reinterpret_cast<const float4_t *>(mine + i);
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < left) o[kt][g][e] = mine[i + e];
            }
#pragma unroll
        for (int kt = 0; kt < KP; ++kt)
#pragma unroll
            for (int g = 0; g < KR / 4; ++g) {
                float t = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) t = fmaf(S[kt][4 * g + e] * f, o[kt][g][e], t);
                if (mine_v && 32 * kt + 8 * g < left) sum += (double)t;
            }
        sum = sum_upto(sum);
        if (lane == 63) to[wave] = sum;
    };
    if (chunks > 0) decays(0);

    for (int c = 0; c < chunks; ++c) {
        const int now = c % L::decays;
        int row0, low, count;
        place(c, row0, count, low);
        if (!kAhead) fetch(c);
        if (OUT) rq.store(lds.q[0], lds.q[L::parts - 1], lds.up_q, q + (int64_t)low * qs, reverse, a.q ? count : 0, qs, a.kdim);
        rk.store(lds.k[0], lds.k[L::parts - 1], lds.up_k, k + (int64_t)low * ks, reverse, a.k ? count : 0, ks, a.kdim);
        rv.store(lds.v[0], lds.v[L::parts - 1], lds.up_v, v + (int64_t)low * vs, reverse, a.v ? count : 0, vs, a.vdim);
        __syncthreads();
        if constexpr (L::folds) {
            const float down = ldexpf(1.0f, -(lds.up_k[lane] + lds.up_v[lane])), down_q = OUT ? ldexpf(1.0f, -lds.up_q[lane]) : 0.0f;
            lds.down[lane] = down;
            lds.keep[now][lane] *= down;
            if (OUT) lds.far[now][lane] *= down_q;
            if (OUT && lds.mild[now]) {
                lds.between[now].from[lane] *= down;
                lds.between[now].to[lane] *= down_q;
            }
            __syncthreads();
        }
        const double all = lds.total[now];
        whole += all;
        if (c + 1 < chunks) {
            if (kAhead && !OUT) fetch(c + 1);
            if (WAVES > 1) decays(c + 1);
        }

        const bool mild = OUT && __builtin_amdgcn_readfirstlane(lds.mild[now]);
        // scores of rows 32 tt .. (lanes) with rows 32 ss .. (registers), the decay between them (without the later row's part where mild), and the
        // power of two they are brought up by; what is the same for a row is left to the sums over ss
        [[maybe_unused]] auto score = [&](const int tt, const int ss, acc_t &p, float &own) -> int {
            p = zero();
            own = 0.0f;
            if constexpr (!OUT) return 0;
            const int qa = (32 * tt + col) * L::kstride + 8 * half, ka = (32 * ss + col) * L::kstride + 8 * half;
#pragma unroll
            for (int s = 0; s < KW / 16; ++s) {
                const half8_t kf = read8(lds.k[0] + ka + 16 * s), qf = read8(lds.q[0] + qa + 16 * s);
                p = mfma(kf, qf, p);
                if constexpr (kLow) {
                    p = mfma(read8(lds.k[1] + ka + 16 * s), qf, p);
                    p = mfma(kf, read8(lds.q[1] + qa + 16 * s), p);
                }
            }
            float most = 0.0f;
            if (mild) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int s = 32 * ss + 8 * (r >> 2) + 4 * half + (r & 3);
                    p[r] *= lds.between[now].from[s];
                    if constexpr (kLow && !L::folds) p[r] = ldexpf(p[r], -(lds.up_k[s] + lds.up_v[s]));
                }
            } else {
                const double Ft = lds.between[now].F[32 * tt + col];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int s = 32 * ss + 8 * (r >> 2) + 4 * half + (r & 3);
                    p[r] *= __builtin_amdgcn_exp2f((float)(Ft - lds.between[now].F[s]));
                    if constexpr (L::folds) p[r] *= lds.down[s];
                    else if constexpr (kLow) p[r] = ldexpf(p[r], -(lds.up_k[s] + lds.up_v[s]));
                }
            }
            if (ss == tt) {
                const int t = anew(col - 4 * half), last = kDots ? t - 1 : t;
                if (kDots)
#pragma unroll
                    for (int r = 0; r < 16; ++r) own = 8 * (r >> 2) + (r & 3) == t ? p[r] : own;
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] = 8 * (r >> 2) + (r & 3) <= last ? p[r] : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(p[r]));
            return lift_of(most);
        };
        if constexpr (L::scores) {
            for (int tile = wave; tile < (count > 32 ? 3 : 1); tile += WAVES) {
                acc_t p;
                float own;
                const int   lift = score(tile > 0, tile > 1, p, own);
                if (kDots && tile != 1 && half == (col >> 2 & 1)) lds.own[tile ? 32 + col : col] = own;
                const float f = power_of_two(lift);
                if (lane == 0) lds.lift[tile] = lift;
                _Float16 *to = lds.p[0] + (tile * 32 + col) * L::pstride + 4 * half;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    half4_t hi, lo;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        hi[e] = (_Float16)(p[4 * g + e] * f);
                        lo[e] = (_Float16)fmaf(p[4 * g + e], f, -(float)hi[e]);
                    }
                    *reinterpret_cast<half4_t *>(to + 8 * g) = hi;
                    *reinterpret_cast<half4_t *>(to + 3 * 32 * L::pstride + 8 * g) = lo;
                }
            }
            apart();
        }

        int lift = 0;                    // brings the state into the range of its fp16 parts
        if (OUT) {
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < 8 * KS; ++i) most = fmaxf(most, fabsf(S[i >> 4][i & 15]));
            lift = lift_of(mine_v ? most : 0.0f);
        }
        // what rows 32 tt .. take from this wavefront's part of the state
        const float lifted = power_of_two(lift);
        auto part_of_state = [&](const int tt) -> acc_t {
            acc_t far = zero();
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = S[s >> 1][8 * (s & 1) + i];
                half8_t hi, lo;
                split(x, lifted, hi, lo);
                const int     at = (32 * tt + col) * L::kstride + 16 * (KS * kh + s) + 4 * half;
                const half8_t b = read4_4(lds.q[0] + at);
                far = mfma(hi, b, far);
                far = mfma(lo, b, far);
                if constexpr (kLow) far = mfma(hi, read4_4(lds.q[1] + at), far);
            }
            const float f = ldexpf(lds.far[now][32 * tt + col], -(up + lift + (kLow && !L::folds ? lds.up_q[32 * tt + col] : 0)));
#pragma unroll
            for (int r = 0; r < VR; ++r) far[r] *= f;
            return far;
        };
        acc_t far, other;                // of this wavefront's rows, and of the other half's
        if constexpr (OUT && HALVES == 2) {
            far = part_of_state(kh);
            other = part_of_state(1 - kh);
            apart();
        }

        auto state_behind = [&]() {
            if (kDots && a.anchors && !reverse) leave_anchor(chunk0 + c);
            // rows 16 s + 8 half .. + 7 of this lane's column, decayed to the chunk's end
            float x[4][8];
            float most = 0.0f;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const half8_t b = read_column(lds.v[0], L::vstride, 16 * s, 32 * vt, lane);
                half8_t l = b;
                if constexpr (kLow) l = read_column(lds.v[1], L::vstride, 16 * s, 32 * vt, lane);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int t = 16 * s + 8 * half + i;
                    x[s][i] = L::folds ? ((float)b[i] + (float)l[i]) * lds.keep[now][t] : kLow ? ((float)b[i] + (float)l[i]) * ldexpf(lds.keep[now][t], -(lds.up_k[t] + lds.up_v[t])) : (float)b[i] * lds.keep[now][t];
                    most = fmaxf(most, fabsf(x[s][i]));
                }
            }
            const uint32_t in = wave_top(mine_v ? most : 0.0f);
            const int      to = in ? lift_from(in, 60) : up;
            const float    scale = power_of_two(to), tot = ldexpf(__builtin_amdgcn_exp2f((float)all), to - up);
            up = to;
#pragma unroll
            for (int kt = 0; kt < KP; ++kt)
#pragma unroll
                for (int r = 0; r < KR; ++r) S[kt][r] *= tot;
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s && 16 * s >= count) break;            // (no rows there)
                half8_t hi, lo;
                split(x[s], scale, hi, lo);
#pragma unroll
                for (int kt = 0; kt < KP; ++kt) {
                    const half8_t w = read_column(lds.k[0], L::kstride, 16 * s, 32 * (KP * kh + kt), lane);
                    S[kt] = mfma(w, hi, S[kt]);
                    S[kt] = mfma(w, lo, S[kt]);
                    if constexpr (kLow) S[kt] = mfma(read_column(lds.k[1], L::kstride, 16 * s, 32 * (KP * kh + kt), lane), hi, S[kt]);
                }
            }
            if (kDots && a.anchors && reverse) {
                const int number = chunk0 + chunks - 1 - c;
                if (number || a.met) meet(number != 0, number, a.products + ((size_t)chunk_number(span.begin, seq, number) * a.heads + h) * WAVES);
            }
            apart();
        };
        if (!OUT || HALVES == 2) state_behind();
        if (kAhead && c + 1 < chunks && OUT) fetch(c + 1);

        if constexpr (OUT) {
            if (WAVES > 1) __syncthreads();                 // the scores are there; q and k have been used
            if constexpr (HALVES == 2) {
#pragma unroll
                for (int r = 0; r < VR; ++r) lds.far_half[wave][r][lane] = other[r];
            }
            const int os = a.heads * a.vdim, xs = a.heads / a.x_div * a.vdim;
            const int t0 = reverse ? kChunk - 1 - col : col, j0 = 32 * vt + 4 * half, left = anew(a.vdim - j0);      // columns from j0 on
#pragma unroll 1
            for (int tt = HALVES == 2 ? kh : 0; tt < (HALVES == 2 ? kh + 1 : count > 32 ? 2 : 1); ++tt) {
                acc_t near = zero();
                if constexpr (HALVES == 1) far = part_of_state(tt);
                const int   t = 32 * tt + col;
                [[maybe_unused]] float own = 0.0f;           // score of the row with itself
                const float of_row = ldexpf(mild ? a.pair_scale * lds.between[now].to[t] : a.pair_scale, kLow && !(L::folds && mild) ? -lds.up_q[t] : 0);
#pragma unroll 1
                for (int ss = 0; ss <= tt && 32 * tt < count; ++ss) {
                    acc_t sum = zero(), p;
                    int   lift;
                    if constexpr (L::scores) lift = __builtin_amdgcn_readfirstlane(lds.lift[tt + ss]);
                    else lift = score(tt, ss, p, own);
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        half8_t hi, lo;
                        if constexpr (L::scores) {
                            const _Float16 *from = lds.p[0] + ((tt + ss) * 32 + col) * L::pstride + 16 * s + 8 * half;
                            hi = read8(from);
                            lo = read8(from + 3 * 32 * L::pstride);
                        } else {
                            float y[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) y[i] = p[8 * s + i];
                            split(y, power_of_two(lift), hi, lo);
                        }
                        const half8_t w = read_column<!L::scores>(lds.v[0], L::vstride, 32 * ss + 16 * s, 32 * vt, lane);
                        sum = mfma(w, hi, sum);
                        sum = mfma(w, lo, sum);
                        if constexpr (kLow) sum = mfma(read_column<!L::scores>(lds.v[1], L::vstride, 32 * ss + 16 * s, 32 * vt, lane), hi, sum);
                    }
                    const float down = power_of_two(-lift) * of_row;
#pragma unroll
                    for (int r = 0; r < VR; ++r) near[r] = fmaf(sum[r], down, near[r]);
                    apart();
                }
                if constexpr (HALVES == 2) {
                    __syncthreads();
#pragma unroll
                    for (int r = 0; r < VR; ++r) far[r] += lds.far_half[wave < VT ? wave + VT : wave - VT][r][lane];
                }
                if (kDots) {
                    if constexpr (L::scores) own = lds.own[t];
                    else own += __shfl_xor(own, 32, 64);
                    own *= of_row;
                }
                const bool there = t < count;
                const int  base = low + (reverse ? -32 * tt : 32 * tt);
                float dot = 0.0f;
                if (kDots && a.x && there) {
                    const T *x = (const T *)a.x + h / a.x_div * a.vdim + (int64_t)base * xs;
                    const uint32_t mine = (uint32_t)(t0 * xs + j0);
#pragma unroll
                    for (int g = 0; g < VR / 4; ++g) {
                        float w[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        if (WHOLE) {
                            if (8 * g < left) {
                                T e4[4];
                                __builtin_memcpy(e4, (x + 8 * g) + mine, sizeof e4);
#pragma unroll
                                for (int e = 0; e < 4; ++e) w[e] = (float)e4[e];
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (8 * g + e < left) w[e] = (float)(x + 8 * g + e)[mine];
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (8 * g + e < left) dot = fmaf(near[4 * g + e] + far[4 * g + e], w[e], dot);
                    }
                }
                if (there) {
                    const uint32_t mine = (uint32_t)(t0 * os + j0);
                    float    *to32 = (float *)a.out + h * a.vdim + (int64_t)base * os;
                    _Float16 *to16 = (_Float16 *)a.out + h * a.vdim + (int64_t)base * os;
#pragma unroll
                    for (int g = 0; g < VR / 4; ++g) {
                        float o[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] = near[4 * g + e] + far[4 * g + e];
                        if (kDots) {
                            const _Float16 *mine_v = lds.v[0] + t * L::vstride + j0 + 8 * g;
                            const half4_t   hi = *reinterpret_cast<const half4_t *>(mine_v), lo = *reinterpret_cast<const half4_t *>(mine_v + (kLow ? kChunk * L::vstride : 0));
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[e] = fmaf(own, kLow ? (float)hi[e] + (float)lo[e] : (float)hi[e], o[e]);
                        }
                        if (WHOLE) {
                            if (8 * g < left) {
                                if (kLow || a.out_f32) *reinterpret_cast<float4_t *>((to32 + 8 * g) + mine) = float4_t{o[0], o[1], o[2], o[3]};
                                else *reinterpret_cast<half4_t *>((to16 + 8 * g) + mine) = half4_t{(_Float16)o[0], (_Float16)o[1], (_Float16)o[2], (_Float16)o[3]};
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (8 * g + e < left) {
                                    if (kLow || a.out_f32) (to32 + 8 * g + e)[mine] = o[e];
                                    else (to16 + 8 * g + e)[mine] = (_Float16)o[e];
                                }
                        }
                    }
                }
                if (kDots && a.x) {
                    dot += __shfl_xor(dot, 32, 64);
                    if (VT == 1) {
                        if (half == 0 && there) a.dot[(size_t)h * a.N + (size_t)(row0 + t * dir)] = dot;
                    } else if (half == 0) lds.dots[vt][t] = dot;
                }
                apart();
            }
            if (HALVES == 1) state_behind();
            if (kDots && VT > 1 && a.x) {
                __syncthreads();
                if (threadIdx.x < kChunk && (int)threadIdx.x < count) {
                    float dot = 0.0f;
#pragma unroll
                    for (int w = 0; w < VT; ++w) dot += lds.dots[w][threadIdx.x];
                    a.dot[(size_t)h * a.N + (size_t)(row0 + (int)threadIdx.x * dir)] = dot;
                }
            }
        }
        if (c + 1 < chunks) {
            if (WAVES == 1) decays(c + 1);
            __syncthreads();                                // the tiles may be written again
        }
    }
    if (kDots && a.anchors && !reverse && a.met && chunks > 0 && end == span.end) meet(false, 0, a.products + ((size_t)seq * a.heads + h) * WAVES);
    if (a.total && threadIdx.x == 0) a.total[state_at] = (float)whole;
    if (a.final && mine_v) {
        char     *to = (char *)a.final + state_at * state_bytes;
        uint32_t  at = (uint32_t)((32 * KP * kh + 4 * half) * a.final_i + j * a.final_j) * 4;
        const int left = anew(a.kdim - 32 * KP * kh - 4 * half);
        const float f = power_of_two(-up);
#pragma unroll
        for (int kt = 0; kt < KP; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (32 * kt + 8 * (r >> 2) + (r & 3) < left) *reinterpret_cast<float *>(to + at) = S[kt][r] * f;
                at += (uint32_t)(r % 4 == 3 ? 5 : 1) * (uint32_t)a.final_i * 4;
            }
    }
}

template <typename T, int KW, int VW, Mode MODE, bool WHOLE>
int launch_walk(const WalkArgs &a, hipStream_t s) {
    using L = Lds<T, KW, VW, MODE>;
    static_assert(L::waves == walk_waves(KW, VW), "the host counts them alike");
    if (sizeof(L) > 64 * 1024)
        if (hipError_t e = hipFuncSetAttribute((const void *)attend_walk_kernel<T, KW, VW, MODE, WHOLE>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(L)))
            return record_hip_failure(e, "hipFuncSetAttribute(MaxDynamicSharedMemorySize)");
    // a workgroup goes over one piece: a loop over pieces would have the addresses of the states' entries formed before it and kept in registers
    const int most = (int)(kMostGroups256 / 2 / a.heads);   // (workgroups of up to 512)
    for (int first = 0; first < a.segments; first += most) {
        WalkArgs part = a;
        part.piece0 = first;
        LaunchTimer t(s, MODE == STATES ? K_ATTEND_STATES : K_ATTEND_WALK);
        attend_walk_kernel<T, KW, VW, MODE, WHOLE><<<(unsigned)a.heads * (unsigned)std::min(a.segments - first, most), 64 * L::waves, sizeof(L), s>>>(part);
        if (int rc = launch_status("attend_walk_kernel")) return rc;
    }
    return CNGP_OK;
}

template <typename T, int KW, int VW, Mode MODE>
int launch(const WalkArgs &a, hipStream_t s) { return a.whole ? launch_walk<T, KW, VW, MODE, true>(a, s) : launch_walk<T, KW, VW, MODE, false>(a, s); }

template <typename T, Mode MODE, int KW>
int launch_columns(const WalkArgs &a, hipStream_t s) {
    return a.vdim <= 16 ? launch<T, KW, 16, MODE>(a, s) : a.vdim <= 32 ? launch<T, KW, 32, MODE>(a, s) : a.vdim <= 64 ? launch<T, KW, 64, MODE>(a, s) : launch<T, KW, 128, MODE>(a, s);
}
template <typename T, Mode MODE>
int launch_mode(const WalkArgs &a, hipStream_t s) {
    return a.kdim <= 16 ? launch_columns<T, MODE, 16>(a, s) : a.kdim <= 32 ? launch_columns<T, MODE, 32>(a, s) : a.kdim <= 64 ? launch_columns<T, MODE, 64>(a, s)
                                                                                                           : launch_columns<T, MODE, 128>(a, s);
}
template <typename T>
int launch_tiles(const WalkArgs &a, bool states_only, hipStream_t s) {
    return states_only ? launch_mode<T, STATES>(a, s) : a.own ? launch_mode<T, GRADIENTS>(a, s) : launch_mode<T, OUTPUTS>(a, s);
}

}  // namespace attend
}  // namespace cngp
