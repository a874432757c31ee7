// Balance of the probing candidates: winners per candidate, the loss N_p sum_k f_k P_k of every level and its gradient.
//
// With sigma = softmax of a row, f and P the means over a level's rows of "candidate k won" and of sigma_k:
//     d loss / d logit_rk = N_p / W * sigma_rk (f_k - sum_j f_j sigma_rj)
// The gradient of every row needs the level's f, so two launches: one reads the logits and leaves sums per workgroup, the other
// adds those up (in a fixed order), reads the logits again and writes the gradient.  A level that one workgroup can hold in registers
// takes one launch.  16 levels x 2^18 rows x 16 logits, the four largest kept: 181 us, 105 + 96 where each launch is profiled by itself; reading
// 268 MB twice and writing it once is 805 MB, 113 us at the rates of a large read and a large fill.  The first launch is bound by the vector
// ALU (the ranks), the second by memory.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include <hip/hip_runtime.h>

#include "cngp_launch.h"

namespace {

using namespace cngp;

constexpr int kBalBlock = 256;
constexpr int kMostChunks = 128;         // workgroups per level: the second launch reads this many partial sums per candidate
constexpr int kLevelBlock = 1024, kLevelGroups = 2;      // one launch: groups of a lane

struct BalArgs {
    const float   *logits;
    const uint8_t *rows;
    float         *grad;
    float         *loss;
    int32_t       *counts;
    float         *part_p;               // [L][chunks][NP]
    int32_t       *part_n;               // [L][chunks][NP] winners
    uint16_t      *kept;                 // [L][groups] which logits keep weight, top_k < N_p
    uint32_t       N_c, groups;          // rows of a level, lanes' worth of them
    uint32_t       chunks, per_chunk;    // groups per workgroup
    uint32_t       top_k;
    float          weight;
    int            accumulate;
};

template <int N>
struct Run { float e[N]; };

// What a lane holds: a row of NP logits, or four logits of 4 / NP rows.
template <int NP>
struct Group {
    static constexpr int E = NP >= 4 ? NP : 4, R = E / NP;
    float v[E];
    bool  counted[R];

    // Group g of the level, or nothing.  A level's last group may reach behind its rows (NP < 4).
    __device__ __forceinline__ void load(const BalArgs &a, const uint32_t level, const uint32_t g, const bool there) {
        const size_t base = (size_t)level * a.N_c * NP, i = (size_t)g * E;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t row = g * (uint32_t)R + (uint32_t)r;
            counted[r] = there && (R == 1 || row < a.N_c) && (!a.rows || a.rows[(size_t)level * a.N_c + row]);
        }
        if (R == 1 || i + E <= (size_t)a.N_c * NP) {
            Run<E> run;
            __builtin_memcpy(&run, a.logits + base + (there ? i : 0), sizeof run);       // some row in the place of none
#pragma unroll
            for (int k = 0; k < E; ++k) v[k] = run.e[k];
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) v[k] = there && i + k < (size_t)a.N_c * NP ? a.logits[base + i + k] : 0.0f;
        }
    }
};

// Batcher's odd-even merge sort of N values: the pairs that are compared, in order (63 of 16, 19 of 8, 5 of 4).
template <int N>
struct Network {
    int lo[64], hi[64], n;
    constexpr Network() : lo(), hi(), n(0) {
        for (int p = 1; p < N; p *= 2)
            for (int k = p; k >= 1; k /= 2)
                for (int j = k % p; j + k < N; j += 2 * k)
                    for (int i = 0; i < k && i + j + k < N; ++i)
                        if ((i + j) / (2 * p) == (i + j + k) / (2 * p)) { lo[n] = i + j; hi[n] = i + j + k; ++n; }
    }
};

// Bit k: entry k is among the top_k largest of the row (equal values by lowest index, any number before a NaN).  Values are compared as
// integers in the order of the numbers, a NaN below all.  The top_k-th largest comes out of a sorting network, and what is not below it is
// kept (195 instructions for 16 against 408 for the rank of each); where that is more than top_k in some row of the wavefront, values equal
// to it among them, every entry is ranked: a pair is compared once, and the earlier of two equal ones is ahead.
template <int NP>
__device__ __forceinline__ uint32_t largest(const float *v, const uint32_t top_k) {
    static constexpr Network<NP> net{};
    uint32_t key[NP], sorted[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v[k] + 0.0f);      // -0 is 0
        key[k] = v[k] == v[k] ? u ^ (uint32_t)((int32_t)u >> 31 | (int32_t)0x80000000) : 0u;      // minus infinity is 0x7fffff
        sorted[k] = key[k];
    }
#pragma unroll
    for (int i = 0; i < net.n; ++i) {
        const uint32_t a = sorted[net.lo[i]], b = sorted[net.hi[i]];
        sorted[net.lo[i]] = max(a, b);
        sorted[net.hi[i]] = min(a, b);
    }
    uint32_t bar = sorted[NP - 1], kept = 0;
#pragma unroll
    for (int k = 0; k < NP - 1; ++k) bar = top_k == (uint32_t)(k + 1) ? sorted[k] : bar;
#pragma unroll
    for (int k = 0; k < NP; ++k) kept |= (key[k] >= bar ? 1u : 0u) << k;
    if (!__any((uint32_t)__popc(kept) != top_k)) return kept;

    int ahead[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) ahead[k] = NP - 1 - k;
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int k = j + 1; k < NP; ++k) {
            const int first = key[j] >= key[k] ? 1 : 0;
            ahead[k] += first;
            ahead[j] -= first;
        }
    kept = 0;
#pragma unroll
    for (int k = 0; k < NP; ++k) kept |= (ahead[k] < (int)top_k ? 1u : 0u) << k;
    return kept;
}

// The logits become their rows' softmax weights.  WINNERS: won[r] is the entry of row r that wins by the rule of the bake: the first that
// equals the largest number; without a number, 0.  SPARSE: bit k of `kept` says whether entry k keeps weight: found here with
// WINNERS, else given.
template <int NP, bool SPARSE, bool WINNERS>
__device__ __forceinline__ void weigh(Group<NP> &g, const uint32_t top_k, uint32_t &kept, uint32_t (&won)[Group<NP>::R]) {
    constexpr int R = Group<NP>::R;
    if (WINNERS && SPARSE) kept = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float *v = g.v + r * NP;
        if (WINNERS && SPARSE) kept |= largest<NP>(v, top_k) << (r * NP);
        float m = v[0];
#pragma unroll
        for (int k = 1; k < NP; ++k) m = fmaxf(m, v[k]);
        if (WINNERS) {
            won[r] = 0;
#pragma unroll
            for (int k = NP - 1; k > 0; --k) won[r] = v[k] == m ? (uint32_t)k : won[r];
            won[r] = v[0] == m ? 0u : won[r];
        }
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            v[k] = !SPARSE || ((kept >> (r * NP + k)) & 1u) ? expf(v[k] - m) : 0.0f;
            s += v[k];
        }
        s = 1.0f / s;
#pragma unroll
        for (int k = 0; k < NP; ++k) v[k] *= s;
    }
}

// n[k]: rows of the wavefront so far that k won, the same in every lane.
template <int NP>
__device__ __forceinline__ void add_up(const Group<NP> &g, const uint32_t (&won)[Group<NP>::R], float (&p)[NP], uint32_t (&n)[NP]) {
#pragma unroll
    for (int r = 0; r < Group<NP>::R; ++r)
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            p[k] += g.counted[r] ? g.v[r * NP + k] : 0.0f;
            n[k] += (uint32_t)__popcll(__ballot(g.counted[r] && won[r] == (uint32_t)k));
        }
}

// Sums over the workgroup's lanes, in sum_p[0][k] and sum_n[0][k] for everybody after the barrier at the end.  Of NP sums over the lanes of a
// wavefront each step adds half as many: a lane hands its neighbour one half of what it still holds and takes the other.
template <int NP, int HELD, int BIT>
__device__ __forceinline__ void over_wavefront(float *p, const int lane) {
    if constexpr (HELD > 1) {
        const bool upper = lane & BIT;
#pragma unroll
        for (int k = 0; k < HELD / 2; ++k) {
            const float give = upper ? p[k] : p[k + HELD / 2], keep = upper ? p[k + HELD / 2] : p[k];
            p[k] = keep + __shfl_xor(give, BIT, 64);
        }
        over_wavefront<NP, HELD / 2, BIT * 2>(p, lane);
    } else if constexpr (BIT < 64) {
        p[0] += __shfl_xor(p[0], BIT, 64);
        over_wavefront<NP, 1, BIT * 2>(p, lane);
    }
}
// p: the sum over the wavefront that this lane ended up with.
template <int NP, int W>
__device__ __forceinline__ void over_workgroup(const float p, const uint32_t (&n)[NP], float (&sum_p)[W][NP], uint32_t (&sum_n)[W][NP]) {
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    int mine = 0;                                              // which of the sums this lane ended up with
#pragma unroll
    for (int half = NP / 2, bit = 1; half; half >>= 1, bit <<= 1) mine += lane & bit ? half : 0;
    if (lane < NP) sum_p[w][mine] = p;
#pragma unroll
    for (int k = 0; k < NP; ++k)
        if (lane == k) sum_n[w][k] = n[k];
    __syncthreads();
    if (t < NP) {
        float    s = 0.0f;
        uint32_t c = 0;
        for (int i = 0; i < W; ++i) { s += sum_p[i][t]; c += sum_n[i][t]; }
        sum_p[0][t] = s;
        sum_n[0][t] = c;
    }
    __syncthreads();
}

// From a level's sums: the share f of each candidate (in place of its sum), the factor of the gradient, and, where asked, the outputs.
// One wavefront.
template <int NP>
__device__ __forceinline__ float level_shares(const BalArgs &a, const uint32_t level, float (&sum_p)[NP], const uint32_t (&sum_n)[NP], const bool writes) {
    const int      t = threadIdx.x;
    const uint32_t c = t < NP ? sum_n[t] : 0u;
    uint32_t       total = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) total += (uint32_t)__shfl_xor((int)total, o, 64);
    const float per_row = total ? 1.0f / (float)total : 0.0f;
    const float share = (float)c * per_row;
    float       l = total && t < NP ? share * (sum_p[t < NP ? t : 0] * per_row) : 0.0f;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o, 64);
    if (t < NP) sum_p[t] = share;
    if (writes) {
        if (t < NP) a.counts[(size_t)level * NP + t] = (int32_t)c;
        if (t == 0) a.loss[level] = (float)NP * l;
    }
    return a.weight * (float)NP * per_row;
}

template <int NP>
__device__ __forceinline__ void put_gradient(const BalArgs &a, const uint32_t level, const uint32_t at, const Group<NP> &g, const float (&share)[NP], const float w) {
    constexpr int E = Group<NP>::E;
    Run<E> out;
#pragma unroll
    for (int r = 0; r < Group<NP>::R; ++r) {
        float inner = 0.0f;
#pragma unroll
        for (int k = 0; k < NP; ++k) inner += share[k] * g.v[r * NP + k];
#pragma unroll
        for (int k = 0; k < NP; ++k) out.e[r * NP + k] = g.counted[r] ? w * g.v[r * NP + k] * (share[k] - inner) : 0.0f;
    }
    float       *grad = a.grad + (size_t)level * a.N_c * NP;
    const size_t i = (size_t)at * E;
    if (E == NP || i + E <= (size_t)a.N_c * NP) {
        if (a.accumulate) {
            Run<E> old;
            __builtin_memcpy(&old, grad + i, sizeof old);
#pragma unroll
            for (int k = 0; k < E; ++k) out.e[k] += old.e[k];
        }
        __builtin_memcpy(grad + i, &out, sizeof out);
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (i + k < (size_t)a.N_c * NP) grad[i + k] = a.accumulate ? grad[i + k] + out.e[k] : out.e[k];
    }
}

// A lane has a whole row here: nothing of the row is computed twice and its softmax needs no other lane.  With four lanes to a row of 16 the
// sparse variant took 171 us at 16 x 2^18 x 16, with every entry of a lane's row ranked 133, with the network 105.  The next row is on its
// way while one is worked on.
// A lane adds 64 rows in fp32, then the wavefront's sum goes to one in fp64: equal weights that are no power of two round the same way row after
// row, and 4096 rows of 1/5 one after the other in fp32 were 540 half steps off.
template <int NP>
constexpr uint32_t kHeldEvery = 64 / Group<NP>::R;                 // groups of a lane
template <int NP, bool SPARSE>
__global__ __launch_bounds__(kBalBlock) void balance_sums_kernel(const BalArgs a)
{
    constexpr int W = kBalBlock / 64;
    __shared__ float    sum_p[W][NP];
    __shared__ uint32_t sum_n[W][NP];
    const uint32_t t = threadIdx.x, level = blockIdx.y, g0 = blockIdx.x * a.per_chunk;
    const uint32_t g1 = g0 + a.per_chunk < a.groups ? g0 + a.per_chunk : a.groups;
    float    p[NP];
    uint32_t n[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) { p[k] = 0.0f; n[k] = 0u; }
    Group<NP> g, next;
    double held = 0.0;                                             // the wavefront's sums so far, one to a lane
    next.load(a, level, g0 + t, g0 + t < g1);
    for (uint32_t base = g0; base < g1;) {
        const uint32_t until = g1 - base > kHeldEvery<NP> * kBalBlock ? base + kHeldEvery<NP> * kBalBlock : g1;
        for (; base < until; base += kBalBlock) {                  // whole wavefronts stay: they count by ballots
            const uint32_t at = base + t;
            uint32_t       kept = 0, won[Group<NP>::R];
            g = next;
            next.load(a, level, at + kBalBlock, at + kBalBlock < g1);      // under way while this one is worked on
            weigh<NP, SPARSE, true>(g, a.top_k, kept, won);
            if (SPARSE && a.grad && at < g1) a.kept[(size_t)level * a.groups + at] = (uint16_t)kept;
            add_up<NP>(g, won, p, n);
        }
        over_wavefront<NP, NP, 1>(p, (int)t & 63);
        held += (double)p[0];
#pragma unroll
        for (int k = 0; k < NP; ++k) p[k] = 0.0f;
    }
    over_workgroup<NP, W>((float)held, n, sum_p, sum_n);
    if (t < NP) {
        const size_t o = ((size_t)level * a.chunks + blockIdx.x) * NP + t;
        a.part_p[o] = sum_p[0][t];
        a.part_n[o] = (int32_t)sum_n[0][t];
    }
}

// The second launch moves twice what the first does and computes little: here four lanes share a row of 16 (two one of 8), so that loads
// and stores run over whole lines (one lane to a row: 130 us at 16 x 2^18 x 16, this 96), and exchange sums by lane permutations.
template <int X>
__device__ __forceinline__ float across(const float v) {
    static_assert(X == 1 || X == 2, "a quad of lanes");
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), X == 1 ? 0xB1 : 0x4E, 0xf, 0xf, true));
}
template <int G>
__device__ __forceinline__ float row_sum(float s) {
    if (G >= 2) s += across<1>(s);
    if (G >= 4) s += across<2>(s);
    return s;
}
template <int G>
__device__ __forceinline__ float row_max(float m) {
    if (G >= 2) m = fmaxf(m, across<1>(m));
    if (G >= 4) m = fmaxf(m, across<2>(m));
    return m;
}

template <int NP, bool SPARSE>
__global__ __launch_bounds__(kBalBlock) void balance_grad_kernel(const BalArgs a)
{
    constexpr int PARTS = kBalBlock / NP;
    constexpr int G = NP >= 4 ? NP / 4 : 1;                        // lanes of a row
    constexpr int H = NP >= 4 ? 4 : NP;                            // candidates of a lane
    __shared__ float    sum_p[PARTS][NP];
    __shared__ uint32_t sum_n[PARTS][NP];
    __shared__ float    scale;                                     // weight * N_p / W, 0 for a level without counted rows
    const uint32_t t = threadIdx.x, level = blockIdx.y, sub = t % G;
    const uint32_t g0 = blockIdx.x * a.per_chunk, g1 = g0 + a.per_chunk < a.groups ? g0 + a.per_chunk : a.groups;
    // lane's group of four logits q; rows of NP >= 4 are seen as rows of four whose sums are completed across lanes
    const uint32_t q0 = g0 * G, q1 = g1 * G;
    const auto fetch = [&](Group<H> &g, const uint32_t q, const bool there) {
        if constexpr (NP >= 4) {
            Run<4> run;
            const uint32_t row = there ? q / G : 0u;
            __builtin_memcpy(&run, a.logits + (size_t)level * a.N_c * NP + (size_t)(there ? q : 0u) * 4, sizeof run);
#pragma unroll
            for (int k = 0; k < 4; ++k) g.v[k] = run.e[k];
            g.counted[0] = there && (!a.rows || a.rows[(size_t)level * a.N_c + row]);
        } else {
            g.load(a, level, q, there);
        }
    };
    Group<H> g, next;
    if (a.grad) fetch(next, q0 + t, q0 + t < q1);                  // under way while the sums are added up
    {
        const uint32_t k = t % NP, part = t / NP;
        float          s = 0.0f;
        uint32_t       c = 0;
        for (uint32_t i = part; i < a.chunks; i += PARTS) {
            const size_t o = ((size_t)level * a.chunks + i) * NP + k;
            s += a.part_p[o];
            c += (uint32_t)a.part_n[o];
        }
        sum_p[part][k] = s;
        sum_n[part][k] = c;
    }
    __syncthreads();
    if (t < 64) {
        if (t < NP) {
            float    s = 0.0f;
            uint32_t c = 0;
            for (int i = 0; i < PARTS; ++i) { s += sum_p[i][t]; c += sum_n[i][t]; }
            sum_p[0][t] = s;
            sum_n[0][t] = c;
        }
        const float w = level_shares<NP>(a, level, sum_p[0], sum_n[0], blockIdx.x == 0);
        if (t == 0) scale = w;
    }
    if (!a.grad) return;
    __syncthreads();
    float share[H];
#pragma unroll
    for (int k = 0; k < H; ++k) share[k] = sum_p[0][sub * 4 % NP + k];
    const float w = scale;
    for (uint32_t base = q0; base < q1; base += kBalBlock) {       // whole wavefronts stay: the lanes of a row exchange
        const uint32_t q = base + t, at = q < q1 ? q : q0;
        uint32_t       kept = 0, won[Group<H>::R];
        if (SPARSE) kept = a.kept[(size_t)level * a.groups + at / G] >> (NP >= 4 ? 4 * sub : 0u);
        g = next;
        fetch(next, q + kBalBlock, q + kBalBlock < q1);
        if constexpr (NP >= 4) {
            const float m = row_max<G>(fmaxf(fmaxf(g.v[0], g.v[1]), fmaxf(g.v[2], g.v[3])));
#pragma unroll
            for (int k = 0; k < 4; ++k) g.v[k] = !SPARSE || ((kept >> k) & 1u) ? expf(g.v[k] - m) : 0.0f;
            const float s = 1.0f / row_sum<G>((g.v[0] + g.v[1]) + (g.v[2] + g.v[3]));
#pragma unroll
            for (int k = 0; k < 4; ++k) g.v[k] *= s;
            float inner = 0.0f;
#pragma unroll
            for (int k = 0; k < 4; ++k) inner += share[k] * g.v[k];
            inner = row_sum<G>(inner);
            if (q >= q1) continue;
            Run<4> out;
#pragma unroll
            for (int k = 0; k < 4; ++k) out.e[k] = g.counted[0] ? w * g.v[k] * (share[k] - inner) : 0.0f;
            float *to = a.grad + (size_t)level * a.N_c * NP + (size_t)q * 4;
            if (a.accumulate) {
                Run<4> old;
                __builtin_memcpy(&old, to, sizeof old);
#pragma unroll
                for (int k = 0; k < 4; ++k) out.e[k] += old.e[k];
            }
            __builtin_memcpy(to, &out, sizeof out);
        } else {
            weigh<NP, SPARSE, false>(g, a.top_k, kept, won);
            if (q < q1) put_gradient<NP>(a, level, q, g, share, w);
        }
    }
}

// A level of at most kLevelBlock * kLevelGroups groups: its weights stay in registers between the sums and the gradient, and the second launch
// is saved: 4 levels x 256 rows x 4 take 4.6 us, bound by latency.
template <int NP, bool SPARSE>
__global__ __launch_bounds__(kLevelBlock) void balance_level_kernel(const BalArgs a)
{
    constexpr int W = kLevelBlock / 64;
    __shared__ float    sum_p[W][NP];
    __shared__ uint32_t sum_n[W][NP];
    __shared__ float    scale;
    const uint32_t t = threadIdx.x, level = blockIdx.x;
    float    p[NP];
    uint32_t n[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) { p[k] = 0.0f; n[k] = 0u; }
    Group<NP> g[kLevelGroups];
#pragma unroll
    for (int i = 0; i < kLevelGroups; ++i) g[i].load(a, level, i * kLevelBlock + t, i * kLevelBlock + t < a.groups);
#pragma unroll
    for (int i = 0; i < kLevelGroups; ++i) {
        uint32_t kept = 0, won[Group<NP>::R];
        weigh<NP, SPARSE, true>(g[i], a.top_k, kept, won);
        add_up<NP>(g[i], won, p, n);
    }
    over_wavefront<NP, NP, 1>(p, (int)t & 63);
    over_workgroup<NP, W>(p[0], n, sum_p, sum_n);
    if (t < 64) {
        const float w = level_shares<NP>(a, level, sum_p[0], sum_n[0], true);
        if (t == 0) scale = w;
    }
    if (!a.grad) return;
    __syncthreads();
    float share[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) share[k] = sum_p[0][k];
    const float w = scale;
#pragma unroll
    for (int i = 0; i < kLevelGroups; ++i)
        if (i * kLevelBlock + t < a.groups) put_gradient<NP>(a, level, i * kLevelBlock + t, g[i], share, w);
}

uint64_t groups_of(const cngp_config *c) { return c->N_p >= 4 ? c->N_c : ((uint64_t)c->N_c * c->N_p + 3) / 4; }
bool     one_launch(const cngp_config *c) { return groups_of(c) <= (uint64_t)kLevelBlock * kLevelGroups; }

// A group per lane before a level gets another workgroup, and at most kMostChunks workgroups per level.
uint32_t chunks_of(const cngp_config *c) {
    const uint64_t want = (groups_of(c) + kBalBlock - 1) / kBalBlock;
    return (uint32_t)std::min<uint64_t>(std::max<uint64_t>(want, 1), kMostChunks);
}
size_t sums_bytes(const cngp_config *c) { return ((size_t)c->L * chunks_of(c) * c->N_p * 8 + 255) / 256 * 256; }

template <int NP, bool SPARSE>
int run(const BalArgs &a, const int L, const bool one, hipStream_t s) {
    if (one) {
        LaunchTimer t(s, K_BALANCE);
        balance_level_kernel<NP, SPARSE><<<(unsigned)L, kLevelBlock, 0, s>>>(a);
        return launch_status("balance_level_kernel");
    }
    {
        LaunchTimer t(s, K_BALANCE);
        balance_sums_kernel<NP, SPARSE><<<dim3(a.chunks, (unsigned)L), kBalBlock, 0, s>>>(a);
        if (int rc = launch_status("balance_sums_kernel")) return rc;
    }
    LaunchTimer t(s, K_BALANCE);
    balance_grad_kernel<NP, SPARSE><<<dim3(a.grad ? a.chunks : 1, (unsigned)L), kBalBlock, 0, s>>>(a);
    return launch_status("balance_grad_kernel");
}

}  // namespace

extern "C" {

size_t cngp_probe_balance_workspace_bytes(const cngp_config *cfg) {
    if (validate(cfg) || one_launch(cfg)) return 0;
    const bool sparse = cfg->top_k && cfg->top_k < cfg->N_p;
    return sums_bytes(cfg) + (sparse ? ((size_t)cfg->L * groups_of(cfg) * 2 + 255) / 256 * 256 : 0);
}

int cngp_probe_balance(const cngp_config *cfg, const float *Dhat_c, const uint8_t *rows, float weight, float *loss, int32_t *counts,
                       float *grad_Dhat_c, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = validate(cfg)) return rc;
    if (!Dhat_c || !loss || !counts) return CNGP_ERR_NULL;
    if (!std::isfinite(weight)) return CNGP_ERR_INVALID;
    const size_t need = cngp_probe_balance_workspace_bytes(cfg);
    if (need && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return CNGP_ERR_WORKSPACE;
    if (groups_of(cfg) * std::max(1u, cfg->N_p / 4) > 0xfff00000ull) return CNGP_ERR_UNSUPPORTED;      // fours of a level are counted in 32 bits
    BalArgs a{};
    a.logits = Dhat_c; a.rows = rows; a.grad = grad_Dhat_c; a.loss = loss; a.counts = counts;
    a.N_c = cfg->N_c;
    a.chunks = chunks_of(cfg);
    a.part_p = (float *)workspace;
    a.part_n = (int32_t *)workspace + (size_t)cfg->L * a.chunks * cfg->N_p;
    a.kept = (uint16_t *)((char *)workspace + sums_bytes(cfg));
    a.groups = (uint32_t)groups_of(cfg);                       // N_c <= 2^30
    a.per_chunk = (a.groups + a.chunks - 1) / a.chunks;
    a.top_k = cfg->top_k;
    a.weight = weight;
    a.accumulate = (cfg->flags & CNGP_ZERO_GRADS) ? 0 : 1;
    hipStream_t s = (hipStream_t)stream;
    const bool sparse = cfg->top_k && cfg->top_k < cfg->N_p, one = one_launch(cfg);
    switch (cfg->N_p) {
    case 1:  return run<1, false>(a, cfg->L, one, s);
    case 2:  return sparse ? run<2, true>(a, cfg->L, one, s) : run<2, false>(a, cfg->L, one, s);
    case 4:  return sparse ? run<4, true>(a, cfg->L, one, s) : run<4, false>(a, cfg->L, one, s);
    case 8:  return sparse ? run<8, true>(a, cfg->L, one, s) : run<8, false>(a, cfg->L, one, s);
    default: return sparse ? run<16, true>(a, cfg->L, one, s) : run<16, false>(a, cfg->L, one, s);
    }
}

}  // extern "C"
