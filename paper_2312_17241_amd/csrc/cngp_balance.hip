// Balance of the probing candidates: winners per candidate, the loss N_p sum_k f_k P_k of every level and its gradient.
//
// With sigma = softmax of a row, f and P the means over a level's rows of "candidate k won" and of sigma_k:
//     d loss / d logit_rk = N_p / W * sigma_rk (f_k - sum_j f_j sigma_rj)
// The gradient of every row needs the level's f, so two launches: one reads the logits and leaves sums per workgroup, the other
// adds those up (in a fixed order), reads the logits again and writes the gradient.  Both stream: a lane holds four neighbouring
// logits, so a row of sixteen is four lanes that exchange their maximum and sums with two lane permutations each.  The sparse variant ranks
// a row's logits once, in the first launch, and leaves four bits per lane for the second.
#include <cmath>
#include <cstdint>

#include <hip/hip_runtime.h>

#include "cngp_launch.h"

namespace {

using namespace cngp;

constexpr int kBalBlock = 256;
constexpr int kMostChunks = 64;          // workgroups per level: the second launch reads this many partial sums per candidate

struct BalArgs {
    const float   *logits;
    const uint8_t *rows;
    float         *grad;
    float         *loss;
    int32_t       *counts;
    float         *part_p;               // [L][chunks][NP]
    int32_t       *part_n;               // [L][chunks][NP] winners
    uint8_t       *kept;                 // [L][quads] which of four logits keep weight, top_k < N_p
    uint32_t       N_c, quads;           // rows and groups of four logits per level
    uint32_t       chunks, per_chunk;    // groups of four logits per workgroup
    uint32_t       top_k;
    float          weight;
    int            accumulate, aligned;  // aligned: a level starts on a 16-byte boundary in both arrays
};

// What a lane holds of the rows: four logits, of one row (NP >= 4, G lanes to a row) or of R whole rows.
template <int NP>
struct Quad {
    static constexpr int G = NP >= 4 ? NP / 4 : 1, R = NP >= 4 ? 1 : 4 / NP;
    float v[4];
    bool  counted[R];

    __device__ __forceinline__ void load(const BalArgs &a, const uint32_t level, const uint32_t q) {
        const size_t   base = (size_t)level * a.N_c * NP;
        const bool     live = q < a.quads;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t row = NP >= 4 ? q / (uint32_t)G : q * (uint32_t)R + (uint32_t)r;
            counted[r] = live && row < a.N_c && (!a.rows || a.rows[(size_t)level * a.N_c + row]);
        }
        if (live && a.aligned) {
            const float4 t = *reinterpret_cast<const float4 *>(a.logits + base + (size_t)q * 4);
            v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const size_t i = (size_t)q * 4 + k;
                v[k] = live && i < (size_t)a.N_c * NP ? a.logits[base + i] : 0.0f;
            }
        }
    }
};

// The value of lane ^ X among four neighbouring lanes.
template <int X, typename T>
__device__ __forceinline__ T across(const T v) {
    static_assert(X >= 1 && X <= 3 && sizeof(T) == 4, "a quad of lanes");
    constexpr int perm = X == 1 ? 0xB1 : X == 2 ? 0x4E : 0x1B;
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), perm, 0xf, 0xf, true));
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

// Which entry of a row wins by the rule of the bake, given its largest number: the first that equals it; none does if there is no
// number, and that gives 0.
template <int NP>
__device__ __forceinline__ uint32_t winner(const float (&v)[4], const int first, const float top) {
    uint32_t best = 255;
#pragma unroll
    for (int k = 3; k >= 0; --k) best = v[k] == top ? (uint32_t)(first + k) : best;
    if (NP >= 8) best = min(best, across<1>(best));
    if (NP >= 16) best = min(best, across<2>(best));
    return best == 255 ? 0 : best;
}

// Bit k: entry k of this lane is among the top_k largest of its row (equal values by lowest index, any number before a NaN).  Values are
// compared as integers in the order of the numbers, a NaN below all; one that comes earlier counts from equality on.
template <int X, int NP>
__device__ __forceinline__ void count_ahead(const uint32_t (&key)[4], const int sub, uint32_t (&ahead)[4]) {
    const uint32_t earlier = (sub ^ X) < sub ? 1u : 0u;
    uint32_t       bar[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) bar[k] = key[k] - earlier;     // keys are at least 1
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t o = across<X>(key[j]);
#pragma unroll
        for (int k = 0; k < 4; ++k) ahead[k] += o > bar[k] ? 1u : 0u;
    }
}
template <int NP>
__device__ __forceinline__ uint32_t largest(const float (&v)[4], const int sub, const uint32_t top_k) {
    uint32_t key[4], ahead[4] = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t u = __builtin_bit_cast(uint32_t, v[k] + 0.0f);      // -0 is 0
        key[k] = v[k] == v[k] ? ((u >> 31) ? ~u : u | 0x80000000u) : 1u;   // minus infinity is 0x7fffff
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (j != k) ahead[k] += (j < k ? key[j] >= key[k] : key[j] > key[k]) ? 1u : 0u;
    if (NP >= 8) count_ahead<1, NP>(key, sub, ahead);
    if (NP >= 16) {
        count_ahead<2, NP>(key, sub, ahead);
        count_ahead<3, NP>(key, sub, ahead);
    }
    uint32_t kept = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) kept |= (ahead[k] < top_k ? 1u : 0u) << k;
    return kept;
}

// The four logits become their softmax weights; WINNERS: win[k] says whether entry k won its row.  With SPARSE, bit k of `kept` says
// whether entry k keeps weight: found here with WINNERS, else given.  All lanes of a wavefront call this together.
template <int NP, bool SPARSE, bool WINNERS>
__device__ __forceinline__ void weigh(Quad<NP> &q, const int first, const uint32_t top_k, uint32_t &kept, bool (&win)[4]) {
    using Q = Quad<NP>;
    if constexpr (NP >= 4) {
        if (SPARSE && WINNERS) kept = largest<NP>(q.v, first / 4, top_k);
        const float m = row_max<Q::G>(fmaxf(fmaxf(q.v[0], q.v[1]), fmaxf(q.v[2], q.v[3])));
        if (WINNERS) {
            const uint32_t best = winner<NP>(q.v, first, m);
#pragma unroll
            for (int k = 0; k < 4; ++k) win[k] = best == (uint32_t)(first + k);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) q.v[k] = !SPARSE || ((kept >> k) & 1u) ? expf(q.v[k] - m) : 0.0f;
        const float s = 1.0f / row_sum<Q::G>((q.v[0] + q.v[1]) + (q.v[2] + q.v[3]));
#pragma unroll
        for (int k = 0; k < 4; ++k) q.v[k] *= s;
    } else if constexpr (NP == 2) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float     &a = q.v[2 * r], &b = q.v[2 * r + 1];
            const bool second = b == b && (!(a == a) || b > a);
            win[2 * r] = !second;
            win[2 * r + 1] = second;
            if (SPARSE) {                                      // the one that stays has all the weight
                (second ? a : b) = 0.0f;
                float &stays = second ? b : a;
                stays = expf(stays - stays);
                continue;
            }
            const float m = fmaxf(a, b);
            a = expf(a - m);
            b = expf(b - m);
            const float s = 1.0f / (a + b);
            a *= s;
            b *= s;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) { q.v[k] = expf(q.v[k] - q.v[k]); win[k] = true; }      // one, or NaN
    }
}

template <int NP, bool SPARSE>
__global__ __launch_bounds__(kBalBlock) void balance_sums_kernel(const BalArgs a)
{
    using Q = Quad<NP>;
    __shared__ float    sum_p[kBalBlock / 64][NP];
    __shared__ uint32_t sum_n[kBalBlock / 64][NP];
    const int      t = threadIdx.x, lane = t & 63;
    const uint32_t level = blockIdx.y, q0 = blockIdx.x * a.per_chunk;
    const uint32_t q1 = q0 + a.per_chunk < a.quads ? q0 + a.per_chunk : a.quads;
    const int      first = NP >= 4 ? (lane & (Q::G - 1)) * 4 : 0;
    float    p[4] = {0, 0, 0, 0};
    uint32_t n[4] = {0, 0, 0, 0};
    for (uint32_t base = q0; base < q1; base += kBalBlock) {      // whole wavefronts stay: the lanes exchange
        const uint32_t at = base + t < q1 ? base + t : 0xffffffffu;
        Q        q;
        bool     win[4];
        uint32_t kept = 15u;
        q.load(a, level, at);
        weigh<NP, SPARSE, true>(q, first, a.top_k, kept, win);
        if (SPARSE && NP >= 4 && a.grad && at != 0xffffffffu) a.kept[(size_t)level * a.quads + at] = (uint8_t)kept;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool c = q.counted[k / (4 / Q::R)];
            p[k] += c ? q.v[k] : 0.0f;
            n[k] += c && win[k] ? 1u : 0u;
        }
    }
    // lanes that hold the same candidates add up: over the rows of a lane, over the lanes of a wavefront, over the wavefronts
    constexpr int K = NP >= 4 ? 4 : NP;
#pragma unroll
    for (int k = K; k < 4; ++k) { p[k % K] += p[k]; n[k % K] += n[k]; }
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int o = Q::G; o < 64; o <<= 1) {
            p[k] += __shfl_xor(p[k], o, 64);
            n[k] += (uint32_t)__shfl_xor((int)n[k], o, 64);
        }
        if (lane < Q::G) { sum_p[t >> 6][first + k] = p[k]; sum_n[t >> 6][first + k] = n[k]; }
    }
    __syncthreads();
    if (t < NP) {
        float    s = 0.0f;
        uint32_t c = 0;
#pragma unroll
        for (int w = 0; w < kBalBlock / 64; ++w) { s += sum_p[w][t]; c += sum_n[w][t]; }
        const size_t o = ((size_t)level * a.chunks + blockIdx.x) * NP + t;
        a.part_p[o] = s;
        a.part_n[o] = (int32_t)c;
    }
}

template <int NP, bool SPARSE>
__global__ __launch_bounds__(kBalBlock) void balance_grad_kernel(const BalArgs a)
{
    using Q = Quad<NP>;
    constexpr int PARTS = kBalBlock / NP;
    __shared__ float    sum_p[PARTS][NP];
    __shared__ uint32_t sum_n[PARTS][NP];
    __shared__ float    f[NP];
    __shared__ float    scale;                                    // weight * N_p / W, 0 for a level without counted rows
    const int      t = threadIdx.x, lane = t & 63;
    const uint32_t level = blockIdx.y;
    {
        const int k = t % NP, part = t / NP;
        float     s = 0.0f;
        uint32_t  c = 0;
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
        float    s = 0.0f;
        uint32_t c = 0;
        if (t < NP)
            for (int i = 0; i < PARTS; ++i) { s += sum_p[i][t]; c += sum_n[i][t]; }
        uint32_t total = c;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) total += (uint32_t)__shfl_xor((int)total, o, 64);
        const float per_row = total ? 1.0f / (float)total : 0.0f;
        const float share = (float)c * per_row;
        float       l = total ? share * (s * per_row) : 0.0f;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o, 64);
        if (t < NP) f[t] = share;
        if (t == 0) scale = a.weight * (float)NP * per_row;
        if (blockIdx.x == 0) {
            if (t < NP) a.counts[(size_t)level * NP + t] = (int32_t)c;
            if (t == 0) a.loss[level] = (float)NP * l;
        }
    }
    if (!a.grad) return;
    __syncthreads();
    const uint32_t q0 = blockIdx.x * a.per_chunk;
    const uint32_t q1 = q0 + a.per_chunk < a.quads ? q0 + a.per_chunk : a.quads;
    const int      first = NP >= 4 ? (lane & (Q::G - 1)) * 4 : 0;
    float share[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) share[k] = f[(first + k) % NP];
    const float w = scale;
    float      *grad = a.grad + (size_t)level * a.N_c * NP;
    for (uint32_t base = q0; base < q1; base += kBalBlock) {
        const bool     live = base + t < q1;
        const uint32_t at = live ? base + t : 0xffffffffu;
        Q        q;
        bool     win[4];
        uint32_t kept = 15u;
        q.load(a, level, at);
        if (SPARSE && NP >= 4 && live) kept = a.kept[(size_t)level * a.quads + at];
        weigh<NP, SPARSE, false>(q, first, a.top_k, kept, win);
        float g[4];
#pragma unroll
        for (int r = 0; r < Q::R; ++r) {
            constexpr int E = 4 / Q::R;                           // entries of a row that this lane holds
            float inner = 0.0f;
#pragma unroll
            for (int k = 0; k < E; ++k) inner += share[r * E + k] * q.v[r * E + k];
            inner = row_sum<Q::G>(inner);
#pragma unroll
            for (int k = 0; k < E; ++k) g[r * E + k] = q.counted[r] ? w * q.v[r * E + k] * (share[r * E + k] - inner) : 0.0f;
        }
        if (!live) continue;
        if (a.aligned) {
            float4 *o = reinterpret_cast<float4 *>(grad + (size_t)at * 4);
            if (a.accumulate) { const float4 b = *o; g[0] += b.x; g[1] += b.y; g[2] += b.z; g[3] += b.w; }
            *o = make_float4(g[0], g[1], g[2], g[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const size_t i = (size_t)at * 4 + k;
                if (i < (size_t)a.N_c * NP) grad[i] = a.accumulate ? grad[i] + g[k] : g[k];
            }
        }
    }
}

uint64_t quads_of(const cngp_config *c) { return ((uint64_t)c->N_c * c->N_p + 3) / 4; }
bool     sparse_rows(const cngp_config *c) { return c->N_p >= 4 && c->top_k && c->top_k < c->N_p; }

// Four groups of logits per lane before a level gets another workgroup, and at most kMostChunks workgroups per level.
uint32_t chunks_of(const cngp_config *c) {
    const uint64_t quads = quads_of(c), per = (uint64_t)kBalBlock * 4;
    const uint64_t want = (quads + per - 1) / per;
    return (uint32_t)(want < 1 ? 1 : want > (uint64_t)kMostChunks ? (uint64_t)kMostChunks : want);
}

size_t sums_bytes(const cngp_config *c) { return ((size_t)c->L * chunks_of(c) * c->N_p * 8 + 255) / 256 * 256; }

template <int NP, bool SPARSE>
int run(const BalArgs &a, const int L, hipStream_t s) {
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
    if (validate(cfg)) return 0;
    return sums_bytes(cfg) + (sparse_rows(cfg) ? (((size_t)cfg->L * quads_of(cfg)) + 255) / 256 * 256 : 0);
}

int cngp_probe_balance(const cngp_config *cfg, const float *Dhat_c, const uint8_t *rows, float weight, float *loss, int32_t *counts,
                       float *grad_Dhat_c, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = validate(cfg)) return rc;
    if (!Dhat_c || !loss || !counts) return CNGP_ERR_NULL;
    if (!std::isfinite(weight)) return CNGP_ERR_INVALID;
    const size_t need = cngp_probe_balance_workspace_bytes(cfg);
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need) return CNGP_ERR_WORKSPACE;
    BalArgs a{};
    a.logits = Dhat_c; a.rows = rows; a.grad = grad_Dhat_c; a.loss = loss; a.counts = counts;
    a.N_c = cfg->N_c;
    a.chunks = chunks_of(cfg);
    a.part_p = (float *)workspace;
    a.part_n = (int32_t *)workspace + (size_t)cfg->L * a.chunks * cfg->N_p;
    a.kept = (uint8_t *)workspace + sums_bytes(cfg);
    const uint64_t quads = quads_of(cfg);                      // at most 2^32: N_c <= 2^30, N_p <= 16
    if (quads > 0xfffffff0ull - (uint64_t)kBalBlock * kMostChunks) return CNGP_ERR_UNSUPPORTED;
    a.quads = (uint32_t)quads;
    // a multiple of a workgroup's step, so that the lanes of a row stay together
    a.per_chunk = (uint32_t)((((quads + a.chunks - 1) / a.chunks) + kBalBlock - 1) / kBalBlock * kBalBlock);
    a.top_k = cfg->top_k;
    a.weight = weight;
    a.accumulate = (cfg->flags & CNGP_ZERO_GRADS) ? 0 : 1;
    a.aligned = ((uint64_t)cfg->N_c * cfg->N_p) % 4 == 0 && !((uintptr_t)Dhat_c & 15u) && !((uintptr_t)grad_Dhat_c & 15u);
    hipStream_t s = (hipStream_t)stream;
    const bool sparse = cfg->top_k && cfg->top_k < cfg->N_p;
    switch (cfg->N_p) {
    case 1:  return run<1, false>(a, cfg->L, s);
    case 2:  return sparse ? run<2, true>(a, cfg->L, s) : run<2, false>(a, cfg->L, s);
    case 4:  return sparse ? run<4, true>(a, cfg->L, s) : run<4, false>(a, cfg->L, s);
    case 8:  return sparse ? run<8, true>(a, cfg->L, s) : run<8, false>(a, cfg->L, s);
    default: return sparse ? run<16, true>(a, cfg->L, s) : run<16, false>(a, cfg->L, s);
    }
}

}  // extern "C"
