// Norms of queries and keys for each head and the rotation by their positions in one pass, with its gradient.
//
//     y = turn(gamma * x / sqrt(mean(x^2) + eps)),    turn: pair p of a head's components by the angle position[axis of p] * omega[p]
//
// One group of lanes takes a row and some of its heads; a lane holds the same components of every head, so the row's angles are formed
// once for all of them: the product in 64 bits, whole turns taken off there, sine and cosine of what is left in fp32.  Bound by memory: x is
// read and y written once, in 16-byte pieces where rows allow (2^15 rows, 20 heads of 128, fp16: 86 us forward, 3.9 TB/s, 131 backward with the gains',
// 3.8; 2^18 rows, 5 heads of 36, fp32, no norms: 80, 4.7).
#include <algorithm>
#include <cmath>

#include "cngp_launch.h"

using namespace cngp;

namespace {

constexpr int kBlock = 256, kMostDim = 512, kMostGroups = 1024;
inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct RotateArgs {
    const void  *x[2];                   // queries, keys: [N, heads, dim]
    void        *y[2];
    const void  *dy[2];                  // backward: gradients of y in, of x out (in y)
    const float *gamma[2];
    float       *part;                   // backward: [groups, 2, dim] sums of the gains' gradient, or NULL
    const float *position, *omega;       // [N, axes], [pairs]
    int64_t      N;
    int32_t      heads[2], dim, axes, pairs, ends[4];   // ends: first pair of the next axis
    int32_t      split, each;            // a row's heads (queries then keys) in `split` parts of `each`
    float        eps, inverse_dim;
};

// Components of an item: VEC of them (next: VEC / 2 pairs beside each other), or VEC and the VEC that lie `pairs` further on (halves).  Items that
// begin behind the pairs are passed on as they are, 2 VEC side by side in the second form.
template <typename T, int VEC> struct alignas(sizeof(T) * VEC) Piece { T v[VEC]; };

typedef uint32_t words_t __attribute__((ext_vector_type(4)));
template <typename T, int VEC, bool NEXT>
struct Item {
    static constexpr int kValues = NEXT ? (VEC == 1 ? 2 : VEC) : 2 * VEC, kAngles = kValues / 2;
    int  at0, at1;                       // where the two runs of kValues / 2 begin
    int  pair;                           // first pair, or -1: none
    __device__ __forceinline__ Item(const int i, const int dim, const int pairs) {
        if (NEXT) {
            at0 = i * kValues;
            at1 = at0 + kAngles;
            pair = i * kAngles;
        } else {
            const int turned = (pairs + VEC - 1) / VEC, rest = 2 * pairs + (i - turned) * 2 * VEC;
            at0 = i < turned ? i * VEC : rest;
            at1 = i < turned ? pairs + i * VEC : rest + VEC;
            pair = i < turned ? i * VEC : -1;
        }
    }
    __device__ __forceinline__ bool there(const int j, const int dim) const { return (j < kAngles ? at0 + j : at1 + j - kAngles) < dim; }
    __device__ __forceinline__ int component(const int j) const { return j < kAngles ? at0 + j : at1 + j - kAngles; }
    // what is on its way from memory: pieces of 16 bytes as they are, or values
    struct Raw { words_t piece[VEC > 1 ? (NEXT ? 1 : 2) : 1]; float value[VEC > 1 ? 1 : kValues]; };
    __device__ __forceinline__ void load(const T *p, const int dim, Raw &r) const {
        if constexpr (VEC > 1) {
            r.piece[0] = *reinterpret_cast<const words_t *>(p + (at0 < dim ? at0 : 0));
            if constexpr (!NEXT) r.piece[1] = *reinterpret_cast<const words_t *>(p + (at1 < dim ? at1 : 0));
        } else {
#pragma unroll
            for (int j = 0; j < kValues; ++j) r.value[j] = there(j, dim) ? (float)p[component(j)] : 0.0f;
        }
    }
    __device__ __forceinline__ void unpack(const Raw &r, const int dim, float (&v)[kValues]) const {
        if constexpr (VEC > 1) {
            typedef T values_t __attribute__((ext_vector_type(VEC)));
#pragma unroll
            for (int i = 0; i < (NEXT ? 1 : 2); ++i) {
                const values_t x = __builtin_bit_cast(values_t, r.piece[i]);
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i * VEC + j] = (i ? at1 : at0) < dim ? (float)x[j] : 0.0f;
            }
        } else {
#pragma unroll
            for (int j = 0; j < kValues; ++j) v[j] = r.value[j];
        }
    }
    __device__ __forceinline__ void store(T *p, const int dim, const float (&v)[kValues]) const {
        if constexpr (VEC > 1) {
            Piece<T, VEC> a;
#pragma unroll
            for (int j = 0; j < VEC; ++j) a.v[j] = (T)v[j];
            if (at0 < dim) *reinterpret_cast<Piece<T, VEC> *>(p + at0) = a;
            if constexpr (!NEXT) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) a.v[j] = (T)v[VEC + j];
                if (at1 < dim) *reinterpret_cast<Piece<T, VEC> *>(p + at1) = a;
            }
        } else {
#pragma unroll
            for (int j = 0; j < kValues; ++j)
                if (there(j, dim)) p[component(j)] = (T)v[j];
        }
    }
    // which two of the values make up pair k of the item
    static __device__ __forceinline__ constexpr int first(const int k) { return NEXT ? 2 * k : k; }
    static __device__ __forceinline__ constexpr int second(const int k) { return NEXT ? 2 * k + 1 : kAngles + k; }
};

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// LANES side by side hold a head, ITEMS items each.
template <typename T, int VEC, bool NEXT, int LANES, int ITEMS, bool NORM, bool BWD>
__global__ __launch_bounds__(kBlock) void rotate_kernel(const RotateArgs a)
{
    using I = Item<T, VEC, NEXT>;
    constexpr int V = I::kValues, A = I::kAngles, kGroups = kBlock / LANES;
    // heads on their way, as they lie in memory (with the norm registers for more cost waves: 211, 213, 248 us for one, two, three, forward and backward of
    // 2^15 rows, 20 heads of 128, fp16; without it three: 170, 164, 157, 2^18 rows, 5 heads of 36, fp32)
    constexpr int AHEAD = NORM ? 1 : 3;
    const int lane = (int)threadIdx.x % LANES, group = (int)threadIdx.x / LANES, H = a.heads[0] + a.heads[1];
    float sums[2][ITEMS][V];
    if (BWD && NORM)
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int n = 0; n < ITEMS; ++n)
#pragma unroll
                for (int j = 0; j < V; ++j) sums[w][n][j] = 0.0f;
    const int64_t parts = a.N * a.split, step = (int64_t)gridDim.x * kGroups;
    // all groups of a wavefront go round together: those without work repeat the last part and write nothing
    for (int64_t first = (int64_t)blockIdx.x * kGroups; first < parts; first += step) {
        const bool    work = first + group < parts;
        const int64_t part = work ? first + group : parts - 1, row = part / a.split;
        const int     h0 = (int)(part % a.split) * a.each, h1 = h0 + a.each < H ? h0 + a.each : H;
        float c[ITEMS][A], s[ITEMS][A];
#pragma unroll
        for (int n = 0; n < ITEMS; ++n) {
            const I it(lane + n * LANES, a.dim, a.pairs);
#pragma unroll
            for (int k = 0; k < A; ++k) {
                const int p = it.pair + k;
                c[n][k] = 1.0f;
                s[n][k] = 0.0f;
                if (it.pair >= 0 && p < a.pairs) {
                    const int    axis = (p >= a.ends[0]) + (p >= a.ends[1]) + (p >= a.ends[2]);
                    const double turns = (double)a.position[row * a.axes + axis] * (double)a.omega[p] * 0.15915494309189533577;
                    sincospif(2.0f * (float)(turns - rint(turns)), &s[n][k], &c[n][k]);
                    if (BWD) s[n][k] = -s[n][k];
                }
            }
        }
        // queries, then keys; the next heads are loaded while one is worked on
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int n0 = w ? a.heads[0] : 0, first_h = (h0 > n0 ? h0 : n0) - n0, last_h = (h1 < n0 + a.heads[w] ? h1 : n0 + a.heads[w]) - n0;
            if (first_h >= last_h) continue;
            float gain[ITEMS][V];
#pragma unroll
            for (int n = 0; n < ITEMS; ++n) {
                const I it(lane + n * LANES, a.dim, a.pairs);
#pragma unroll
                for (int j = 0; j < V; ++j) gain[n][j] = NORM && a.gamma[w] && it.there(j, a.dim) ? a.gamma[w][it.component(j)] : 1.0f;
            }
            const T *from = (const T *)a.x[w] + (size_t)row * a.heads[w] * a.dim, *up = (const T *)a.dy[w] + (size_t)row * a.heads[w] * a.dim;
            T       *to = (T *)a.y[w] + (size_t)row * a.heads[w] * a.dim;
            float x[ITEMS][V], u[ITEMS][V];
            typename I::Raw rx[AHEAD][ITEMS], ru[AHEAD][ITEMS];
            auto load = [&](const int h, typename I::Raw (&xo)[ITEMS], typename I::Raw (&uo)[ITEMS]) {
                if (h >= last_h) return;
#pragma unroll
                for (int n = 0; n < ITEMS; ++n) {
                    const I it(lane + n * LANES, a.dim, a.pairs);
                    if (!BWD || NORM) it.load(from + h * a.dim, a.dim, xo[n]);
                    if (BWD) it.load(up + h * a.dim, a.dim, uo[n]);
                }
            };
#pragma unroll
            for (int d = 0; d < AHEAD; ++d) load(first_h + d, rx[d], ru[d]);
            for (int h = first_h; h < last_h; ++h) {
#pragma unroll
                for (int n = 0; n < ITEMS; ++n) {
                    const I it(lane + n * LANES, a.dim, a.pairs);
                    if (!BWD || NORM) it.unpack(rx[0][n], a.dim, x[n]);
                    if (BWD) it.unpack(ru[0][n], a.dim, u[n]);
                }
#pragma unroll
                for (int d = 0; d + 1 < AHEAD; ++d)
#pragma unroll
                    for (int n = 0; n < ITEMS; ++n) {
                        rx[d][n] = rx[d + 1][n];
                        ru[d][n] = ru[d + 1][n];
                    }
                load(h + AHEAD, rx[AHEAD - 1], ru[AHEAD - 1]);
                float r = 1.0f;
                if (NORM) {
                    float t = 0.0f;
#pragma unroll
                    for (int n = 0; n < ITEMS; ++n)
#pragma unroll
                        for (int j = 0; j < V; ++j) t = fmaf(x[n][j], x[n][j], t);
                    r = rsqrtf(fmaf(lanes_sum<LANES>(t), a.inverse_dim, a.eps));
                }
                float dot = 0.0f;
#pragma unroll
                for (int n = 0; n < ITEMS; ++n) {
                    if (!BWD) {
#pragma unroll
                        for (int j = 0; j < V; ++j) u[n][j] = NORM ? x[n][j] * r * gain[n][j] : x[n][j];
                    }
#pragma unroll
                    for (int k = 0; k < A; ++k) {
                        // (a sine of 0: passed on, also next to what is not finite)
                        const float p = u[n][I::first(k)], q = u[n][I::second(k)];
                        u[n][I::first(k)] = s[n][k] != 0.0f ? fmaf(p, c[n][k], -(q * s[n][k])) : p * c[n][k];
                        u[n][I::second(k)] = s[n][k] != 0.0f ? fmaf(p, s[n][k], q * c[n][k]) : q * c[n][k];
                    }
                    if (BWD && NORM) {
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            x[n][j] *= r;
                            sums[w][n][j] += work ? u[n][j] * x[n][j] : 0.0f;
                            u[n][j] *= gain[n][j];
                            dot = fmaf(u[n][j], x[n][j], dot);
                        }
                    }
                }
                if (BWD && NORM) dot = lanes_sum<LANES>(dot) * a.inverse_dim;
#pragma unroll
                for (int n = 0; n < ITEMS; ++n) {
                    const I it(lane + n * LANES, a.dim, a.pairs);
                    if (BWD && NORM)
#pragma unroll
                        for (int j = 0; j < V; ++j) u[n][j] = r * fmaf(-x[n][j], dot, u[n][j]);
                    if (work) it.store(to + h * a.dim, a.dim, u[n]);
                }
            }
        }
    }
    if constexpr (BWD && NORM) {
        if (!a.part) return;
        __shared__ float all[kGroups][LANES * V];
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int n = 0; n < ITEMS; ++n) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < V; ++j) all[group][lane * V + j] = sums[w][n][j];
                __syncthreads();
                for (int e = threadIdx.x; e < LANES * V; e += kBlock) {
                    const I it(e / V + n * LANES, a.dim, a.pairs);
                    float t = 0.0f;
                    for (int g = 0; g < kGroups; ++g) t += all[g][e];
                    if (it.there(e % V, a.dim)) a.part[((size_t)blockIdx.x * 2 + w) * a.dim + it.component(e % V)] = t;
                }
            }
    }
}

// The gains' gradient from the workgroups' sums, in a fixed order: a wavefront per component.
__global__ __launch_bounds__(64) void rotate_gain_kernel(const float *__restrict__ part, float *dq, float *dk, const int groups, const int dim, const int add)
{
    const int w = (int)blockIdx.x / dim, j = (int)blockIdx.x % dim;
    float    *out = w ? dk : dq;
    if (!out) return;
    float t = 0.0f;
    for (int g = threadIdx.x; g < groups; g += 64) t += part[((size_t)g * 2 + w) * dim + j];
    t = lanes_sum<64>(t);
    if (threadIdx.x == 0) out[j] = (add ? out[j] : 0.0f) + t;
}

int check(const cngp_rotate_config *c, int64_t N) {
    if (!c) return CNGP_ERR_NULL;
    if (c->heads < 0 || c->heads > 4096 || c->kv_heads < 0 || c->kv_heads > 4096 || c->heads + c->kv_heads < 1) return CNGP_ERR_INVALID;
    if (c->dim < 1 || c->dim > kMostDim || c->axes < 1 || c->axes > 4) return CNGP_ERR_INVALID;
    int pairs = 0;
    for (int a = 0; a < 4; ++a) {
        if (c->pairs[a] < 0 || c->pairs[a] > kMostDim / 2 || (a >= c->axes && c->pairs[a])) return CNGP_ERR_INVALID;
        pairs += c->pairs[a];
    }
    if (2 * pairs > c->dim) return CNGP_ERR_INVALID;
    if (c->io_dtype != CNGP_F32 && c->io_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (!std::isfinite(c->eps) || c->eps < 0.0f) return CNGP_ERR_INVALID;
    if (c->flags & ~(uint32_t)(CNGP_ROTATE_NORM | CNGP_ROTATE_NEXT | CNGP_ZERO_GRADS)) return CNGP_ERR_INVALID;
    if (N < 0 || N > 0x7fffffffll - 65536) return CNGP_ERR_INVALID;
    return CNGP_OK;
}

struct Shape { int vec, lanes, items; };

template <typename T, int VEC, bool NEXT, int LANES, int ITEMS>
int launch(const RotateArgs &a, bool norm, bool bwd, unsigned blocks, hipStream_t s) {
    LaunchTimer t(s, bwd ? K_ROTATE_BWD : K_ROTATE);
    if (norm) bwd ? rotate_kernel<T, VEC, NEXT, LANES, ITEMS, true, true><<<blocks, kBlock, 0, s>>>(a)
                  : rotate_kernel<T, VEC, NEXT, LANES, ITEMS, true, false><<<blocks, kBlock, 0, s>>>(a);
    else bwd ? rotate_kernel<T, VEC, NEXT, LANES, ITEMS, false, true><<<blocks, kBlock, 0, s>>>(a)
             : rotate_kernel<T, VEC, NEXT, LANES, ITEMS, false, false><<<blocks, kBlock, 0, s>>>(a);
    return launch_status("rotate_kernel");
}
template <typename T, int VEC, bool NEXT>
int launch_lanes(const RotateArgs &a, int lanes, int items, bool norm, bool bwd, unsigned blocks, hipStream_t s) {
    constexpr int kMost = kMostDim / Item<T, VEC, NEXT>::kValues;
    switch (lanes) {
        case 4: return launch<T, VEC, NEXT, 4, 1>(a, norm, bwd, blocks, s);
        case 8: return launch<T, VEC, NEXT, 8, 1>(a, norm, bwd, blocks, s);
        case 16: return launch<T, VEC, NEXT, 16, 1>(a, norm, bwd, blocks, s);
        case 32: return launch<T, VEC, NEXT, 32, 1>(a, norm, bwd, blocks, s);
        default:                         // (vectors of a head of at most 512 are fewer)
            if constexpr (kMost > 128)
                if (items > 2) return launch<T, VEC, NEXT, 64, 4>(a, norm, bwd, blocks, s);
            if constexpr (kMost > 64)
                if (items > 1) return launch<T, VEC, NEXT, 64, 2>(a, norm, bwd, blocks, s);
            if constexpr (kMost > 32) return launch<T, VEC, NEXT, 64, 1>(a, norm, bwd, blocks, s);
            return CNGP_ERR_INVALID;
    }
}

int run(const cngp_rotate_config *c, RotateArgs a, bool bwd, unsigned *groups, hipStream_t s) {
    const bool half = c->io_dtype == CNGP_F16, next = c->flags & CNGP_ROTATE_NEXT, norm = c->flags & CNGP_ROTATE_NORM;
    const int  full = half ? 8 : 4;
    bool whole = c->dim % full == 0 && (next || a.pairs % full == 0);
    for (int w = 0; w < 2; ++w)
        whole = whole && ((uintptr_t)a.x[w] & 15u) == 0 && ((uintptr_t)a.y[w] & 15u) == 0 && ((uintptr_t)a.dy[w] & 15u) == 0;
    const int vec = whole ? full : 1;
    const int items = next ? (c->dim + (vec == 1 ? 2 : vec) - 1) / (vec == 1 ? 2 : vec)
                           : (a.pairs + vec - 1) / vec + (c->dim - 2 * a.pairs + 2 * vec - 1) / (2 * vec);
    int lanes = 4;
    while (lanes < items && lanes < 64) lanes *= 2;
    const int64_t H = c->heads + c->kv_heads, per = kBlock / lanes;
    // a group per row shares its angles among all heads; few rows are split by heads, so that the chip has work
    int64_t split = 1;
    while (split < H && a.N * split < 256 * 8 * per) split *= 2;
    a.each = (int32_t)((H + split - 1) / split);
    a.split = (int32_t)((H + a.each - 1) / a.each);
    int64_t blocks = (a.N * a.split + per - 1) / per;
    if (bwd && norm) blocks = std::min<int64_t>(blocks, kMostGroups);
    blocks = std::min<int64_t>(blocks, kMostGroups256);
    if (groups) *groups = (unsigned)blocks;
    const int n = (items + lanes - 1) / lanes;
    if (half) {
        if (vec > 1) return next ? launch_lanes<_Float16, 8, true>(a, lanes, n, norm, bwd, (unsigned)blocks, s) : launch_lanes<_Float16, 8, false>(a, lanes, n, norm, bwd, (unsigned)blocks, s);
        return next ? launch_lanes<_Float16, 1, true>(a, lanes, n, norm, bwd, (unsigned)blocks, s) : launch_lanes<_Float16, 1, false>(a, lanes, n, norm, bwd, (unsigned)blocks, s);
    }
    if (vec > 1) return next ? launch_lanes<float, 4, true>(a, lanes, n, norm, bwd, (unsigned)blocks, s) : launch_lanes<float, 4, false>(a, lanes, n, norm, bwd, (unsigned)blocks, s);
    return next ? launch_lanes<float, 1, true>(a, lanes, n, norm, bwd, (unsigned)blocks, s) : launch_lanes<float, 1, false>(a, lanes, n, norm, bwd, (unsigned)blocks, s);
}

RotateArgs args_of(const cngp_rotate_config *c, int64_t N, const float *position, const float *omega) {
    RotateArgs a{};
    a.position = position; a.omega = omega; a.N = N;
    a.heads[0] = c->heads; a.heads[1] = c->kv_heads;
    a.dim = c->dim; a.axes = c->axes;
    for (int i = 0; i < 4; ++i) a.ends[i] = a.pairs += c->pairs[i];
    a.eps = c->eps; a.inverse_dim = 1.0f / (float)c->dim;
    return a;
}

}  // namespace

extern "C" {

int cngp_rotate_fwd(const cngp_rotate_config *cfg, const void *q, const void *k, int64_t N, const float *position, const float *omega, const float *gamma_q,
                    const float *gamma_k, void *q_out, void *k_out, void *stream) {
    if (int rc = check(cfg, N)) return rc;
    if (N == 0) return CNGP_OK;
    RotateArgs a = args_of(cfg, N, position, omega);
    if ((cfg->heads && (!q || !q_out)) || (cfg->kv_heads && (!k || !k_out)) || (a.pairs && (!position || !omega))) return CNGP_ERR_NULL;
    a.x[0] = q; a.x[1] = k; a.y[0] = q_out; a.y[1] = k_out; a.gamma[0] = gamma_q; a.gamma[1] = gamma_k;
    return run(cfg, a, false, nullptr, (hipStream_t)stream);
}

size_t cngp_rotate_workspace_bytes(const cngp_rotate_config *cfg, int64_t N) {
    if (check(cfg, N) || N == 0 || !(cfg->flags & CNGP_ROTATE_NORM)) return 0;
    return align256((size_t)kMostGroups * 2 * cfg->dim * 4);
}

int cngp_rotate_bwd(const cngp_rotate_config *cfg, const void *q, const void *k, int64_t N, const float *position, const float *omega, const float *gamma_q,
                    const float *gamma_k, const void *dq_out, const void *dk_out, void *dq, void *dk, float *dgamma_q, float *dgamma_k, void *workspace,
                    size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N)) return rc;
    const bool norm = cfg->flags & CNGP_ROTATE_NORM, gains = norm && (dgamma_q || dgamma_k);       // without norms they are zeros
    hipStream_t s = (hipStream_t)stream;
    unsigned groups = 0;
    if (N) {
        RotateArgs a = args_of(cfg, N, position, omega);
        if ((cfg->heads && (!dq_out || !dq || (norm && !q))) || (cfg->kv_heads && (!dk_out || !dk || (norm && !k))) || (a.pairs && (!position || !omega)))
            return CNGP_ERR_NULL;
        const size_t need = cngp_rotate_workspace_bytes(cfg, N);
        if (gains && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return CNGP_ERR_WORKSPACE;
        if (norm) { a.x[0] = q; a.x[1] = k; }
        a.dy[0] = dq_out; a.dy[1] = dk_out; a.y[0] = dq; a.y[1] = dk; a.gamma[0] = gamma_q; a.gamma[1] = gamma_k;
        a.part = gains ? (float *)workspace : nullptr;
        if (int rc = run(cfg, a, true, &groups, s)) return rc;
    }
    if (!gains && !((dgamma_q || dgamma_k) && (cfg->flags & CNGP_ZERO_GRADS))) return CNGP_OK;
    if (!norm) groups = 0;
    LaunchTimer t(s, K_ROTATE_BWD);
    rotate_gain_kernel<<<(unsigned)(2 * cfg->dim), 64, 0, s>>>((const float *)workspace, cfg->heads ? dgamma_q : nullptr, cfg->kv_heads ? dgamma_k : nullptr,
                                                                 (int)groups, cfg->dim, !(cfg->flags & CNGP_ZERO_GRADS));
    return launch_status("rotate_gain_kernel");
}

}  // extern "C"
