// Orthogonalised update of matrices by products of a polynomial.  X [m, n], m <= n (a taller matrix is taken transposed):
//     X = G / (|G| + eps);      each step   A = X X^T,   B = b A + c A A,   X <- a X + B X
// The products run on the matrix cores.  One fp16 number per value would not do: the polynomial lifts small singular values by 3.4 in each
// step and with them what a rounding put into their directions, so that 11 bits leave errors of a tenth of an entry.  Every operand is two fp16
// numbers, and a product three (high by high and both mixed ones, into the same sums): 22 bits.  (Low parts scaled apart, with sums of their own, took
// 16464 us for 4096 x 4096 and five steps, this form 5833, registers being short.)  Small matrices take four, with sums of their own for the low parts (multiply).
// A and B are symmetric: tiles on and below the diagonal are computed and written twice.
#include <algorithm>
#include <cmath>

#include "cngp_launch.h"
#include "cngp_matrix.h"

using namespace cngp;
using namespace cngp::mat;

namespace {

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
constexpr int kBlock = 256, kTile = 128, kDepth = 32;       // matrices are padded to tiles of 128; how much of a contraction a workgroup has in LDS at a time
constexpr int kPad = 8;                                     // halves between rows in LDS: 16-byte reads of neighbouring rows fall into different banks
// X, A and B are kept times these: singular values of 1 spread over rows of thousands, and their low parts, would be subnormal fp16 numbers.  What
// is left above: entries of X below 4 (so its singular values may be), of A below 16, of B below 64.
constexpr float kScaleX = 16384.0f, kScaleA = 4096.0f, kScaleB = 1024.0f;
constexpr int kNormParts = 1024;
constexpr int64_t kEnoughTiles = 256;                       // of 128 x 128: a CU each (1024 x 4096, 256 tiles: 471 us, by tiles of 64 x 64 529; 6 of 1000 x 333, 144: 254 and 237)
constexpr int kSlots = 512, kLeastShare = 256;              // ... that run at a time; least length of a share of a contraction

// High and low parts of a matrix, rows of `stride` values.
struct Pair {
    _Float16 *hi, *lo;
    size_t    stride, each;                                 // each: values of one matrix of the batch
};

__device__ __forceinline__ void put(const Pair &p, const size_t at, const float v) {
    const _Float16 h = (_Float16)v;
    p.hi[at] = h;
    p.lo[at] = (_Float16)(v - (float)h);
}
__device__ __forceinline__ void put4(const Pair &p, const size_t at, const float (&v)[4]) {
    half4_t h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        h[e] = (_Float16)v[e];
        l[e] = (_Float16)(v[e] - (float)h[e]);
    }
    *reinterpret_cast<half4_t *>(p.hi + at) = h;
    *reinterpret_cast<half4_t *>(p.lo + at) = l;
}
__device__ __forceinline__ void get4(const Pair &p, const size_t at, float (&v)[4]) {
    const half4_t h = *reinterpret_cast<const half4_t *>(p.hi + at), l = *reinterpret_cast<const half4_t *>(p.lo + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)h[e] + (float)l[e];
}

// ---------------------------------------------------------------- what is orthogonalised, and what becomes of it
// A matrix of its own, or the momentum of an optimiser step: then the norm's pass takes the gradient into it, and the result moves the weights.
struct Step {
    float    *m, *grad, *master;         // m NULL: a plain matrix
    _Float16 *half;
    float     momentum, scale, lr, keep; // keep: 1 - lr * weight decay
    int       nesterov, clear;
};
__device__ __forceinline__ float direction(const Step &st, const size_t at) {
    return st.nesterov ? fmaf(st.momentum, st.m[at], st.grad[at] * st.scale) : st.m[at];
}
template <typename T>
__device__ __forceinline__ float entry(const T *g, const Step &st, const size_t at) { return st.m ? direction(st, at) : (float)g[at]; }
// U entries `step` apart, those before `end`, the gradient taken into the momentum; all loads before the first store.
template <int U, typename T>
__device__ __forceinline__ void take(const T *g, const Step &st, const size_t first, const int64_t i, const int64_t step, const int64_t end, float (&v)[U]) {
    float gr[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool in = i + u * step < end;
        v[u] = !in ? 0.0f : st.m ? st.m[first + i + u * step] : (float)g[first + i + u * step];
        gr[u] = in && st.m ? st.grad[first + i + u * step] * st.scale : 0.0f;
    }
    if (!st.m) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        v[u] = fmaf(st.momentum, v[u], gr[u]);
        if (i + u * step < end) st.m[first + i + u * step] = v[u];
        if (st.nesterov) v[u] = fmaf(st.momentum, v[u], gr[u]);
    }
}
__device__ __forceinline__ void moved(const Step &st, const size_t at, const float v) {
    const float w = fmaf(-st.lr, v, st.master[at] * st.keep);
    st.master[at] = w;
    if (st.half) st.half[at] = (_Float16)w;
    if (st.clear) st.grad[at] = 0.0f;
}

__device__ __forceinline__ void moved4(const Step &st, const size_t at, const float (&v)[4]) {
    const float4 from = *reinterpret_cast<const float4 *>(st.master + at);
    const float  w[4] = {fmaf(-st.lr, v[0], from.x * st.keep), fmaf(-st.lr, v[1], from.y * st.keep), fmaf(-st.lr, v[2], from.z * st.keep), fmaf(-st.lr, v[3], from.w * st.keep)};
    *reinterpret_cast<float4 *>(st.master + at) = make_float4(w[0], w[1], w[2], w[3]);
    if (st.half) {
        half4_t h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = (_Float16)w[e];
        *reinterpret_cast<half4_t *>(st.half + at) = h;
    }
    if (st.clear) *reinterpret_cast<float4 *>(st.grad + at) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}

// ---------------------------------------------------------------- norm, start, no steps
__device__ __forceinline__ double block_sum(double v, double *room) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    return room[0] + room[1] + room[2] + room[3];
}

// Bound by its reads: eight to a lane are under way (4096 x 4096 fp32: 16 us; one: 98).
template <typename T>
__global__ __launch_bounds__(kBlock) void ortho_norm_kernel(const T *__restrict__ g, const Step st, const int64_t n, double *__restrict__ parts)
{
    __shared__ double room[4];
    const size_t first = (size_t)blockIdx.y * n;
    double sums[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) sums[u] = 0.0;
    const int64_t step = (int64_t)gridDim.x * kBlock;
    for (int64_t i = blockIdx.x * (int64_t)kBlock + threadIdx.x; i < n; i += 8 * step) {
        float v[8];
        take(g, st, first, i, step, n, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) sums[u] = fma((double)v[u], (double)v[u], sums[u]);
    }
    double t = 0.0;
#pragma unroll
    for (int u = 0; u < 8; ++u) t += sums[u];
    t = block_sum(t, room);
    if (threadIdx.x == 0) parts[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = t;
}

// In 64 bits, as the products with it: norms of fp32 matrices and their inverses leave fp32's range.
__device__ __forceinline__ double inverse(const double squares, const float eps) {
    const double norm = sqrt(squares) + (double)eps;
    return norm > 0.0 || norm != norm ? 1.0 / norm : 0.0;
}
__device__ __forceinline__ double inverse_norm(const double *parts, const int count, const float eps, double *room) {
    double t = 0.0;
    for (int i = threadIdx.x; i < count; i += kBlock) t += parts[(size_t)blockIdx.z * count + i];
    return inverse(block_sum(t, room), eps);
}

// X from G (transposed where `turned`), with zeros behind its edges: 64 x 64 tiles, bound by its reads and writes (4096 x 4096 fp32: 30 us).
template <typename T>
__global__ __launch_bounds__(kBlock) void ortho_start_kernel(const T *__restrict__ g, const Step st, const int rows, const int cols, const bool turned, const double *__restrict__ parts,
                                                             const int count, const float eps, const float scale, const Pair X)
{
    __shared__ double room[4];
    __shared__ float  tile[64][65];
    const double inv = inverse_norm(parts, count, eps, room) * (double)scale;
    const size_t first = (size_t)blockIdx.z * rows * cols;
    const int m0 = (int)blockIdx.y * 64, n0 = (int)blockIdx.x * 64;     // of X
    const int c = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < 64; r += 4) {
        const int row = (turned ? n0 : m0) + r, col = (turned ? m0 : n0) + c;
        const float v = row < rows && col < cols ? (float)((double)entry(g, st, first + (size_t)row * cols + col) * inv) : 0.0f;
        if (turned) tile[c][r] = v;
        else tile[r][c] = v;
    }
    __syncthreads();
    const int c4 = (threadIdx.x & 15) * 4;
    for (int r = threadIdx.x >> 4; r < 64; r += 16) {
        const float v[4] = {tile[r][c4], tile[r][c4 + 1], tile[r][c4 + 2], tile[r][c4 + 3]};
        put4(X, blockIdx.z * X.each + (size_t)(m0 + r) * X.stride + n0 + c4, v);
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void ortho_scale_kernel(const T *g, const Step st, T *out, const int64_t n, const double *__restrict__ parts, const int count, const float eps)
{
    __shared__ double room[4];
    const double inv = inverse_norm(parts, count, eps, room);
    for (int64_t i = blockIdx.x * (int64_t)kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock)
    {
        const size_t at = (size_t)blockIdx.z * n + i;
        const float  v = (float)((double)entry(g, st, at) * inv);
        if (st.m) moved(st, at, v);
        else out[at] = (T)v;
    }
}

// ---------------------------------------------------------------- products
// Short sums, of small matrices, show what long ones bury in their own rounding: there the products with low parts have sums of their own, low by
// low among them, added to those of the high parts at the end.  (14 x 53: 1.3e-6 off after five steps, so 1.0, fp32 arithmetic 0.7; 2 of 15 x 821: 1.6, 0.8, 0.8.  In
// tiles of 64 and in one launch, where it costs little: 6 of 1000 x 333 237 us, so 240, 64 x 64 17.0 and 18.2.)
__device__ __forceinline__ void multiply(const half8_t ah, const half8_t al, const half8_t bh, const half8_t bl, acc_t &sum, acc_t &fine) {
    fine = mfma(bl, al, fine);
    sum = mfma(bh, ah, sum);
    fine = mfma(bh, al, fine);
    fine = mfma(bl, ah, fine);
}

enum : int { GRAM, POLY, UPDATE, LAST };
struct ProductArgs {
    Pair   A, B, C, D;                   // C = epilogue(A B^T, or A B for updates; D)
    int    depth, tiles_m, tiles_n, tiles;
    int    whole, parts;                 // tiles (of all matrices) by one workgroup each; the others by `parts`, each a share of the contraction
    float *sums;                         // ... into here, as their lanes hold them: [tile, part, subtiles of 32 x 32, 4, lanes, 4]
    float  of_sum, of_d;                 // C = of_sum * product + of_d * D
    void  *out;                          // LAST: the result
    int    m, n, turned, out_f16, wide;  // wide: four neighbouring results go as one
    Step   step;
};

struct Tile { int i, j; size_t z; };
template <bool BACK>
__device__ __forceinline__ Tile tile_of(const ProductArgs &a, const int number) {
    Tile t;
    t.z = (size_t)(number / a.tiles);
    const int n = number % a.tiles;
    if (BACK) {
        t.i = n % a.tiles_m;
        t.j = n / a.tiles_m;
    } else {                             // the triangle's tiles, row after row
        t.i = (int)((sqrtf(8.0f * (float)n + 1.0f) - 1.0f) * 0.5f);
        while ((t.i + 1) * (t.i + 2) / 2 <= n) ++t.i;
        while (t.i * (t.i + 1) / 2 > n) --t.i;
        t.j = n - t.i * (t.i + 1) / 2;
    }
    return t;
}

// What becomes of four neighbouring sums, row i, columns j ..
template <int WHAT>
__device__ __forceinline__ void finish(const ProductArgs &a, const Tile &t, const int i, const int j, const float (&sum)[4]) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = sum[e] * a.of_sum;
    if (WHAT != GRAM) {
        float d[4];
        get4(a.D, t.z * a.D.each + (size_t)i * a.D.stride + j, d);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(a.of_d, d[e], v[e]);
    }
    if (WHAT != LAST) put4(a.C, t.z * a.C.each + (size_t)i * a.C.stride + j, v);
    if ((WHAT == GRAM || WHAT == POLY) && t.i != t.j)
#pragma unroll
        for (int e = 0; e < 4; ++e) put(a.C, t.z * a.C.each + (size_t)(j + e) * a.C.stride + i, v[e]);
    if (WHAT == LAST && i < a.m && j < a.n) {
        const size_t first = t.z * (size_t)a.m * a.n;
        if (a.wide) {
            const size_t at = first + (size_t)i * a.n + j;
            if (a.step.m) moved4(a.step, at, v);
            else if (a.out_f16) {
                half4_t h;
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = (_Float16)v[e];
                *reinterpret_cast<half4_t *>((_Float16 *)a.out + at) = h;
            } else *reinterpret_cast<float4 *>((float *)a.out + at) = make_float4(v[0], v[1], v[2], v[3]);
        } else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < a.n) {
                    const size_t at = first + (a.turned ? (size_t)(j + e) * a.m + i : (size_t)i * a.n + j + e);
                    if (a.step.m) moved(a.step, at, v[e]);
                    else if (a.out_f16) ((_Float16 *)a.out)[at] = (_Float16)v[e];
                    else ((float *)a.out)[at] = v[e];
                }
    }
}

// A tile of 64 U x 64 U of a product by four wavefronts of 32 U x 32 U; computed transposed (a lane has a row of C and four neighbouring columns in
// four registers).  The next piece of the contraction is fetched into registers while one is multiplied from LDS, two buffers, so one barrier a piece.
// 4096 x 4096: 460 us the last product, 235 and 255 the triangles', 870 TFLOP/s of fp16 operations where a library product reaches 1200.  Bound by what is
// exposed around the barriers: wavefronts wait for the matrix instructions' queue half of the time, for barriers and loads a quarter.  One buffer and three
// workgroups to a CU took 6116 us in place of 5000 for the five steps, pieces fetched further ahead (64 x 64 tiles) 244 for 236.
template <int WHAT, int U>
__global__ __launch_bounds__(kBlock, 2) void ortho_product_kernel(const ProductArgs a)
{
    constexpr bool kBack = WHAT == UPDATE || WHAT == LAST;              // the right factor lies by rows of the contraction
    constexpr int  TILE = 64 * U, kRowA = kDepth, kRowB = kBack ? TILE + 32 : kDepth, kSizeA = TILE * kRowA, kSizeB = kBack ? kDepth * kRowB : TILE * kRowB;
    constexpr int  kBackRow = TILE / 8, kStepA = kBlock / 4, kStepB = kBack ? kBlock / kBackRow : kStepA;
    __shared__ __align__(16) _Float16 lds[2][2 * kSizeA + 2 * kSizeB];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    int number = (int)blockIdx.x, part = -1, k0 = 0, k_end = a.depth;
    if (number >= a.whole) {
        const int share = (a.depth / kDepth + a.parts - 1) / a.parts * kDepth;
        part = number - a.whole;
        number = a.whole + part / a.parts;
        k0 = part % a.parts * share;
        k_end = k0 + share < a.depth ? k0 + share : a.depth;
    }
    const Tile t = tile_of<kBack>(a, number);
    const int i0 = t.i * TILE, j0 = t.j * TILE, wi = 32 * U * (wave & 1), wj = 32 * U * (wave >> 1);

    words_t r[4 * U];
    const _Float16 *pa = a.A.hi + t.z * a.A.each + (size_t)(i0 + ((int)threadIdx.x >> 2)) * a.A.stride + k0 + ((int)threadIdx.x & 3) * 8;
    const _Float16 *pb = a.B.hi + t.z * a.B.each + (kBack ? (size_t)(k0 + (int)threadIdx.x / kBackRow) * a.B.stride + j0 + (int)threadIdx.x % kBackRow * 8
                                                          : (size_t)(j0 + ((int)threadIdx.x >> 2)) * a.B.stride + k0 + ((int)threadIdx.x & 3) * 8);
    const ptrdiff_t la = a.A.lo - a.A.hi, lb = a.B.lo - a.B.hi;
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const _Float16 *qa = pa + (size_t)(kStepA * i) * a.A.stride, *qb = pb + (size_t)(kStepB * i) * a.B.stride;
            r[i] = *reinterpret_cast<const words_t *>(qa);
            r[U + i] = *reinterpret_cast<const words_t *>(qa + la);
            r[2 * U + i] = *reinterpret_cast<const words_t *>(qb);
            r[3 * U + i] = *reinterpret_cast<const words_t *>(qb + lb);
        }
        pa += kDepth;
        pb += kBack ? (size_t)kDepth * a.B.stride : (size_t)kDepth;
    };
    // Banks: rows along the contraction are 64 bytes, their 16-byte pieces turned by (row / 4) % 4 (sixteen lanes' pieces of sixteen rows, or of four whole rows,
    // then lie in different ones); rows across it are 64 bytes more than a multiple of 256 (a transposing read takes 64 bytes of four rows).
    const int oa = ((int)threadIdx.x >> 2) * kRowA + (((int)threadIdx.x & 3) ^ ((int)threadIdx.x >> 4 & 3)) * 8, ob = kBack ? (int)threadIdx.x / kBackRow * kRowB + (int)threadIdx.x % kBackRow * 8 : oa;
    auto keep = [&](_Float16 *to) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int qa = oa + kStepA * i * kRowA, qb = ob + kStepB * i * kRowB;
            *reinterpret_cast<words_t *>(to + qa) = r[i];
            *reinterpret_cast<words_t *>(to + kSizeA + qa) = r[U + i];
            *reinterpret_cast<words_t *>(to + 2 * kSizeA + qb) = r[2 * U + i];
            *reinterpret_cast<words_t *>(to + 2 * kSizeA + kSizeB + qb) = r[3 * U + i];
        }
    };

    constexpr bool kFine = U == 1;       // products with low parts in sums of their own, low by low among them (see multiply)
    acc_t sum[U][U], fine = zero();
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int w = 0; w < U; ++w) sum[u][w] = zero();
    if (k0 < k_end) fetch();
    for (int b = 0; k0 < k_end; k0 += kDepth, b ^= 1) {
        keep(lds[b]);
        __syncthreads();
        if (k0 + kDepth < k_end) fetch();
        const _Float16 *A = lds[b], *B = lds[b] + 2 * kSizeA;
#pragma unroll
        for (int s = 0; s < kDepth / 16; ++s) {
            half8_t ah[U], al[U], bh[U], bl[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int       turned = 8 * ((2 * s + half) ^ (col >> 2 & 3));
                const _Float16 *p = A + (wi + 32 * u + col) * kRowA + turned;
                ah[u] = read8(p);
                al[u] = read8(p + kSizeA);
                if constexpr (kBack) {
                    bh[u] = read_column(B, kRowB, 16 * s, wj + 32 * u, lane);
                    bl[u] = read_column(B + kSizeB, kRowB, 16 * s, wj + 32 * u, lane);
                } else {
                    const _Float16 *q = B + (wj + 32 * u + col) * kRowB + turned;
                    bh[u] = read8(q);
                    bl[u] = read8(q + kSizeB);
                }
            }
            if constexpr (kFine) {
                multiply(ah[0], al[0], bh[0], bl[0], sum[0][0], fine);
                continue;
            }
#pragma unroll
            for (int which = 0; which < 3; ++which)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int w = 0; w < U; ++w) sum[u][w] = mfma(which == 2 ? bl[w] : bh[w], which == 1 ? al[u] : ah[u], sum[u][w]);
        }
    }
    if constexpr (kFine) sum[0][0] += fine;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int w = 0; w < U; ++w)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float v[4] = {sum[u][w][4 * g], sum[u][w][4 * g + 1], sum[u][w][4 * g + 2], sum[u][w][4 * g + 3]};
                if (part >= 0)
                    *reinterpret_cast<float4 *>(a.sums + ((((size_t)part * (U * U) + u * U + w) * 4 + g) * kBlock + threadIdx.x) * 4) = make_float4(v[0], v[1], v[2], v[3]);
                else finish<WHAT>(a, t, i0 + wi + 32 * u + col, j0 + wj + 32 * w + 8 * g + 4 * half, v);
            }
}

// Shares of a contraction added up, in their order: a workgroup for eight columns of one of each wavefront's 32 x 32.  Bound by its reads (thirds of 144 tiles,
// 28 MB: 13 us).
template <int WHAT, int U>
__global__ __launch_bounds__(kBlock) void ortho_join_kernel(const ProductArgs a)
{
    constexpr bool kBack = WHAT == UPDATE || WHAT == LAST;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    const int each = U * U * 4, tail = (int)blockIdx.x / each, piece = (int)blockIdx.x % each, u = piece / (4 * U), w = piece / 4 % U, g = piece & 3;
    const Tile t = tile_of<kBack>(a, a.whole + tail);
    const float *p = a.sums + (((size_t)tail * a.parts * each + piece) * kBlock + threadIdx.x) * 4;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int k = 0; k < a.parts; ++k) {
        const float4 x = *reinterpret_cast<const float4 *>(p + (size_t)k * each * kBlock * 4);
        v[0] += x.x;
        v[1] += x.y;
        v[2] += x.z;
        v[3] += x.w;
    }
    finish<WHAT>(a, t, 64 * U * t.i + 32 * U * (wave & 1) + 32 * u + col, 64 * U * t.j + 32 * U * (wave >> 1) + 32 * w + 8 * g + 4 * half, v);
}

// How a product's tiles are shared out.  A card has room for two workgroups of 128 x 128 on each of its 256 CUs: what is left after whole turns of
// 512 is cut along the contraction, into as many parts as there is room for (of 256 at least), and joined by a second launch.  (528 tiles of a
// triangle of 4096: the last 16 alone took more than half of what the 512 before them did, 5683 us in place of 5007 for the five steps.  Tiles that do not
// fill the card go in parts of 1024 at least: 4 of 1024 x 4096, thirds of 1365, 95 + 13 us in place of 141 by 64 x 64; of 341, 26 + 23 in place of 36.)
struct Cut {
    int U, tiles, whole, parts;
    int64_t rest() const { return (int64_t)tiles - whole; }
};
Cut cut_of(bool back, int mp, int np, int depth, int batch) {
    auto count = [&](int64_t tile) { const int64_t tm = mp / tile, tn = np / tile; return (int)((back ? tm * tn : tm * (tm + 1) / 2) * batch); };
    Cut c{2, count(kTile), 0, 1};
    c.whole = c.tiles / kSlots * kSlots;
    const int most = c.rest() ? (int)std::min<int64_t>(kSlots / c.rest(), depth / (c.whole ? kLeastShare : 4 * kLeastShare)) : 1;
    if (most > 1 && c.whole + c.rest() * most >= kEnoughTiles) {
        c.parts = most;
        return c;
    }
    if (c.tiles < kEnoughTiles) {
        c = Cut{1, count(kTile / 2), 0, 1};
        c.parts = depth >= 4 * kLeastShare ? (int)std::min<int64_t>(std::max(kSlots / c.tiles, 1), depth / kLeastShare) : 1;
    }
    c.whole = c.parts > 1 ? 0 : c.tiles;
    return c;
}
size_t sums_bytes(const Cut &c) { return (size_t)c.rest() * c.parts * (64 * c.U) * (64 * c.U) * 4; }

template <int WHAT>
int product(const ProductArgs &p, int mp, int np, int batch, hipStream_t st) {
    constexpr bool kBack = WHAT == UPDATE || WHAT == LAST;
    ProductArgs a = p;
    const Cut   c = cut_of(kBack, mp, np, a.depth, batch);
    a.tiles_m = mp / (64 * c.U);
    a.tiles_n = np / (64 * c.U);
    a.tiles = c.tiles / batch;
    a.whole = c.whole;
    a.parts = c.parts;
    LaunchTimer t(st, K_ORTHO_PRODUCT);
    const unsigned groups = (unsigned)(c.whole + c.rest() * c.parts);
    if (c.U == 2) ortho_product_kernel<WHAT, 2><<<groups, kBlock, 0, st>>>(a);
    else ortho_product_kernel<WHAT, 1><<<groups, kBlock, 0, st>>>(a);
    if (int rc = launch_status("ortho_product_kernel")) return rc;
    if (!c.rest()) return CNGP_OK;
    if (c.U == 2) ortho_join_kernel<WHAT, 2><<<(unsigned)(c.rest() * 16), kBlock, 0, st>>>(a);
    else ortho_join_kernel<WHAT, 1><<<(unsigned)(c.rest() * 4), kBlock, 0, st>>>(a);
    return launch_status("ortho_join_kernel");
}

// ---------------------------------------------------------------- matrices of at most 64 x 128
// One workgroup does everything in one launch: X in registers (fp32, as the tiles of the last product come out), its two parts and those of A and
// B in LDS.  Bound by the chain of products (four barriers a step): 64 x 64, five steps 18 us; by the kernels above 262.
struct SmallArgs {
    const void *g;
    void       *out;
    int   rows, cols, turned, m, n, steps;
    float a, b, c, eps;
    Step  step;
};
template <typename T, int NP>
__global__ __launch_bounds__(kBlock) void ortho_small_kernel(const SmallArgs a)
{
    constexpr int kTiles = NP / 64, kRowX = NP + kPad, kRowA = 64 + kPad;   // column tiles to a wavefront: two row tiles by NP / 32
    __shared__ __align__(16) _Float16 X[2][64 * kRowX], A[2][64 * kRowA], B[2][64 * kRowA];
    __shared__ double room[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, col = lane & 31;
    const int i = 32 * (wave & 1) + col, jw = 32 * (wave >> 1);           // this lane's row; the wavefront's first column (the next tile 64 further on)
    const size_t count = (size_t)a.rows * a.cols;
    const size_t first = blockIdx.x * count;
    const T *g = (const T *)a.g;
    double t = 0.0;
    for (int e = threadIdx.x; e < (int)count; e += 8 * kBlock) {
        float v[8];
        take(g, a.step, first, e, kBlock, (int64_t)count, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) t = fma((double)v[u], (double)v[u], t);
    }
    const double scale = inverse(block_sum(t, room), a.eps);
    float x[kTiles][16];
    auto place = [&](const int r, const int j) -> size_t { return a.turned ? (size_t)j * a.m + r : (size_t)r * a.n + j; };
#pragma unroll
    for (int k = 0; k < kTiles; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int j = jw + 64 * k + 8 * (r >> 2) + 4 * half + (r & 3);
            x[k][r] = i < a.m && j < a.n ? (float)((double)entry(g, a.step, first + place(i, j)) * scale) : 0.0f;
        }
    auto keep4 = [&](_Float16 *hi, _Float16 *lo, const int at, const float (&v)[4]) {
        half4_t h, l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[e] = (_Float16)v[e];
            l[e] = (_Float16)(v[e] - (float)h[e]);
        }
        *reinterpret_cast<half4_t *>(hi + at) = h;
        *reinterpret_cast<half4_t *>(lo + at) = l;
    };
    for (int step = 0; step < a.steps; ++step) {
#pragma unroll
        for (int k = 0; k < kTiles; ++k)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = x[k][4 * q + e] * kScaleX;
                keep4(X[0], X[1], i * kRowX + jw + 64 * k + 8 * q + 4 * half, v);
            }
        __syncthreads();
        acc_t s = zero(), f = zero();    // A: rows i, columns jw ..
#pragma unroll
        for (int k = 0; k < NP / 16; ++k) {
            const int pi = i * kRowX + 16 * k + 8 * half, pj = (jw + col) * kRowX + 16 * k + 8 * half;
            multiply(read8(X[0] + pi), read8(X[1] + pi), read8(X[0] + pj), read8(X[1] + pj), s, f);
        }
        s += f;
        float y[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[4 * q + e] = v[e] = s[4 * q + e] * (kScaleA / (kScaleX * kScaleX));
            keep4(A[0], A[1], i * kRowA + jw + 8 * q + 4 * half, v);
        }
        __syncthreads();
        s = zero();
        f = zero();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int pi = i * kRowA + 16 * k + 8 * half, pj = (jw + col) * kRowA + 16 * k + 8 * half;
            multiply(read8(A[0] + pi), read8(A[1] + pi), read8(A[0] + pj), read8(A[1] + pj), s, f);
        }
        s += f;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(a.b * (kScaleB / kScaleA), y[4 * q + e], s[4 * q + e] * (a.c * (kScaleB / (kScaleA * kScaleA))));
            keep4(B[0], B[1], i * kRowA + jw + 8 * q + 4 * half, v);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kTiles; ++k) {
            s = zero();
            f = zero();
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const int pi = i * kRowA + 16 * d + 8 * half;
                multiply(read8(B[0] + pi), read8(B[1] + pi), read_column(X[0], kRowX, 16 * d, jw + 64 * k, lane), read_column(X[1], kRowX, 16 * d, jw + 64 * k, lane), s, f);
            }
            s += f;
#pragma unroll
            for (int r = 0; r < 16; ++r) x[k][r] = fmaf(a.a, x[k][r], s[r] * (1.0f / (kScaleB * kScaleX)));
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kTiles; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int j = jw + 64 * k + 8 * (r >> 2) + 4 * half + (r & 3);
            if (i < a.m && j < a.n) {
                const size_t at = first + place(i, j);
                if (a.step.m) moved(a.step, at, x[k][r]);
                else ((T *)a.out)[at] = (T)x[k][r];
            }
        }
}

struct Shape {
    int    m, n, mp, np, parts;
    bool   turned, small;
    size_t x[2], a, b, norm, sums, bytes;
};
Shape shape_of(const cngp_ortho_config *c) {
    Shape s{};
    s.turned = c->rows > c->cols;
    s.m = std::min(c->rows, c->cols);
    s.n = std::max(c->rows, c->cols);
    s.mp = (s.m + kTile - 1) / kTile * kTile;
    s.np = (s.n + kTile - 1) / kTile * kTile;
    s.parts = (int)std::max<int64_t>(1, std::min<int64_t>((int64_t)s.m * s.n / 4096, kNormParts / std::min(c->batch, 16)));
    s.small = s.m <= 64 && s.n <= 128;
    if (s.small) return s;
    size_t at = 0;
    auto take = [&](bool wanted, size_t bytes) { const size_t o = at; if (wanted) at += align256(bytes); return o; };
    const size_t batch = (size_t)c->batch, x = batch * s.mp * s.np * 4, a = batch * s.mp * s.mp * 4;
    s.norm = take(true, batch * s.parts * 8);
    s.x[0] = take(c->steps > 0, x);
    s.x[1] = take(c->steps > 1, x);
    s.a = take(c->steps > 0, a);
    s.b = take(c->steps > 0, a);
    if (c->steps > 0) {
        size_t most = 0;
        for (const Cut &k : {cut_of(false, s.mp, s.np, s.np, c->batch), cut_of(false, s.mp, s.np, s.mp, c->batch), cut_of(true, s.mp, s.np, s.mp, c->batch)})
            most = std::max(most, sums_bytes(k));
        s.sums = take(most > 0, most);
    }
    s.bytes = at;
    return s;
}

int check(const cngp_ortho_config *c) {
    if (!c) return CNGP_ERR_NULL;
    if (c->rows < 1 || c->rows > 16384 || c->cols < 1 || c->cols > 16384 || c->batch < 1 || c->batch > 65535) return CNGP_ERR_INVALID;
    if (c->io_dtype != CNGP_F32 && c->io_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->steps < 0 || c->steps > 32 || c->flags) return CNGP_ERR_INVALID;
    if (!std::isfinite(c->eps) || c->eps < 0.0f) return CNGP_ERR_INVALID;
    for (float v : {c->a, c->b, c->c})
        if (!(std::fabs(v) <= 16.0f)) return CNGP_ERR_INVALID;
    return CNGP_OK;
}

Pair pair_of(char *ws, size_t at, int rows, int cols, int batch) {
    Pair p;
    p.stride = (size_t)cols;
    p.each = (size_t)rows * cols;
    p.hi = (_Float16 *)(ws + at);
    p.lo = p.hi + p.each * batch;
    return p;
}

template <typename T>
int norm_and_start(const cngp_ortho_config *c, const Shape &s, const T *g, const Step &step, T *out, char *ws, hipStream_t st) {
    LaunchTimer t(st, K_ORTHO);
    double *parts = (double *)(ws + s.norm);
    const int64_t n = (int64_t)s.m * s.n;
    ortho_norm_kernel<T><<<dim3((unsigned)s.parts, (unsigned)c->batch), kBlock, 0, st>>>(g, step, n, parts);
    if (int rc = launch_status("ortho_norm_kernel")) return rc;
    if (c->steps == 0) {
        ortho_scale_kernel<T><<<dim3((unsigned)std::min<int64_t>((n + 1023) / 1024, 1024), 1, (unsigned)c->batch), kBlock, 0, st>>>(g, step, out, n, parts, s.parts, c->eps);
        return launch_status("ortho_scale_kernel");
    }
    ortho_start_kernel<T><<<dim3((unsigned)(s.np / 64), (unsigned)(s.mp / 64), (unsigned)c->batch), kBlock, 0, st>>>(g, step, c->rows, c->cols, s.turned, parts, s.parts, c->eps,
                                                                                                                  kScaleX, pair_of(ws, s.x[0], s.mp, s.np, c->batch));
    return launch_status("ortho_start_kernel");
}

template <typename T>
void launch_small(const SmallArgs &a, int batch, hipStream_t st) {
    if (a.n <= 64) ortho_small_kernel<T, 64><<<(unsigned)batch, kBlock, 0, st>>>(a);
    else ortho_small_kernel<T, 128><<<(unsigned)batch, kBlock, 0, st>>>(a);
}
int small(const cngp_ortho_config *c, const Shape &s, const void *g, const Step &step, void *out, hipStream_t st) {
    SmallArgs a{g, out, c->rows, c->cols, s.turned, s.m, s.n, c->steps, c->a, c->b, c->c, c->eps, step};
    LaunchTimer t(st, K_ORTHO);
    if (c->io_dtype == CNGP_F16) launch_small<_Float16>(a, c->batch, st);
    else launch_small<float>(a, c->batch, st);
    return launch_status("ortho_small_kernel");
}

int run(const cngp_ortho_config *cfg, const void *g, const Step &step, void *out, void *workspace, size_t workspace_bytes, hipStream_t st) {
    const Shape s = shape_of(cfg);
    if (s.small) return small(cfg, s, g, step, out, st);
    if (s.bytes && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < s.bytes)) return CNGP_ERR_WORKSPACE;
    char *ws = (char *)workspace;
    if (int rc = cfg->io_dtype == CNGP_F16 ? norm_and_start(cfg, s, (const _Float16 *)g, step, (_Float16 *)out, ws, st)
                                           : norm_and_start(cfg, s, (const float *)g, step, (float *)out, ws, st)) return rc;
    const Pair A = pair_of(ws, s.a, s.mp, s.mp, cfg->batch), B = pair_of(ws, s.b, s.mp, s.mp, cfg->batch);
    for (int i = 0; i < cfg->steps; ++i) {
        const bool last = i + 1 == cfg->steps;
        const Pair X = pair_of(ws, s.x[i & 1], s.mp, s.np, cfg->batch), Y = last ? X : pair_of(ws, s.x[1 - (i & 1)], s.mp, s.np, cfg->batch);
        ProductArgs p{};
        p.sums = (float *)(ws + s.sums);
        p.A = X; p.B = X; p.C = A; p.D = A;
        p.depth = s.np; p.of_sum = kScaleA / (kScaleX * kScaleX);
        if (int rc = product<GRAM>(p, s.mp, s.np, cfg->batch, st)) return rc;
        p.A = A; p.B = A; p.C = B; p.D = A;
        p.depth = s.mp; p.of_sum = cfg->c * kScaleB / (kScaleA * kScaleA); p.of_d = cfg->b * kScaleB / kScaleA;
        if (int rc = product<POLY>(p, s.mp, s.np, cfg->batch, st)) return rc;
        p.A = B; p.B = X; p.C = Y; p.D = X;
        p.depth = s.mp; p.of_sum = 1.0f / kScaleB; p.of_d = cfg->a;
        if (last) {
            p.of_sum /= kScaleX; p.of_d /= kScaleX;
            p.out = out; p.m = s.m; p.n = s.n; p.turned = s.turned; p.out_f16 = cfg->io_dtype == CNGP_F16; p.step = step;
            const auto on = [](const void *q, uintptr_t bytes) { return ((uintptr_t)q & (bytes - 1)) == 0; };
            p.wide = !s.turned && s.n % 4 == 0 && (step.m ? on(step.master, 16) && on(step.grad, 16) && on(step.half, 8) : on(out, p.out_f16 ? 8 : 16));
        }
        if (int rc = last ? product<LAST>(p, s.mp, s.np, cfg->batch, st) : product<UPDATE>(p, s.mp, s.np, cfg->batch, st)) return rc;
    }
    return CNGP_OK;
}

}  // namespace

extern "C" {

size_t cngp_orthogonalise_workspace_bytes(const cngp_ortho_config *cfg) { return check(cfg) ? 0 : shape_of(cfg).bytes; }

int cngp_orthogonalise(const cngp_ortho_config *cfg, const void *g, void *out, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg)) return rc;
    if (!g || !out) return CNGP_ERR_NULL;
    return run(cfg, g, Step{}, out, workspace, workspace_bytes, (hipStream_t)stream);
}

int cngp_muon_step(const cngp_ortho_config *cfg, const cngp_muon *opt, float *master, void *half_copy, float *m, float *grad, int clear_grad, void *workspace,
                   size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg)) return rc;
    if (!opt || !master || !m || !grad) return CNGP_ERR_NULL;
    if (cfg->io_dtype != CNGP_F32) return CNGP_ERR_UNSUPPORTED;
    if (!(opt->lr >= 0.0f) || !std::isfinite(opt->lr) || !(opt->momentum >= 0.0f && opt->momentum < 1.0f) || !(opt->weight_decay >= 0.0f) ||
        !std::isfinite(opt->weight_decay) || !std::isfinite(opt->grad_scale) || (opt->nesterov != 0 && opt->nesterov != 1))
        return CNGP_ERR_INVALID;
    const Step step{m, grad, master, (_Float16 *)half_copy, opt->momentum, opt->grad_scale, opt->lr, 1.0f - opt->lr * opt->weight_decay, opt->nesterov, clear_grad != 0};
    return run(cfg, m, step, nullptr, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
