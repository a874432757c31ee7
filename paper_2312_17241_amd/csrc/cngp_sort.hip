// Optional reordering of a batch of query points by Morton code (the interleaved bits of the quantised
// coordinates), so that points that are close in space are close in the batch.  Not part of the paper's
// method: its hash tables leave no locality between neighbouring vertices, but neighbouring POINTS share
// the vertices of the coarse levels.
//
// The sort is a stable least-significant-digit radix sort of (code, index) pairs, 7 bits per pass, three
// passes for the 20- or 21-bit codes (10, 7 and 5 bits per axis for d = 2, 3, 4), written for 64-lane wavefronts:
//   keys     one workgroup per tile of 8192 points: codes from x, and the tile's histogram of the first digit
//   count    (passes 2, 3) the tile histograms of the next digit in the order the previous pass left
//   row scan one workgroup per digit value: exclusive prefix over the tiles, the digit's total beside it
//   scatter  one workgroup per tile.  A wavefront walks its eighth of the tile 64 elements at a time; the lanes
//            that hold the same digit find each other with seven ballots, which gives every element its rank
//            among the equal digits before it without an atomic, so the order of equal digits is the order of
//            the input.  The tile is then laid out by digit in LDS and leaves in runs of consecutive addresses
//            (64 elements of a digit per tile on average: whole cache lines instead of 64 lines per store).
// No kernel waits for another workgroup; every pass is three ordinary launches.
#include <cstdint>
#include <cstring>

#include <hip/hip_runtime.h>

#include "../../include/cngp.h"
#include "cngp_radix.h"

namespace cngp { int record_hip_failure(hipError_t e, const char *what); }   // cngp_api.hip

namespace {

constexpr int kSortBlock = 256;          // gather kernel

// Bits per axis: more than these change nothing measurable (the finer levels have no reuse to find).
constexpr int morton_bits(int d) { return d == 3 ? 7 : d == 4 ? 5 : 10; }

// code = bit b of coordinate j at position b * D + j; coordinates quantised as floor(x * 2^B) clamped to
// [0, 2^B - 1] (the scaling by a power of two is exact; a NaN counts as 0).
template <int D>
__device__ __forceinline__ uint32_t morton_code(const float *__restrict__ x, const int64_t n)
{
    constexpr int B = morton_bits(D);
    uint32_t code = 0;
#pragma unroll
    for (int j = 0; j < D; ++j) {
        const float    v = fminf(fmaxf(x[n * D + j] * (float)(1 << B), 0.0f), (float)((1 << B) - 1));
        const uint32_t q = (uint32_t)v;
#pragma unroll
        for (int b = 0; b < B; ++b) code |= ((q >> b) & 1u) << (b * D + j);
    }
    return code;
}

template <int D>
__global__ __launch_bounds__(kTileBlock) void morton_keys_kernel(const float *__restrict__ x, const int64_t N,
                                                                 uint32_t *__restrict__ keys, uint32_t *__restrict__ counts,
                                                                 const int64_t tiles)
{
    __shared__ uint32_t hist[kTileWaves * kDigits];
    const int     t = threadIdx.x, w = t >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * kTile;
    for (int i = t; i < kTileWaves * kDigits; i += kTileBlock) hist[i] = 0;
    __syncthreads();
#pragma unroll 4
    for (int r = 0; r < kRounds; ++r) {
        const int64_t n = n0 + (int64_t)r * kTileBlock + t;
        if (n < N) {
            const uint32_t code = morton_code<D>(x, n);
            keys[n] = code;
            atomicAdd(&hist[w * kDigits + (code & (kDigits - 1))], 1u);
        }
    }
    __syncthreads();
    flush_tile_histogram(hist, counts, tiles, blockIdx.x, t);
}

// x_sorted[n] = x[perm[n]].  Every read fetches a whole 128-byte line for 4d bytes of it, and that line traffic (2.1 GB
// for 2^24 points) is what the kernel waits for: more loads in flight per lane, non-temporal loads or doing the reads
// inside the last scatter pass were all slower (measured).
template <int D>
__global__ __launch_bounds__(kSortBlock) void gather_points_kernel(const float *__restrict__ x, const int32_t *__restrict__ perm,
                                                                   const int64_t N, float *__restrict__ x_sorted)
{
    const int64_t n = (int64_t)blockIdx.x * kSortBlock + threadIdx.x;
    if (n >= N) return;
    const int64_t from = perm[n];
#pragma unroll
    for (int j = 0; j < D; ++j) x_sorted[n * D + j] = x[from * D + j];
}

struct SortSpace {
    size_t keys_a, keys_b, index, counts, totals, bytes;
};
SortSpace sort_space(int64_t N) {
    SortSpace s{};
    const size_t col = align256((size_t)N * 4);
    s.keys_a = 0;
    s.keys_b = col;
    s.index = 2 * col;
    s.counts = 3 * col;
    s.totals = s.counts + align256((size_t)kDigits * (size_t)tiles_of(N) * 4);
    s.bytes = s.totals + align256((size_t)kDigits * 4);
    return s;
}

template <int D>
int morton_sort(const float *x, int64_t N, int32_t *perm, float *x_sorted, char *ws, hipStream_t s) {
    const SortSpace sp = sort_space(N);
    uint32_t *keys_a = (uint32_t *)(ws + sp.keys_a), *keys_b = (uint32_t *)(ws + sp.keys_b);
    int32_t  *index = (int32_t *)(ws + sp.index);
    uint32_t *counts = (uint32_t *)(ws + sp.counts), *totals = (uint32_t *)(ws + sp.totals);
    const int64_t  tiles = tiles_of(N);
    const unsigned grid = (unsigned)tiles;
    constexpr int  bits = morton_bits(D) * D, passes = (bits + kDigitBits - 1) / kDigitBits;
    static_assert(passes == 3, "the buffers below are laid out for three passes");

    morton_keys_kernel<D><<<grid, kTileBlock, 0, s>>>(x, N, keys_a, counts, tiles);
    if (hipError_t e = hipGetLastError()) return cngp::record_hip_failure(e, "morton_keys_kernel");
    // pass 0: keys_a, identity -> keys_b, perm (as scratch); 1: keys_b, perm -> keys_a, index; 2: keys_a, index -> perm
    const uint32_t *k_in[3] = {keys_a, keys_b, keys_a};
    uint32_t       *k_out[3] = {keys_b, keys_a, nullptr};
    const int32_t  *i_in[3] = {nullptr, perm, index};
    int32_t        *i_out[3] = {perm, index, perm};
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * kDigitBits;
        if (pass) {
            digit_count_kernel<kRounds><<<grid, kTileBlock, 0, s>>>(k_in[pass], N, shift, counts, tiles);
            if (hipError_t e = hipGetLastError()) return cngp::record_hip_failure(e, "digit_count_kernel");
        }
        digit_row_scan_kernel<<<kDigits, kScanBlock, 0, s>>>(counts, tiles, totals);
        if (hipError_t e = hipGetLastError()) return cngp::record_hip_failure(e, "digit_row_scan_kernel");
        digit_scatter_kernel<kRounds><<<grid, kTileBlock, 0, s>>>(k_in[pass], i_in[pass], N, shift, counts, tiles, totals, k_out[pass], i_out[pass]);
        if (hipError_t e = hipGetLastError()) return cngp::record_hip_failure(e, "digit_scatter_kernel");
    }
    if (x_sorted) {
        gather_points_kernel<D><<<(unsigned)((N + kSortBlock - 1) / kSortBlock), kSortBlock, 0, s>>>(x, perm, N, x_sorted);
        if (hipError_t e = hipGetLastError()) return cngp::record_hip_failure(e, "gather_points_kernel");
    }
    return CNGP_OK;
}

}  // namespace

extern "C" {

size_t cngp_morton_sort_workspace_bytes(int32_t d, int64_t N) {
    if (d < 2 || d > 4 || N <= 0 || N > 0x7fffffffLL) return 0;
    return sort_space(N).bytes;
}

int cngp_morton_sort(int32_t d, const float *x, int64_t N, int32_t *perm, float *x_sorted,
                     void *workspace, size_t workspace_bytes, void *stream) {
    if (d < 2 || d > 4) return CNGP_ERR_INVALID;
    if (N < 0 || N > 0x7fffffffLL) return CNGP_ERR_INVALID;
    if (N == 0) return CNGP_OK;
    if (!x || !perm) return CNGP_ERR_NULL;
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < sort_space(N).bytes) return CNGP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    return d == 3 ? morton_sort<3>(x, N, perm, x_sorted, (char *)workspace, s)
         : d == 4 ? morton_sort<4>(x, N, perm, x_sorted, (char *)workspace, s)
                  : morton_sort<2>(x, N, perm, x_sorted, (char *)workspace, s);
}

}  // extern "C"
