// Stable radix sort of (32-bit key, index) pairs, 7 bits per pass, written for 64-lane wavefronts: the kernels that the sort of the
// points by Morton code and the sort of the ids of a lookup share.  cngp_sort.hip describes a pass.
#pragma once
#include <cstdint>

#include <hip/hip_runtime.h>

namespace {

constexpr int kDigitBits = 7;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kTileBlock = 512;          // 8 wavefronts per tile
constexpr int kTileWaves = kTileBlock / 64;
constexpr int kRounds = 16;              // elements per lane, where a batch fills the chip with such tiles
constexpr int kTile = kTileBlock * kRounds;
constexpr int kScanBlock = 1024;

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int64_t tiles_of(int64_t N) { return (N + kTile - 1) / kTile; }

// Sum of a tile's per-wavefront histograms, written as column `tile` of counts[digit][tiles], or with PREFIX as row `tile` of
// counts[tiles][digit] (what digit_scatter_kernel adds up itself).
template <bool PREFIX = false>
__device__ __forceinline__ void flush_tile_histogram(const uint32_t *hist, uint32_t *__restrict__ counts,
                                                     const int64_t tiles, const int64_t tile, const int t)
{
    if (t < kDigits) {
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < kTileWaves; ++w) sum += hist[w * kDigits + t];
        counts[PREFIX ? (size_t)tile * kDigits + (size_t)t : (size_t)t * (size_t)tiles + (size_t)tile] = sum;
    }
}

template <int ROUNDS, bool PREFIX = false>
__global__ __launch_bounds__(kTileBlock) void digit_count_kernel(const uint32_t *__restrict__ keys, const int64_t N, const int shift,
                                                                 uint32_t *__restrict__ counts, const int64_t tiles)
{
    __shared__ uint32_t hist[kTileWaves * kDigits];
    const int     t = threadIdx.x, w = t >> 6;
    const int64_t n0 = (int64_t)blockIdx.x * (kTileBlock * ROUNDS);
    for (int i = t; i < kTileWaves * kDigits; i += kTileBlock) hist[i] = 0;
    __syncthreads();
    uint32_t key[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t n = n0 + (int64_t)r * kTileBlock + t;
        key[r] = n < N ? keys[n] : 0u;
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t n = n0 + (int64_t)r * kTileBlock + t;
        if (n < N) atomicAdd(&hist[w * kDigits + ((key[r] >> shift) & (kDigits - 1))], 1u);
    }
    __syncthreads();
    flush_tile_histogram<PREFIX>(hist, counts, tiles, blockIdx.x, t);
}

// Exclusive prefix of v over the 64 lanes of a wavefront; *total = the sum.
__device__ __forceinline__ uint32_t wave_exclusive_scan(const uint32_t v, uint32_t *total)
{
    const int lane = threadIdx.x & 63;
    uint32_t  inc = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(inc, o, 64);
        if (lane >= o) inc += up;
    }
    *total = __shfl(inc, 63, 64);
    return inc - v;
}

// Row `digit` of counts[digit][tiles] -> its exclusive prefix over the tiles, in place; totals[digit] = the row's sum.
__global__ __launch_bounds__(kScanBlock) void digit_row_scan_kernel(uint32_t *__restrict__ counts, const int64_t tiles,
                                                                    uint32_t *__restrict__ totals)
{
    __shared__ uint32_t wave_sum[kScanBlock / 64];
    uint32_t *row = counts + (size_t)blockIdx.x * (size_t)tiles;
    const int t = threadIdx.x, w = t >> 6, lane = t & 63;
    uint32_t  carry = 0;
    for (int64_t base = 0; base < tiles; base += kScanBlock) {
        const int64_t  i = base + t;
        const uint32_t v = i < tiles ? row[i] : 0u;
        uint32_t       wtotal;
        const uint32_t in_wave = wave_exclusive_scan(v, &wtotal);
        if (lane == 0) wave_sum[w] = wtotal;
        __syncthreads();
        uint32_t before = 0, all = 0;
#pragma unroll
        for (int k = 0; k < kScanBlock / 64; ++k) {
            const uint32_t s = wave_sum[k];
            before += k < w ? s : 0u;
            all += s;
        }
        if (i < tiles) row[i] = carry + before + in_wave;
        carry += all;
        __syncthreads();
    }
    if (t == 0) totals[blockIdx.x] = carry;
}

// One pass of the sort for one tile.  keys_in in the order of the previous pass; index_in NULL = the identity
// (first pass).  keys_out NULL on the last pass (nobody reads them).  Element n of the input goes to
//   sum of totals of smaller digits + counts[digit][tile] (prefix over earlier tiles) + its rank inside the tile.
// PREFIX, for up to kPrefixTiles tiles: `counts` holds the tiles' own counts, whose prefix every workgroup adds up itself (`totals` is not read):
// a launch less per pass.
constexpr int kPrefixTiles = 128;
template <int ROUNDS, bool PREFIX = false>
__global__ __launch_bounds__(kTileBlock) void digit_scatter_kernel(
    const uint32_t *__restrict__ keys_in, const int32_t *__restrict__ index_in, const int64_t N, const int shift,
    const uint32_t *__restrict__ counts, const int64_t tiles, const uint32_t *__restrict__ totals,
    uint32_t *__restrict__ keys_out, int32_t *__restrict__ index_out)
{
    __shared__ uint32_t wave_count[kTileWaves * kDigits];   // per wavefront and digit: running count, then base inside the digit's run
    __shared__ uint32_t tile_start[kDigits];                // first slot of the digit in the sorted tile
    __shared__ uint32_t dest[kDigits];                      // global position of that slot
    __shared__ uint32_t stage[kTileBlock * ROUNDS];          // the tile in sorted order: first its keys, then its indices
    __shared__ uint32_t carry[2];
    const int     t = threadIdx.x, w = t >> 6, lane = t & 63;
    const int64_t tile = blockIdx.x;
    constexpr int TILE = kTileBlock * ROUNDS;
    const int64_t n0 = tile * TILE;
    const int     tile_n = (int)((N - n0 < TILE) ? N - n0 : TILE);
    uint32_t     *mine = wave_count + w * kDigits;
    for (int i = t; i < kTileWaves * kDigits; i += kTileBlock) wave_count[i] = 0;
    uint32_t part_all = 0, part_before = 0;                 // PREFIX: lane t adds every fourth tile's count of digit t mod 128
    if constexpr (PREFIX) {
#pragma unroll 8
        for (int64_t i = t >> kDigitBits; i < tiles; i += kTileBlock / kDigits) {
            const uint32_t c = counts[(size_t)i * kDigits + (size_t)(t & (kDigits - 1))];
            part_all += c;
            part_before += i < tile ? c : 0u;
        }
    }
    __syncthreads();

    // rank of every element among the equal digits before it in this wavefront's eighth of the tile
    uint32_t key[ROUNDS], rank[ROUNDS];
    int32_t  index[ROUNDS];
    const int64_t  w0 = n0 + (int64_t)w * (ROUNDS * 64);
    const uint64_t below = lane ? (~0ull >> (64 - lane)) : 0ull;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t n = w0 + r * 64 + lane;
        key[r] = n < N ? keys_in[n] : 0u;
        index[r] = n < N ? (index_in ? index_in[n] : (int32_t)n) : 0;
    }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t  n = w0 + r * 64 + lane;
        const bool     valid = n < N;
        const uint32_t digit = (key[r] >> shift) & (kDigits - 1);
        uint64_t       peers = __ballot(valid);
#pragma unroll
        for (int b = 0; b < kDigitBits; ++b) {
            const bool     bit = (digit >> b) & 1u;
            const uint64_t has = __ballot(bit);
            peers &= bit ? has : ~has;
        }
        rank[r] = 0;
        if (valid) {
            const uint32_t seen = mine[digit];                        // same address for all peers: one broadcast read
            rank[r] = seen + (uint32_t)__popcll(peers & below);
            if ((peers & below) == 0) mine[digit] = seen + (uint32_t)__popcll(peers);   // the first peer moves the count on
        }
        __builtin_amdgcn_wave_barrier();                              // the next round's read stays behind this write
    }
    __syncthreads();

    // per digit: counts of the wavefronts -> bases inside the digit's run; runs laid end to end; global targets
    uint32_t count = 0, total = 0;
    if (t < kDigits) {                                                 // wavefronts 0 and 1 hold the 128 digits
#pragma unroll
        for (int k = 0; k < kTileWaves; ++k) {
            const uint32_t c = wave_count[k * kDigits + t];
            wave_count[k * kDigits + t] = count;
            count += c;
        }
        if constexpr (!PREFIX) total = totals[t];
    }
    uint32_t earlier = 0;                                   // the digit's elements in earlier tiles
    if constexpr (PREFIX) {
        __syncthreads();
        stage[t] = part_all;
        stage[kTileBlock + t] = part_before;
        __syncthreads();
        if (t < kDigits) {
#pragma unroll
            for (int k = 0; k < kTileBlock / kDigits; ++k) { total += stage[k * kDigits + t]; earlier += stage[kTileBlock + k * kDigits + t]; }
        }
    } else if (t < kDigits) {
        earlier = counts[(size_t)t * (size_t)tiles + (size_t)tile];
    }
    uint32_t       count_sum, total_sum;
    const uint32_t count_before = wave_exclusive_scan(count, &count_sum);
    const uint32_t total_before = wave_exclusive_scan(total, &total_sum);
    if (t == 0) { carry[0] = count_sum; carry[1] = total_sum; }        // digits 0..63, for wavefront 1
    __syncthreads();
    if (t < kDigits) {
        tile_start[t] = (w ? carry[0] : 0u) + count_before;
        dest[t] = (w ? carry[1] : 0u) + total_before + earlier;
    }
    __syncthreads();

    // keys: into LDS in sorted order (rank[] becomes the slot), out in runs of consecutive addresses;
    // slot j of the sorted tile is element (j - tile_start[digit]) of its digit's run
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t  n = w0 + r * 64 + lane;
        const uint32_t digit = (key[r] >> shift) & (kDigits - 1);
        rank[r] = n < N ? tile_start[digit] + mine[digit] + rank[r] : (uint32_t)TILE;
        if (rank[r] < (uint32_t)TILE) stage[rank[r]] = key[r];
    }
    __syncthreads();
    uint32_t to[ROUNDS];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
        const int j = t + i * kTileBlock;
        to[i] = 0xffffffffu;
        if (j < tile_n) {
            const uint32_t k = stage[j];
            const uint32_t digit = (k >> shift) & (kDigits - 1);
            to[i] = dest[digit] + ((uint32_t)j - tile_start[digit]);
            if (keys_out && (int64_t)to[i] < N) keys_out[to[i]] = k;
        }
    }
    __syncthreads();
    // indices: the same way through the same buffer
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if (rank[r] < (uint32_t)TILE) stage[rank[r]] = (uint32_t)index[r];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
        const int j = t + i * kTileBlock;
        if (j < tile_n && (int64_t)to[i] < N) index_out[to[i]] = (int32_t)stage[j];
    }
}

}  // namespace
