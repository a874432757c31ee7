// Lookup of codes with scaling, and its gradient by sorted ids.
//
//     y[n] = base[n] + scale * table[ids[n]]          grad[r] += scale * sum over n with ids[n] == r of dy[n]
//
// The gradient needs, per row of the table, the points that chose it.  Float atomics would give sums whose order, hence bits, change
// from call to call, and frequent ids would queue at one address; so the ids are sorted (stable, with their positions), and the rows
// of dy that belong to one id are added up in the order of the points.
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

template <typename Id, typename Table, typename Io>
__global__ __launch_bounds__(kEmbBlock) void embed_fwd_kernel(const Id *__restrict__ ids, const Table *__restrict__ table, const Io *base, Io *y,
                                                              const int64_t N, const int64_t rows, const int dim, const float scale)
{
    const int64_t i = (int64_t)blockIdx.x * kEmbBlock + threadIdx.x;
    if (i >= N * dim) return;
    const int64_t  n = i / dim;
    const uint32_t r = row_of(ids[n], rows);
    const float    b = base ? load(base, i) : 0.0f;
    store(y, i, (int64_t)r < rows ? b + scale * load(table, (int64_t)r * dim + (i - n * dim)) : b);
}

template <typename Id>
__global__ __launch_bounds__(kEmbBlock) void embed_keys_kernel(const Id *__restrict__ ids, uint32_t *__restrict__ keys, const int64_t N, const int64_t rows)
{
    const int64_t n = (int64_t)blockIdx.x * kEmbBlock + threadIdx.x;
    if (n < N) keys[n] = row_of(ids[n], rows);
}

// First position of the sorted keys that is not below `key`.
__device__ __forceinline__ int64_t first_at(const uint32_t *__restrict__ keys, const int64_t N, const uint32_t key) {
    int64_t lo = 0, hi = N;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (keys[mid] < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// A wavefront per row of the table.
template <typename Io>
__global__ __launch_bounds__(kEmbBlock) void embed_sums_kernel(const uint32_t *__restrict__ keys, const int32_t *__restrict__ from,
                                                               const Io *__restrict__ dy, float *__restrict__ grad, const int64_t N,
                                                               const int64_t rows, const int dim, const float scale, const int accumulate)
{
    const int64_t r = ((int64_t)blockIdx.x * kEmbBlock + threadIdx.x) >> 6;
    if (r >= rows) return;
    const int64_t p0 = first_at(keys, N, (uint32_t)r), p1 = first_at(keys, N, (uint32_t)r + 1u);
    if (p0 == p1 && accumulate) return;
    for (int c = threadIdx.x & 63; c < dim; c += 64) {
        float sum = 0.0f;
        for (int64_t p = p0; p < p1; ++p) sum += load(dy, (int64_t)from[p] * dim + c);
        const int64_t o = r * dim + c;
        grad[o] = accumulate ? grad[o] + scale * sum : scale * sum;
    }
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

struct EmbedSpace { size_t keys_a, keys_b, from_a, from_b, counts, totals, bytes; };
EmbedSpace space_of(int64_t N) {
    EmbedSpace s{};
    const size_t col = align256((size_t)N * 4);
    s.keys_a = 0; s.keys_b = col; s.from_a = 2 * col; s.from_b = 3 * col;
    s.counts = 4 * col;
    s.totals = s.counts + align256((size_t)kDigits * (size_t)tiles_of(N) * 4);
    s.bytes = N ? s.totals + align256((size_t)kDigits * 4) : 0;
    return s;
}

}  // namespace

extern "C" {

size_t cngp_embed_workspace_bytes(const cngp_embed_config *cfg, int64_t N) {
    return check(cfg, N) ? 0 : space_of(N).bytes;
}

int cngp_embed_fwd(const cngp_embed_config *cfg, const void *ids, int64_t N, const void *table, const void *base, void *y, void *stream) {
    if (int rc = check(cfg, N)) return rc;
    if (N == 0) return CNGP_OK;
    if (!ids || !table || !y) return CNGP_ERR_NULL;
    const int64_t blocks = (N * cfg->dim + kEmbBlock - 1) / kEmbBlock;
    if (blocks > 0x7fffffffLL) return CNGP_ERR_INVALID;
    hipStream_t s = (hipStream_t)stream;
    LaunchTimer t(s, K_EMBED_FWD);
#define CNGP_EMBED(Id, Table, Io) embed_fwd_kernel<Id, Table, Io><<<(unsigned)blocks, kEmbBlock, 0, s>>>( \
        (const Id *)ids, (const Table *)table, (const Io *)base, (Io *)y, N, cfg->rows, cfg->dim, cfg->scale)
    switch (cfg->id_dtype * 4 + cfg->table_dtype * 2 + cfg->io_dtype) {
    case 0: CNGP_EMBED(int32_t, float, float); break;
    case 1: CNGP_EMBED(int32_t, float, __half); break;
    case 2: CNGP_EMBED(int32_t, __half, float); break;
    case 3: CNGP_EMBED(int32_t, __half, __half); break;
    case 4: CNGP_EMBED(int64_t, float, float); break;
    case 5: CNGP_EMBED(int64_t, float, __half); break;
    case 6: CNGP_EMBED(int64_t, __half, float); break;
    default: CNGP_EMBED(int64_t, __half, __half); break;
    }
#undef CNGP_EMBED
    return launch_status("embed_fwd_kernel");
}

int cngp_embed_bwd(const cngp_embed_config *cfg, const void *ids, int64_t N, const void *dy, float *grad_table,
                   void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N)) return rc;
    if (!grad_table) return CNGP_ERR_NULL;
    const int accumulate = (cfg->flags & CNGP_ZERO_GRADS) ? 0 : 1;
    if (N == 0 && accumulate) return CNGP_OK;
    if (N && (!ids || !dy)) return CNGP_ERR_NULL;
    const EmbedSpace sp = space_of(N);
    if (sp.bytes && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < sp.bytes)) return CNGP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    char     *ws = (char *)workspace;
    uint32_t *keys[2] = {(uint32_t *)(ws + sp.keys_a), (uint32_t *)(ws + sp.keys_b)};
    int32_t  *from[2] = {(int32_t *)(ws + sp.from_a), (int32_t *)(ws + sp.from_b)};
    uint32_t *counts = (uint32_t *)(ws + sp.counts), *totals = (uint32_t *)(ws + sp.totals);
    int       at = 0;
    if (N) {
        LaunchTimer t(s, K_EMBED_SORT);
        const unsigned lanes = (unsigned)((N + kEmbBlock - 1) / kEmbBlock), tiles = (unsigned)tiles_of(N);
        if (cfg->id_dtype == CNGP_I32) embed_keys_kernel<int32_t><<<lanes, kEmbBlock, 0, s>>>((const int32_t *)ids, keys[0], N, cfg->rows);
        else embed_keys_kernel<int64_t><<<lanes, kEmbBlock, 0, s>>>((const int64_t *)ids, keys[0], N, cfg->rows);
        if (int rc = launch_status("embed_keys_kernel")) return rc;
        bool first = true;
        for (int shift = 0; shift < 32 && ((uint64_t)cfg->rows >> shift); shift += kDigitBits, at ^= 1, first = false) {
            digit_count_kernel<<<tiles, kTileBlock, 0, s>>>(keys[at], N, shift, counts, tiles);
            if (int rc = launch_status("digit_count_kernel")) return rc;
            digit_row_scan_kernel<<<kDigits, kScanBlock, 0, s>>>(counts, tiles, totals);
            if (int rc = launch_status("digit_row_scan_kernel")) return rc;
            digit_scatter_kernel<<<tiles, kTileBlock, 0, s>>>(keys[at], first ? nullptr : from[at], N, shift, counts, tiles, totals, keys[at ^ 1], from[at ^ 1]);
            if (int rc = launch_status("digit_scatter_kernel")) return rc;
        }
    }
    LaunchTimer t(s, K_EMBED_SUMS);
    const unsigned blocks = (unsigned)((cfg->rows + kEmbBlock / 64 - 1) / (kEmbBlock / 64));
    if (cfg->io_dtype == CNGP_F16)
        embed_sums_kernel<__half><<<blocks, kEmbBlock, 0, s>>>(keys[at], from[at], (const __half *)dy, grad_table, N, cfg->rows, cfg->dim, cfg->scale, accumulate);
    else
        embed_sums_kernel<float><<<blocks, kEmbBlock, 0, s>>>(keys[at], from[at], (const float *)dy, grad_table, N, cfg->rows, cfg->dim, cfg->scale, accumulate);
    return launch_status("embed_sums_kernel");
}

}  // extern "C"
