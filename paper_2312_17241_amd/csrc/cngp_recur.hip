// Gated linear recurrence h_t = a_t h_{t-1} + v_t over the rows of sequences, and its gradient.
//
//     dh_t = dy_t + a_{t+1} dh_{t+1} (+ dlast at the last row)      dx = dh, or (1 - a) dh with mixed inputs
//     da_t = dh_t (h_{t-1} [- x_t])     log gates: times a_t        dh0 = a_0 dh_0
#include <algorithm>
#include <cstdint>

#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "cngp_launch.h"

namespace {

using namespace cngp;

constexpr int kRecurBlock = 256;

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct RecurArgs {
    const void    *gate, *x;
    const int32_t *offsets;
    const float   *h0, *dlast;
    const void    *y, *dy;               // backward; y_f32: y is the workspace's fp32 copy
    void          *out_y, *dgate, *dx;
    float         *last, *dh0;
    float         *slope;                // backward of a gate shared by the channels: dL/dgate per channel, fp32 [N, C]
    int64_t        N, S, rows_each;
    int32_t        C, G;
    uint32_t       flags;
    int32_t        y_f32;
};

__device__ __forceinline__ float load(const float *p, const int64_t i) { return p[i]; }
__device__ __forceinline__ float load(const __half *p, const int64_t i) { return __half2float(p[i]); }
__device__ __forceinline__ void store(float *p, const int64_t i, const float v) { p[i] = v; }
__device__ __forceinline__ void store(__half *p, const int64_t i, const float v) { p[i] = __float2half_rn(v); }

// Rows [lo, hi) of sequence s, inside [0, N) whatever the offsets hold.
__device__ __forceinline__ void bounds(const RecurArgs &a, const int64_t s, int64_t &lo, int64_t &hi) {
    if (!a.offsets) { lo = s * a.rows_each; hi = lo + a.rows_each; return; }
    const int64_t p = a.offsets[s], q = a.offsets[s + 1];
    lo = p < 0 ? 0 : p > a.N ? a.N : p;
    hi = q < lo ? lo : q > a.N ? a.N : q;
}

// The gate of a row and how much of the input it lets in.
__device__ __forceinline__ void gate_of(const uint32_t flags, const float g, float &a, float &in) {
    a = flags & CNGP_RECUR_LOG_GATE ? expf(g) : g;
    in = !(flags & CNGP_RECUR_MIX) ? 1.0f : flags & CNGP_RECUR_LOG_GATE ? -expm1f(g) : 1.0f - g;
}

// One lane per sequence and channel.
template <typename Io, typename Gate, typename Y>
__global__ __launch_bounds__(kRecurBlock) void recur_fwd_kernel(const RecurArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * kRecurBlock + threadIdx.x;
    if (i >= a.S * a.C) return;
    const int64_t s = i / a.C;
    const int     c = (int)(i - s * a.C);
    int64_t lo, hi;
    bounds(a, s, lo, hi);
    float h = a.h0 ? a.h0[i] : 0.0f;
    for (int64_t k = lo; k < hi; ++k) {
        const int64_t r = a.flags & CNGP_RECUR_REVERSE ? lo + hi - 1 - k : k;
        float gate, in;
        gate_of(a.flags, load((const Gate *)a.gate, a.G == 1 ? r : r * a.C + c), gate, in);
        h = gate * h + in * load((const Io *)a.x, r * a.C + c);
        if (a.out_y) store((Y *)a.out_y, r * a.C + c, h);
    }
    if (a.last) a.last[i] = h;
}

template <typename Io, typename Gate>
__global__ __launch_bounds__(kRecurBlock) void recur_bwd_kernel(const RecurArgs a)
{
    const int64_t i = (int64_t)blockIdx.x * kRecurBlock + threadIdx.x;
    if (i >= a.S * a.C) return;
    const int64_t s = i / a.C;
    const int     c = (int)(i - s * a.C);
    int64_t lo, hi;
    bounds(a, s, lo, hi);
    const bool    rev = a.flags & CNGP_RECUR_REVERSE;
    float         u = a.dlast ? a.dlast[i] : 0.0f;           // what reaches the state after the row
    for (int64_t k = lo; k < hi; ++k) {
        const int64_t r = rev ? k : lo + hi - 1 - k, e = r * a.C + c, prev = rev ? r + 1 : r - 1;
        float gate, in;
        gate_of(a.flags, load((const Gate *)a.gate, a.G == 1 ? r : e), gate, in);
        const bool  inner = k + 1 < hi;
        const float before = !inner ? (a.h0 ? a.h0[i] : 0.0f)
                             : a.y_f32 ? ((const float *)a.y)[prev * a.C + c] : load((const Io *)a.y, prev * a.C + c);
        const float dh = u + (a.dy ? load((const Io *)a.dy, e) : 0.0f);
        float       da = dh * (a.flags & CNGP_RECUR_MIX ? before - load((const Io *)a.x, e) : before);
        if (a.flags & CNGP_RECUR_LOG_GATE) da *= gate;
        if (a.slope) a.slope[e] = da;
        else store((Gate *)a.dgate, e, da);
        store((Io *)a.dx, e, in * dh);
        u = gate * dh;
    }
    if (a.dh0) a.dh0[i] = u;
}

// dgate of a gate that all channels share: the sum over a row's channels.  A wavefront per row.
template <typename Gate>
__global__ __launch_bounds__(kRecurBlock) void recur_slope_kernel(const RecurArgs a)
{
    const int64_t r = ((int64_t)blockIdx.x * kRecurBlock + threadIdx.x) >> 6;
    int64_t lo = 0, hi = a.N, unused;
    if (a.offsets) { bounds(a, 0, lo, unused); bounds(a, a.S - 1, unused, hi); }
    if (r < lo || r >= hi) return;
    float sum = 0.0f;
    for (int c = threadIdx.x & 63; c < a.C; c += 64) sum += a.slope[r * a.C + c];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
    if ((threadIdx.x & 63) == 0) store((Gate *)a.dgate, r, sum);
}

int check(const cngp_recur_config *c, int64_t N, int64_t S, bool ragged) {
    if (!c) return CNGP_ERR_NULL;
    if (c->channels < 1 || c->channels > 65536) return CNGP_ERR_INVALID;
    if (c->gate_channels != 1 && c->gate_channels != c->channels) return CNGP_ERR_INVALID;
    if (c->io_dtype != CNGP_F32 && c->io_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->gate_dtype != CNGP_F32 && c->gate_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->longest < 0) return CNGP_ERR_INVALID;
    if (c->flags & ~(uint32_t)(CNGP_RECUR_REVERSE | CNGP_RECUR_LOG_GATE | CNGP_RECUR_MIX)) return CNGP_ERR_INVALID;
    if (N < 0 || N > 0x7fffffffLL || S < 0 || S > 0x7ffffffeLL) return CNGP_ERR_INVALID;
    if (!ragged && (S == 0 ? N != 0 : N % S != 0)) return CNGP_ERR_INVALID;
    return CNGP_OK;
}

RecurArgs args_of(const cngp_recur_config *c, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t S, const float *h0) {
    RecurArgs a{};
    a.gate = gate; a.x = x; a.offsets = offsets; a.h0 = h0;
    a.N = N; a.S = S; a.rows_each = S ? N / S : 0;
    a.C = c->channels; a.G = c->gate_channels; a.flags = c->flags;
    return a;
}

// Where the parts of a workspace lie.
struct RecurSpace { size_t y, slope, bytes; };
RecurSpace space_of(const cngp_recur_config *c, int64_t N, uint32_t call) {
    RecurSpace s{};
    const size_t rows = align256((size_t)N * (size_t)c->channels * 4);
    if (!(call & CNGP_RECUR_CALL_BWD)) return s;
    s.y = 0;
    s.slope = call & CNGP_RECUR_CALL_NO_Y ? rows : 0;
    s.bytes = s.slope + (c->gate_channels != c->channels ? rows : 0);
    return s;
}

int launch_fwd(const cngp_recur_config *c, const RecurArgs &a, bool y_f32, hipStream_t s) {
    const int64_t blocks = (a.S * a.C + kRecurBlock - 1) / kRecurBlock;
    if (blocks > 0x7fffffffLL) return CNGP_ERR_INVALID;
    LaunchTimer t(s, K_RECUR_FWD);
    const bool io16 = c->io_dtype == CNGP_F16, g16 = c->gate_dtype == CNGP_F16;
#define CNGP_RECUR(Io, Gate) \
    if (y_f32) recur_fwd_kernel<Io, Gate, float><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a); \
    else       recur_fwd_kernel<Io, Gate, Io><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a)
    if (io16 && g16) { CNGP_RECUR(__half, __half); } else if (io16) { CNGP_RECUR(__half, float); }
    else if (g16) { CNGP_RECUR(float, __half); } else { CNGP_RECUR(float, float); }
#undef CNGP_RECUR
    return launch_status("recur_fwd_kernel");
}

}  // namespace

extern "C" {

size_t cngp_recur_workspace_bytes(const cngp_recur_config *cfg, int64_t N, int64_t sequences, uint32_t call) {
    if (check(cfg, N, sequences, call & CNGP_RECUR_CALL_RAGGED)) return 0;
    return space_of(cfg, N, call).bytes;
}

int cngp_recur_fwd(const cngp_recur_config *cfg, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t sequences,
                   const float *h0, void *y, float *last, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N, sequences, offsets != nullptr)) return rc;
    if (sequences == 0) return CNGP_OK;
    if (N && (!gate || !x)) return CNGP_ERR_NULL;
    if (!last && !y) return N ? CNGP_ERR_NULL : CNGP_OK;
    (void)workspace; (void)workspace_bytes;
    RecurArgs a = args_of(cfg, gate, x, N, offsets, sequences, h0);
    a.out_y = y; a.last = last;
    return launch_fwd(cfg, a, false, (hipStream_t)stream);
}

int cngp_recur_bwd(const cngp_recur_config *cfg, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t sequences,
                   const float *h0, const void *y, const void *dy, const float *dlast, void *dgate, void *dx, float *dh0,
                   void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N, sequences, offsets != nullptr)) return rc;
    if (sequences == 0) return CNGP_OK;
    if (N && (!gate || !x || !dgate || !dx || (!dy && !dlast))) return CNGP_ERR_NULL;
    const uint32_t   call = CNGP_RECUR_CALL_BWD | (offsets ? CNGP_RECUR_CALL_RAGGED : 0) | (y ? 0 : CNGP_RECUR_CALL_NO_Y);
    const RecurSpace sp = space_of(cfg, N, call);
    if (sp.bytes && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < sp.bytes)) return CNGP_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    RecurArgs a = args_of(cfg, gate, x, N, offsets, sequences, h0);
    if (!y && N) {
        a.out_y = (char *)workspace + sp.y;
        if (int rc = launch_fwd(cfg, a, true, s)) return rc;
        a.y = a.out_y;
        a.y_f32 = 1;
    } else {
        a.y = y;
    }
    a.dy = dy; a.dlast = dlast; a.dgate = dgate; a.dx = dx; a.dh0 = dh0;
    const bool shared = cfg->gate_channels != cfg->channels;
    a.slope = shared ? (float *)((char *)workspace + sp.slope) : nullptr;
    const int64_t blocks = (a.S * a.C + kRecurBlock - 1) / kRecurBlock;
    if (blocks > 0x7fffffffLL) return CNGP_ERR_INVALID;
    const bool io16 = cfg->io_dtype == CNGP_F16, g16 = cfg->gate_dtype == CNGP_F16;
    {
        LaunchTimer t(s, K_RECUR_BWD);
        if (io16 && g16) recur_bwd_kernel<__half, __half><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a);
        else if (io16) recur_bwd_kernel<__half, float><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a);
        else if (g16) recur_bwd_kernel<float, __half><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a);
        else recur_bwd_kernel<float, float><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a);
        if (int rc = launch_status("recur_bwd_kernel")) return rc;
    }
    if (!shared || !N) return CNGP_OK;
    LaunchTimer t(s, K_RECUR_BWD);
    const int64_t sums = (N + kRecurBlock / 64 - 1) / (kRecurBlock / 64);
    if (g16) recur_slope_kernel<__half><<<(unsigned)sums, kRecurBlock, 0, s>>>(a);
    else recur_slope_kernel<float><<<(unsigned)sums, kRecurBlock, 0, s>>>(a);
    return launch_status("recur_slope_kernel");
}

}  // extern "C"
