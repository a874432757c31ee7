// Gated linear recurrence: entry points, how a call is cut, the small kernels beside the scan (cngp_recur_scan.h).
#include <type_traits>

#include "cngp_recur.h"

using namespace cngp;

namespace {

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// The state that reaches each window, from the windows' maps: a wavefront per channel, a lane with up to 16 neighbouring windows, held in
// registers between composing them and walking them with the state.
constexpr int kCarryEach = 16, kMostWindows = 64 * kCarryEach;
__global__ __launch_bounds__(64) void recur_carry_kernel(const Cut cut, const int C)
{
    const int      lane = threadIdx.x, c = (int)blockIdx.x;
    const uint32_t per = (cut.K + 63) / 64, k0 = lane * per;
    float a[kCarryEach], b[kCarryEach];
    int   f[kCarryEach];
#pragma unroll
    for (int i = 0; i < kCarryEach; ++i) {
        const uint32_t k = k0 + i;
        const bool     there = (uint32_t)i < per && k < cut.K;
        f[i] = there ? cut.piece_cut[k] : 0;
        a[i] = there ? cut.piece_a[(size_t)k * C + c] : 1.0f;
        b[i] = there ? cut.piece_b[(size_t)k * C + c] : 0.0f;
    }
    float A = 1.0f, B = 0.0f;
    int   gone = 0;
#pragma unroll
    for (int i = 0; i < kCarryEach; ++i) {
        B = f[i] ? b[i] : fmaf(a[i], B, b[i]);
        A *= a[i];
        gone |= f[i];
    }
    const uint64_t cuts = __ballot(gone);
    const uint64_t upto = cuts & (~0ull >> (63 - lane));
    const int      since = upto ? 63 - __clzll(upto) : -1;     // last lane, up to this one, with a window that forgets
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const float Al = __shfl_up(A, d, 64), Bl = __shfl_up(B, d, 64);
        if (lane >= d && since <= lane - d) {
            B = fmaf(A, Bl, B);
            A *= Al;
        }
    }
    const float before = __shfl_up(B, 1, 64);
    float       h = lane ? before : 0.0f;                      // the first window's state is 0
#pragma unroll
    for (int i = 0; i < kCarryEach; ++i) {
        const uint32_t k = k0 + i;
        if ((uint32_t)i < per && k < cut.K) cut.carry[(size_t)k * C + c] = h;
        h = f[i] ? b[i] : fmaf(a[i], h, b[i]);
    }
}

__global__ __launch_bounds__(kRecurBlock) void recur_copy_kernel(const float *__restrict__ from, float *__restrict__ to, const int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * kRecurBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kRecurBlock) to[i] = from ? from[i] : 0.0f;
}

// dgate of a gate that all channels share, from the sums of the channel tiles.
template <typename Gate>
__global__ __launch_bounds__(kRecurBlock) void recur_slope_kernel(const RecurArgs a, const int tiles)
{
    const int64_t r = (int64_t)blockIdx.x * kRecurBlock + threadIdx.x;
    const Order   o{a.offsets, a.N, a.S, a.rows_each, false};
    if (r >= a.N || r < o.at(0) || r >= o.at(a.S)) return;
    float sum = 0.0f;
    for (int i = 0; i < tiles; ++i) sum += a.slope[(int64_t)i * a.N + r];
    store((Gate *)a.dgate, r, sum);
}

// One row to each sequence, forward: nothing to scan, h = a h0 + v value by value.  A workgroup takes kStepEach neighbouring values of the
// [N, C] array, a lane four of them at once; with one gate to a row, the rows of its values by a division in 32 bits.  64 rows of 1024 in fp16:
// 2.4 us in place of the scan's 7.0.
constexpr int kStepEach = kRecurBlock * 4;
template <typename Io, typename Gate, bool SHARED, bool LOG, bool MIX>
__global__ __launch_bounds__(kRecurBlock) void recur_step_kernel(const RecurArgs a)
{
    const int64_t  n = (int64_t)a.N * a.C, start = (int64_t)blockIdx.x * kStepEach, i0 = start + threadIdx.x * 4;
    const int64_t  row = start / a.C;                          // the same for the workgroup
    const uint32_t at = (uint32_t)(start - row * a.C) + threadIdx.x * 4;
    const auto work = [&](auto many, const int64_t i, const uint32_t at_i) {
        constexpr int M = decltype(many)::value;
        float x[M], h[M], g[M];
        load_vec<Io, M>(x, (const Io *)a.x + i);
        if (SHARED) {
#pragma unroll
            for (int v = 0; v < M; ++v) g[v] = load((const Gate *)a.gate, row + (at_i + v) / (uint32_t)a.C);
        } else {
            load_vec<Gate, M>(g, (const Gate *)a.gate + i);
        }
#pragma unroll
        for (int v = 0; v < M; ++v) h[v] = 0.0f;
        if (a.h0) load_vec<float, M>(h, a.h0 + i);
#pragma unroll
        for (int v = 0; v < M; ++v) {
            float gate, in;
            gate_of<LOG, MIX>(g[v], gate, in);
            h[v] = fmaf(gate, h[v], MIX ? in * x[v] : x[v]);
        }
        if (a.out_y) store_vec<Io, M>((Io *)a.out_y + i, h);
        if (a.last) store_vec<float, M>(a.last + i, h);
    };
    if (i0 + 4 <= n) work(std::integral_constant<int, 4>{}, i0, at);
    else for (int v = 0; i0 + v < n; ++v) work(std::integral_constant<int, 1>{}, i0 + v, at + v);
}

template <typename Io, typename Gate>
int step(const RecurArgs &a, hipStream_t s) {
    const int64_t blocks = ((int64_t)a.N * a.C + kStepEach - 1) / kStepEach;
    const bool shared = a.G == 1 && a.C > 1, log = a.flags & CNGP_RECUR_LOG_GATE, mix = a.flags & CNGP_RECUR_MIX;
    LaunchTimer t(s, K_RECUR_FWD);
#define CNGP_STEP(SHARED)                                                                                                             \
    if (log) mix ? recur_step_kernel<Io, Gate, SHARED, true, true><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a)                        \
                 : recur_step_kernel<Io, Gate, SHARED, true, false><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a);                      \
    else     mix ? recur_step_kernel<Io, Gate, SHARED, false, true><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a)                       \
                 : recur_step_kernel<Io, Gate, SHARED, false, false><<<(unsigned)blocks, kRecurBlock, 0, s>>>(a)
    if (shared) { CNGP_STEP(true); }
    else { CNGP_STEP(false); }
#undef CNGP_STEP
    return launch_status("recur_step_kernel");
}

int check(const cngp_recur_config *c, int64_t N, int64_t S, bool ragged) {
    if (!c) return CNGP_ERR_NULL;
    if (c->channels < 1 || c->channels > 65536) return CNGP_ERR_INVALID;
    if (c->gate_channels != 1 && c->gate_channels != c->channels) return CNGP_ERR_INVALID;
    if (c->io_dtype != CNGP_F32 && c->io_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->gate_dtype != CNGP_F32 && c->gate_dtype != CNGP_F16) return CNGP_ERR_INVALID;
    if (c->longest < 0) return CNGP_ERR_INVALID;
    if (c->flags & ~(uint32_t)(CNGP_RECUR_REVERSE | CNGP_RECUR_LOG_GATE | CNGP_RECUR_MIX)) return CNGP_ERR_INVALID;
    if (N < 0 || N > kMostRows || S < 0 || S > kMostRows) return CNGP_ERR_INVALID;
    if (!ragged && (S == 0 ? N != 0 : N % S != 0)) return CNGP_ERR_INVALID;
    return CNGP_OK;
}

RecurArgs args_of(const cngp_recur_config *c, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t S, const float *h0) {
    RecurArgs a{};
    a.gate = gate; a.x = x; a.offsets = offsets; a.h0 = h0;
    a.N = (pos)N; a.S = (pos)S; a.rows_each = (pos)(S ? N / S : 0);
    a.C = c->channels; a.G = c->gate_channels; a.flags = c->flags;
    return a;
}

// How a call is cut.  CL lanes side by side hold V channels each: as many as there are channels, at most 32 (a row of a tile is then a
// 128-byte line of fp32).  Eight lanes in place of sixteen for 5 to 8 channels: 45306 sequences of 10 rows of 8 fp16, forward and backward
// with the states computed again, 91 and 121 us; 40000 with 400000 rows of 5 fp32 74 and 112.
constexpr int64_t kEnoughGroups = 2048;               // workgroups that fill the chip's 256 CUs with eight each

RecurPlan plan_of(const cngp_recur_config *c, int64_t N, int64_t S, bool ragged) {
    RecurPlan p{};
    const int C = c->channels;
    p.CL = C <= 4 ? 1 : C <= 8 ? 8 : C <= 16 ? 16 : 32;
    p.V = C <= 4 ? C : C > 32 && C % 2 == 0 ? 2 : 1;
    p.block = p.CL == 1 ? kNarrowBlock : kRecurBlock;
    p.tiles = (C + p.CL * p.V - 1) / (p.CL * p.V);
    const int64_t tile_rows = p.CL == 1 ? kNarrowBlock * kRowsNarrow : p.block / p.CL * kRowsEach;
    const int64_t mean = S ? (N + S - 1) / S : 0;
    // Ragged ones are of unknown length here (the offsets lie on the device).  Cutting wherever one might be long costs ordinary batches two
    // launches; a single long sequence among short ones that is not known of costs 280 times what it takes cut (2^20 rows of three channels).
    const int64_t longest = !ragged ? mean : c->longest ? std::min<int64_t>(c->longest, N) : 4 * mean;
    // windows that give every CU eight workgroups, of whole tiles; single wavefronts four times as many (a frame of 1920 x 1080 rays with 8192 of
    // them 102.6 us, 4096 114, 16384 105)
    const int64_t enough = kEnoughGroups * (kRecurBlock / std::min(p.block, kRecurBlock));
    int64_t       R = (N * p.tiles + enough - 1) / enough;
    R = std::max<int64_t>((R + tile_rows - 1) / tile_rows * tile_rows, tile_rows);
    // sequences that are no longer than a few windows stay whole: one launch, every input read once.  Longer ones are cut
    // (a tile after the other takes 1.5 to 2 us; the two launches more of a cut sequence take what a dozen tiles do)
    p.exact = longest > std::max(4 * R, 12 * tile_rows);
    if (p.exact && p.V == 2 && !ragged && S * ((C + 31) / 32) >= 192) {
        // enough sequences by channels to give most CUs one of 32 channels, walked by eight wavefronts: whole after all
        p.CL = 16;
        p.block = kWideBlock;
        p.tiles = (C + 31) / 32;
        p.exact = false;
        R = mean;
    }
    if (p.exact) R = std::max(R, ((N + kMostWindows - 1) / kMostWindows + tile_rows - 1) / tile_rows * tile_rows);
    else if (!ragged) R = std::max<int64_t>((R + mean / 2) / std::max<int64_t>(mean, 1), 1) * mean;
    // a window's last sequence reaches over its edge: room for it in the window's tiles, but no more windows than twice as many (16.7 M rows in
    // sequences of about 1023, all but 2 rows of a window taken off: 1092 us, this 129; 2^18 rows in sequences of 127: 36 and 8.3)
    else if (2 * mean < R) R = std::max(R - 2 * mean, R / 2);
    p.R = std::max<int64_t>(R, 1);
    p.K = (uint32_t)std::max<int64_t>((N + p.R - 1) / p.R, 1);
    return p;
}

// Where the backward pass has the states from, a factor of the gates' gradient (less x, with mixed inputs: what rounding them to fp16 takes
// off is relative to the states, not to that difference).  Kept ones serve as they are in fp32.  In fp16 a launch computes them again:
// into the workspace; or, with fp16 gates, only what their rounding took off, into dx, whose rows are overwritten after they were read, so
// that the call needs no workspace (8 sequences of 4096 rows of 1024: 162 us, 61 + 101; by the 134 MB workspace 160, 70 + 90).  Not so for rows that a
// wavefront computes again by itself (up to four channels), nor for cut sequences, whose last row in a window has its state in the next one.
int states_of(const cngp_recur_config *c, const RecurPlan &p, bool given) {
    if (given && c->io_dtype == CNGP_F32) return STATES_Y;
    return given && c->gate_dtype == CNGP_F16 && p.CL > 1 && !p.exact ? STATES_LOW : STATES_F32;
}

RecurSpace space_of(const cngp_recur_config *c, const RecurPlan &p, int64_t N, int64_t S, uint32_t call) {
    RecurSpace s{};
    size_t at = 0;
    auto take = [&](bool wanted, size_t bytes) { const size_t o = at; if (wanted) at += align256(bytes); return o; };
    const size_t C = (size_t)c->channels;
    const bool   bwd = call & CNGP_RECUR_CALL_BWD;
    s.y = take(bwd && states_of(c, p, !(call & CNGP_RECUR_CALL_NO_Y)) == STATES_F32, (size_t)N * C * 4);
    s.slope = take(bwd && c->gate_channels == 1 && p.tiles > 1, (size_t)N * (size_t)p.tiles * 4);
    s.piece_a = take(p.exact, p.K * C * 4);
    s.piece_b = take(p.exact, p.K * C * 4);
    s.carry = take(p.exact, p.K * C * 4);
    s.piece_cut = take(p.exact, p.K * 4);
    s.state = take(p.exact, (size_t)S * C * 4);
    s.bytes = at;
    return s;
}

}  // namespace

int cngp::recur_copy(const float *from, float *to, int64_t n, hipStream_t s) {
    LaunchTimer t(s, K_RECUR_CARRY);
    recur_copy_kernel<<<(unsigned)std::min<int64_t>((n + kRecurBlock - 1) / kRecurBlock, kMostGroups256), kRecurBlock, 0, s>>>(from, to, n);
    return launch_status("recur_copy_kernel");
}

int cngp::recur_carry(const Cut &cut, int C, hipStream_t s) {
    LaunchTimer t(s, K_RECUR_CARRY);
    recur_carry_kernel<<<(unsigned)C, 64, 0, s>>>(cut, C);
    return launch_status("recur_carry_kernel");
}

namespace {
int pass_states(const float *in, float *out, int64_t n, hipStream_t s) {      // no rows at all
    if (!out || in == out || n == 0) return CNGP_OK;
    return recur_copy(in, out, n, s);
}

}  // namespace

extern "C" {

size_t cngp_recur_workspace_bytes(const cngp_recur_config *cfg, int64_t N, int64_t sequences, uint32_t call) {
    if (check(cfg, N, sequences, call & CNGP_RECUR_CALL_RAGGED)) return 0;
    return space_of(cfg, plan_of(cfg, N, sequences, call & CNGP_RECUR_CALL_RAGGED), N, sequences, call).bytes;
}

int cngp_recur_fwd(const cngp_recur_config *cfg, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t sequences,
                   const float *h0, void *y, float *last, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N, sequences, offsets != nullptr)) return rc;
    if (sequences == 0) return CNGP_OK;
    if (N && (!gate || !x || (!last && !y))) return CNGP_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    if (N == 0) return pass_states(h0, last, sequences * cfg->channels, s);
    const RecurPlan  p = plan_of(cfg, N, sequences, offsets != nullptr);
    const RecurSpace sp = space_of(cfg, p, N, sequences, offsets ? CNGP_RECUR_CALL_RAGGED : 0);
    if (sp.bytes && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < sp.bytes)) return CNGP_ERR_WORKSPACE;
    RecurArgs a = args_of(cfg, gate, x, N, offsets, sequences, h0);
    a.out_y = y; a.last = last;
    if (!offsets && N == sequences && (N * cfg->channels + kStepEach - 1) / kStepEach <= kMostGroups256) {      // 2^34 values; above by the scan
        const bool io16 = cfg->io_dtype == CNGP_F16, g16 = cfg->gate_dtype == CNGP_F16;
        return io16 ? (g16 ? step<__half, __half>(a, s) : step<__half, float>(a, s)) : (g16 ? step<float, __half>(a, s) : step<float, float>(a, s));
    }
    return recur_launch<false>(cfg, a, p, sp, (char *)workspace, s);
}

int cngp_recur_bwd(const cngp_recur_config *cfg, const void *gate, const void *x, int64_t N, const int32_t *offsets, int64_t sequences,
                   const float *h0, const void *y, const void *dy, const float *dlast, void *dgate, void *dx, float *dh0,
                   void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = check(cfg, N, sequences, offsets != nullptr)) return rc;
    if (sequences == 0) return CNGP_OK;
    if (N && (!gate || !x || !dgate || !dx || (!dy && !dlast))) return CNGP_ERR_NULL;
    hipStream_t s = (hipStream_t)stream;
    if (N == 0) return pass_states(dlast, dh0, sequences * cfg->channels, s);
    const RecurPlan  p = plan_of(cfg, N, sequences, offsets != nullptr);
    const uint32_t   call = CNGP_RECUR_CALL_BWD | (offsets ? CNGP_RECUR_CALL_RAGGED : 0) | (y ? 0 : CNGP_RECUR_CALL_NO_Y);
    const RecurSpace sp = space_of(cfg, p, N, sequences, call);
    char            *ws = (char *)workspace;
    if (sp.bytes && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < sp.bytes)) return CNGP_ERR_WORKSPACE;
    RecurArgs a = args_of(cfg, gate, x, N, offsets, sequences, h0);
    a.states = states_of(cfg, p, y != nullptr);
    a.y = y;
    if (a.states != STATES_Y) {
        a.out_y = a.states == STATES_LOW ? dx : ws + sp.y;
        if (a.states == STATES_F32) a.y = a.out_y;
        if (p.CL > 1 || p.exact) {                             // else the backward launch computes them (recur_narrow_again_kernel)
            if (int rc = recur_launch<false>(cfg, a, p, sp, ws, s)) return rc;
            a.out_y = nullptr;
        }
    }
    a.dy = dy; a.dlast = dlast; a.dgate = dgate; a.dx = dx; a.dh0 = dh0;
    const bool sums = cfg->gate_channels == 1 && p.tiles > 1;
    a.slope = sums ? (float *)(ws + sp.slope) : nullptr;
    if (int rc = recur_launch<true>(cfg, a, p, sp, ws, s)) return rc;
    if (!sums) return CNGP_OK;
    LaunchTimer t(s, K_RECUR_BWD);
    const unsigned blocks = (unsigned)((N + kRecurBlock - 1) / kRecurBlock);
    if (cfg->gate_dtype == CNGP_F16) recur_slope_kernel<__half><<<blocks, kRecurBlock, 0, s>>>(a, p.tiles);
    else recur_slope_kernel<float><<<blocks, kRecurBlock, 0, s>>>(a, p.tiles);
    return launch_status("recur_slope_kernel");
}

}  // extern "C"
