"""The gradient of linear attention's decays in 64 bits as the library puts it together, and how far fp32 sums may be from it.

Row t's is what reaches over it: with near = the products of a row inside its chunk of 64 (its own with itself left out), far = those with states, D = <state,
gradient of the state> at the start of a stretch of 1024 rows, counted from the sequence's start,
    sum over its chunk's rows s >= t of (q.dq near - k.dk near + q.dq far) + sum over s < t of k.dk far + what crosses the whole chunk,
the last D with k.dk far - q.dq far of the stretch's rows before added, less the chunk's q.dq far.

Errors: every number here is a sum of products of inputs, and a rounding is u = 2^-24 of what is rounded, of either sign.  The same recurrences over squares
give the sum of the squares of all products: roundings of random signs add up as the root of it.  Roundings to a product: 24 for the operands in
two parts (three factors, off by 2 u each, as squares), a quarter of key_dim + value_dim + 64 (a matrix instruction takes 16 products, at most four roundings), 6 for
each chunk that a state passes, 64 for the decays (exponents rounded to fp32: two of 8 u relative, as squares halved).  Six times the root of
that many is the bound: a result is off by less unless roundings conspire."""
import numpy as np

import mixer_ref as R

CHUNK, STRETCH = 64, 1024


def heads_of(q, k, v):
    G = q.shape[1] // k.shape[1]
    return np.repeat(k, G, 1), np.repeat(v, G, 1)


def assembled(q, k, v, g, spans, h0, scale, dy, dlast, without_D=None, carried=True):
    """The gradient [N, heads] by the formula above.  without_D: number of the stretch whose D is left out; carried: whether D goes on from chunk to chunk."""
    N, H, dk = q.shape
    k, v = heads_of(q, k, v)
    dv = v.shape[2]
    e = np.exp(np.maximum(g, -700.0))
    dg = np.zeros((N, H))
    for s, (lo, hi) in enumerate(spans):
        starts = list(range(lo, hi, CHUNK))
        before, st = [], np.zeros((H, dk, dv)) if h0 is None else h0[s].copy()
        for r in range(lo, hi):
            if (r - lo) % CHUNK == 0:
                before.append(st)
            st = e[r][:, None, None] * st + k[r][:, :, None] * v[r][:, None, :]
        behind, d = {}, np.zeros((H, dk, dv)) if dlast is None else dlast[s].copy()
        for r in range(hi - 1, lo - 1, -1):
            if r == hi - 1 or (r + 1 - lo) % CHUNK == 0:
                behind[(r - lo) // CHUNK] = d
            if dy is not None:
                d = d + scale * q[r][:, :, None] * dy[r][:, None, :]
            d = e[r][:, None, None] * d
            if (r - lo) % CHUNK == 0:
                behind["start", (r - lo) // CHUNK] = d
        D = None
        for c, a in enumerate(starts):
            rows = slice(a, min(a + CHUNK, hi))
            F = np.cumsum(np.maximum(g[rows], -700.0), 0)                            # [rows, H]
            n = F.shape[0]
            W = np.zeros((n, n, H))                                                   # products of rows t > s
            if dy is not None:
                W = scale * np.einsum("thk,shk->tsh", q[rows], k[rows]) * np.einsum("thv,shv->tsh", dy[rows], v[rows]) * \
                    np.where(np.tril(np.ones((n, n)), -1)[:, :, None] > 0, np.exp(np.minimum(F[:, None] - F[None], 0.0)), 0.0)
            near = W.sum(1) - W.sum(0)
            qf = np.zeros((n, H)) if dy is None else scale * np.exp(F) * np.einsum("thk,hkv,thv->th", q[rows], before[c], dy[rows])
            kf = np.exp(F[-1] - F) * np.einsum("thk,hkv,thv->th", k[rows], behind[c], v[rows])
            if (c * CHUNK) % STRETCH == 0:
                D = (before[c] * behind["start", c]).sum((1, 2)) * (0.0 if without_D == c * CHUNK // STRETCH else 1.0)
            T = D - qf.sum(0)
            dg[rows] = np.cumsum((near + qf)[::-1], 0)[::-1] + np.cumsum(kf, 0) - kf + T
            if carried:
                D = T + kf.sum(0)
    return dg


def bounds(q, k, v, g, spans, h0, scale, dy, dlast):
    """(of each row's gradient [N, heads], of the sum over all rows [heads])."""
    N, H, dk = q.shape
    k, v = heads_of(q, k, v)
    sq = lambda t: None if t is None else t * t
    m = R.attend(sq(q), sq(k), sq(v), 2 * g, spans, sq(h0), scale * scale, sq(dy), sq(dlast))
    own = 0.0 if dy is None else scale * scale * (sq(q) * sq(k)).sum(2) * (sq(v) * sq(dy)).sum(2)
    each = np.maximum((sq(q) * m["dq"]).sum(2) + (sq(k) * m["dk"]).sum(2) - 2 * own, 0.0)
    b, total = np.zeros((N, H)), np.zeros(H)
    for lo, hi in spans:
        n = 24 + (dk + v.shape[2] + CHUNK) / 4 + 6 * ((hi - lo) // CHUNK + 1) + 64
        for a in range(lo, hi, STRETCH):
            z = min(a + STRETCH, hi)
            b[a:z] = 6 * R.U * np.sqrt(n * (m["dg"][a] + each[a:z].sum(0)))           # m["dg"][a]: squares of D, from before the row
            total += ((z - a) * b[a]) ** 2                                            # a stretch's rows share their errors
    return b, np.sqrt(total)


def inputs(lengths, H, K, dk, dv, rows, seed, slow, half=False, lead=0, trail=0):
    """(q, k, v, decay [N, H] or [H], h0, dy, dlast, offsets) as 64-bit arrays of numbers that the library's types hold."""
    g = np.random.default_rng(seed)
    S, N = len(lengths), lead + sum(lengths) + trail
    decay = -np.log1p(np.exp(g.normal(size=(N, H) if rows else (H,)) * 1.5 - (7 if slow else 3)))
    if rows:
        decay[g.random((N, H)) < 0.001] = -np.inf
    held = lambda t, dtype: t.astype(dtype).astype(np.float64)
    io = np.float16 if half else np.float32
    shapes = ((N, H, dk), io), ((N, K, dk), io), ((N, K, dv), io), ((S, H, dk, dv), np.float32), ((N, H, dv), io), ((S, H, dk, dv), np.float32)
    q, k, v, h0, dy, dlast = (held(g.normal(size=shape), dtype) for shape, dtype in shapes)
    return q, k, v, held(decay, np.float32), h0, dy, dlast, np.concatenate([[lead], lead + np.cumsum(lengths)]).astype(np.int32)
