"""The gradient of linear attention's decays in 64 bits as the library puts it together, and how far fp32 sums may be from it.

Row t's is what reaches over it, g_t = <state before row t, its gradient there>, and g_{t+1} = g_t + k_t . dk_t - q_t . dq_t.  In chunks of 64 rows, counted from the
sequence's start: g at both ends of a chunk from the states there (0 before a sequence without a first state, and behind one whose last is not used), rows between by
the products, what is left over at the end taken off evenly.

Errors: every number here is a sum of products of inputs, and a rounding is u = 2^-24 of what is rounded, of either sign.  The same recurrences over squares
give the sum of the squares of all products: roundings of random signs add up as the root of it.  Roundings to a product: 24 for the operands in
two parts (three factors, off by 2 u each, as squares), a quarter of key_dim + value_dim + 64 (a matrix instruction takes 16 products, at most four roundings), 6 for
each chunk that a state passes, 64 for the decays (exponents rounded to fp32: two of 8 u relative, as squares halved).  Six times the root of
that many is the bound: a result is off by less unless roundings conspire.  A row takes errors from its chunk alone, no part of them more than once."""
import numpy as np

import mixer_ref as R

CHUNK = 64


def heads_of(q, k, v):
    G = q.shape[1] // k.shape[1]
    return np.repeat(k, G, 1), np.repeat(v, G, 1)


def assembled(q, k, v, g, spans, h0, scale, dy, dlast, lost=()):
    """The gradient [N, heads] by the formula above.  lost: numbers of chunks at whose starts g is taken for 0, "end" for behind the last row."""
    N, H, dk = q.shape
    k, v = heads_of(q, k, v)
    dv = v.shape[2]
    e = np.exp(g)
    out = np.zeros((N, H))
    all_ = R.attend(q, k, v, g, spans, h0, scale, dy, dlast)
    step = (k * all_["dk"]).sum(2) - (q * all_["dq"]).sum(2)
    for s, (lo, hi) in enumerate(spans):
        if lo == hi:
            continue
        states, st = [], np.zeros((H, dk, dv)) if h0 is None else h0[s].copy()
        for r in range(lo, hi):
            if (r - lo) % CHUNK == 0:
                states.append(st)
            st = e[r][:, None, None] * st + k[r][:, :, None] * v[r][:, None, :]
        d = np.zeros((H, dk, dv)) if dlast is None else dlast[s].copy()
        known = {"end": (st * d).sum((1, 2))}
        for r in range(hi - 1, lo - 1, -1):
            if dy is not None:
                d = d + scale * q[r][:, :, None] * dy[r][:, None, :]
            d = e[r][:, None, None] * d
            if (r - lo) % CHUNK == 0:
                known[(r - lo) // CHUNK] = (states[(r - lo) // CHUNK] * d).sum((1, 2))
        known = {n: t * (n not in lost) for n, t in known.items()}
        for c, a in enumerate(range(lo, hi, CHUNK)):
            z = min(a + CHUNK, hi)
            upto = np.cumsum(step[a:z], 0)
            rest = known[c + 1 if z < hi else "end"] - known[c] - upto[-1]
            out[a:z] = known[c] + upto - step[a:z] + rest * (np.arange(z - a) / (z - a))[:, None]
    return out


def bounds(q, k, v, g, spans, h0, scale, dy, dlast):
    """(of each row's gradient [N, heads], of the sum over all rows [heads])."""
    N, H, dk = q.shape
    k, v = heads_of(q, k, v)
    sq = lambda t: None if t is None else t * t
    m = R.attend(sq(q), sq(k), sq(v), 2 * g, spans, sq(h0), scale * scale, sq(dy), sq(dlast))
    own = 0.0 if dy is None else scale * scale * (sq(q) * sq(k)).sum(2) * (sq(v) * sq(dy)).sum(2)
    each = np.maximum((sq(q) * m["dq"]).sum(2) + (sq(k) * m["dk"]).sum(2) - 2 * own, 0.0)
    b, total = np.zeros((N, H)), np.zeros(H)
    for s, (lo, hi) in enumerate(spans):
        n = 24 + (dk + v.shape[2] + CHUNK) / 4 + 6 * ((hi - lo) // CHUNK + 1) + 64
        behind = np.zeros(H) if dlast is None else (m["last"][s] * sq(dlast[s])).sum((1, 2))
        for a in range(lo, hi, CHUNK):
            z = min(a + CHUNK, hi)
            ends, products = m["dg"][a] + (m["dg"][z] if z < hi else behind), each[a:z].sum(0)                      # m["dg"][a]: squares of g there
            b[a:z] = 6 * R.U * np.sqrt(n * (ends + products))
            # summed up: an end's error falls to nothing over the chunk at either side of it, a product's weighs by its distance from the chunk's middle
            total += (6 * R.U * (z - a)) ** 2 * n * (ends / 2 + products / 12)
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
