"""Linear attention with decays, norms with rotation and orthogonalised updates in 64 bits, with the error that the library's arithmetic may make.

Attention row by row: S_t = e^{g_t} S_{t-1} + k_t v_t^T, y_t = scale S_t^T q_t, backward by the transposed recurrence.  The magnitudes next to
every result are the same recurrences over absolute values; every rounding is u = 2^-24 of a magnitude, so an error is at most
rounds * u * magnitude with, per result: a product over key_dim and one over value_dim (as many roundings as terms), 128 for the rows of a chunk
(scores and state), 2 for every chunk a state passes through, 160 for the decays (an exponent below 110 rounded to fp32 and taken as a power of
two: 110 * 1.45), 16 for two fp16 numbers in place of one value (2^-22 each, twice, for both factors), 32 for the rest."""
import numpy as np

U = 2.0 ** -24


def half_step(dtype):
    return 2.0 ** -11 if dtype == np.float16 else U


def smallest(dtype):
    return 2.0 ** -25 if dtype == np.float16 else 2.0 ** -140


def spans(N, S, offsets):
    if offsets is None:
        return [(s * (N // S), (s + 1) * (N // S)) for s in range(S)]
    o = np.clip(np.asarray(offsets, np.int64), 0, N)
    return [(int(o[s]), max(int(o[s]), int(o[s + 1]))) for s in range(len(o) - 1)]


def rounds(dk, dv, longest):
    return dk + dv + 128 + 2 * (longest // 64 + 1) + 160 + 16 + 32


def attend(q, k, v, g, spans_, h0, scale, dy=None, dlast=None):
    """All results in a dict; q [N, H, dk], k [N, K, dk], v [N, K, dv], g [N, H]; h0, dlast [S, H, dk, dv] or None."""
    N, H, dk = q.shape
    K, dv = v.shape[1], v.shape[2]
    G, S = H // K, len(spans_)
    kk, vv = np.repeat(k, G, 1), np.repeat(v, G, 1)
    e = np.exp(g)
    y, last = np.zeros((N, H, dv)), np.zeros((S, H, dk, dv))
    out = dict(dq=np.zeros((N, H, dk)), dk=np.zeros((N, H, dk)), dv=np.zeros((N, H, dv)), dg=np.zeros((N, H)), dh0=np.zeros((S, H, dk, dv)))
    for s, (lo, hi) in enumerate(spans_):
        st = np.zeros((H, dk, dv)) if h0 is None else h0[s].copy()
        states = [st]
        for r in range(lo, hi):
            st = e[r][:, None, None] * st + kk[r][:, :, None] * vv[r][:, None, :]
            states.append(st)
            y[r] = scale * np.einsum("hkv,hk->hv", st, q[r])
        last[s] = st
        if dy is not None or dlast is not None:
            d = np.zeros((H, dk, dv)) if dlast is None else dlast[s].copy()
            for r in range(hi - 1, lo - 1, -1):
                st = states[r - lo + 1]
                if dy is not None:
                    out["dq"][r] = scale * np.einsum("hkv,hv->hk", st, dy[r])
                    d = d + scale * q[r][:, :, None] * dy[r][:, None, :]
                out["dk"][r] = np.einsum("hkv,hv->hk", d, vv[r])
                out["dv"][r] = np.einsum("hkv,hk->hv", d, kk[r])
                d = e[r][:, None, None] * d
                out["dg"][r] = (d * states[r - lo]).sum((1, 2))
            out["dh0"][s] = d
    out["dk"] = out["dk"].reshape(N, K, G, dk).sum(2)
    out["dv"] = out["dv"].reshape(N, K, G, dv).sum(2)
    return dict(out, y=y, last=last)


def attend_bounds(q, k, v, g, spans_, h0, scale, dy=None, dlast=None):
    """Magnitude times roundings for every result of attend()."""
    a = lambda t: None if t is None else np.abs(t)
    m = attend(a(q), a(k), a(v), g, spans_, a(h0), abs(scale), a(dy), a(dlast))
    longest = max([hi - lo for lo, hi in spans_] + [1])
    c = rounds(q.shape[2], v.shape[2], longest) * U
    G = q.shape[1] // k.shape[1]
    b = {n: t * (c + G * U) for n, t in m.items()}
    # The gradient of a row's decay is put together from sums over its 64 rows and the product of two states up to 16 chunks away: what
    # is rounded are those, not the result.  The largest of them in the stretch; products of q and dq, k and dk include the row's own.
    near = (np.abs(q) * m["dq"]).sum(2) + (np.repeat(np.abs(k) * m["dk"], G, 1).sum(2))
    for s, (lo, hi) in enumerate(spans_):
        for h in range(q.shape[1]):
            top = (np.abs(h0[s, h]) * m["dh0"][s, h]).sum() if h0 is not None else 0.0
            b["dg"][lo:hi, h] = c * 3 * (m["dg"][lo:hi, h].max(initial=0.0) + top + near[lo:hi, h].sum())
    return b


def within(name, got, want, bound, dtype=np.float32):
    slack = bound + half_step(dtype) * (np.abs(want) + bound) + smallest(dtype)
    off = np.abs(got.astype(np.float64) - want)
    bad = ~(off <= slack)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} outside, worst {np.nanmax(off / slack):.3g} x the bound at {np.argwhere(bad)[0]}"


def turn(x, angle, nxt, sign=1.0):
    """Pairs of the last dimension turned; angle [N, pairs]."""
    p = angle.shape[1]
    c, s = np.cos(angle)[:, None], sign * np.sin(angle)[:, None]
    out = x.copy()
    a, b = (x[..., 0:2 * p:2], x[..., 1:2 * p:2]) if nxt else (x[..., :p], x[..., p:2 * p])
    if nxt:
        out[..., 0:2 * p:2], out[..., 1:2 * p:2] = a * c - b * s, a * s + b * c
    else:
        out[..., :p], out[..., p:2 * p] = a * c - b * s, a * s + b * c
    return out


def rotate(x, angle, nxt, gamma, eps, norm, du=None):
    """(y, dx, dgamma) of one of the two arrays [N, heads, dim] in 64 bits."""
    if not norm:
        return turn(x, angle, nxt), None if du is None else turn(du, angle, nxt, -1.0), None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    hat = x * r
    y = turn(hat * gamma, angle, nxt)
    if du is None:
        return y, None, None
    u = turn(du, angle, nxt, -1.0)
    w = u * gamma
    return y, r * (w - hat * (w * hat).mean(-1, keepdims=True)), (u * hat).sum((0, 1))


def orthogonalise(g, steps, coefficients, eps):
    a, b, c = coefficients
    out = []
    for m in g:
        x = m / (np.linalg.norm(m) + eps)
        if m.shape[0] > m.shape[1]:
            x = x.T
        for _ in range(steps):
            A = x @ x.T
            x = a * x + (b * A + c * A @ A) @ x
        out.append(x.T if m.shape[0] > m.shape[1] else x)
    return np.stack(out)
