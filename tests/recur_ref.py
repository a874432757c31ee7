"""The gated linear recurrence and its gradient in 64 bits, row by row, with the error that fp32 arithmetic may make.

`bound` next to every result: the recurrence of the magnitudes m_t = |a| m_{t-1} + |v| carries a rounding error of at most
c u m_t per row (u = 2^-24: the gate's exponential, one product, one sum), and errors travel through the gates like the state,
E_t = |a| E_{t-1} + c u m_t.  A product of k gates that a piece of a sequence is joined with has k roundings, and the k rows it
spans put k c u m into E: any way of cutting the sequence stays inside.  c = 8: two for the exponential, one for 1 - a, one for
the product, one for the sum, doubled for a piece that is scanned twice."""
import numpy as np

U, C_ROUND = 2.0 ** -24, 8.0


def half_step(dtype):
    return 2.0 ** -11 if dtype == np.float16 else 0.0


def spans(N, S, offsets):
    if offsets is None:
        return [(s * (N // S), (s + 1) * (N // S)) for s in range(S)]
    o = np.clip(np.asarray(offsets, np.int64), 0, N)
    return [(int(o[s]), max(int(o[s]), int(o[s + 1]))) for s in range(len(o) - 1)]


def forward(gate, x, spans_, h0, reverse, log_gate, mix):
    """{y, last and their bounds}; gate [N, G], x [N, C] in 64 bits."""
    N, C = x.shape
    a = np.exp(gate) if log_gate else gate
    share = (-np.expm1(gate) if log_gate else 1.0 - gate) if mix else np.ones_like(a)
    y, Ey, M = (np.zeros((N, C)) for _ in range(3))
    last, El = np.zeros((len(spans_), C)), np.zeros((len(spans_), C))
    for s, (lo, hi) in enumerate(spans_):
        h = np.zeros(C) if h0 is None else h0[s].astype(np.float64)
        m, e = np.abs(h), np.zeros(C)
        for r in (range(hi - 1, lo - 1, -1) if reverse else range(lo, hi)):
            v = share[r] * x[r]
            # 1 - a from a rounded exponential or gate is exact to u of 1 (log gates: of itself)
            m = np.abs(a[r]) * m + np.abs(v) + (0.0 if log_gate or not mix else 0.25 * np.abs(x[r]))
            e = np.abs(a[r]) * e + C_ROUND * U * m
            h = a[r] * h + v
            y[r], Ey[r], M[r] = h, e, m
        last[s], El[s] = h, e
    return dict(y=y, Ey=Ey, M=M, last=last, El=El, a=a, share=share)


def backward(gate, x, spans_, h0, dy, dlast, reverse, log_gate, mix, y_rounding=0.0):
    N, C = x.shape
    f = forward(gate, x, spans_, h0, reverse, log_gate, mix)
    a, share = f["a"], f["share"]
    G = gate.shape[1]
    dx, Ex, slope, Es, mags = (np.zeros((N, C)) for _ in range(5))
    dh0, E0 = np.zeros((len(spans_), C)), np.zeros((len(spans_), C))
    for s, (lo, hi) in enumerate(spans_):
        start = np.zeros(C) if h0 is None else h0[s].astype(np.float64)
        u = np.zeros(C) if dlast is None else dlast[s].astype(np.float64)
        mu, eu = np.abs(u), np.zeros(C)
        rows = list(range(hi - 1, lo - 1, -1) if reverse else range(lo, hi))
        for i in range(len(rows) - 1, -1, -1):
            r = rows[i]
            prev = f["y"][rows[i - 1]] if i else start
            eprev = f["Ey"][rows[i - 1]] + y_rounding * np.abs(prev) + (2.0 ** -25 if y_rounding else 0.0) if i else np.zeros(C)
            dh = u + (0.0 if dy is None else dy[r])
            md = mu + (0.0 if dy is None else np.abs(dy[r]))
            ed = eu + C_ROUND * U * md
            k = a[r] if log_gate else np.ones(G)
            left = prev - x[r] if mix else prev
            mleft = np.abs(prev) + (np.abs(x[r]) if mix else 0.0)
            slope[r] = dh * left * k
            mags[r] = md * mleft * np.abs(k)
            Es[r] = (ed * mleft + md * eprev) * np.abs(k) + C_ROUND * U * mags[r]
            dx[r] = share[r] * dh
            Ex[r] = np.abs(share[r]) * ed + C_ROUND * U * md * (np.abs(share[r]) + (0.25 if mix and not log_gate else 0.0))
            u = a[r] * dh
            mu = np.abs(a[r]) * md
            eu = np.abs(a[r]) * ed + C_ROUND * U * mu
        dh0[s], E0[s] = u, eu
    if G == 1 and C > 1:      # the sum over channels: C more roundings of the magnitudes
        dgate = slope.sum(1, keepdims=True)
        Eg = (Es + C * U * mags).sum(1, keepdims=True)
    else:
        dgate, Eg = slope, Es
    return dict(dgate=dgate, Eg=Eg, dx=dx, Ex=Ex, dh0=dh0, E0=E0, **{k: f[k] for k in ("y", "Ey", "last", "El")})


def within(name, got, want, bound, dtype=np.float32):
    """got (as float64) within the bound and the rounding to its storage type (half a step; fp16 has a smallest step of 2^-24)."""
    slack = bound + half_step(dtype) * (np.abs(want) + bound) + (2.0 ** -25 if dtype == np.float16 else 2.0 ** -140)
    off = np.abs(got - want)
    bad = ~(off <= slack)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} outside, worst {np.nanmax(off / slack):.3g} x the bound at {np.argwhere(bad)[0]}"
