"""Orthogonalising with operands of two fp16 numbers, on the host: what the library computes but for the order of its sums, and the same with one of a
product's three parts left out.

Inputs whose entries are all of one magnitude, with signs of rank one, in some rows and columns (how many decides the magnitude after the norm: such that X, A
and B all have low parts that count).  Then X, A and B = b A + c A A have entries of one magnitude each, low parts stand to high ones in one ratio everywhere,
and what is left out of a product comes out in that ratio, whatever the length of its sums; between random low parts it would average out.

Tolerance relative to the result (a + b + c) X, an error d of a product entering by w d with w = 1 of A (b + 2 c, over a + b + c), 2.9 of A A (c), 3.9 of
B X (b + c): a product's operands are off by 2^-23 each and low times low is below 2^-22, together 2^-21, times 7.8; fp32 sums take 16 products at a time,
roundings of 2^-24 / sqrt(3) of random signs, six times the root of their number."""
import numpy as np

COEFFICIENTS = (3.4445, -4.7750, 2.0315)
SCALES = (16384.0, 4096.0, 1024.0)        # of X, A and B


def tolerance(m, n):
    return 7.8 * 2.0 ** -21 + 6 / np.sqrt(3) * 2.0 ** -24 * np.sqrt(n / 16 + (2.9 ** 2 + 3.9 ** 2) * m / 16 + 6)


def tolerance_of(m, n, steps):
    """A second step carries the first one's error on (the slope of the polynomial at 0.701, relative: 0.72) and has smaller weights (0.86, 0.31, 1.17)."""
    return tolerance(min(m, n), max(m, n)) * (1.0 if steps == 1 else 2.0)


def low(v):
    """Share of a value that one fp16 number leaves."""
    return abs(float(v) - float(np.float16(v))) / abs(float(v))


def matrices(batch, m, n, seed):
    if m > n:
        return matrices(batch, n, m, seed).transpose(0, 2, 1).copy()
    b, c = COEFFICIENTS[1:]
    best = lambda count, score: max(range(max(1, count * 3 // 4), count + 1), key=score)
    p = best(m, lambda p: min(low(SCALES[1] / p), low((b + c) * SCALES[2] / p)))
    q = best(n, lambda q: low(SCALES[0] / np.sqrt(p * q)))
    g = np.random.default_rng(seed)
    signs = lambda count, used: np.where(g.permutation(count) < used, g.choice((-1.0, 1.0), count), 0.0)
    return np.stack([np.outer(signs(m, p), signs(n, q)) for _ in range(batch)]).astype(np.float32)


def parts(x):
    hi = x.astype(np.float16).astype(np.float64)
    return hi, (x - hi).astype(np.float16).astype(np.float64)


def wide(G):
    return G if G.shape[0] <= G.shape[1] else G.T


def step(G, without=()):
    """One step of a wide matrix in the library's parts.  without: names of what is left out, "gram", "poly" or "update" with "hl" or "lh", or "lows": one
    fp16 number to an operand."""
    a, b, c = (np.float64(np.float32(v)) for v in COEFFICIENTS)
    X0 = G.astype(np.float64)
    X0 = (X0 / np.linalg.norm(X0)).astype(np.float32).astype(np.float64)

    def product(which, p, q):
        (ph, pl), (qh, ql) = p, q
        if "lows" in without:
            return ph @ qh
        out = ph @ qh
        if which + " hl" not in without:
            out = out + ph @ ql
        if which + " lh" not in without:
            out = out + pl @ qh
        return out

    t = lambda p: (p[0].T, p[1].T)
    X = parts(X0 * SCALES[0])
    A = (product("gram", X, t(X)) * (SCALES[1] / SCALES[0] ** 2)).astype(np.float32).astype(np.float64)
    Ap = parts(A)
    whole = lambda p: p[0] + p[1]
    B = parts((b * SCALES[2] / SCALES[1] * whole(Ap) + c * SCALES[2] / SCALES[1] ** 2 * product("poly", Ap, t(Ap))).astype(np.float32).astype(np.float64))
    return a / SCALES[0] * whole(X) + product("update", B, X) / (SCALES[2] * SCALES[0])


def exact(G, steps=1):
    a, b, c = (np.float64(np.float32(v)) for v in COEFFICIENTS)
    X = G.astype(np.float64)
    X = X / np.linalg.norm(X)
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
    return X


def off_by(got, want):
    """Of the largest entry."""
    return float(np.abs(got.astype(np.float64) - want).max() / np.abs(want).max())


# how the library shares out tiles (cngp_ortho.hip): side of a tile, whether contractions are cut
def cut(back, m, n, depth, batch):
    up = lambda v: -(-v // 128) * 128
    m, n, depth = up(m), up(n), up(depth)
    count = lambda t: (m // t * (n // t) if back else m // t * (m // t + 1) // 2) * batch
    rest = count(128) % 512
    most = min(512 // rest, depth // (256 if count(128) >= 512 else 1024)) if rest else 1
    if most > 1 and count(128) - rest + rest * most >= 256:
        return 128, True
    if count(128) < 256:
        return 64, depth >= 1024 and min(max(512 // count(64), 1), depth // 256) > 1
    return 128, False


def tiles(batch, m, n):
    return dict(gram=cut(False, m, n, n, batch), poly=cut(False, m, n, m, batch), update=cut(True, m, n, m, batch))
