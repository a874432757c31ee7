"""Operators around the encoding as cases that can be timed and compared: the gated linear recurrence that composites the samples of
a ray (and scans any sequence of rows), the lookup of per-image codes with its gradient, and the balance loss of the probing
confidences.  Every case has a plain form in elementary torch operations and the package's own calls (`own`).

A case is a dict of plain values: `path` names the calls (see run), the rest are sizes and types.  Sizes are those of workloads.py
(4096 rays of 64 samples, 32 encoded columns, 16 levels of 2^14 confidence rows ...) or generic ones of sequence models; ragged and
odd ones stand for batches that no power of two decides.
"""
import functools
import math

import torch

own = False

_TORCH = {"f16": torch.float16, "f32": torch.float32, "i32": torch.int32, "i64": torch.int64}
_BYTES = {"f16": 2, "f32": 4, "i32": 4, "i64": 8}


def _recur(name, path, S, N, C, shared, io, gate, ragged, form, keep):
    """path: "recur" (forward) or "recur_train" (forward and backward); form: "rays" (log gates, mixed inputs, back to front) or "plain";
    keep: whether the states of all rows are an output, or only the last ones."""
    c = dict(path=path, S=S, N=N, C=C, shared=shared, io=io, gate=gate, ragged=ragged, form=form, keep=keep)
    return dict(c, name=name) if name else c


def _embed(name, path, N, rows, dim, table, io, ids, base, hot):
    """path: "embed" (lookup) or "embed_train" (lookup and gradient); hot: how the ids are spread, "rays" (64 samples of a ray share one),
    "zipf" or "even"."""
    c = dict(path=path, N=N, rows=rows, dim=dim, table=table, io=io, ids=ids, base=base, hot=hot)
    return dict(c, name=name) if name else c


def _balance(name, L, N_c, N_p, top_k, masked):
    c = dict(path="balance", L=L, N_c=N_c, N_p=N_p, top_k=top_k, masked=masked)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new row for each of 64 running sequences: a single step of a recurrent layer while serving
        _recur("recur_step", "recur", 64, 64, 1024, False, "f16", "f16", False, "plain", True),
        # training a radiance field: 4096 rays of 64 samples each on average (an occupancy grid has dropped some, a few rays have none)
        _recur("rays_train", "recur_train", 4096, 2**18, 3, True, "f32", "f32", True, "rays", False),
        # compositing a 1920 x 1080 frame, eight samples to a ray on average
        _recur("rays_frame", "recur", 1920 * 1080, 8 * 1920 * 1080, 3, True, "f32", "f32", True, "rays", False),
        # a recurrent layer in training: 8 sequences of 4096 rows, a gate for every channel, everything fp16
        _recur("recur_layer", "recur_train", 8, 8 * 4096, 1024, False, "f16", "f16", False, "plain", True),
        # one long odd sequence of few channels, fp32: there are too few rows of work to fill the chip without cutting the sequence
        _recur("recur_long", "recur_train", 1, 100003, 96, False, "f32", "f32", False, "plain", True),
        # the code of one image added to the encodings of an interactive query
        _embed("code_query", "embed", 1001, 100, 32, "f32", "f16", "i32", True, "even"),
        # training with a code per image: 100 images, the 64 samples of a ray share the code
        _embed("code_train", "embed_train", 2**18, 100, 32, "f32", "f16", "i32", True, "rays"),
        # token embedding of a batch: frequent and rare ids, wide rows, scaled by the root of the width
        _embed("token_train", "embed_train", 16381, 50000, 1024, "f16", "f16", "i64", False, "zipf"),
        # a code for every ray of a large capture, more rows than a chip's caches hold
        _embed("wide_train", "embed_train", 1000003, 2**20, 64, "f32", "f32", "i32", False, "even"),
        # balance of the smallest model's probing confidences
        _balance("balance_tiny2d", 4, 2**8, 4, 0, False),
        # ... of the headline model's
        _balance("balance_nerf3d", 16, 2**14, 16, 0, False),
        # ... of large index codebooks, the sparse backward, rows that the batch did not touch left out
        _balance("balance_large", 16, 2**18, 16, 4, True),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    path = rng.choice(("recur", "recur_train", "recur_train", "embed", "embed_train", "embed_train", "balance"))
    if path.startswith("recur"):
        form = rng.choice(("rays", "plain", "plain"))
        C = rng.choice((1, 2, 3, 3, 4, 8)) if form == "rays" else _log(rng, 1, 2048)
        N = _log(rng, 64, min(2**24, 2**25 // C))
        S = min(N, rng.choice((1, _log(rng, 1, N), _log(rng, 1, N), N)))
        ragged = rng.random() < 0.5
        N = N if ragged else N // S * S
        return _recur(None, path, S, N, C, form == "rays" or rng.random() < 0.2, rng.choice(("f16", "f32")), rng.choice(("f16", "f32")), ragged,
                      form, form == "plain" or rng.random() < 0.3)
    if path.startswith("embed"):
        dim = _log(rng, 1, 2048)
        N, rows = _log(rng, 1, min(2**20, 2**26 // dim)), _log(rng, 1, min(2**20, 2**26 // dim))
        return _embed(None, path, N, rows, dim, rng.choice(("f16", "f32")), rng.choice(("f16", "f32")), rng.choice(("i32", "i64")),
                      rng.random() < 0.5, rng.choice(("rays", "zipf", "even")))
    N_p = 1 << rng.randint(1, 4)
    return _balance(None, rng.randint(1, 16), 1 << rng.randint(0, 18), N_p, rng.choice((0, 0, rng.randint(1, N_p))), rng.random() < 0.5)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")
    s = dict(case=dict(c))
    if c["path"].startswith("recur"):
        S, N, C, G = c["S"], c["N"], c["C"], 1 if c["shared"] else c["C"]
        s["offsets"] = None
        if c["ragged"]:            # lengths that scatter around their mean, a few sequences empty; some rows behind the last sequence
            used = N - min(N // 16, 7)
            cuts = torch.randint(0, used + 1, (S - 1,), generator=g, device="cuda").sort().values
            s["offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), used)]).int()
        if c["form"] == "rays":    # optical depths of samples: free space mostly, then a surface; the background behind it
            gate = -torch.relu(randn(N, G) * 0.4 - 0.2)
        else:                      # gates of a trained layer: most of them close to one
            gate = torch.sigmoid(randn(N, G) * 1.5 + 3.0)
        s["gate"] = gate.to(_TORCH[c["gate"]])
        s["x"] = (rand(N, C) if c["form"] == "rays" else randn(N, C) * 0.1).to(_TORCH[c["io"]])
        s["h0"] = randn(S, C) * 0.3
        if c["path"] == "recur_train":
            s["dy"] = randn(N, C).to(_TORCH[c["io"]]) if c["keep"] else None
            s["dlast"] = randn(S, C)
        return s
    if c["path"].startswith("embed"):
        N, rows, dim = c["N"], c["rows"], c["dim"]
        if c["hot"] == "rays":
            ids = torch.randint(0, rows, ((N + 63) // 64, 1), generator=g, device="cuda").expand(-1, 64).reshape(-1)[:N]
        elif c["hot"] == "zipf":   # frequencies that fall with the rank, ranks spread over the table
            ids = (torch.exp(rand(N) * math.log(rows + 1.0)) - 1.0).long().clamp(0, rows - 1) * 7919 % rows
        else:
            ids = torch.randint(0, rows, (N,), generator=g, device="cuda")
        s["ids"] = torch.where(rand(N) < 0.01, -1, ids).to(_TORCH[c["ids"]]).contiguous()      # one in a hundred is padding
        s["table"] = (randn(rows, dim) * 0.1).to(_TORCH[c["table"]])
        s["base"] = (randn(N, dim) * 0.1).to(_TORCH[c["io"]]) if c["base"] else None
        if c["path"] == "embed_train":
            s["dy"] = randn(N, dim).to(_TORCH[c["io"]])
        return s
    L, N_c, N_p = c["L"], c["N_c"], c["N_p"]
    s["Dhat"] = randn(L, N_c, N_p) + randn(L, 1, N_p) * 0.3
    s["rows"] = (rand(L, N_c) < 0.7).to(torch.uint8) if c["masked"] else None
    s["weight"] = 0.01
    return s


def _scale(c):
    return math.sqrt(c["dim"]) if c["hot"] == "zipf" else 0.5


@functools.lru_cache(maxsize=64)
def _config(kind, *values):
    """The package's description of an operator, which a program keeps."""
    import paper_2312_17241_amd as cngp
    dtype = {"f16": cngp.F16, "f32": cngp.F32, "i32": cngp.I32, "i64": cngp.I64}
    if kind == "recur":
        C, G, io, gate, rays = values
        flags = cngp.RECUR_LOG_GATE | cngp.RECUR_MIX | cngp.RECUR_REVERSE if rays else 0
        return cngp.RecurConfig(channels=C, gate_channels=G, io_dtype=dtype[io], gate_dtype=dtype[gate], flags=flags)
    if kind == "embed":
        rows, dim, table, io, ids, scale = values
        return cngp.EmbedConfig(rows=rows, dim=dim, table_dtype=dtype[table], io_dtype=dtype[io], id_dtype=dtype[ids], scale=scale,
                                flags=cngp.ZERO_GRADS)
    L, N_c, N_p, top_k = values
    return cngp.Config(d=3, L=L, F=2, N_f=2**16, N_c=N_c, N_p=N_p, N_min=16, N_max=2048, top_k=top_k, flags=cngp.ZERO_GRADS)


def _run_own(s):
    import paper_2312_17241_amd as cngp
    c = s["case"]
    if c["path"].startswith("recur"):
        cfg = _config("recur", c["C"], 1 if c["shared"] else c["C"], c["io"], c["gate"], c["form"] == "rays")
        where = dict(h0=s["h0"], offsets=s["offsets"], sequences=c["S"])
        y, last = cngp.recur_fwd(cfg, s["gate"], s["x"], y=c["keep"], **where)
        rows = slice(None) if s["offsets"] is None else slice(0, c["N"] - min(c["N"] // 16, 7))
        outs = [last] + ([y[rows]] if c["keep"] else [])
        if c["path"] == "recur_train":
            dgate, dx, dh0 = cngp.recur_bwd(cfg, s["gate"], s["x"], dy=s["dy"], dlast=s["dlast"], y=y, **where)
            outs += [dgate[rows], dx[rows], dh0]
        return outs
    if c["path"].startswith("embed"):
        cfg = _config("embed", c["rows"], c["dim"], c["table"], c["io"], c["ids"], _scale(c))
        y = cngp.embed_fwd(cfg, s["ids"], s["table"], base=s["base"])
        return [y, cngp.embed_bwd(cfg, s["ids"], s["dy"])] if c["path"] == "embed_train" else [y]
    cfg = _config("balance", c["L"], c["N_c"], c["N_p"], c["top_k"])
    return list(cngp.probe_balance(cfg, s["Dhat"], s["weight"], rows=s["rows"]))


def _scan(a, b):
    """States of h[t] = a[t] h[t-1] + b[t] along the first dimension: pairs joined, the half as many scanned, the rest filled in."""
    n = b.shape[0]
    if n == 1:
        return b
    m = n // 2
    odd = _scan(a[1::2] * a[0::2][:m], a[1::2] * b[0::2][:m] + b[1::2])
    h = torch.empty_like(b)
    h[1::2] = odd
    h[0] = b[0]
    h[2::2] = a[2::2] * odd[: (n - 1) // 2] + b[2::2]
    return h


def _ends(s):
    """First and last row of the sequences that have rows, and which ones they are."""
    c = s["case"]
    if s["offsets"] is None:
        first = torch.arange(c["S"], device="cuda") * (c["N"] // c["S"])
        return first, first + (c["N"] // c["S"] - 1), torch.arange(c["S"], device="cuda")
    off = s["offsets"].long()
    full = torch.nonzero(off[1:] > off[:-1]).flatten()
    return off[:-1][full], off[1:][full] - 1, full


def _plain_recur(s):
    c = s["case"]
    rays = c["form"] == "rays"
    used = c["N"] if s["offsets"] is None else c["N"] - min(c["N"] // 16, 7)
    g, x, h0 = s["gate"][:used].float(), s["x"][:used].float(), s["h0"]
    first, final, which = _ends(s)
    if rays:                               # back to front: as a forward recurrence over the rows turned round
        g, x = g.flip(0), x.flip(0)
        first, final = used - 1 - final, used - 1 - first
    a = g.exp() if rays else g
    keep_in = -torch.expm1(g) if rays else None
    v = keep_in * x if rays else x.clone()
    v[first] += a[first] * h0[which]
    inner = a.clone()
    inner[first] = 0
    h = _scan(inner, v)
    last = h0.clone()
    last[which] = h[final]
    io, gate = s["x"].dtype, s["gate"].dtype
    back = (lambda t: t.flip(0)) if rays else (lambda t: t)
    outs = [last] + ([back(h).to(io)] if c["keep"] else [])
    if c["path"] == "recur_train":
        dy = back(s["dy"][:used].float()) if c["keep"] else torch.zeros_like(x)
        dy = dy.clone()
        dy[final] += s["dlast"][which]
        into = torch.zeros_like(a)         # the gate through which the next row's gradient comes back
        into[:-1] = inner[1:]
        dh = _scan(into.flip(0), dy.flip(0)).flip(0)
        before = torch.empty_like(h)
        before[1:] = h[:-1]
        before[first] = h0[which]
        da = dh * (before - x) if rays else dh * before
        if c["shared"]:
            da = da.sum(1, keepdim=True)
        dh0 = s["dlast"].clone()           # a sequence without rows passes its state on
        dh0[which] = a[first] * dh[first]
        outs += [back(da * a if rays else da).to(gate), back(keep_in * dh if rays else dh).to(io), dh0]
    return outs


def _plain_embed(s):
    c = s["case"]
    ids = s["ids"].long()
    real = (ids >= 0) & (ids < c["rows"])
    at = torch.where(real, ids, 0)
    rows = torch.where(real[:, None], s["table"][at].float() * _scale(c), 0.0)
    y = rows if s["base"] is None else s["base"].float() + rows
    outs = [y.to(_TORCH[c["io"]])]
    if c["path"] == "embed_train":
        grad = torch.zeros((c["rows"], c["dim"]), device="cuda")
        outs.append(grad.index_add_(0, at, torch.where(real[:, None], s["dy"].float(), 0.0)) * _scale(c))
    return outs


def _plain_balance(s):
    c = s["case"]
    v, N_p = s["Dhat"], c["N_p"]
    counted = torch.ones(v.shape[:2], device="cuda", dtype=torch.bool) if s["rows"] is None else s["rows"] != 0
    order = torch.arange(N_p, device="cuda")
    top = v.max(dim=2, keepdim=True).values
    winner = torch.where(v == top, order, N_p).min(dim=2).values             # equal values: the lowest index
    counts = ((winner[:, :, None] == order) & counted[:, :, None]).sum(1).int()
    if c["top_k"]:
        rest = v                                                             # the largest taken away top_k times
        for _ in range(c["top_k"]):
            place = torch.where(rest == rest.max(dim=2, keepdim=True).values, order, N_p).min(dim=2, keepdim=True).values
            rest = rest.scatter(2, place, -math.inf)
        v = torch.where(rest == v, -math.inf, v)
    e = (v - top).exp()
    sigma = e / e.sum(dim=2, keepdim=True)
    used = counted.sum(1, keepdim=True).clamp(min=1).float()                 # [L, 1]
    f = counts / used
    P = torch.where(counted[:, :, None], sigma, 0.0).sum(1) / used
    loss = N_p * (f * P).sum(1)
    grad = (s["weight"] * N_p / used)[:, :, None] * sigma * (f[:, None, :] - (sigma * f[:, None, :]).sum(2, keepdim=True))
    return [loss, counts, torch.where(counted[:, :, None], grad, 0.0)]


def run(state):
    if own:
        return _run_own(state)
    path = state["case"]["path"]
    return _plain_recur(state) if path.startswith("recur") else _plain_embed(state) if path.startswith("embed") else _plain_balance(state)


def work(case):
    c = case
    if c["path"].startswith("recur"):
        N, C, G, S = c["N"], c["C"], 1 if c["shared"] else c["C"], c["S"]
        x, gate, state = N * C * _BYTES[c["io"]], N * G * _BYTES[c["gate"]], S * C * 4
        offsets = (S + 1) * 4 if c["ragged"] else 0
        extra = 2 * N * C if c["form"] == "rays" else 0
        bytes_, flops = x + gate + 2 * state + offsets + (x if c["keep"] else 0), 2 * N * C + extra
        if c["path"] == "recur_train":   # the incoming gradients in; those of gates, inputs and states out
            bytes_ += (x if c["keep"] else 0) + state + gate + x + state
            flops += 4 * N * C + extra
        return {"bytes": bytes_, "flops": flops}
    if c["path"].startswith("embed"):
        N, rows, dim = c["N"], c["rows"], c["dim"]
        y = N * dim * _BYTES[c["io"]]
        groups = (N + 63) // 64 if c["hot"] == "rays" else N
        touched = rows * (1.0 - (1.0 - 1.0 / rows) ** groups) if c["hot"] != "zipf" else min(rows, N) * 0.5
        bytes_, flops = N * _BYTES[c["ids"]] + touched * dim * _BYTES[c["table"]] + (2 * y if c["base"] else y), 2 * N * dim
        if c["path"] == "embed_train":
            bytes_ += y + rows * dim * 4
            flops += N * dim + rows * dim
        return {"bytes": bytes_, "flops": flops}
    n = c["L"] * c["N_c"] * c["N_p"]
    return {"bytes": 2 * n * 4 + (c["L"] * c["N_c"] if c["masked"] else 0) + c["L"] * (c["N_p"] + 1) * 4, "flops": 12 * n}


def _doubled(a, b, longest):
    """The same recurrence by doubling: after k steps row t has taken in the 2^k rows up to it."""
    a, b, step = a.expand_as(b).clone(), b.clone(), 1
    while step < longest:
        b[step:] = b[step:] + a[step:] * b[:-step]
        a[step:] = a[step:] * a[:-step]
        step *= 2
    return b


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["path"].startswith("embed"):
        table, ids = s["table"].double(), s["ids"].long()
        keep = ((ids >= 0) & (ids < c["rows"])).double()[:, None]
        picked = keep * _scale(c) * table.index_select(0, ids.clamp(0, c["rows"] - 1))
        out = [picked + (0 if s["base"] is None else s["base"].double())]
        if c["path"] == "embed_train":
            order = torch.where(keep[:, 0] > 0, ids, c["rows"]).sort(stable=True)
            total = torch.zeros((c["N"] + 1, c["dim"]), dtype=torch.float64, device="cuda")
            torch.cumsum(s["dy"].double()[order.indices], 0, out=total[1:])
            edge = torch.searchsorted(order.values, torch.arange(c["rows"] + 1, device="cuda"))
            out.append(_scale(c) * (total[edge[1:]] - total[edge[:-1]]))
        return out
    if c["path"] == "balance":
        v = s["Dhat"].double()
        kept = torch.full_like(v, -math.inf)
        places = v.sort(dim=2, descending=True, stable=True).indices[..., : c["top_k"] or c["N_p"]]
        kept.scatter_(2, places, v.gather(2, places))
        sigma = kept.softmax(2)
        w = torch.ones(v.shape[:2], dtype=torch.float64, device="cuda") if s["rows"] is None else s["rows"].double()
        n = w.sum(1).clamp(min=1)
        wins = torch.zeros((c["L"], c["N_p"]), dtype=torch.float64, device="cuda").scatter_add_(1, places[..., 0], w)
        loss = c["N_p"] * (wins / n[:, None] * (sigma * w[..., None]).sum(1) / n[:, None]).sum(1)
        inner = torch.matmul(sigma, (wins / n[:, None])[:, :, None])
        grad = sigma * (wins[:, None, :] / n[:, None, None] - inner) * (w * s["weight"] * c["N_p"] / n[:, None])[..., None]
        return [loss, None, grad]
    rays, train = c["form"] == "rays", c["path"] == "recur_train"
    off = torch.arange(c["S"] + 1, device="cuda") * (c["N"] // c["S"]) if s["offsets"] is None else s["offsets"].long()
    length = off[1:] - off[:-1]
    used, longest, some = int(off[-1]), int(length.max()), length > 0
    turn = (lambda t: t.flip(0)) if rays else (lambda t: t)
    gate, x = turn(s["gate"][:used].double()), turn(s["x"][:used].double())
    begin, end = (used - off[1:], used - 1 - off[:-1]) if rays else (off[:-1], off[1:] - 1)
    begin, end = begin[some], end[some]
    a = torch.exp(gate) if rays else gate
    share = 1 - a if rays else torch.ones_like(a)
    prior = s["h0"].double()
    starts = torch.zeros((used, 1), dtype=torch.bool, device="cuda")
    starts[begin] = True
    entering = torch.zeros_like(x)
    entering[begin] = prior[some]
    inside = torch.where(starts, 0.0, a)
    h = _doubled(inside, share * x + a * entering, longest)
    last = prior.clone()
    last[some] = h[end]
    out = [last] + ([turn(h)] if c["keep"] else [])
    if train:
        d = torch.zeros_like(x) if s["dy"] is None else turn(s["dy"][:used].double()).clone()
        d[end] += s["dlast"].double()[some]
        after = torch.cat([inside[1:], torch.zeros_like(inside[:1])])
        dh = _doubled(after.flip(0), d.flip(0), longest).flip(0)
        previous = torch.where(starts, entering, torch.cat([torch.zeros_like(h[:1]), h[:-1]]))
        slope = dh * (previous - x if rays else previous)
        slope = slope.sum(1, keepdim=True) if c["shared"] else slope
        dstate = s["dlast"].double().clone()
        dstate[some] = (a * dh)[begin]
        out += [turn(slope * a if rays else slope), turn(share * dh), dstate]
    return out
