"""What the operators at the ends of the stack of layers are timed on: token embeddings with their gradient, the norm of rows (root mean
square or layer norm) with its gradients, and the loss of the kept tokens straight from the head's input, without logits in memory,
with its gradients towards that input and the head's table.

They are what a training step does below the lowest layer (embeddings forward; their gradient from the compact dx of that layer) and above the
highest one (the last norm and the loss, on kept rows).  Embeddings and norms are bound by HBM traffic from some hundred rows on and by launch
latency below; the loss by its matrix products, and by the table's traffic for few rows.

`run` computes the plain form, elementary torch operations in fp32, or, where `own` is set, makes the calls of
paper_2502_00340_amd.binding that a program makes.  `exact` is the same in fp64, written apart from the plain form.
"""
import math

import torch

own = False

DEV = "cuda:0"
BF, F32, F64, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int64
DT = {"bf16": BF, "f32": F32}

WIDTHS = (256, 768, 840, 2048, 4096, 8192)
VOCABS = (32000, 50257, 128256, 151936)
EPS = 1e-5
CLIP_LO, CLIP_HI, KL = 0.2, 0.28, 0.04


def listed():
    return [
        # single tokens of 16 sequences (generation): launch latency
        dict(name="embed_fwd_tokens", kind="embed_fwd", rows=16, V=128256, H=4096, dtype="bf16", scaled=False),
        # every token of a training batch at the 8B width
        dict(name="embed_fwd_8b", kind="embed_fwd", rows=8192, V=128256, H=4096, dtype="bf16", scaled=False),
        # gradient from the kept half of that batch into an fp32 main gradient
        dict(name="embed_bwd_8b", kind="embed_bwd", rows=8192, rho=0.5, V=128256, H=4096, dtype="bf16", scaled=False, main=True),
        # an odd vocabulary and width in fp32, scaled embeddings, few rows kept, the whole table's gradient written
        dict(name="embed_bwd_odd_f32", kind="embed_bwd", rows=4593, rho=0.3, V=50257, H=840, dtype="f32", scaled=True, main=False),
        # layer norm of single tokens of 16 sequences: launch latency
        dict(name="norm_fwd_tokens", kind="norm_fwd", rows=16, rho=1.0, H=4096, dtype="bf16", layer=True),
        # the last norm of a training batch at the 8B width, on the kept half
        dict(name="norm_fwd_8b", kind="norm_fwd", rows=8192, rho=0.5, H=4096, dtype="bf16", layer=False),
        # its backward, gains into an fp32 main gradient
        dict(name="norm_bwd_8b", kind="norm_bwd", rows=8192, rho=0.5, H=4096, dtype="bf16", layer=False, main=True),
        # layer norm with biases of an odd width in fp32, every row of a ragged batch
        dict(name="norm_bwd_layer_odd_f32", kind="norm_bwd", rows=4593, rho=1.0, H=840, dtype="f32", layer=True, main=False),
        # log probabilities of one short answer under a reference model: 64 rows of a large vocabulary, no gradient
        dict(name="head_logp_few", kind="head", loss="nll", grads="none", rows=64, rho=1.0, H=4096, V=128256, dtype="bf16"),
        # the method's own loss, the mean NLL of kept tokens, at TinyLlama's width and vocabulary, with both gradients
        dict(name="head_nll_32k", kind="head", loss="nll", grads="both", rows=8192, rho=0.5, H=2048, V=32000, dtype="bf16"),
        # policy update of a batch whose kept half are answers, large vocabulary at the 8B width: the largest
        dict(name="head_policy_128k", kind="head", loss="policy", grads="both", rows=8192, rho=0.5, H=4096, V=128256, dtype="bf16"),
        # odd vocabulary, width and number of rows in fp32
        dict(name="head_policy_odd_f32", kind="head", loss="policy", grads="both", rows=301, rho=1.0, H=840, V=50257, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        k = c["kind"][:4], c["dtype"] if c["kind"] == "head" else ""
        w = work(c)
        most[k] = max(most.get(k, 0.0), w["flops"] if c["kind"] == "head" else w["bytes"])
    while True:
        kind = rng.choice(("embed_fwd", "embed_bwd", "embed_bwd", "norm_fwd", "norm_bwd", "head", "head", "head"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        H = rng.choice(WIDTHS + (8 * _log(rng, 2, 1024),))
        V = rng.choice(VOCABS + (_log(rng, 300, 200000),))
        rows, rho = _log(rng, 1, 8192), rng.choice((1.0, round(rng.uniform(0.1, 0.9), 3)))
        c = dict(kind=kind, rows=rows, H=H, dtype=dtype)
        if kind[:5] == "embed":
            c.update(V=V, scaled=rng.random() < 0.3)
        if kind != "embed_fwd":
            c.update(rho=rho)
        if kind in ("embed_bwd", "norm_bwd"):
            c.update(main=rng.random() < 0.5)
        if kind[:4] == "norm":
            c.update(layer=rng.random() < 0.4)
        if kind == "head":
            c.update(V=V, loss=rng.choice(("nll", "policy")), grads=rng.choice(("none", "dx", "both", "both")))
        w = work(c)
        if (w["flops"] if kind == "head" else w["bytes"]) <= most[kind[:4], dtype if kind == "head" else ""]:
            return c


# ---- inputs -----------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(gen, *shape, std=1.0, mean=0.0, dtype=F32):
    return torch.randn(shape, generator=gen, device=DEV, dtype=F32).mul_(std).add_(mean).to(dtype)


def _kept(c):
    return max(1, int(math.floor(c["rho"] * c["rows"] + 0.5)))


def _kept_rows(gen, T, n):
    """int32, ascending: n of T rows, by the highest of uniform scores; None for all."""
    return None if n == T else torch.rand(T, generator=gen, device=DEV).topk(n).indices.sort().values.to(torch.int32)


def _tokens(gen, rows, V):
    """Some tokens are far more frequent than others (log-uniform ranks, spread over the table); one in fifty is padding."""
    rank = torch.exp(torch.rand(rows, generator=gen, device=DEV, dtype=F64) * math.log(V)).long() - 1
    t = (rank.clamp(0, V - 1) * 7919 + 17) % V
    t[torch.rand(rows, generator=gen, device=DEV) < 0.02] = -1
    return t


def _embed(c, gen):
    dt, s = DT[c["dtype"]], dict(tokens=_tokens(gen, c["rows"], c["V"]), scale=math.sqrt(c["H"]) if c["scaled"] else 1.0)
    if c["kind"] == "embed_fwd":
        s["table"] = _randn(gen, c["V"], c["H"], std=0.02, dtype=dt)
        return s
    n = _kept(c)
    s["idx"], s["dx"], s["main"] = _kept_rows(gen, c["rows"], n), _randn(gen, n, c["H"], dtype=dt), None
    if c["main"]:            # what earlier micro-batches left
        s["main"] = _randn(gen, c["V"], c["H"], std=0.5)
    return s


def _norm(c, gen):
    dt, n, H = DT[c["dtype"]], _kept(c), c["H"]
    s = dict(idx=_kept_rows(gen, c["rows"], n), n=n, x=_randn(gen, c["rows"], H, std=1.5, mean=0.3, dtype=dt))
    s["g"] = _randn(gen, H, std=0.3, mean=1.0, dtype=dt)
    s["b"] = _randn(gen, H, std=0.3, dtype=dt) if c["layer"] else None
    s["dg"] = s["db"] = None
    if c["kind"] == "norm_bwd":
        s["dy"] = _randn(gen, n, H, dtype=dt)
        if c["main"]:
            s["dg"], s["db"] = _randn(gen, H, std=30.0), _randn(gen, H, std=30.0) if c["layer"] else None
    return s


def _head(c, gen):
    R, V, H, n, dt = c["rows"], c["V"], c["H"], _kept(c), DT[c["dtype"]]
    s = dict(idx=_kept_rows(gen, R, n), n=n)
    s["table"] = _randn(gen, V, H, std=2.5 / math.sqrt(H), dtype=dt)             # logits of some 2.5 from inputs of size 1
    s["targets"] = torch.randint(0, V, (R,), generator=gen, device=DEV, dtype=I64)
    rows = torch.arange(n, device=DEV) if s["idx"] is None else s["idx"].long()
    y = s["targets"][rows]
    # a model knows its next token in part
    s["x"] = (_randn(gen, n, H) + s["table"][y].float() * _randn(gen, n, 1, std=0.4, mean=1.28)).to(dt)
    if c["loss"] == "nll":
        s["targets"][torch.rand(R, generator=gen, device=DEV) < 0.02] = -100
        return s
    lp = torch.empty(n, dtype=F64, device=DEV)
    t = s["table"].float()
    for a in range(0, n, 512):
        l = s["x"][a:a + 512].float() @ t.T
        lp[a:a + 512] = (l.gather(1, y[a:a + 512, None]).squeeze(1) - torch.logsumexp(l, 1)).to(F64)
    # log ratios of a few off-policy steps, none within 1e-3 of a border of the clipping, where the gradient jumps
    x = _randn(gen, n, std=0.25).to(F64)
    for border in (math.log(1.0 - CLIP_LO), math.log(1.0 + CLIP_HI)):
        x = torch.where((x - border).abs() < 1e-3, x + 4e-3, x)
    s["old"], s["ref"] = torch.zeros(R, device=DEV), torch.zeros(R, device=DEV)
    s["old"][rows], s["ref"][rows] = (lp - x).to(F32), (lp + _randn(gen, n, std=0.3)).to(F32)
    s["adv"] = _randn(gen, R)
    s["weight"] = torch.rand(R, generator=gen, device=DEV).add_(0.5)         # one over the answers' lengths, say
    s["weight"][torch.rand(R, generator=gen, device=DEV) < 0.01] = 0.0
    return s


def _inputs(case, seed):
    gen = _gen(seed)
    return {"embe": _embed, "norm": _norm, "head": _head}[case["kind"][:4]](case, gen)


def prepare(case, seed):
    return _inputs(case, seed) | {"case": case}


# ---- one pass ---------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    if own:
        return _own(c, s)
    return {"embed_fwd": _run_embed_fwd, "embed_bwd": _run_embed_bwd, "norm_fwd": _run_norm_fwd, "norm_bwd": _run_norm_bwd, "head": _run_head}[c["kind"]](c, s)


def _own(c, s):
    from paper_2502_00340_amd import binding as cf
    if c["kind"] == "embed_fwd":
        return cf.embed_fwd(s["table"], s["tokens"], scale=s["scale"])
    if c["kind"] == "embed_bwd":
        return cf.embed_bwd(s["tokens"], s["dx"], c["V"], scale=s["scale"], idx=s["idx"], main_grad=s["main"])
    if c["kind"] == "norm_fwd":
        return cf.norm_fwd(s["x"], s["g"], s["b"], eps=EPS, layer=c["layer"], idx=s["idx"])
    if c["kind"] == "norm_bwd":
        return cf.norm_bwd(s["x"], s["g"], s["dy"], eps=EPS, layer=c["layer"], idx=s["idx"], main_grads=(s["dg"], s["db"]) if c["main"] else None)
    pol = dict(old_logp=s["old"], ref_logp=s["ref"], advantages=s["adv"], weights=s["weight"], clip=(CLIP_LO, CLIP_HI),
               kl_coef=KL) if c["loss"] == "policy" else {}
    return cf.head_loss(s["x"], s["table"], s["targets"], idx=s["idx"], need_dx=c["grads"] != "none", need_dtable=c["grads"] == "both", **pol)


def _run_embed_fwd(c, s):
    t = s["tokens"]
    live = ((t >= 0) & (t < c["V"]))[:, None]
    y = s["table"][t.clamp(0, c["V"] - 1)].float() * s["scale"]
    return torch.where(live, y, 0.0).to(s["table"].dtype)


def _run_embed_bwd(c, s):
    t = s["tokens"] if s["idx"] is None else s["tokens"][s["idx"].long()]
    live = (t >= 0) & (t < c["V"])
    d = torch.where(live[:, None], s["dx"].float() * s["scale"], 0.0)
    out = s["main"] if s["main"] is not None else torch.zeros((c["V"], c["H"]), device=DEV)
    out.index_add_(0, t.clamp(0, c["V"] - 1), d)
    return out if s["main"] is not None else out.to(s["dx"].dtype)


def _stats(c, x):
    mu = x.mean(-1, keepdim=True) if c["layer"] else 0.0
    x = x - mu
    return x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt(), (x.square().mean(-1, keepdim=True) + EPS).rsqrt()


def _run_norm_fwd(c, s):
    x = (s["x"] if s["idx"] is None else s["x"][s["idx"].long()]).float()
    y = _stats(c, x)[0] * s["g"].float()
    return (y + s["b"].float() if c["layer"] else y).to(s["x"].dtype)


def _run_norm_bwd(c, s):
    x, dy = (s["x"] if s["idx"] is None else s["x"][s["idx"].long()]).float(), s["dy"].float()
    n, rstd = _stats(c, x)
    u = dy * s["g"].float()
    dx = u - n * (u * n).mean(-1, keepdim=True)
    if c["layer"]:
        dx = dx - u.mean(-1, keepdim=True)
    dg, db = (dy * n).sum(0), dy.sum(0) if c["layer"] else None
    to = lambda t, acc: None if t is None else t.to(s["g"].dtype) if acc is None else acc.add_(t)
    return (dx * rstd).to(s["dy"].dtype), to(dg, s["dg"]), to(db, s["db"])


def _run_head(c, s):
    n, V = s["n"], c["V"]
    rows = torch.arange(n, device=DEV) if s["idx"] is None else s["idx"].long()
    xf, t, y = s["x"].float(), s["table"].float(), s["targets"][rows]
    l = xf @ t.T
    live = (y >= 0) & (y < V)
    if c["loss"] == "policy":
        w = s["weight"][rows]
        live &= w != 0
    else:
        w = torch.ones(n, device=DEV)
    y = y.clamp(0, V - 1)[:, None]
    m = l.max(1, keepdim=True).values
    ly = l.gather(1, y) - m
    e = l.sub_(m).exp_()
    z = e.sum(1, keepdim=True)
    lp = (ly - z.log()).squeeze(1)
    if c["loss"] == "policy":
        A, k = s["adv"][rows], s["ref"][rows] - lp
        r = (lp - s["old"][rows]).exp()
        rc = r.clamp(1.0 - CLIP_LO, 1.0 + CLIP_HI)
        clipped = r * A > rc * A
        pl, kl = -torch.minimum(r * A, rc * A), torch.expm1(k) - k
        coef = torch.where(clipped, 0.0, -r * A) - KL * torch.expm1(k)
    else:
        pl, kl, coef, clipped = -lp, torch.zeros_like(lp), -torch.ones_like(lp), torch.zeros_like(live)
    w = torch.where(live, w, 0.0) / n
    zero = torch.zeros((), device=DEV)
    mean = lambda v: torch.where(live, w * v, zero).double().sum()
    pm, km = mean(pl), mean(kl)
    stats = torch.stack((pm + (KL if c["loss"] == "policy" else 0.0) * km, pm, km, mean(clipped.float()))).float()
    lp = torch.where(live, lp, zero)
    if c["grads"] == "none":
        return stats, lp, None, None
    coef = torch.where(live, w * coef, zero)[:, None]
    d = e.mul_(-coef / z)
    d.scatter_add_(1, y, coef)
    dx = (d @ t).to(s["x"].dtype)
    return stats, lp, dx, (d.T @ xf).to(s["table"].dtype) if c["grads"] == "both" else None


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    c, kind = case, case["kind"]
    e, H = 2.0 if c["dtype"] == "bf16" else 4.0, float(c["H"])
    # rows of the table that are read or added to: V distinct tokens of log-uniform ranks, n draws
    touched = lambda n: min(n, c["V"] * 1.0, sum((1.0 - (1.0 - 1.0 / (k * math.log(c["V"]))) ** n) * w for k, w in _bands(c["V"])))
    if kind == "embed_fwd":
        n = float(c["rows"])
        return {"bytes": touched(n) * H * e + n * (H * e + 8.0), "flops": n * H}
    n = float(_kept(c))
    index = 0.0 if c["rho"] == 1.0 else 4.0
    if kind == "embed_bwd":
        out = touched(n) * H * 8.0 if c["main"] else c["V"] * H * e
        return {"bytes": n * (H * e + 8.0 + index) + out, "flops": 2.0 * n * H}
    if kind == "norm_fwd":
        return {"bytes": n * (2.0 * H * e + index) + H * e * (2.0 if c["layer"] else 1.0), "flops": n * H * (8.0 if c["layer"] else 5.0)}
    if kind == "norm_bwd":
        return {"bytes": n * (3.0 * H * e + index) + H * (e + (8.0 if c["main"] else e) * (2.0 if c["layer"] else 1.0)),
                "flops": n * H * (18.0 if c["layer"] else 13.0)}
    V, products = float(c["V"]), {"none": 1.0, "dx": 2.0, "both": 3.0}[c["grads"]]
    per_row = 12.0 + (16.0 if c["loss"] == "policy" else 0.0) + index
    moved = (n + V) * H * e + (n * H * e if c["grads"] != "none" else 0.0) + (V * H * e if c["grads"] == "both" else 0.0)
    return {"bytes": moved + n * per_row, "flops": 2.0 * n * H * V * products}


def _bands(V):
    """Ranks 1 .. V in bands (a rank of the band, its number of ranks)."""
    out, a = [], 1
    while a <= V:
        b = min(V + 1, max(a + 1, a + a // 8))
        out.append(((a + b - 1) / 2.0, float(b - a)))
        a = b
    return out


# ---- the same in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"embe": _exact_embed, "norm": _exact_norm, "head": _exact_head}[case["kind"][:4]](case, s)


def _exact_embed(c, s):
    if c["kind"] == "embed_fwd":
        padded = torch.cat((s["table"], s["table"].new_zeros(1, c["H"])))          # a row of zeros for what is no token
        t = torch.where((s["tokens"] < 0) | (s["tokens"] >= c["V"]), c["V"], s["tokens"])
        return padded.index_select(0, t).double() * s["scale"]
    t = s["tokens"] if s["idx"] is None else s["tokens"].index_select(0, s["idx"].long())
    rows = (t >= 0).nonzero().squeeze(1)
    out = s["main"].double() if c["main"] else torch.zeros((c["V"], c["H"]), dtype=F64, device=DEV)
    order = rows[torch.argsort(t[rows], stable=True)]
    which, count = torch.unique_consecutive(t[order], return_counts=True)
    # sums of runs of equal tokens, as differences would lose digits: the k-th row of every run in turn
    first = torch.cumsum(count, 0) - count
    for k in range(int(count.max()) if count.numel() else 0):
        have = count > k
        out[which[have]] += s["dx"][order[first[have] + k]].double() * s["scale"]
    return out


def _exact_norm(c, s):
    x = (s["x"] if s["idx"] is None else s["x"].index_select(0, s["idx"].long())).double()
    H = c["H"]
    if c["layer"]:
        x = x - torch.sum(x, 1, keepdim=True) / H
    inv = 1.0 / torch.sqrt(torch.sum(x * x, 1, keepdim=True) / H + EPS)
    g = s["g"].double()
    if c["kind"] == "norm_fwd":
        y = x * inv * g
        return y + s["b"].double() if c["layer"] else y
    dy = s["dy"].double()
    a = dy * g
    dx = inv * a - x * inv ** 3 * torch.sum(a * x, 1, keepdim=True) / H
    if c["layer"]:
        dx = dx - inv * torch.sum(a, 1, keepdim=True) / H
    dg, db = torch.sum(dy * x * inv, 0), torch.sum(dy, 0) if c["layer"] else None
    if c["main"]:
        dg, db = dg + s["dg"].double(), None if db is None else db + s["db"].double()
    return dx, dg, db


def _exact_head(c, s):
    V, n, H = c["V"], s["n"], c["H"]
    rows = torch.arange(n, device=DEV) if s["idx"] is None else s["idx"].long()
    table = s["table"].double()
    lp, loss = torch.zeros(n, dtype=F64, device=DEV), torch.zeros(4, dtype=F64, device=DEV)
    dx = torch.zeros((n, H), dtype=F64, device=DEV) if c["grads"] != "none" else None
    dt = torch.zeros((V, H), dtype=F64, device=DEV) if c["grads"] == "both" else None
    step = max(1, (1 << 27) // V)
    for a in range(0, n, step):
        at = rows[a:a + step]
        t = s["targets"][at]
        w = torch.ones(at.numel(), dtype=F64, device=DEV) if c["loss"] == "nll" else s["weight"][at].double()
        use = ((t != -100) & (w > 0)).nonzero().squeeze(1)
        at, t, w, x = at[use], t[use], w[use] / n, s["x"][a + use].double()
        this = torch.arange(at.numel(), device=DEV)
        p = torch.log_softmax(torch.mm(x, table.t()), 1)
        l = p[this, t]
        lp[a + use] = l
        if c["loss"] == "nll":
            first, kl, cut, slope = -l, torch.zeros_like(l), torch.zeros_like(l), -torch.ones_like(l)
        else:
            A, r, q = s["adv"][at].double(), torch.exp(l - s["old"][at].double()), s["ref"][at].double() - l
            over = torch.where(A > 0, r > 1.0 + CLIP_HI, (A < 0) & (r < 1.0 - CLIP_LO))
            bound = torch.where(A > 0, 1.0 + CLIP_HI, 1.0 - CLIP_LO).double()
            first, kl, cut = -torch.where(over, bound, r) * A, torch.exp(q) - q - 1.0, over.double()
            slope = torch.where(over, 0.0, -r * A) + KL * (1.0 - torch.exp(q))
        loss += torch.stack(((w * (first + (KL if c["loss"] == "policy" else 0.0) * kl)).sum(), (w * first).sum(), (w * kl).sum(), (w * cut).sum()))
        if dx is None:
            continue
        p.exp_().neg_()
        p[this, t] += 1.0
        p *= (w * slope)[:, None]
        dx[a + use] = torch.mm(p, table)
        if dt is not None:
            dt.addmm_(p.t(), x)
    return loss, lp, dx, dt
