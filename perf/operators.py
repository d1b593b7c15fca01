"""What the operators around the layer backward are timed on: the query/key norm with rotary embedding, the token losses with
their gradient towards the logits, and the AdamW step.

They are what a training step does before the filtered layer backward (query/key norm and rotation, forward), inside it (their
backward on kept rows), ahead of it (the loss of the kept tokens and its gradient) and behind it (global gradient norm and
parameter update).  All are bound by HBM traffic from some hundred rows on and by launch latency below.

`run` computes the plain form, elementary torch operations in fp32, or, where `own` is set, makes the calls of
paper_2502_00340_amd.binding that a program makes.  `exact` is the same in fp64, written apart from the plain form.
"""
import math

import torch

own = False

DEV = "cuda:0"
BF, F32, F64, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int64
E4M3 = torch.float8_e4m3fn
DT = {"bf16": BF, "f32": F32}

HEADS = ((32, 8, 128), (32, 4, 64), (64, 8, 128), (16, 8, 128), (4, 1, 128), (12, 4, 64))
# (H, Nq, Nkv, F) of layers whose parameters are updated: TinyLlama and 8B shapes, a narrow one with odd sizes
LAYERS = {"1b": (2048, 2048, 256, 5632), "8b": (4096, 4096, 1024, 14336), "8b_tp8": (4096, 512, 128, 1792),
          "narrow": (840, 768, 256, 2312)}
EPS_N = 1e-6
CLIP_LO, CLIP_HI, KL = 0.2, 0.28, 0.04
LR, B1, B2, EPS, WD, MAX_NORM, SEED = 3e-4, 0.9, 0.95, 1e-8, 0.1, 1.0, 20240
BLOCK = 256                  # elements that share a scale of an 8-bit state


def listed():
    return [
        # single tokens of 16 sequences at their own positions (generation): launch latency
        dict(name="qk_fwd_tokens", kind="qk_fwd", B=16, S=1, table=32768, Hq=32, Hkv=8, d=128, dtype="bf16", fused=False, tokens=True),
        # forward of a training batch at the 8B head layout, q and k read out of one fused projection
        dict(name="qk_fwd_8b", kind="qk_fwd", B=2, S=4096, table=4096, Hq=32, Hkv=8, d=128, dtype="bf16", fused=True, tokens=False),
        # backward on the kept half of that batch
        dict(name="qk_bwd_8b", kind="qk_bwd", B=2, S=4096, table=4096, Hq=32, Hkv=8, d=128, dtype="bf16", rho=0.5, main=False),
        # head size 64, odd length, few rows kept, gains into fp32 main gradients
        dict(name="qk_bwd_ragged_d64", kind="qk_bwd", B=3, S=1531, table=1531, Hq=32, Hkv=4, d=64, dtype="bf16", rho=0.3, main=True),
        # reference log probabilities of one short answer: 64 rows of a large vocabulary, forward only, few rows
        dict(name="loss_logp_few", kind="loss", loss="nll", grad=False, rows=64, rho=1.0, V=128256, dtype="bf16"),
        # the method's own loss, the mean NLL of kept tokens, at TinyLlama's vocabulary, with its gradient
        dict(name="loss_nll_32k", kind="loss", loss="nll", grad=True, rows=8192, rho=0.5, V=32000, dtype="bf16"),
        # policy update of a batch whose kept half are answers, large vocabulary: the largest
        dict(name="loss_policy_128k", kind="loss", loss="policy", grad=True, rows=8192, rho=0.5, V=128256, dtype="bf16"),
        # fp32 logits of an odd vocabulary (rows not on a 16-byte boundary), odd number of rows, every row kept
        dict(name="loss_policy_odd_f32", kind="loss", loss="policy", grad=True, rows=701, rho=1.0, V=50257, dtype="f32"),
        # adapters of rank 64 on the q, k, v, o projections of an 8B layer, bf16 without a master copy: launch latency
        dict(name="adamw32_adapters", kind="adamw", layer="8b", rank=64, bits=32, p="bf16", master=False, g="bf16"),
        # a TinyLlama layer, bf16 with fp32 master copies and fp32 main gradients
        dict(name="adamw32_1b", kind="adamw", layer="1b", rank=0, bits=32, p="bf16", master=True, g="f32"),
        # the 8B layer with states in 8 bits
        dict(name="adamw8_8b", kind="adamw", layer="8b", rank=0, bits=8, p="bf16", master=True, g="f32"),
        # fp32 parameters of a narrow layer (sizes that end inside a block of the 8-bit states' scales)
        dict(name="adamw8_narrow_f32", kind="adamw", layer="narrow", rank=0, bits=8, p="f32", master=False, g="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        k = c["kind"][:2]
        most[k] = max(most.get(k, 0.0), work(c)["bytes"])
    while True:
        kind = rng.choice(("qk_fwd", "qk_bwd", "loss", "loss", "adamw", "adamw"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if kind in ("qk_fwd", "qk_bwd"):
            Hq, Hkv, d = rng.choice(HEADS)
            tokens = kind == "qk_fwd" and rng.random() < 0.4
            S = 1 if tokens else _log(rng, 2, 8192)
            B = _log(rng, 1, 512) if tokens else rng.randint(1, max(1, min(8, 8192 // S)))
            c = dict(kind=kind, B=B, S=S, table=_log(rng, 64, 65536) if tokens else S, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype)
            c.update(dict(fused=rng.random() < 0.5, tokens=tokens) if kind == "qk_fwd" else
                     dict(rho=round(rng.uniform(0.1, 1.0), 3), main=rng.random() < 0.5))
        elif kind == "loss":
            V = rng.choice((32000, 50257, 128256, 151936, _log(rng, 300, 200000)))
            c = dict(kind=kind, loss=rng.choice(("nll", "policy")), grad=rng.random() < 0.75, rows=_log(rng, 1, 8192),
                     rho=rng.choice((1.0, round(rng.uniform(0.1, 0.9), 3))), V=V, dtype=dtype)
        else:
            c = dict(kind=kind, layer=rng.choice(sorted(LAYERS)), rank=rng.choice((0, 0, 8, 24, 64)), bits=rng.choice((8, 32)), p=dtype,
                     master=dtype == "bf16" and rng.random() < 0.6, g=rng.choice(("bf16", "f32")))
        if work(c)["bytes"] <= most[kind[:2]] and c not in [{k: v for k, v in x.items() if k != "name"} for x in listed()]:
            return c


# ---- inputs -----------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(gen, *shape, std=1.0, mean=0.0, dtype=F32):
    return torch.randn(shape, generator=gen, device=DEV, dtype=F32).mul_(std).add_(mean).to(dtype)


def _kept(c):
    T = c["B"] * c["S"] if "B" in c else c["rows"]
    return max(1, int(math.floor(c["rho"] * T + 0.5)))


def _kept_rows(gen, T, n):
    """int32, ascending: n of T rows, by the highest of uniform scores."""
    return torch.rand(T, generator=gen, device=DEV).topk(n).indices.sort().values.to(torch.int32)


def _tables(n_pos, d):
    f = 500000.0 ** (-torch.arange(0, d // 2, device=DEV, dtype=F64) * 2.0 / d)
    a = torch.arange(n_pos, device=DEV, dtype=F64)[:, None] * f[None, :]        # in 64 bits: angles of far positions
    return a.cos().to(F32), a.sin().to(F32)


def _qk(c, gen):
    dt, Nq, Nkv, T = DT[c["dtype"]], c["Hq"] * c["d"], c["Hkv"] * c["d"], c["B"] * c["S"]
    s = dict(gq=_randn(gen, c["d"], std=0.3, mean=1.0, dtype=dt), gk=_randn(gen, c["d"], std=0.3, mean=1.0, dtype=dt))
    s["cos"], s["sin"] = _tables(c["table"], c["d"])
    s["positions"] = None
    if c["kind"] == "qk_fwd":
        if c["fused"]:
            qkv = _randn(gen, T, Nq + 2 * Nkv, std=1.5, dtype=dt)
            s["q"], s["k"] = qkv[:, :Nq], qkv[:, Nq:Nq + Nkv]
        else:
            s["q"], s["k"] = _randn(gen, T, Nq, std=1.5, dtype=dt), _randn(gen, T, Nkv, std=1.5, dtype=dt)
        if c["tokens"]:
            s["positions"] = torch.randint(0, c["table"], (T,), generator=gen, device=DEV, dtype=torch.int32)
        return s
    n = _kept(c)
    s["q"], s["k"] = _randn(gen, T, Nq, std=1.5, dtype=dt), _randn(gen, T, Nkv, std=1.5, dtype=dt)
    s["dq"], s["dk"] = _randn(gen, n, Nq, dtype=dt), _randn(gen, n, Nkv, dtype=dt)
    s["idx"] = _kept_rows(gen, T, n)
    if c["main"]:            # what earlier micro-batches left
        s["dgq"], s["dgk"] = _randn(gen, c["d"], std=30.0), _randn(gen, c["d"], std=30.0)
    return s


def _loss(c, gen):
    R, V, n = c["rows"], c["V"], _kept(c)
    s = dict(idx=None if n == R else _kept_rows(gen, R, n), n=n)
    s["logits"] = _randn(gen, R, V, std=2.5, dtype=DT[c["dtype"]])
    s["targets"] = torch.randint(0, V, (R,), generator=gen, device=DEV, dtype=I64)
    # a model knows its next token in part
    s["logits"].scatter_add_(1, s["targets"][:, None], _randn(gen, R, 1, std=3.0, mean=8.0, dtype=s["logits"].dtype))
    if c["loss"] == "nll":
        s["targets"][torch.rand(R, generator=gen, device=DEV) < 0.02] = -100
        return s
    lp = (s["logits"].gather(1, s["targets"][:, None]).squeeze(1).to(F64) - torch.logsumexp(s["logits"].float(), 1).to(F64))
    # log ratios of a few off-policy steps, none within 1e-3 of a border of the clipping, where the gradient jumps
    x = _randn(gen, R, std=0.25).to(F64)
    for border in (math.log(1.0 - CLIP_LO), math.log(1.0 + CLIP_HI)):
        x = torch.where((x - border).abs() < 1e-3, x + 4e-3, x)
    s["old"] = (lp - x).to(F32)
    s["ref"] = (lp + _randn(gen, R, std=0.3)).to(F32)
    s["adv"] = _randn(gen, R)
    s["weight"] = torch.rand(R, generator=gen, device=DEV).add_(0.5)         # one over the answers' lengths, say
    s["weight"][torch.rand(R, generator=gen, device=DEV) < 0.01] = 0.0
    return s


def _sizes(c):
    H, Nq, Nkv, F = LAYERS[c["layer"]]
    r = c["rank"]
    if r:
        return [(H, r), (r, Nq), (H, r), (r, Nkv), (H, r), (r, Nkv), (Nq, r), (r, H)]
    return [(H, Nq), (H, Nkv), (H, Nkv), (Nq, H), (H, F), (H, F), (F, H), (H,), (H,)]


def _adamw(c, gen):
    s = dict(p=[], master=[], g=[], m=[], v=[], ms=[], vs=[], step=120, kinds=c)
    for shape in _sizes(c):
        w = _randn(gen, *shape, std=0.02)
        s["p"].append(w.to(DT[c["p"]]))
        if c["master"]:
            s["master"].append(w)
        s["g"].append(_randn(gen, *shape, std=2e-3, dtype=DT[c["g"]]))
        m, v = _randn(gen, *shape, std=5e-4), _randn(gen, *shape, std=2e-3).square_().add_(1e-7)
        if c["bits"] == 8:
            (m8, ms), (v8, vs) = _quant(m, E4M3), _quant(v.sqrt_(), E4M3)
            s["m"].append(m8), s["v"].append(v8), s["ms"].append(ms), s["vs"].append(vs)
        else:
            s["m"].append(m), s["v"].append(v)
    return s


def prepare(case, seed):
    gen, kind = _gen(seed), case["kind"]
    s = _loss(case, gen) if kind == "loss" else _adamw(case, gen) if kind == "adamw" else _qk(case, gen)
    s["case"] = case
    if own:
        from paper_2502_00340_amd import binding as Bn
        s["Bn"] = Bn
        if kind == "adamw":          # the plan that a program keeps: pointers, hyperparameters, a workspace
            s["plan"] = Bn.AdamW(s["p"], s["g"], lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, max_norm=MAX_NORM, seed=SEED,
                                 master=s["master"] or None, state=(s["m"], s["v"], s["ms"], s["vs"]) if case["bits"] == 8 else (s["m"], s["v"]))
        elif kind != "loss":
            s["desc"] = Bn.make_desc(1, case["table"], 256, case["Hq"], case["Hkv"], case["d"], 256, case["dtype"], rms_eps=EPS_N)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    return {"qk_fwd": _run_qk_fwd, "qk_bwd": _run_qk_bwd, "loss": _run_loss, "adamw": _run_adamw}[c["kind"]](c, s)


def _positions(c, s, rows):
    return rows % c["table"] if s["positions"] is None else s["positions"][rows].long()


def _rotate(x, cos, sin):
    """x [n, heads, d]; cos, sin [n, d/2]"""
    lo, hi = x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:]
    cos, sin = cos[:, None], sin[:, None]
    return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1)


def _run_qk_fwd(c, s):
    if own:
        return s["Bn"].qk_norm_rope_fwd(s["desc"], s["q"], s["k"], s["gq"], s["gk"], s["cos"], s["sin"], positions=s["positions"])
    pos = _positions(c, s, torch.arange(c["B"] * c["S"], device=DEV))
    cos, sin = s["cos"][pos], s["sin"][pos]

    def one(x, g):
        y = x.float().reshape(x.shape[0], -1, c["d"])
        y = y * (y.square().mean(-1, keepdim=True) + EPS_N).rsqrt() * g.float()
        return _rotate(y, cos, sin).reshape(x.shape).to(x.dtype)
    return one(s["q"], s["gq"]), one(s["k"], s["gk"])


def _run_qk_bwd(c, s):
    if own:
        return s["Bn"].qk_norm_rope_bwd(s["desc"], s["q"], s["k"], s["gq"], s["gk"], s["dq"], s["dk"], s["cos"], s["sin"], idx=s["idx"],
                                        main_grads=(s["dgq"], s["dgk"]) if c["main"] else None)
    rows = s["idx"].long()
    pos = _positions(c, s, rows)
    cos, sin = s["cos"][pos], s["sin"][pos]

    def one(x, dy, g, acc):
        y = x[rows].float().reshape(dy.shape[0], -1, c["d"])
        rstd = (y.square().mean(-1, keepdim=True) + EPS_N).rsqrt()
        n, u = y * rstd, _rotate(dy.float().reshape(y.shape), cos, -sin)
        dg = (u * n).sum((0, 1))
        ug = u * g.float()
        dx = rstd * (ug - n * (ug * n).mean(-1, keepdim=True))
        return dx.reshape(dy.shape).to(dy.dtype), dg.to(g.dtype) if acc is None else acc.add_(dg)
    dq, dgq = one(s["q"], s["dq"], s["gq"], s.get("dgq"))
    dk, dgk = one(s["k"], s["dk"], s["gk"], s.get("dgk"))
    return dq, dk, dgq, dgk


def _run_loss(c, s):
    if own:
        pol = dict(old_logp=s["old"], ref_logp=s["ref"], advantages=s["adv"], weights=s["weight"], clip=(CLIP_LO, CLIP_HI),
                   kl_coef=KL) if c["loss"] == "policy" else {}
        return s["Bn"].token_loss(s["logits"], s["targets"], idx=s["idx"], need_grad=c["grad"], **pol)
    rows = torch.arange(c["rows"], device=DEV) if s["idx"] is None else s["idx"].long()
    x, y = s["logits"][rows].float(), s["targets"][rows]
    live = (y >= 0) & (y < c["V"])
    if c["loss"] == "policy":
        w = s["weight"][rows]
        live &= w != 0
    else:
        w = torch.ones(rows.numel(), device=DEV)
    y = y.clamp(0, c["V"] - 1)[:, None]
    m = x.max(1, keepdim=True).values
    e = (x - m).exp()
    z = e.sum(1, keepdim=True)
    lp = ((x.gather(1, y) - m) - z.log()).squeeze(1)
    if c["loss"] == "policy":
        A, k = s["adv"][rows], s["ref"][rows] - lp
        r = (lp - s["old"][rows]).exp()
        rc = r.clamp(1.0 - CLIP_LO, 1.0 + CLIP_HI)
        clipped = r * A > rc * A
        pl, kl = -torch.minimum(r * A, rc * A), torch.expm1(k) - k
        coef = torch.where(clipped, 0.0, -r * A) - KL * torch.expm1(k)
    else:
        pl, kl, coef, clipped = -lp, torch.zeros_like(lp), -torch.ones_like(lp), torch.zeros_like(live)
    w = torch.where(live, w, 0.0) / rows.numel()
    zero = torch.zeros((), device=DEV)
    mean = lambda t: torch.where(live, w * t, zero).double().sum()
    pm, km = mean(pl), mean(kl)
    stats = torch.stack((pm + (KL if c["loss"] == "policy" else 0.0) * km, pm, km, mean(clipped.float()))).float()
    lp = torch.where(live, lp, zero)
    if not c["grad"]:
        return stats, lp, None
    coef = torch.where(live, w * coef, zero)[:, None]
    d = e.mul_(-coef / z)
    d.scatter_add_(1, y, coef)
    return stats, lp, d.to(s["logits"].dtype)


def _blocks(x):
    """[n/256, 256], zeros behind the last element"""
    x = x.reshape(-1)
    out = torch.zeros(-(-x.numel() // BLOCK) * BLOCK, dtype=x.dtype, device=DEV)
    out[:x.numel()] = x
    return out.view(-1, BLOCK)


def _quant(x, dtype, u=None):
    """x in e4m3 with a scale for every 256 elements; u: uniform numbers in [0, 1), one an element, that round x (which is not
    negative then) up where what is cut off reaches 1 - u, and what is not zero to no less than the smallest value."""
    b = _blocks(x)
    top = b.abs().amax(1, keepdim=True).clamp(min=2.0 ** -100)
    y = b * (448.0 / top)
    if u is not None:
        ulp = (y.clamp(min=2.0 ** -6).view(torch.int32) & 0x7F800000).view(F32) * 0.125
        y = torch.where(b > 0, (torch.floor(y / ulp + _blocks(u)) * ulp).clamp(2.0 ** -9, 448.0), y)
    return y.to(dtype).view(-1)[:x.numel()].view(x.shape), (top / 448.0).squeeze(1)


def _value(q, scale):
    return (_blocks(q.to(scale.dtype)) * scale[:, None]).view(-1)[:q.numel()].view(q.shape)


def _uniform(n, tensor, step):
    """20 random bits of every element of a tensor: a hash of its number, the step, the tensor's number and the seed"""
    M = 0xFFFFFFFF
    i = torch.arange(n, device=DEV, dtype=I64)
    key = (SEED + 0x85EBCA77 * (tensor + 1) + 0xC2B2AE3D * step) & M
    h = ((i & M) * 0x9E3779B1 + (i >> 32) * 0x27D4EB2F + key) & M
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & M
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & M
    return (h ^ (h >> 16)) >> 12


def _run_adamw(c, s):
    if own:
        s["plan"].step(step=s["step"])
        norm = s["plan"].grad_norm
    else:
        norm = _plain_adamw(c, s)
    return {k: s[k] for k in ("p", "master", "m", "v", "ms", "vs")} | {"norm": norm}


def _plain_adamw(c, s):
    t = s["step"]
    norm = torch.stack([g.double().square().sum() for g in s["g"]]).sum().sqrt().float().view(1)
    clip = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
    size, root = LR / (1.0 - B1 ** t), math.sqrt(1.0 - B2 ** t)

    def one(i):
        g = s["g"][i].float() * clip
        w = s["master"][i] if c["master"] else s["p"][i].float()
        if c["bits"] == 8:
            m, v = _value(s["m"][i], s["ms"][i]), _value(s["v"][i], s["vs"][i]).square()
        else:
            m, v = s["m"][i], s["v"][i]
        m = B1 * m + (1.0 - B1) * g
        v = B2 * v + (1.0 - B2) * g.square()
        w = w * (1.0 - LR * WD) - size * m / (v.sqrt() / root + EPS)
        if c["master"]:
            s["master"][i].copy_(w)
        s["p"][i].copy_(w)
        if c["bits"] == 8:
            u = _uniform(g.numel(), i, t).to(F32).mul_(2.0 ** -20)
            for k, (q, sc) in (("m", _quant(m, E4M3)), ("v", _quant(v.sqrt(), E4M3, u))):
                s[k][i].copy_(q), s[k + "s"][i].copy_(sc)
        else:
            s["m"][i].copy_(m), s["v"][i].copy_(v)
    for i in range(len(s["g"])):
        one(i)
    return norm


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    c, kind = case, case["kind"]
    if kind == "adamw":
        n = float(sum(math.prod(x) for x in _sizes(c)))
        e = (10.0 if c["master"] else 4.0) if c["p"] == "bf16" else 8.0
        state = 16.0 if c["bits"] == 32 else 4.0 + 16.0 / BLOCK
        return {"bytes": n * (e + state + (2.0 if c["g"] == "bf16" else 4.0)), "flops": 16.0 * n}
    e = 2.0 if c["dtype"] == "bf16" else 4.0
    if kind == "loss":
        n = _kept(c)
        per_row = 8.0 + 4.0 + (16.0 if c["loss"] == "policy" else 0.0) + (0.0 if c["rho"] == 1.0 else 4.0)
        return {"bytes": n * (c["V"] * e * (2.0 if c["grad"] else 1.0) + per_row), "flops": n * c["V"] * (8.0 if c["grad"] else 4.0)}
    n, cols = (c["B"] * c["S"], (c["Hq"] + c["Hkv"]) * c["d"]) if kind == "qk_fwd" else (_kept(c), (c["Hq"] + c["Hkv"]) * c["d"])
    tables = 4.0 * c["d"] * min(n, c["table"])
    return {"bytes": n * cols * e * (2.0 if kind == "qk_fwd" else 3.0) + tables + 4.0 * n * (kind == "qk_bwd"),
            "flops": n * cols * (9.0 if kind == "qk_fwd" else 18.0)}


# ---- the same in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    c, gen = case, _gen(seed)
    if c["kind"] == "adamw":
        return _exact_adamw(c, _adamw(c, gen))
    return _exact_loss(c, _loss(c, gen)) if c["kind"] == "loss" else _exact_qk(c, _qk(c, gen))


def _exact_qk(c, s):
    d, h = c["d"], c["d"] // 2
    rows = s["idx"].long() if c["kind"] == "qk_bwd" else torch.arange(c["B"] * c["S"], device=DEV)
    pos = s["positions"].long() if s["positions"] is not None else torch.remainder(rows, c["table"])
    # the rotation of a pair (i, i + d/2) as a product of complex numbers
    turn = torch.complex(s["cos"].double()[pos], s["sin"].double()[pos])[:, None]
    pairs = lambda x: torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous())
    flat = lambda z, like: torch.cat((z.real, z.imag), -1).reshape(like)
    out = []
    for x, g, dy, acc in ((s["q"], s["gq"], s.get("dq"), s.get("dgq")), (s["k"], s["gk"], s.get("dk"), s.get("dgk"))):
        x = x[rows].double().unflatten(1, (-1, d))
        inv = 1.0 / torch.sqrt(torch.sum(x * x, -1, keepdim=True) / d + EPS_N)
        if dy is None:
            out.append(flat(pairs(x * inv * g.double()) * turn, (rows.numel(), -1)))
            continue
        u = flat(pairs(dy.double().unflatten(1, (-1, d))) * turn.conj(), x.shape)
        dg = torch.einsum("nhd,nhd->d", u, x * inv)
        a = u * g.double()
        dx = inv * a - x * inv ** 3 * torch.sum(a * x, -1, keepdim=True) / d
        out.append((dx.reshape(dy.shape), dg if acc is None else dg + acc.double()))
    return tuple(out) if c["kind"] == "qk_fwd" else (out[0][0], out[1][0], out[0][1], out[1][1])


def _exact_loss(c, s):
    V, n = c["V"], s["n"]
    rows = torch.arange(c["rows"], device=DEV) if s["idx"] is None else s["idx"].long()
    lp, loss = torch.zeros(n, dtype=F64, device=DEV), torch.zeros(4, dtype=F64, device=DEV)
    grad = torch.zeros((n, V), dtype=F64, device=DEV) if c["grad"] else None
    step = max(1, (1 << 27) // V)
    for a in range(0, n, step):
        at = rows[a:a + step]
        t = s["targets"][at]
        w = torch.ones(at.numel(), dtype=F64, device=DEV) if c["loss"] == "nll" else s["weight"][at].double()
        use = ((t != -100) & (w > 0)).nonzero().squeeze(1)
        at, t, w = at[use], t[use], w[use] / n
        p = torch.softmax(s["logits"][at].double(), 1)
        l = torch.log(p[torch.arange(at.numel(), device=DEV), t])
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
        if grad is not None:
            p.neg_()
            p[torch.arange(at.numel(), device=DEV), t] += 1.0
            grad[a + use] = p * (w * slope)[:, None]
    return loss, lp, grad


def _exact_adamw(c, s):
    t, out = s["step"], {k: [] for k in ("p", "master", "m", "v", "ms", "vs")}
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in s["g"]))
    clip = min(1.0, MAX_NORM / (norm + 1e-6))
    for i, g in enumerate(s["g"]):
        g = g.double() * clip
        w = (s["master"][i] if c["master"] else s["p"][i]).double()
        if c["bits"] == 8:
            at = torch.arange(g.numel(), device=DEV).view(g.shape) // BLOCK
            m, r = s["m"][i].double() * s["ms"][i].double()[at], s["v"][i].double() * s["vs"][i].double()[at]
            v = r * r
        else:
            m, v = s["m"][i].double(), s["v"][i].double()
        m, v = m + (g - m) * (1.0 - B1), v + (g * g - v) * (1.0 - B2)
        w = w - LR * WD * w - LR * (m / (1.0 - B1 ** t)) / (torch.sqrt(v / (1.0 - B2 ** t)) + EPS)
        out["p"].append(w)
        if c["master"]:
            out["master"].append(w)
        if c["bits"] == 32:
            out["m"].append(m), out["v"].append(v)
            continue
        for k, x in (("m", m), ("v", torch.sqrt(v))):       # what is rounded to 8 bits, in units of its block's scale
            n, x = x.numel(), x.reshape(-1)
            x = torch.cat((x, x.new_zeros(-n % BLOCK))).view(-1, BLOCK)
            scale = x.abs().amax(1).clamp(min=2.0 ** -100) / 448.0
            out[k].append((x / scale[:, None]).view(-1)[:n].view(g.shape)), out[k + "s"].append(scale)
    return out | {"norm": torch.tensor([norm], dtype=F64, device=DEV)}
