"""What stands at the ends of the stack of layers in a training step: token embeddings with their gradient, the norm of rows with its gradients, the loss
straight from the head's input.  Each against a plain implementation in 64 bits, whose own gradients are pinned by differences.

Tolerances count roundings: a stored value is off by half a step of its type (EPS: half of finfo.eps, relative), an fp32 sum of n
terms by (its depth, at most n) * 2^-24 of the sum of their absolute values, a function of the hardware or the library by a few 2^-24."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2502_00340_amd import binding as Bn
from tests import harness as Hn
from tests.test_step_ops import BF, DEV, EPS, EPS_N, F32, F64, FAKE, U, _layer_qk_device, _layer_qk_problem, close, gen, gpu, loss_ref, qk_ref, randn, say


@pytest.fixture(scope="module")
def L():
    import os
    if not os.path.exists(Bn.LIB_PATH):
        from paper_2502_00340_amd import build
        build.build_library(verbose=False)
    return Bn.lib()


# ---- plain forms in 64 bits --------------------------------------------------------------------------------

def norm_ref(x, g, b, eps, layer):
    x = x.to(F64)
    mu = x.mean(1, keepdim=True) if layer else torch.zeros((), dtype=F64, device=x.device)
    n = (x - mu) / ((x - mu).square().mean(1, keepdim=True) + eps).sqrt()
    return n * g.to(F64) + (b.to(F64) if b is not None else 0.0)


def norm_ref_bwd(x, g, dy, eps, layer):
    """dx, dg, db and the absolute sums that bound their rounding."""
    x, g, dy = x.to(F64), g.to(F64), dy.to(F64)
    mu = x.mean(1, keepdim=True) if layer else torch.zeros((), dtype=F64, device=x.device)
    r = 1.0 / ((x - mu).square().mean(1, keepdim=True) + eps).sqrt()
    n, u = (x - mu) * r, dy * g
    dx = r * (u - n * (u * n).mean(1, keepdim=True) - (u.mean(1, keepdim=True) if layer else 0.0))
    big = r * (u.abs() + n.abs() * (u * n).abs().mean(1, keepdim=True) + (u.abs().mean(1, keepdim=True) if layer else 0.0))
    return dx, (dy * n).sum(0), dy.sum(0), big, (dy * n).abs().sum(0), dy.abs().sum(0)


def embed_ref_bwd(tokens, dx, V, scale, main=None):
    """The gradient and the absolute values of its terms, summed."""
    live = (tokens >= 0) & (tokens < V)
    d = dx[live].to(F64) * scale
    out = torch.zeros((V, dx.shape[1]), dtype=F64, device=dx.device).index_add_(0, tokens[live], d)
    mag = torch.zeros_like(out).index_add_(0, tokens[live], d.abs())
    return (out if main is None else out + main.to(F64)), mag


def head_ref(x, table, y, policy=None, w=None, scale=1.0, norm=0.0):
    """(stats, logp, dx, dtable, d, coef): loss_ref behind the product, and the gradients towards its operands."""
    x, t = x.to(F64), table.to(F64)
    dead = (y < 0) | (y >= t.shape[0])
    if w is not None:
        dead = dead | (w == 0)
    x = torch.where(dead[:, None], torch.zeros((), dtype=F64, device=x.device), x)       # whatever such a row holds
    stats, lp, d, coef = loss_ref(x @ t.T, y, policy, w, scale, norm)
    return stats, lp, d @ t, d.T @ x, d, coef


# ---- the plain forms' gradients against differences (CPU) ---------------------------------------------------

def _differences(f, ts, grads, h=1e-5, tol=1e-7):
    for k, (t, grad) in enumerate(zip(ts, grads)):
        for i in range(t.numel()):
            e = torch.zeros(t.numel(), dtype=F64)
            e[i] = h
            moved = [[u + s * e.view(t.shape) if j == k else u for j, u in enumerate(ts)] for s in (1.0, -1.0)]
            assert abs(float(f(*moved[0]) - f(*moved[1])) / (2 * h) - float(grad.reshape(-1)[i])) < tol


@pytest.mark.parametrize("layer", [False, True])
def test_norm_reference_gradients_against_differences(layer):
    g0 = gen(1)
    x, g, b, dy = (randn(g0, *s, dtype=F64, device="cpu") for s in ((4, 6), (6,), (6,), (4, 6)))
    dx, dg, db = norm_ref_bwd(x, g, dy, 1e-3, layer)[:3]
    f = lambda x_, g_, b_: (norm_ref(x_, g_, b_, 1e-3, layer) * dy).sum()
    _differences(f, (x, g, b), (dx, dg, db))


@pytest.mark.parametrize("policy", [False, True])
def test_head_reference_gradients_against_differences(policy):
    g0, n, H, V = gen(2), 5, 4, 6
    x, t = randn(g0, n, H, dtype=F64, device="cpu"), randn(g0, V, H, dtype=F64, device="cpu")
    y, w = torch.tensor([1, 5, -1, 0, 2]), torch.tensor([1.0, 0.5, 1.0, 0.0, 2.0], dtype=F64)
    pol = None
    if policy:
        lp = loss_ref(x @ t.T, y)[1]
        pol = (lp - torch.tensor([0.1, 0.6, 0.0, 0.2, -0.5], dtype=F64), randn(g0, n, dtype=F64, device="cpu"), lp + 0.2, 0.2, 0.3, 0.1)
    _, _, dx, dt, _, _ = head_ref(x, t, y, pol, w, 1.3)
    _differences(lambda x_, t_: head_ref(x_, t_, y, pol, w, 1.3)[0][0], (x, t), (dx, dt))


def test_embedding_reference_gradient_against_differences():
    g0 = gen(3)
    e, dy, tok = randn(g0, 5, 3, dtype=F64, device="cpu"), randn(g0, 6, 3, dtype=F64, device="cpu"), torch.tensor([0, 4, 0, -1, 7, 2])
    live = (tok >= 0) & (tok < 5)
    _differences(lambda e_: (2.0 * e_[tok[live]] * dy[live]).sum(), (e,), (embed_ref_bwd(tok, dy, 5, 2.0)[0],))


# ---- refusals (CPU) ----------------------------------------------------------------------------------------

def test_embedding_refusals(L):
    f = lambda table=FAKE, V=10, H=16, dt=0, tok=FAKE, n=4, s=1.0, out=2 * FAKE: L.cf_embed_fwd(table, V, H, dt, tok, n, s, out, None)
    assert f(table=None) == f(tok=None) == f(out=None) == 1
    assert f(dt=2) == 3
    assert f(V=0) == f(V=(1 << 30) + 1) == f(H=0) == f(H=12) == f(H=-8) == f(n=-1) == f(n=1 << 60) == 2
    assert f(s=math.inf) == f(s=math.nan) == f(table=FAKE + 2) == f(out=FAKE + 8) == f(tok=FAKE + 4) == f(dt=1, H=6) == 2
    assert f(out=FAKE + 32) == f(out=FAKE) == 2             # overlaps
    assert f(n=0) == 0
    need = L.cf_embed_bwd_workspace_bytes
    assert need(0, 4) == need(16, -1) == need(1 << 21, 4) == need(16, (1 << 30) + 1) == 0
    assert need(16, 0) > 0 and need(16, 8192) < need(16, 8193)
    b = lambda tok=FAKE, dx=FAKE, V=10, H=16, dt=0, idx=None, nd=None, n=4, s=1.0, out=2 * FAKE, main=0, ws=FAKE, wsb=1 << 20: \
        L.cf_embed_bwd(tok, dx, V, H, dt, idx, nd, n, s, out, main, ws, wsb, None)
    assert b(tok=None) == b(dx=None) == b(out=None) == 1
    assert b(dt=-1) == 3
    assert b(V=0) == b(H=4) == b(n=-1) == b(n=(1 << 30) + 1) == b(main=2) == b(s=math.inf) == b(idx=FAKE + 2) == b(nd=FAKE + 1) == b(dx=FAKE + 4) == 2
    assert b(out=FAKE + 64) == b(dx=2 * FAKE + 304) == 2 and b(dx=2 * FAKE + 320, main=1, ws=None) == 2
    assert b(ws=None) == b(ws=FAKE + 16) == b(wsb=need(16, 4) - 1) == 4


def test_norm_refusals(L):
    D = lambda H=16, dt=0, layer=0, eps=1e-5: C.byref(Bn.NormDesc(H, dt, layer, eps))
    f = lambda d=D(), x=FAKE, g=FAKE, b=None, idx=None, nd=None, n=4, y=2 * FAKE: L.cf_norm_fwd(d, x, g, b, idx, nd, n, y, None)
    assert f(d=None) == f(x=None) == f(g=None) == f(y=None) == 1
    assert f(d=D(dt=3)) == 3
    assert f(d=D(H=0)) == f(d=D(H=12)) == f(d=D(layer=2)) == f(d=D(eps=-1.0)) == f(d=D(eps=math.nan)) == f(d=D(eps=math.inf)) == 2
    assert f(n=-1) == f(b=FAKE) == f(x=FAKE + 8) == f(y=FAKE + 32) == f(idx=FAKE + 2) == f(x=FAKE, y=FAKE, idx=FAKE) == 2
    assert f(d=D(H=32776)) == f(d=D(H=16388, dt=1)) == 5
    assert f(n=0) == 0
    need = L.cf_norm_bwd_workspace_bytes
    assert need(D(H=12), 4) == need(D(), -1) == need(D(H=32776), 4) == 0
    assert need(D(layer=1), 4096) == 2 * need(D(), 4096) > 0
    b = lambda d=D(), x=FAKE, g=FAKE, dy=2 * FAKE, idx=None, nd=None, n=4, dx=3 * FAKE, dg=FAKE, db=None, main=0, ws=FAKE, wsb=1 << 20: \
        L.cf_norm_bwd(d, x, g, dy, idx, nd, n, dx, dg, db, main, ws, wsb, None)
    assert b(d=None) == b(x=None) == b(g=None) == b(dy=None) == b(dx=None) == 1
    assert b(db=FAKE) == b(d=D(layer=1), dg=None, db=FAKE) == b(main=-1) == b(dx=2 * FAKE + 64) == b(dx=FAKE, idx=FAKE) == b(dx=FAKE + 64) == 2
    assert b(d=D(layer=1), db=FAKE + 16) == b(dg=3 * FAKE + 96) == 2
    assert b(dg=FAKE + 4) == b(nd=FAKE + 2) == b(n=(1 << 30) + 1) == 2
    assert b(ws=None) == b(ws=FAKE + 128) == b(wsb=need(D(), 4) - 1) == 4


def test_head_loss_refusals(L):
    T = lambda kind=0, V=300, dt=0, s=1.0, lo=0.2, hi=0.2, kl=0.0, norm=0.0: C.byref(Bn.LossDesc(kind, V, dt, s, lo, hi, kl, norm))
    need = L.cf_head_loss_workspace_bytes
    f = lambda d=T(), H=16, x=FAKE, t=8 * FAKE, y=FAKE, old=None, ref=None, adv=None, w=None, idx=None, nd=None, n=4, dx=2 * FAKE, dt=16 * FAKE, main=0, lp=FAKE, \
        st=FAKE, ws=FAKE, wsb=1 << 30: L.cf_head_loss(d, H, x, t, y, old, ref, adv, w, idx, nd, n, dx, dt, main, lp, st, ws, wsb, None)
    assert f(d=None) == f(x=None) == f(t=None) == f(y=None) == f(dx=None, dt=None, lp=None, st=None) == 1
    assert f(d=T(kind=1)) == f(d=T(kind=1), old=FAKE) == 1
    assert f(d=T(dt=2)) == 3
    assert f(d=T(kind=2)) == f(d=T(V=0)) == f(d=T(V=(1 << 30) + 1)) == f(d=T(s=-1.0)) == f(d=T(s=3e38)) == f(d=T(norm=math.inf)) == 2
    assert f(H=0) == f(H=12) == f(n=-1) == f(n=(1 << 30) + 1) == f(main=2) == f(x=FAKE + 8) == f(y=FAKE + 4) == f(lp=FAKE + 2) == f(dt=FAKE + 4) == 2
    assert f(dx=FAKE + 64) == f(dx=8 * FAKE) == f(dt=8 * FAKE + 1600) == f(dt=FAKE) == f(dt=2 * FAKE) == 2        # overlaps
    assert f(d=T(kind=1, lo=1.5), old=FAKE, adv=FAKE) == f(d=T(kind=1, kl=0.1), old=FAKE, adv=FAKE) == 2
    assert f(n=1 << 27) == f(n=(1 << 22) + 1) == f(d=T(V=1 << 30), n=1 << 20) == f(H=1 << 21) == 5
    assert f(ws=None) == f(ws=FAKE + 64) == f(wsb=need(T(), 16, 4, 1, 1, 0) - 1) == 4
    assert need(T(), 12, 4, 1, 1, 0) == need(T(V=0), 16, 4, 1, 1, 0) == need(T(), 16, 1 << 27, 1, 1, 0) == 0
    # as much as is of use, at most the limit, never less than will do
    big = T(V=100000)
    least, most = need(big, 16, 4096, 1, 1, 0), need(big, 16, 4096, 1, 1, 1 << 40)
    assert need(big, 16, 4096, 0, 0, 1 << 40) < least < most < 1 << 30
    mid = (least + most) // 2
    assert mid - 4096 * 512 - 256 <= need(big, 16, 4096, 1, 1, mid) <= mid


def test_binding_refuses_what_the_library_cannot_see(L):
    z = lambda *s, dt=F32: torch.zeros(s, dtype=dt)
    i64, i32 = torch.int64, torch.int32
    bad = [
        lambda: Bn.embed_fwd(z(4, 8).T, z(3, dt=i64)),
        lambda: Bn.embed_fwd(z(4, 8), z(3, dt=i32)),
        lambda: Bn.embed_fwd(z(4, 8), z(3, dt=i64), out=z(3, 4)),
        lambda: Bn.embed_fwd(z(4, 8), z(3, dt=i64)),                                             # not on a GPU
        lambda: Bn.embed_bwd(z(3, dt=i64), z(4, 8), 10),                                         # more rows than tokens
        lambda: Bn.embed_bwd(z(9, dt=i64), z(4, 8), 10, idx=z(3, dt=i32)),
        lambda: Bn.embed_bwd(z(9, dt=i64), z(4, 8), 10, idx=z(4, dt=i64)),
        lambda: Bn.embed_bwd(z(4, dt=i64), z(4, 8), 10, main_grad=z(10, 8, dt=BF)),
        lambda: Bn.embed_bwd(z(4, dt=i64), z(4, 8), 10, main_grad=z(9, 8)),
        lambda: Bn.embed_bwd(z(4, dt=i64), z(4, 16)[:, :8], 10),
        lambda: Bn.norm_fwd(z(4, 8), z(4)),
        lambda: Bn.norm_fwd(z(4, 8), z(8), z(8)),                                                # biases without layer
        lambda: Bn.norm_fwd(z(4, 8), z(8, dt=BF)),
        lambda: Bn.norm_fwd(z(4, 8), z(8), max_kept=5),
        lambda: Bn.norm_bwd(z(4, 8), z(8), z(5, 8)),
        lambda: Bn.norm_bwd(z(4, 8), z(8), z(4, 8, dt=BF)),
        lambda: Bn.norm_bwd(z(4, 8), z(8), z(4, 8), main_grads=(z(8, dt=BF), None)),
        lambda: Bn.norm_bwd(z(4, 8), z(8), z(4, 8), main_grads=(z(8), z(8))),
        lambda: Bn.head_loss(z(4, 8), z(6, 9), z(4, dt=i64)),
        lambda: Bn.head_loss(z(4, 8), z(6, 8, dt=BF), z(4, dt=i64)),
        lambda: Bn.head_loss(z(4, 8), z(6, 8), z(3, dt=i64)),
        lambda: Bn.head_loss(z(4, 8), z(6, 8), z(4, dt=i32)),
        lambda: Bn.head_loss(z(4, 8), z(6, 8), z(4, dt=i64), old_logp=z(4)),
        lambda: Bn.head_loss(z(4, 8), z(6, 8), z(4, dt=i64), advantages=z(3), old_logp=z(4)),
        lambda: Bn.head_loss(z(4, 8), z(6, 8), z(4, dt=i64), main_grad=z(6, 8, dt=BF)),
        lambda: Bn.head_loss(z(4, 8), z(6, 8), z(9, dt=i64), idx=z(3, dt=i32)),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()


# ---- embeddings --------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,V,H", [(1, 1, 8), (16, 300, 4096), (7, 11, 24), (1001, 50257, 840), (3, 40, 8200)])
def test_embedding_forward(dtype, n, V, H):
    say("embed_fwd", dtype, n, V, H)
    g0 = gen(n + H)
    table = randn(g0, V, H, dtype=dtype)
    tok = torch.randint(-1, V + 1, (n,), generator=g0).to(DEV)
    live = ((tok >= 0) & (tok < V))[:, None]
    zero = torch.zeros((), dtype=F64, device=DEV)
    for scale in (1.0, math.sqrt(H)):
        want = torch.where(live, table.to(F64)[tok.clamp(0, V - 1)] * scale, zero)
        got = Bn.embed_fwd(table, tok, scale=scale)
        assert got.dtype is dtype
        close(got, want, (0.0 if scale == 1.0 else EPS[dtype] + 2 * U) * want.abs(), "y")       # the factor itself is rounded to fp32
    out = torch.full((2, n, H), 7.0, dtype=dtype, device=DEV)
    assert Bn.embed_fwd(table, torch.stack((tok, tok.flip(0))), out=out) is out
    assert torch.equal(out[0], out[1].flip(0))
    assert Bn.embed_fwd(table, tok[:0]).shape == (0, H)


# (rows, V, H): one row; rows around a chunk of 8 and a span of 8192; few tokens (long runs); more bits than two passes
EMBED = [(1, 1, 8), (7, 3, 24), (8, 300, 520), (9, 2, 1024), (130, 1, 40), (256, 90, 2056), (257, 90, 2056), (1000, 50257, 840), (8192, 37, 16), (8193, 5000, 24), (20011, 300, 136),
         (500, 1 << 19, 8), (3000, 128256, 2056)]


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,V,H", EMBED)
@pytest.mark.parametrize("main", [False, True])
def test_embedding_backward(dtype, n, V, H, main):
    say("embed_bwd", dtype, n, V, H, main)
    g0 = gen(n + V)
    T = n + n // 3 + 1
    tok = (torch.rand(T, generator=g0) ** 3 * (V + 1)).long().to(DEV) - (torch.rand(T, generator=g0) < 0.05).long().to(DEV) * (V + 5)      # some outside [0, V)
    dx = randn(g0, n, H, dtype=dtype)
    idx = torch.randperm(T, generator=g0)[:n].to(torch.int32).to(DEV)          # any order
    kept = tok[idx.long()]
    dx[(kept < 0) | (kept >= V)] = float("nan")            # counts for nothing
    grad = randn(g0, V, H) if main else None
    before = grad.clone() if main else None
    want, mag = embed_ref_bwd(kept, dx, V, 1.7, before)
    got = Bn.embed_bwd(tok, dx, V, scale=1.7, idx=idx, main_grad=grad)
    count = torch.bincount(kept[(kept >= 0) & (kept < V)], minlength=V).to(F64)[:, None]
    # the sum, times a factor that is itself rounded; added to the old value, or rounded to the type
    tol = mag * U * (count + 4) + want.abs() * (U if main else EPS[dtype])
    close(got, want, tol, "dE")
    if main:
        rest = (count == 0).squeeze(1)
        assert torch.equal(got[rest], before[rest])
        again = Bn.embed_bwd(tok, dx, V, scale=1.7, idx=idx, main_grad=before.clone())
    else:
        again = Bn.embed_bwd(tok, dx, V, scale=1.7, idx=idx, out=torch.full((V, H), float("nan"), dtype=dtype, device=DEV))
    assert torch.equal(got, again)


@gpu
@pytest.mark.parametrize("main", [False, True])
def test_embedding_backward_with_the_count_on_the_device(main):
    g0, V, H, n = gen(5), 50, 264, 9000
    tok, dx = torch.randint(0, V, (n,), generator=g0).to(DEV), randn(g0, n, H, dtype=BF)
    for live in (0, 1, 8, 200, 256, 1500, 8192, 8200, n, n + 7):
        say("embed_bwd count", live)
        m = min(live, n)
        grad = randn(g0, V, H) if main else None
        want, mag = embed_ref_bwd(tok[:m], dx[:m], V, 1.0, grad)
        dev = torch.tensor([live], dtype=torch.int32, device=DEV)
        got = Bn.embed_bwd(tok, dx, V, n_kept_dev=dev, main_grad=grad.clone() if main else None)
        close(got, want, mag * U * (m + 2) + want.abs() * (U if main else EPS[BF]), "dE of %d rows" % live)
        if m > 256:             # fewer, known to the host, are added up in one pass
            known = Bn.embed_bwd(tok, dx[:m].contiguous(), V, main_grad=grad.clone() if main else None)
            assert torch.equal(got, known)
    assert Bn.embed_bwd(tok, dx[:0], V).eq(0).all()
    for live in (0, 3, 40):
        dev = torch.tensor([live], dtype=torch.int32, device=DEV)
        got = Bn.embed_bwd(tok, dx[:40].contiguous(), V, n_kept_dev=dev)
        want, mag = embed_ref_bwd(tok[:live], dx[:live], V, 1.0)
        close(got, want, mag * U * (live + 2) + want.abs() * EPS[BF], "dE of %d of 40 rows" % live)


# ---- norm --------------------------------------------------------------------------------------------------

# rows and widths around a wave's four vectors, a block's four, a block of 1024's; in bf16 (halved in fp32)
NORM = [(1, 8), (5, 24), (33, 504), (300, 512), (70, 2040), (70, 2056), (1500, 4096), (41, 8192), (9, 8200), (3, 16392), (2, 32768), (2100, 840)]


def _norm_case(dtype, n, H, mean=0.3):
    g0 = gen(n + H)
    T = n + n // 2
    x = randn(g0, T, H, std=1.5, mean=mean, dtype=dtype)
    g, b, dy = randn(g0, H, std=0.3, mean=1.0, dtype=dtype), randn(g0, H, std=0.3, dtype=dtype), randn(g0, n, H, dtype=dtype)
    idx = torch.randperm(T, generator=g0)[:n].sort().values.to(torch.int32).to(DEV)
    return x, g, b, dy, idx, g0


def _norm_rounding(x, H, layer):
    """Relative error of n beyond its formula's condition: the sums of H terms (depth at most H / 64 + 12: a lane's terms, its wave, the waves), a root, a few products;
    and how far rounding the mean moves x - mu against the row's spread."""
    depth = H / 64 + 12
    xd = x.to(F64)
    mu = xd.mean(1, keepdim=True) if layer else torch.zeros((), dtype=F64, device=x.device)
    spread = (xd - mu).square().mean(1, keepdim=True).sqrt()
    moved = (depth * U * xd.abs().mean(1, keepdim=True) + U * xd.abs()) / spread if layer else torch.zeros((), dtype=F64, device=x.device)
    return (depth + 8) * U, moved


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,H", NORM)
@pytest.mark.parametrize("layer", [False, True])
def test_norm_forward(dtype, n, H, layer):
    H = H if dtype is BF else H // 2
    say("norm_fwd", dtype, n, H, layer)
    x, g, b, _, idx, _ = _norm_case(dtype, n, H)
    b = b if layer else None
    for i in (idx, None):
        rows = x if i is None else x[i.long()]
        want = norm_ref(rows, g, b, 1e-5, layer)
        rel, moved = _norm_rounding(rows, H, layer)
        bias = torch.zeros((), dtype=F64, device=DEV) if b is None else b.to(F64)
        ng = want - bias
        tol = want.abs() * (EPS[dtype] + U) + ng.abs() * rel + (moved + ng.abs() * moved.mean()) * g.to(F64).abs() * 2 + bias.abs() * U
        close(Bn.norm_fwd(x, g, b, eps=1e-5, layer=layer, idx=i), want, tol, "y")
    y = Bn.norm_fwd(x, g, b, layer=layer)
    x2 = x.clone()
    assert Bn.norm_fwd(x2, g, b, layer=layer, out=x2) is x2 and torch.equal(x2, y)
    if layer:
        assert torch.equal(Bn.norm_fwd(x, g, None, layer=True), Bn.norm_fwd(x, g, torch.zeros_like(b), layer=True))


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,H", NORM)
@pytest.mark.parametrize("layer", [False, True])
def test_norm_backward(dtype, n, H, layer):
    H = H if dtype is BF else H // 2
    say("norm_bwd", dtype, n, H, layer)
    x, g, _, dy, idx, g0 = _norm_case(dtype, n, H)
    rows = x[idx.long()]
    dx, dg, db, big, gmag, bmag = norm_ref_bwd(rows, g, dy, 1e-5, layer)
    rel, moved = _norm_rounding(rows, H, layer)
    tol = dx.abs() * EPS[dtype] + big * 4 * rel + big.mean(1, keepdim=True) * 4 * moved + big * 4 * moved.mean()
    # gains: n's own error in each term, then a sum of n rows
    gtol = gmag * (rel + (n + 8) * U) + 2 * (dy.to(F64).abs() * moved).sum(0) + 2 * gmag * moved.mean()
    btol = bmag * (n + 8) * U
    got = Bn.norm_bwd(x, g, dy, eps=1e-5, layer=layer, idx=idx)
    close(got[0], dx, tol, "dx")
    close(got[1], dg, gtol + dg.abs() * EPS[dtype], "dg")
    assert (got[2] is None) != layer
    if layer:
        close(got[2], db, btol + db.abs() * EPS[dtype], "db")
    main = randn(g0, H, std=20.0), randn(g0, H, std=20.0) if layer else None
    start = [None if t is None else t.clone() for t in main]
    # in place, into fp32 gradients
    dy2 = dy.clone()
    got2 = Bn.norm_bwd(x, g, dy2, eps=1e-5, layer=layer, idx=idx, main_grads=main, out=dy2)
    assert got2[0] is dy2 and torch.equal(dy2, got[0]) and got2[1] is main[0]
    close(main[0], start[0].to(F64) + dg, gtol + (start[0].to(F64) + dg).abs() * U, "dg added")
    if layer:
        close(main[1], start[1].to(F64) + db, btol + (start[1].to(F64) + db).abs() * U, "db added")
    frozen = Bn.norm_bwd(x, g, dy, eps=1e-5, layer=layer, idx=idx, need_gains=False)
    assert frozen[1] is None and frozen[2] is None and torch.equal(frozen[0], got[0])
    if n > 1:           # without idx, dx over x
        x2 = x[:n].clone()
        want = Bn.norm_bwd(x[:n].contiguous(), g, dy, layer=layer)[0]
        assert torch.equal(Bn.norm_bwd(x2, g, dy, layer=layer, out=x2)[0], want)


@gpu
@pytest.mark.parametrize("H", [512, 4096, 16384])
def test_norm_with_the_count_on_the_device(H):
    x, g, b, dy, idx, g0 = _norm_case(BF, 3000, H)
    for live in (0, 1, 5, 2049, 3000, 3005):
        m = min(live, 3000)
        dev = torch.tensor([live], dtype=torch.int32, device=DEV)
        y = torch.full((3000, H), 7.0, dtype=BF, device=DEV)
        Bn.norm_fwd(x, g, b, layer=True, idx=idx, n_kept_dev=dev, out=y)
        assert y[m:].eq(7.0).all() and torch.equal(y[:m], Bn.norm_fwd(x, g, b, layer=True, idx=idx[:m].contiguous()) if m else y[:0])
        out = torch.full((3000, H), 7.0, dtype=BF, device=DEV)
        _, dg, db = Bn.norm_bwd(x, g, dy, layer=True, idx=idx, n_kept_dev=dev, out=out)
        want = Bn.norm_bwd(x, g, dy[:m].contiguous(), layer=True, idx=idx)
        assert out[m:].eq(7.0).all() and torch.equal(out[:m], want[0]) and torch.equal(dg, want[1]) and torch.equal(db, want[2])
        if m == 0:
            assert dg.eq(0).all() and db.eq(0).all()


@gpu
def test_layer_norm_of_rows_far_from_zero():
    """The mean is taken off before anything is squared."""
    g0, n, H = gen(11), 20, 1024
    x = randn(g0, n, H, std=1.0, mean=1000.0)
    g = torch.ones(H, device=DEV)
    rel, moved = _norm_rounding(x, H, True)
    want = norm_ref(x, g, None, 1e-5, True)
    close(Bn.norm_fwd(x, g, layer=True), want, want.abs() * (rel + 2 * U) + 2 * moved + want.abs() * 2 * moved.mean(), "y")


# ---- loss from the head's input ----------------------------------------------------------------------------

def _head_case(seed, dtype, n, H, V, rows=None):
    """x [n, H] whose target's logit stands out, table, targets [rows] and an index; some targets outside [0, V)."""
    g0 = gen(seed)
    rows = n if rows is None else rows
    table = randn(g0, V, H, std=2.0 / math.sqrt(H), dtype=dtype)
    y = torch.randint(0, V, (rows,), generator=g0).to(DEV)
    idx = None if rows == n else torch.randperm(rows, generator=g0)[:n].sort().values.to(torch.int32).to(DEV)
    at = y if idx is None else y[idx.long()]
    x = (randn(g0, n, H) + table[at].float() * randn(g0, n, 1, std=0.3, mean=1.0)).to(dtype)
    if n > 4:
        y[(torch.rand(rows, generator=g0) < 0.05).to(DEV)] = -100
    return x, table, y, idx, g0


def _head_policy(g0, x, table, y, idx, rows, scale=1.0):
    at = torch.arange(rows, device=DEV) if idx is None else idx.long()
    lp = loss_ref(x.to(F64) @ table.to(F64).T, y[at], scale=scale)[1]
    ratio = randn(g0, lp.numel(), std=0.25).to(F64)
    for border in (math.log(0.8), math.log(1.28)):          # no ratio close to where the gradient jumps
        ratio = torch.where((ratio - border).abs() < 2e-3, ratio + 8e-3, ratio)
    old, ref = torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV)
    old[at], ref[at] = (lp - ratio).to(F32), (lp + randn(g0, lp.numel(), std=0.3).to(F64)).to(F32)
    w = torch.rand(rows, generator=g0).to(DEV) + 0.5
    if rows > 8:
        w[3] = 0.0
    return old, randn(g0, rows), ref, w


def _head_check(got, x, table, y, dtype, policy=None, w=None, scale=1.0, norm=0.0, main=None):
    stats, lp, dx, dt, d, coef = head_ref(x, table, y, policy, w, scale, norm)
    n, V, H = x.shape[0], table.shape[0], x.shape[1]
    dead = (y < 0) | (y >= V)
    if w is not None:
        dead = dead | (w == 0)
    ax = torch.where(dead[:, None], torch.zeros((), dtype=F64, device=DEV), x.to(F64)).abs()
    at = table.to(F64).abs()
    # a logit, a sum of H products: its own error and that of the reference, then exponentials and their sum
    big = (ax @ at.T).max(1).values * scale
    dlp = (2 * H + 8) * U * big + (32 + lp.abs() * 4 + math.log2(V + 1)) * U
    if policy is not None:      # old and ref are fp32 values: exact as given; exp(lp - old) moves by its argument's error
        slope = 1.0 + (lp - policy[0].to(F64)).exp() * policy[1].to(F64).abs()
    else:
        slope = torch.ones_like(lp)
    close(got[1], lp, dlp, "logp")
    by = norm if norm else float(n)
    ww = torch.ones(n, dtype=F64, device=DEV) if w is None else w.to(F64)
    kl = 0.0 if policy is None else abs(policy[5])
    moved = (ww.abs() * dlp * slope * (1.0 + kl) * 4).sum() / by + 16 * U * (1.0 + kl)
    close(got[0][:2], stats[:2], moved + stats[:2].abs() * 8 * U, "stats")
    if got[2] is None and got[3] is None:
        return
    # an element of dlogits: its exponential, the row's factor (times a ratio that moves with lp); e and the scaled input are rounded
    rel = 4 * dlp * (1.0 + slope * 0) + 64 * U
    cw = (ww.abs() / by * scale)[:, None]
    extra = cw * (dlp * slope * 4)[:, None]                 # what moves the row's coefficient as a whole
    p = torch.softmax(torch.where(dead[:, None], torch.zeros((), dtype=F64, device=DEV), x.to(F64)) @ table.to(F64).T * scale, 1)
    hot = torch.zeros_like(p)
    ok = (~dead).nonzero().squeeze(1)
    hot[ok, y[ok]] = 1.0
    shape = torch.where(dead[:, None], torch.zeros((), dtype=F64, device=DEV), (p - hot).abs())
    err = d.abs() * rel[:, None] + extra * shape + cw * p * (dlp * slope)[:, None] * ~dead[:, None]
    # bf16: the target's e is exact, with its rounding taken over by the row's factor, so that the other columns have two: that one and their own
    re = torch.where(hot > 0, 0.0, 2 * EPS[dtype]) if dtype is BF else EPS[dtype]
    if got[2] is not None:
        # below 2^-126, the smallest normal number of both types, a stored e (times a factor of at most cw and its row of the table) or a result may be 0
        tol = (d.abs() * (re + V * U) + err + 2.0 ** -126 * cw) @ at + dx.abs() * EPS[dtype] + 2.0 ** -126
        close(got[2], dx, tol, "dx")
    if got[3] is not None:
        # the same for e (times x) and for a scaled input, times an e of at most 2^58 in each of a strip's columns
        tol = (d.abs() * (re + EPS[dtype] + (n + 4) * U) + err + 2.0 ** -126 * cw).T @ ax + n * 2.0 ** (58 - 126) + 2.0 ** -126
        want = dt if main is None else dt + main.to(F64)
        close(got[3], want, tol + want.abs() * (EPS[dtype] if main is None else U), "dtable")


# one row, one column; rows around 16, 32, 64, 128 and tiles of 256; odd vocabularies; a width of one vector; wide; more columns than a least piece
HEAD = [(1, 8, 1), (1, 64, 300), (3, 16, 7), (1, 1032, 5000), (4, 264, 2100), (13, 1096, 3001), (16, 64, 40000), (17, 40, 999), (33, 72, 130), (64, 256, 1003), (65, 328, 4100), (128, 520, 2500), (129, 840, 2049), (300, 264, 5001), (513, 128, 33000), (257, 1032, 257), (200, 8, 600),
        (140, 24, 5000), (3000, 64, 9)]


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,H,V", HEAD)
@pytest.mark.parametrize("policy", [False, True])
def test_head_loss(dtype, n, H, V, policy):
    say("head", dtype, n, H, V, policy)
    x, table, y, _, g0 = _head_case(n + V, dtype, n, H, V)
    kw, ref = {}, {}
    if policy:
        old, adv, rf, w = _head_policy(g0, x, table, y, None, n)
        kw = dict(old_logp=old, advantages=adv, ref_logp=rf, weights=w, clip=(0.2, 0.28), kl_coef=0.04)
        ref = dict(policy=(old, adv, rf, 0.2, 0.28, 0.04), w=w)
    got = Bn.head_loss(x, table, y, **kw)
    _head_check(got, x, table, y, dtype, **ref)
    # no gradient, either one, and pieces of the least size: the same log probabilities and statistics, bit for bit
    a = Bn.head_loss(x, table, y, need_dx=False, need_dtable=False, **kw)
    b = Bn.head_loss(x, table, y, need_dtable=False, **kw)
    c = Bn.head_loss(x, table, y, need_dx=False, **kw)
    p = Bn.head_loss(x, table, y, ws_limit=0, **kw)
    for o in (a, b, c, p):
        assert torch.equal(o[0], got[0]) and torch.equal(o[1], got[1])
    assert a[2] is None and a[3] is None and torch.equal(b[2], got[2]) and b[3] is None and c[2] is None and torch.equal(c[3], got[3])
    _head_check(p, x, table, y, dtype, **ref)
    again = Bn.head_loss(x, table, y, **kw)
    for s, t in zip(again, got):
        assert torch.equal(s, t)


@gpu
def test_widths_of_four_in_fp32():
    for n, H, V in ((70, 20, 333), (300, 12, 2500)):
        x, table, y, _, g0 = _head_case(n, F32, n, H, V)
        _head_check(Bn.head_loss(x, table, y, ws_limit=0), x, table, y, F32)
        g, dy = randn(g0, H), randn(g0, n, H)
        dx, _, _, big, _, _ = norm_ref_bwd(x, g, dy, 1e-5, False)
        close(Bn.norm_bwd(x, g, dy)[0], dx, dx.abs() * U + big * 80 * U, "dx")
        want, mag = embed_ref_bwd(y, dy, V, 1.0)
        close(Bn.embed_bwd(y, dy, V), want, mag * U * (n + 2) + want.abs() * U, "dE")


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_head_loss_on_kept_rows_into_a_main_gradient(dtype):
    n, H, V, rows = 150, 200, 4500, 401
    x, table, y, idx, g0 = _head_case(5, dtype, n, H, V, rows)
    old, adv, rf, w = _head_policy(g0, x, table, y, idx, rows, 0.7)
    at = idx.long()
    kw = dict(old_logp=old, advantages=adv, ref_logp=rf, weights=w, clip=(0.2, 0.28), kl_coef=0.04, idx=idx, logit_scale=0.7, norm=37.0)
    ref = dict(policy=(old[at], adv[at], rf[at], 0.2, 0.28, 0.04), w=w[at], scale=0.7, norm=37.0)
    for limit in (0, 1 << 30):
        main = randn(g0, V, H)
        start = main.clone()
        x2 = x.clone()
        got = Bn.head_loss(x2, table, y, main_grad=main, dx_out=x2, ws_limit=limit, **kw)
        assert got[2] is x2 and got[3] is main
        _head_check(got, x, table, y[at], dtype, main=start, **ref)


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("limit", [0, 1 << 30])
@pytest.mark.parametrize("n", [12, 100, 600])
def test_head_loss_with_the_count_on_the_device(dtype, limit, n):
    H, V = 72, 3001
    x, table, y, _, g0 = _head_case(6, dtype, n, H, V)
    for live in (0, 1, n // 3, n, n + 9) if n <= 100 else (0, 1, 100, 129, 257, 600, 609):
        say("head count", dtype, live, limit)
        m = min(live, n)
        dev = torch.tensor([live], dtype=torch.int32, device=DEV)
        x2 = x.clone()
        x2[m:] = float("nan")
        dx = torch.full((n, H), 7.0, dtype=dtype, device=DEV)
        got = Bn.head_loss(x2, table, y, n_kept_dev=dev, dx_out=dx, ws_limit=limit)
        assert dx[m:].eq(7.0).all()
        if m == 0:
            assert got[0].eq(0).all() and got[3].eq(0).all()
            continue
        _head_check((got[0], got[1][:m], dx[:m], got[3]), x[:m], table, y[:m], dtype)
    none = Bn.head_loss(x[:0], table, y)
    assert none[0].eq(0).all() and none[1].numel() == 0 and none[2].shape == (0, H) and none[3].eq(0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_head_loss_of_rows_that_are_left_out(dtype):
    """Targets outside [0, V), weights of 0: nothing of such a row counts, NaN and infinities included."""
    n, H, V = 300, 64, 2500
    x, table, y, _, g0 = _head_case(8, dtype, n, H, V)
    w = torch.ones(n, device=DEV)
    y[0:40:4], y[1:41:4], y[2] = -1, V, 1 << 40
    w[3:200:16] = 0.0
    dead = (y < 0) | (y >= V) | (w == 0)
    for few in (16, 9, 1):          # the first rows alone
        got = Bn.head_loss(torch.where(dead[:, None], float("nan"), x)[:few].contiguous(), table, y[:few].contiguous(), weights=w[:few].contiguous())
        _head_check(got, x[:few], table, y[:few], dtype, w=w[:few])
    clean = torch.where(dead[:, None], torch.zeros((), dtype=dtype, device=DEV), x)
    want = Bn.head_loss(clean, table, y, weights=w)
    x[dead] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38], device=DEV, dtype=dtype).repeat(H // 4)
    for limit in (0, 1 << 30):
        got = Bn.head_loss(x, table, y, weights=w, ws_limit=limit)
        _head_check(got, x, table, y, dtype, w=w)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert got[2][dead].eq(0).all() and got[1][dead].eq(0).all()
    allout = Bn.head_loss(x, table, torch.full_like(y, -100))
    assert allout[0].eq(0).all() and allout[2].eq(0).all() and allout[3].eq(0).all()


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("gap", [50.0, 200.0, 5000.0])
@pytest.mark.parametrize("n", [12, 100, 600])
def test_head_loss_of_improbable_targets(dtype, gap, n):
    """Targets whose logit lies far below the row's largest: their exponentials leave the range in which the target is the reference."""
    H, V = 64, 3000
    x, table, y, _, g0 = _head_case(9, dtype, n, H, V)
    z = torch.arange(0, n, 37, device=DEV)              # rows of two of the three row tiles
    z = z[z < 300]
    y[z] = torch.randint(0, V - 1, (z.numel(),), generator=g0).to(DEV)
    x[z] = 0.0
    x[z, 0] = 1.0
    table[:, 0] = 0.0
    table[V - 1, 0] = gap
    for limit in (0, 1 << 30):
        got = Bn.head_loss(x, table, y, ws_limit=limit)
        _head_check(got, x, table, y, dtype)
    assert float(got[1][z].max()) < -0.9 * gap
    # a row with NaN: NaN where the formula has it, and nothing else
    x[5, 3] = float("nan")
    y[5] = 1
    got = Bn.head_loss(x, table, y)
    rest = torch.arange(n, device=DEV) != 5
    assert got[1][5].isnan() and got[1][rest].isfinite().all() and got[2][5].isnan().all() and got[2][rest].isfinite().all() and got[0][0].isnan()


@gpu
def test_head_loss_on_policy_ratio_is_one():
    n, H, V = 200, 128, 5000
    x, table, y, _, g0 = _head_case(10, BF, n, H, V)
    old = Bn.head_loss(x, table, y, need_dx=False, need_dtable=False)[1]
    adv = randn(g0, n)
    got = Bn.head_loss(x, table, y, old_logp=old, advantages=adv)
    live = (y >= 0)
    want = -(torch.where(live, adv, torch.zeros((), device=DEV)).to(F64).sum() / n)
    assert float(got[0][3]) == 0.0 and abs(float(got[0][0]) - float(want)) <= 4 * U * float(adv.abs().sum()) / n


@gpu
def test_head_loss_agrees_with_the_loss_from_logits():
    """The same losses as token_loss gives for the product's logits, in fp32."""
    n, H, V = 90, 64, 1200
    x, table, y, _, g0 = _head_case(12, F32, n, H, V)
    old, adv, rf, w = _head_policy(g0, x, table, y, None, n)
    kw = dict(old_logp=old, advantages=adv, ref_logp=rf, weights=w, clip=(0.2, 0.28), kl_coef=0.04)
    a = Bn.head_loss(x, table, y, **kw)
    logits = (x.to(F64) @ table.to(F64).T).to(F32)
    b = Bn.token_loss(logits, y, **kw)
    big = (x.to(F64).abs() @ table.to(F64).abs().T).max(1).values
    assert bool(((a[1] - b[1]).abs().to(F64) <= (2 * H + 40) * U * big + 64 * U).all())
    assert bool(((a[0] - b[0]).abs() <= 1e-4).all())


# ---- the set together --------------------------------------------------------------------------------------

def _step(tok, y, idx, n, emb, g, b, head, main, dev=None):
    """Embeddings, a layer norm on kept rows, the loss, and back, into main gradients (dE, dg, db, dW)."""
    h = Bn.embed_fwd(emb, tok, scale=2.0)
    z = Bn.norm_fwd(h, g, b, layer=True, idx=idx, max_kept=n, n_kept_dev=dev, out=torch.zeros((n, h.shape[1]), dtype=h.dtype, device=h.device))
    stats, logp, dz, _ = Bn.head_loss(z, head, y, idx=idx, n_kept_dev=dev, main_grad=main[3])
    dh, _, _ = Bn.norm_bwd(h, g, dz, layer=True, idx=idx, n_kept_dev=dev, main_grads=(main[1], main[2]))
    Bn.embed_bwd(tok, dh, emb.shape[0], scale=2.0, idx=idx, n_kept_dev=dev, main_grad=main[0])
    return stats, logp


def _step_case(dtype, tied):
    g0, T, H, V = gen(20), 700, 128, 3000
    tok, y = torch.randint(0, V, (T,), generator=g0).to(DEV), torch.randint(0, V, (T,), generator=g0).to(DEV)
    emb = randn(g0, V, H, std=0.3, dtype=dtype)
    head = emb if tied else randn(g0, V, H, std=0.2, dtype=dtype)
    g, b = randn(g0, H, std=0.2, mean=1.0, dtype=dtype), randn(g0, H, std=0.2, dtype=dtype)
    mask = (torch.rand(2, T // 2, generator=g0) < 0.6).to(torch.uint8).to(DEV)
    return tok, y, mask, emb, g, b, head


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tied", [False, True])
def test_ends_of_a_step_together(dtype, tied):
    """Against autograd in 64 bits: norms of the gradients' differences, a few roundings of the type on the way."""
    tok, y, mask, emb, g, b, head = _step_case(dtype, tied)
    V, H = emb.shape
    idx, _, dev, n = Bn.build_keep_index(mask)
    idx = idx[:n].contiguous()
    main = [torch.zeros(s, device=DEV) for s in ((V, H), (H,), (H,))]
    main.append(main[0] if tied else torch.zeros((V, H), device=DEV))       # a tied table's two gradients share one buffer
    stats, _ = _step(tok, y, idx, n, emb, g, b, head, main)
    leaves = [t.to(F64).requires_grad_() for t in (emb, g, b)]
    w = leaves[0] if tied else head.to(F64).requires_grad_()
    h = leaves[0][tok] * 2.0
    z = torch.nn.functional.layer_norm(h[idx.long()], (H,), leaves[1], leaves[2], 1e-5)
    loss = torch.nn.functional.cross_entropy(z @ w.T, y[idx.long()])
    want = torch.autograd.grad(loss, leaves if tied else leaves + [w])
    # roundings on the way to each gradient: embeddings, norm, e, scaled input, dx of the loss, dx of the norm, each EPS, and its effect on p of a logit of some |z||w|
    tol = {BF: 12 * EPS[BF], F32: 200 * U}[dtype]
    for got, ref in zip(main, want):
        assert float((got.to(F64) - ref).norm()) <= tol * float(ref.norm())
    assert abs(float(stats[0]) - loss.item()) <= tol * loss.item()


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_ends_of_a_step_in_a_graph_and_on_another_stream(dtype):
    """Captured with the count on the device and replayed for other inputs of another count, with eager work in between; twice, so that two graphs live."""
    tok, y, mask, emb, g, b, head = _step_case(dtype, False)
    V, H = emb.shape
    T = tok.numel()
    idx, cu, dev = torch.zeros(T, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    bound = 600

    def work(main):
        Bn.build_keep_index_static(mask, idx, cu, dev)
        return _step(tok, y, idx, bound, emb, g, b, head, main, dev)
    zeros = lambda: [torch.zeros(s, device=DEV) for s in ((V, H), (H,), (H,), (V, H))]
    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        main = zeros()
        with torch.cuda.stream(side):
            work(main)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = work(main)
        graphs.append((gr, main, out))
    g0 = gen(33)
    for turn in range(4):
        tok.copy_(torch.randint(-2, V + 2, (T,), generator=g0))
        y.copy_(torch.randint(0, V, (T,), generator=g0))
        mask.copy_((torch.rand(2, T // 2, generator=g0) < (0.2, 0.5, 0.7, 0.0)[turn]).to(torch.uint8))
        gr, main, out = graphs[turn % 2]
        for t in main:
            t.zero_()
        gr.replay()
        torch.cuda.synchronize()
        eager = zeros()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            stats, logp = work(eager)
        torch.cuda.synchronize()
        n = int(dev)
        assert torch.equal(stats, out[0]) and torch.equal(logp[:n], out[1][:n])
        for s, t in zip(main, eager):
            assert torch.equal(s, t)


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tied", [False, True])
def test_whole_model_step(dtype, tied):
    """Embeddings, a layer, the last norm and the loss, and back into main gradients, with every token kept: the gradients of the whole function, which torch
    differentiates in 64 bits."""
    say("model step", dtype, tied)
    V = 520
    shape, W, sv, tabs, rng = _layer_qk_problem(dtype, seed=41)
    B, S, H, Hq, Hkv, d = shape.B, shape.S, shape.H, shape.Hq, shape.Hkv, shape.d
    T = shape.T
    tok = torch.from_numpy(rng.permutation(V)[:T])                      # the layer's input is given: a row of the table each
    table = Hn.quantize(0.05 * rng.standard_normal((V, H)), shape.dtype)
    table[tok.numpy()] = sv["x"]
    wh = table if tied else Hn.quantize(0.05 * rng.standard_normal((V, H)), shape.dtype)
    gf = Hn.quantize(1.0 + 0.2 * rng.standard_normal(H), shape.dtype)
    y = torch.from_numpy(rng.integers(0, V, T))
    # the whole function in 64 bits
    P = {n: torch.from_numpy(v.astype(np.float64)).requires_grad_() for n, v in {**W, "table": table, "gf": gf}.items()}
    head = P["table"] if tied else torch.from_numpy(wh.astype(np.float64)).requires_grad_()
    rms = lambda x, g: x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * g
    x = P["table"][tok]
    cos, sin, pos = torch.from_numpy(tabs[0]), torch.from_numpy(tabs[1]), torch.arange(T) % S
    h1 = rms(x, P["g1"])
    q, k, v = qk_ref(h1 @ P["wq"], P["gq"], d, EPS_N, cos, sin, pos), qk_ref(h1 @ P["wk"], P["gk"], d, EPS_N, cos, sin, pos), h1 @ P["wv"]
    heads = lambda t, n: t.view(B, S, n, d).transpose(1, 2)
    kk, vv = (heads(t, Hkv).repeat_interleave(Hq // Hkv, 1) for t in (k, v))
    sc = (heads(q, Hq) @ kk.transpose(2, 3) / math.sqrt(d)).masked_fill(torch.triu(torch.ones(S, S, dtype=torch.bool), 1), -math.inf)
    r = x + (torch.softmax(sc, -1) @ vv).transpose(1, 2).reshape(T, -1) @ P["wo"]
    h2 = rms(r, P["g2"])
    out = r + (torch.nn.functional.silu(h2 @ P["wg"]) * (h2 @ P["wu"])) @ P["wd"]
    loss = torch.nn.functional.cross_entropy(rms(out, P["gf"]) @ head.T, y)
    loss.backward()
    # the same through the library
    to = lambda a: Hn.to_dev(a, shape.dtype)
    dsv, dW = _layer_qk_device(shape, W, sv, tabs)
    dtab, dgf, dwh, tok, y = to(table), to(gf), to(wh), tok.to(DEV), y.to(DEV)
    assert torch.equal(Bn.embed_fwd(dtab, tok), dsv["x"])
    top = to(Hn.quantize(out.detach().numpy(), shape.dtype))
    idx, cu, nd, n = Bn.build_keep_index(torch.ones((B, S), dtype=torch.uint8, device=DEV))
    plan = Bn.LayerBackward(Bn.make_desc(B, S, H, Hq, Hkv, d, shape.F, shape.dtype), main_grad=True, qk_norm_eps=EPS_N)
    z = lambda *s: torch.zeros(s, device=DEV)
    gtab, ggf = z(V, H), z(H)
    gwh = gtab if tied else z(V, H)
    hz = Bn.norm_fwd(top, dgf, idx=idx, n_kept_dev=nd)
    stats, _, dz, _ = Bn.head_loss(hz, dwh, y, idx=idx, n_kept_dev=nd, main_grad=gwh, dx_out=hz)
    dy, _, _ = Bn.norm_bwd(top, dgf, dz, idx=idx, n_kept_dev=nd, main_grads=(ggf, None), out=dz)
    plan.compact_dev(dsv, dW, dy, idx, cu, nd)
    Bn.embed_bwd(tok, plan.grads["dx"], V, idx=idx, n_kept_dev=nd, main_grad=gtab)
    tol = 4 * Hn.TOL[shape.dtype]           # the layer's, the norm's, the head's and the loss's one after the other
    assert abs(float(stats[0]) - loss.item()) < tol
    want = {"d" + m: t.grad.numpy() for m, t in P.items()}
    got = {m: plan.grads[m] for m in Hn.GRADS + ("dgq", "dgk")} | {"dtable": gtab, "dgf": ggf}
    if not tied:
        want["dhead"], got["dhead"] = head.grad.numpy(), gwh
    for m, t in got.items():
        assert Hn.rel_fro(Hn.to_np(t), want[m]) <= tol, (m, Hn.rel_fro(Hn.to_np(t), want[m]))
