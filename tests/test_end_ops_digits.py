"""Digits and paths of the operators at the ends of the stack of layers that bounds by absolute sums are too wide for: targets that are almost certain, fp32 products
whose exact result fp32 holds, plans of tiles and rings that small sizes do not reach.

Tolerances count roundings: a stored value is off by half a step of its type (EPS: half of finfo.eps, relative), an fp32 sum of n
terms by (its depth, at most n) * 2^-24 of the sum of their absolute values, a function of the hardware or the library by a few 2^-24."""
import ctypes as C
import math

import pytest
import torch

from paper_2502_00340_amd import binding as Bn
from tests.test_end_ops import _head_case, _head_check, embed_ref_bwd
from tests.test_step_ops import BF, DEV, EPS, F32, F64, U, close, gen, gpu, randn, say


# ---- overlaps (CPU) ----------------------------------------------------------------------------------------

def test_norm_refuses_overlaps_of_known_extents():
    """Blocks read the gains, and the backward's last launch writes their gradients, while and after others write rows."""
    L = Bn.lib()
    A, N = 1 << 20, 4 * 16 * 2           # far apart; bytes of four rows of 16
    D = lambda layer=1: C.byref(Bn.NormDesc(16, 0, layer, 1e-5))
    idx = 9 * A
    f = lambda x=A, g=2 * A, b=3 * A, i=None, n=4, y=4 * A: L.cf_norm_fwd(D(), x, g, b, i, None, n, y, None)
    for y in (2 * A, 2 * A + 16, 3 * A, 3 * A - N + 16, 2 * A - N + 16):
        assert f(y=y) == f(y=y, i=idx) == 2
    assert f(i=idx, y=A) == 2 and f(i=idx, y=A + 16) == 2          # the first of the rows that an index may name
    need = L.cf_norm_bwd_workspace_bytes(D(), 4)
    b = lambda x=A, g=2 * A, dy=3 * A, i=None, dx=4 * A, dg=5 * A, db=6 * A, main=0: L.cf_norm_bwd(D(), x, g, dy, i, None, 4, dx, dg, db, main, 7 * A, need, None)
    for i in (None, idx):
        for main in (0, 1):
            wide = 64 if main else 32
            for at, size in ((2 * A, 32), (3 * A, N)):              # the gains, dy
                assert b(dg=at, i=i, main=main) == b(dg=at + size - 16, i=i, main=main) == b(db=at - wide + 16, i=i, main=main) == 2
            assert b(dx=2 * A, i=i, main=main) == b(dx=2 * A - N + 16, i=i, main=main) == 2
    assert b(dg=A) == b(db=A + N - 16) == b(dg=A + 16, i=idx) == b(dx=A + 16, i=idx) == 2


# ---- bounds (CPU) ------------------------------------------------------------------------------------------

def test_head_loss_bounds_of_rows():
    need = lambda n, dx, dt, code=0: Bn.lib().cf_head_loss_workspace_bytes(C.byref(Bn.LossDesc(0, 300, code, 1.0, 0.0, 0.0, 0.0, 0.0)), 8, n, dx, dt, 0)
    most = 1 << 22
    for dx, dt in ((1, 0), (0, 1), (1, 1)):
        assert need(most - 65, dx, dt) > 0 and need(most - 64, dx, dt) == 0
        assert need(most, dx, dt, 1) > 0 and need(most + 1, dx, dt, 1) == 0
    assert need(most, 0, 0) > 0 and need(most + 1, 0, 0) == 0


# ---- targets that are almost certain -----------------------------------------------------------------------

def _dlogits(l, y, n):
    """(logp, dlogits of the mean NLL) for logits l [n, V] in 64 bits, from the other columns' share alone: no digit of 1 - p is lost."""
    at = y[:, None]
    others = (l - l.gather(1, at)).exp().scatter_(1, at, 0.0)
    rest = others.sum(1, keepdim=True)
    d = others / (1.0 + rest)
    return -torch.log1p(rest).squeeze(1), d.scatter(1, at, -rest / (1.0 + rest)) / n


def test_share_of_the_other_columns_reference():
    g0 = gen(1)
    l, y = randn(g0, 5, 7, std=2.0, dtype=F64, device="cpu").requires_grad_(), torch.tensor([0, 6, 3, 3, 1])
    loss = torch.nn.functional.cross_entropy(l, y)
    loss.backward()
    lp, d = _dlogits(l.detach(), y, 5)
    close(d, l.grad, 1e-14, "d")
    assert abs(float(-lp.mean()) - loss.item()) < 1e-14


def _certain_case(dtype, n, H, V, improbable):
    """Rows whose targets have 1 - p of some 1e-2 down to 1e-11.  The first columns of x are the identity, those of the table 0: the table's gradient holds there what
    the logits' gradient is, row by row."""
    g0, K = gen(n + H + V), (n + 7) // 8 * 8
    table = randn(g0, V, H, std=2.0 / math.sqrt(H))
    y = torch.randint(0, V - 1, (n,), generator=g0).to(DEV)
    x = randn(g0, n, H) + table[y] * torch.linspace(3.2, 8.0, n)[torch.randperm(n, generator=g0)][:, None].to(DEV)
    if improbable:          # the first row's tile is gone over again with another reference; its other rows stay what they are
        x[:, 0], table[:, 0] = 0.0, 0.0
        x[0], table[V - 1, 0] = 0.0, 200.0
        x[0, 0] = 1.0
    x = torch.cat((torch.eye(n, K, device=DEV), x), 1).to(dtype).contiguous()
    table = torch.cat((torch.zeros(V, K, device=DEV), table), 1).to(dtype).contiguous()
    return x, table, y


# rows of each form: up to 16, 32, 64 and 128, whole tiles; columns beyond a piece of the least size; more tiles than CUs
@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,H,V", [(1, 264, 3000), (12, 1096, 3000), (24, 1096, 3000), (60, 264, 3001), (100, 264, 2500), (300, 520, 3000), (12, 264, 40000), (24, 264, 40000), (60, 264, 40000),
                                   (100, 264, 40000)])
@pytest.mark.parametrize("improbable", [False, True])
def test_head_loss_of_almost_certain_targets(dtype, n, H, V, improbable):
    say("certain", dtype, n, H, V, improbable)
    x, table, y = _certain_case(dtype, n, H, V, improbable)
    x64, t64 = x.to(F64), table.to(F64)
    l = x64 @ t64.T
    lp, d = _dlogits(l, y, n)
    # the difference of two logits, sums of H products each (the identity adds none), its scaling and its exponential; sums of 64 columns and of these strips
    big = float((x64.abs() @ t64.abs().T).max())
    rel = 2 * (H + 4) * U * big + (4 * float((l - l.gather(1, y[:, None])).abs().max()) + V / 64 + 64) * U
    got = [Bn.head_loss(x, table, y, ws_limit=limit) for limit in (1 << 30, 0)]
    got.append(Bn.head_loss(x, table, y, need_dx=False, need_dtable=False))
    for k, (_, glp, dx, dt) in enumerate(got):
        # 1 - p and its logarithm: both relative to themselves
        close(glp, lp, (2 * rel + 8 * U) * lp.abs() + 2.0 ** -126, "logp")
        if dt is None:
            continue
        # e, the row's factor, the scaled input, the result; bf16: the target's e is exact, its rounding the factor's
        gd = dt[:, :n].T.to(F64)
        hot = torch.zeros_like(d, dtype=torch.bool).scatter_(1, y[:, None], True)
        tol = d.abs() * (2 * rel + 16 * U + 1.01 * EPS[dtype] * torch.where(hot, 2.0, 4.0)) + 2.0 ** -120
        close(gd, d, tol, "dlogits")
        # what a row's gradient adds up to is nothing but roundings
        own = d.abs().sum(1)
        if dtype is F32 and not improbable and k == 0:
            over = gd.sum(1).abs() - own * (V / 64 + 128) * U
        else:
            over = gd.sum(1).abs() - own * (2 * rel + 16 * U + 4.04 * EPS[dtype])
        assert float(over.max()) <= 2.0 ** -120 * V, float((gd.sum(1).abs() / own).max())
        want = d @ t64
        if dtype is F32:
            close(dx, want, (d.abs() * (2 * rel + (V + 16) * U)) @ t64.abs() + 2.0 ** -120, "dx")


# ---- fp32 logits whose contraction is cut into parts --------------------------------------------------------

# few tiles of 128 columns, wide inputs: parts that come out even and that do not, one row more than the streamed form takes, more rows than a flag's
@gpu
@pytest.mark.parametrize("n,H,V", [(33, 8192, 300), (64, 8192, 2400), (100, 4100, 6000), (300, 4096, 2500), (130, 8192, 1), (600, 2052, 130)])
def test_fp32_logits_of_few_tiles(n, H, V):
    say("parts", n, H, V)
    x, table, y, _, _ = _head_case(n + V, F32, n, H, V)
    got = Bn.head_loss(x, table, y)
    _head_check(got, x, table, y, F32)
    for kw in (dict(need_dx=False, need_dtable=False), dict(need_dx=False), dict(ws_limit=0)):
        o = Bn.head_loss(x, table, y, **kw)
        assert torch.equal(o[0], got[0]) and torch.equal(o[1], got[1])
        _head_check(o, x, table, y, F32)
    for s, t in zip(Bn.head_loss(x, table, y), got):
        assert torch.equal(s, t)


@gpu
@pytest.mark.parametrize("improbable", [False, True])
def test_fp32_logits_of_few_tiles_of_live_rows(improbable):
    """The count on the device, rows that are left out whatever they hold, targets far below their row's largest logit."""
    n, H, V = 300, 520, 2500
    x, table, y, _, g0 = _head_case(3, F32, n, H, V)
    if improbable:
        x[:, 0], table[:, 0] = 0.0, 0.0
        table[V - 1, 0] = 300.0
        x[7], y[7] = 0.0, 11
        x[7, 0] = 1.0
    for live in (0, 1, 9, 128, 129, 300, 310):
        m = min(live, n)
        x2, y2 = x.clone(), y.clone()
        x2[m:] = float("nan")
        if m > 20:
            x2[3], y2[3], x2[20], y2[20] = float("nan"), -100, float("inf"), V
        dev = torch.tensor([live], dtype=torch.int32, device=DEV)
        dx = torch.full((n, H), 7.0, device=DEV)
        got = Bn.head_loss(x2, table, y2, n_kept_dev=dev, dx_out=dx)
        assert dx[m:].eq(7.0).all()
        if m == 0:
            assert got[0].eq(0).all() and got[3].eq(0).all()
            continue
        _head_check((got[0], got[1][:m], dx[:m], got[3]), x2[:m], table, y2[:m], F32)
    if improbable:
        assert float(got[1][7]) < -290.0


# ---- fp32 products on operands in bf16 parts ----------------------------------------------------------------

def _ints(g0, bits, *shape, device=DEV):
    """Odd and even whole numbers of so many bits and a sign."""
    return torch.randint(-(1 << bits) + 1, 1 << bits, shape, generator=g0).to(F32).to(device)


def _sparse(g0, bits, n, H, device, k=4):
    """Rows with k whole numbers among H."""
    at = torch.rand(n, H, generator=g0).topk(k, 1).indices.to(device)
    return torch.zeros(n, H, device=device).scatter_(1, at, _ints(g0, bits, n, k, device=device))


def _exact_logits_case(n, H, V, wide_x, device=DEV):
    """Logits that are sums of four products of 19 and 3 bits: whole numbers below 2^24 in units of 2^-20, so that every order of summing them in fp32 is exact.  A 19-bit
    number takes three bf16 parts; without the third a logit is off by up to 16 * 2^-17, a hundred times the bound."""
    g0 = gen(n + H + V)
    x, t = _sparse(g0, 19 if wide_x else 3, n, H, device), _ints(g0, 3 if wide_x else 19, V, H, device=device)
    return x * 2.0 ** -10, t * 2.0 ** -10, torch.randint(0, V, (n,), generator=g0).to(device)


def _exact_logits_want(x, t, y):
    l = x.to(F64) @ t.to(F64).T
    # t = k l - ref: k and ref are rounded, the difference is; then exponentials, sums of 64 columns and of these strips
    tol = (6 * float(l.abs().max()) + t.shape[0] / 64 + 64) * U
    return l, _dlogits(l, y, x.shape[0])[0], tol


# streamed, whole tiles, the contraction in parts
@gpu
@pytest.mark.parametrize("n,H,V", [(20, 264, 3000), (70, 64, 130), (300, 96, 2500), (70, 1024, 300)])
@pytest.mark.parametrize("wide_x", [False, True])
def test_fp32_logits_are_exact_where_fp32_holds_them(n, H, V, wide_x):
    say("exact logits", n, H, V, wide_x)
    x, t, y = _exact_logits_case(n, H, V, wide_x)
    _, lp, tol = _exact_logits_want(x, t, y)
    close(Bn.head_loss(x, t, y, need_dx=False, need_dtable=False)[1], lp, tol, "logp")


def _exact_gradients_case(n, V, bits, device=DEV, H=72):
    """Equal logits: every exponential is 1, the target's V - 1, and the row's factor 1 / (n V), a power of two.  Both gradients are whole numbers below 2^24 times it."""
    g0 = gen(n + V)
    return _ints(g0, bits, n, H, device=device), _ints(g0, bits, V, H, device=device), torch.randint(0, V, (n,), generator=g0).to(device)


def _exact_gradients_want(x, t, y):
    n, V = x.shape[0], t.shape[0]
    d = torch.ones(n, V, dtype=F64, device=x.device).scatter_(1, y[:, None], -(V - 1.0))
    # any order of summing is exact: the absolute values, too, add up to less than 2^24
    assert float((d.abs() @ t.to(F64).abs()).max()) < 2 ** 24 and float((d.T.abs() @ x.to(F64).abs()).max()) < 2 ** 24
    return d @ t.to(F64) / (n * V), d.T @ x.to(F64) / (n * V)


# third parts of one operand beside one part of the other (19 and 18 bits); two parts of each (11 and 12); rows of each form
@gpu
@pytest.mark.parametrize("n", [1, 4, 16, 32, 256])
@pytest.mark.parametrize("V,dx_bits,dt_bits", [(16, 19, 17), (8, 19, 18), (4096, 11, 11)])
def test_fp32_gradients_are_exact_where_fp32_holds_them(n, V, dx_bits, dt_bits):
    say("exact gradients", n, V)
    x, t, y = _exact_gradients_case(n, V, dt_bits if n < 256 else dt_bits - 3)
    z = torch.zeros_like(x)
    got = Bn.head_loss(x, torch.zeros_like(t), y)[3]
    assert torch.equal(got, _exact_gradients_want(x, 0 * t, y)[1].to(F32))
    _, t, y = _exact_gradients_case(n, V, dx_bits)
    got = Bn.head_loss(z, t, y)[2]
    assert torch.equal(got, _exact_gradients_want(z, t, y)[0].to(F32))


def test_fp32_digits_are_seen():
    """On the CPU, products of operands without their third parts, or rounded to bf16, are outside of the bounds of the tests above (and whole operands inside)."""
    part = lambda v, k: v.to(BF).to(F32) if k == 1 else (lambda a: a + part(v - a, k - 1))(v.to(BF).to(F32))
    for wide_x in (False, True):
        x, t, y = _exact_logits_case(70, 64, 130, wide_x, "cpu")
        l, lp, tol = _exact_logits_want(x, t, y)
        assert torch.equal(l.to(F32).to(F64), l) and float(l.abs().max()) < 16.0
        for k, fine in ((3, True), (2, False), (1, False)):
            off = (_dlogits(part(x, k).to(F64) @ part(t, k).to(F64).T, y, 70)[0] - lp).abs().max()
            assert (float(off) <= tol) is fine, (wide_x, k, float(off), tol)
    for n, V, bits, which in ((32, 16, 19, 0), (32, 8, 19, 0), (32, 4096, 11, 0), (32, 8, 18, 1), (32, 4096, 11, 1)):
        x, t, y = _exact_gradients_case(n, V, bits, "cpu")
        want = _exact_gradients_want(x * which, t * (1 - which), y)
        assert torch.equal(want[which].to(F32).to(F64), want[which])
        d = torch.ones(n, V).scatter_(1, y[:, None], -(V - 1.0))
        for k in (1, 2, 3):
            a, b = part(d, k).to(F64), part((t if which == 0 else x), k).to(F64)
            got = (a @ b if which == 0 else a.T @ b) / (n * V)
            assert torch.equal(got, want[which]) is (k == 3 or (k == 2 and V == 4096)), (n, V, which, k)


# ---- plans and rings that small sizes do not reach ----------------------------------------------------------

# dx in tiles of which whole rounds of the CUs are products of their own and the rest are cut into parts: 260 tiles of 256 in bf16, 774 of 128 in fp32 (three blocks a CU)
@gpu
@pytest.mark.parametrize("dtype,H", [(BF, 33032), (F32, 33000)])
@pytest.mark.parametrize("V,limit,live", [(1100, 2 << 30, None), (2500, 0, None), (1100, 2 << 30, 260), (2500, 0, 40)])
def test_input_gradient_of_more_tiles_than_blocks(dtype, H, V, limit, live):
    n = 300
    say("dx plan", dtype, H, V, limit, live)
    x, table, y, _, _ = _head_case(n + V, dtype, n, H, V)
    m = n if live is None else live
    dev = None if live is None else torch.tensor([live], dtype=torch.int32, device=DEV)
    dx = torch.full((n, H), 7.0, dtype=dtype, device=DEV)
    got = Bn.head_loss(x, table, y, n_kept_dev=dev, dx_out=dx, ws_limit=limit)
    assert dx[m:].eq(7.0).all()
    _head_check((got[0], got[1][:m], dx[:m], got[3]), x[:m], table, y[:m], dtype)


# rows of each form that streams the table, with rings that turn (many steps of k) and several tiles a block (more than 256 tiles of 128 columns)
@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,H,V", [(1, 1032, 40000), (16, 200, 70001), (17, 840, 3001), (24, 1096, 40000), (32, 72, 33000), (33, 520, 40000), (64, 264, 33001), (100, 1032, 34000), (128, 136, 40000)])
def test_streamed_logits_of_many_steps_and_tiles(dtype, n, H, V):
    say("rings", dtype, n, H, V)
    x, table, y, _, _ = _head_case(n + V, dtype, n, H, V)
    got = Bn.head_loss(x, table, y)
    _head_check(got, x, table, y, dtype)
    a = Bn.head_loss(x, table, y, need_dx=False, need_dtable=False)
    assert torch.equal(a[0], got[0]) and torch.equal(a[1], got[1])


# more rows than a block sorts, more bits than two passes of nine take; a token that most rows share
@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,V,H,share", [(9001, (1 << 18) + 5, 16, 0.0), (8193, 1 << 18, 24, 0.3), (20000, (1 << 19) + 1, 8, 0.9)])
@pytest.mark.parametrize("main", [False, True])
def test_embedding_backward_of_three_sort_passes(dtype, n, V, H, share, main):
    say("sort", dtype, n, V, H, share, main)
    g0 = gen(n + V)
    tok = torch.randint(0, V, (n,), generator=g0)
    tok[torch.rand(n, generator=g0) < share] = V - 1
    tok[::7] = torch.randint(0, 40, (len(tok[::7]),), generator=g0) * (V // 40)
    tok[3], tok[n - 1] = V, -1
    tok, dx = tok.to(DEV), randn(g0, n, H, dtype=dtype)
    grad = randn(g0, V, H) if main else None
    want, mag = embed_ref_bwd(tok, dx, V, 1.3, grad)
    got = Bn.embed_bwd(tok, dx, V, scale=1.3, main_grad=None if grad is None else grad.clone())
    count = torch.bincount(tok[(tok >= 0) & (tok < V)], minlength=V).to(F64)[:, None]
    close(got, want, mag * U * (count + 4) + want.abs() * (U if main else EPS[dtype]), "dE")
    assert torch.equal(got, Bn.embed_bwd(tok, dx, V, scale=1.3, main_grad=None if grad is None else grad.clone()))
