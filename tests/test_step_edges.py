"""Edges of the operators around the layer calls: states that outlive their gradients, values beyond a type, sizes at the ends of an index,
overlapping tensors.  Plain forms and tolerances as in test_step_ops."""
import ctypes as C
import math

import pytest
import torch

from paper_2502_00340_amd import binding as Bn
from tests import harness as Hn
from tests import test_step_ops as ops
from tests.test_step_ops import AEPS, B1, B2, BF, DEV, EPS_N, F32, F64, LR, U, close, gen, gpu, randn, say


# ---- AdamW: 8-bit states -----------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("b1,b2", [(0.9, 0.95), (0.9, 0.999), (0.95, 0.95), (0.95, 0.999)])
def test_adamw_8_bit_states_come_to_rest_without_a_gradient(b1, b2):
    """Half of the elements of every block lose their gradient after 100 steps, the others keep the scales up.  m is unbiased while it falls: n steps on, the
    mean code of what was at most 448 * 2^9 smallest codes is b1^n times that, 1e-7 of one after the n below (an m is at rest with all but 1e-7 of
    probability, one of 8192 but for 1e-3): then the parameter stands still.  Until then it moves as far as with 32-bit states: an m and a root are off by a step of
    2^-3 at most, their quotient by (1 + 2^-3) / (1 - 2^-3) - 1 < 0.3, and so is the mean of what the elements moved."""
    say("adamw8 rest", b1, b2)
    n, live = 16384, 100
    rest = int(math.log(448 * 512 * 1e7) / -math.log(b1))
    dead = torch.arange(n, device=DEV) % 2 == 1
    g0 = torch.Generator(DEV).manual_seed(11)
    g = torch.empty(n, device=DEV)
    opts = [Bn.AdamW([torch.zeros(n, device=DEV)], [g], lr=1.0, betas=(b1, b2), eps=1e-12, state_bits=bits, seed=5) for bits in (32, 8)]
    at = []
    for step in range(live + rest + 300):
        g.normal_(std=1e-2, generator=g0)
        if step >= live:
            g.masked_fill_(dead, 0.0)
        for o in opts:
            o.step()
        if step + 1 in (live, live + rest):
            at.append([o.params[0].clone() for o in opts])
    assert not bool(opts[1].m[0].float()[dead].any()), "the average of a gradient that ended"
    assert torch.equal(opts[1].params[0][dead], at[1][1][dead]), "a parameter without a gradient"
    far = [float((o.params[0] - a)[dead].double().abs().mean()) for o, a in zip(opts, at[0])]
    assert abs(far[1] / far[0] - 1.0) < 0.3, far
    assert bool((opts[1].v[0].float()[dead] > 0).all())


@gpu
@pytest.mark.parametrize("b1", [0.95, 0.99, 0.999])
def test_adamw_8_bit_averages_fall_without_bias(b1):
    """One step from all kinds of codes, without a gradient but for the one that keeps a block's scale: an m that falls by less than half a step is off by less than
    a step, and by nothing on average.  A step s of e4m3, n elements, errors between -s and s with a variance of at most s^2/4: the mean is within
    6 * s / (2 sqrt(n)), and 2^-12 steps below for the 12 bits that decide.  Those that fall by more are rounded to nearest."""
    say("adamw8 falls", b1)
    n = 1 << 18
    g0 = gen(31)
    q = (torch.randn(n, generator=g0) * torch.exp2(-16 * torch.rand(n, generator=g0)) * 120).clamp(-448, 448)
    q[::256] = 448.0
    q = q.to(torch.float8_e4m3fn).to(DEV)
    scale = torch.full((n // 256,), 2.0 ** -12, device=DEV)
    m0 = q.double() * 2.0 ** -12
    g = torch.zeros(n, device=DEV)
    g[::256] = 448.0 * 2.0 ** -12
    opt = Bn.AdamW([torch.zeros(n, device=DEV)], [g], lr=1e-3, betas=(b1, 0.999), seed=3,
                   state=([q], [torch.full((n,), 448.0, device=DEV).to(torch.float8_e4m3fn)], [scale], [scale.clone()]))
    opt.step(step=50)
    close(opt.m_scale[0], torch.full((n // 256,), 2.0 ** -12), 8 * U * 2.0 ** -12, "scale")
    y = m0.abs() * b1 * 4096.0
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3.0)
    off = (opt.m[0].double() * m0.sign() - y) / step
    free = (g == 0) & (m0 != 0)
    slow = free & ((m0.abs() * 4096.0 - y) < (0.5 - 1e-4) * step)
    assert int(slow.sum()) > n // 10 and float(off[slow].abs().max()) <= 1.0 + 1e-4
    for k in (slow, slow & (y < 2.0 ** -6), slow & (y >= 2.0 ** -6)):
        mean, lim = float(off[k].mean()), 6 * 0.5 / math.sqrt(int(k.sum()))
        assert int(k.sum()) > 1000 and -lim - 2.0 ** -12 < mean < lim, (mean, lim, int(k.sum()))
    fast = free & ((m0.abs() * 4096.0 - y) > (0.5 + 1e-4) * step)
    assert not bool(fast.any()) or float(off[fast].abs().max()) <= 0.5 + 1e-4
    assert not bool(opt.m[0].float()[m0 == 0].any())


@gpu
@pytest.mark.parametrize("bad", [1e30, -1e30, float("inf"), float("-inf"), float("nan")])
def test_adamw_8_bit_block_outlives_a_value_beyond_fp32(bad):
    """Without clipping: what one element does to itself, as with 32-bit states, its block's others do not see."""
    say("adamw8 poison", bad)
    n, at = 700, [5, 300, 699]
    g0 = gen(33)
    first, then = randn(g0, n, std=1e-2), randn(g0, n, std=1e-2)
    ends = []
    for with_bad in (False, True):
        g = first.clone()
        g[at] = bad if with_bad else 0.0
        opt = Bn.AdamW([torch.zeros(n, device=DEV)], [g], lr=LR, betas=(B1, B2), eps=AEPS, state_bits=8, seed=7)
        opt.step()
        moved = opt.params[0].clone()
        g.copy_(then)
        for _ in range(3):
            opt.step()
        ends.append((moved, opt.params[0], opt.m[0].float(), opt.v[0].float(), opt.m_scale[0], opt.v_scale[0]))
    others = torch.ones(n, dtype=torch.bool, device=DEV)
    others[at] = False
    if math.isnan(bad):         # it stays, and takes no part in the scales
        for a, b in zip(ends[0][:4], ends[1][:4]):
            assert bool(b[at].isnan().all()) and bool(a[others].isfinite().all()) and bool(b[others].isfinite().all())
        return
    for a, b in zip(ends[0][:1] + ends[0][2:4], ends[1][:1] + ends[1][2:4]):
        assert torch.equal(a[others], b[others])
    for a, b in zip(ends[0][4:], ends[1][4:]):
        assert torch.equal(a, b)
    assert torch.equal(ends[0][1][others], ends[1][1][others])
    if math.isfinite(bad):      # an update of 0, moments as they were
        assert not bool(ends[1][0][at].any()) and torch.equal(ends[0][1], ends[1][1])
    else:
        assert bool(ends[1][0][at].isnan().all())


# ---- AdamW: the ends of fp32 -------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_root_of_second_moments_below_the_normal_numbers(bits):
    """v from 2^-110 down to 2^-146 with an eps that hides nothing.  A v below the normal numbers is rounded to multiples of 2^-149: three times, of the square, the
    product and the sum, by 2^-150 each.  With 32 bits its root counts as something between itself (2^-64 at least) and 2^-63."""
    say("adamw root", bits)
    e = torch.arange(110, 147, dtype=F64)
    root = torch.exp2(-e / 2)
    n = root.numel()
    p = torch.zeros(n, device=DEV)
    m = (root * 0.5).float().to(DEV)
    if bits == 8:       # a root each of its own block, so that the code is exact: 1.5 times its scale
        root = root.float().double()
        size = n * 256
        q = torch.zeros(size)
        q[::256] = 448.0
        p, g = torch.zeros(size, device=DEV), torch.zeros(size, device=DEV)
        q = q.to(torch.float8_e4m3fn).to(DEV)
        scale = (root / 448).float().to(DEV)
        ms = (root / 896).float().to(DEV)
        state = ([q.clone()], [q.clone()], [ms.clone()], [scale.clone()])
        v0, m0 = (scale.double() * 448).cpu() ** 2, (ms.double() * 448).cpu()
    else:
        g = torch.zeros(n, device=DEV)
        v = torch.exp2(-e).float().to(DEV)
        state = ([m], [v])
        v0, m0 = v.double().cpu(), m.double().cpu()
    opt = Bn.AdamW([p], [g], lr=LR, betas=(0.9, 0.99), eps=1e-30, state=state)
    opt.step(step=5000)
    got = (opt.params[0][::256] if bits == 8 else opt.params[0]).double().cpu()
    v1 = 0.99 * v0
    want = -LR * 0.9 * m0 / (v1.sqrt() + 1e-30)
    off = (1.0 - 3 * 2.0 ** -150 / v1) ** -0.5 - 1.0         # of a quotient by the root of a v that much too small
    far = (32 * U + off) * want.abs()
    if bits == 32:
        few = v1 < 2.0 ** -126
        least, most = (LR * 0.9 * m0 / (r + 1e-30) for r in (torch.full_like(v1, 2.0 ** -63), v1.sqrt().clamp(min=2.0 ** -64)))
        assert bool((-got[few] >= (least - far)[few]).all()) and bool((-got[few] <= (most + far)[few]).all())
        got, want, far = got[~few], want[~few], far[~few]
    close(got, want, far, "parameter")
    if bits == 8:
        close(opt.v_scale[0], v1.sqrt() / 448, (16 * U + off) * v1.sqrt() / 448, "scale")


def test_adamw_refuses_an_eps_below_the_normal_numbers(L):
    """Its reciprocal is infinite: an element without moments would be 0 times that."""
    t = Bn.AdamwTensor(ops.FAKE, None, ops.FAKE, ops.FAKE, ops.FAKE, None, None, 8, 0.0)
    call = lambda eps: L.cf_adamw_step(C.byref(Bn.AdamwDesc(1e-3, 0.9, 0.99, eps, 1, 1, 1, 32, 0, 1.0, 0.0, None, None, None)), C.byref(t), 0, None)
    assert call(1e-39) == 2 and call(2.0 ** -127) == 2 and call(2.0 ** -126) == 0 and call(1e-8) == 0        # of no tensors: nothing is launched


def test_adamw_refuses_tensors_that_overlap_what_it_writes(L):
    """Scales among what is written, views that start elsewhere, gradients that a step would write over."""
    f = torch.zeros(4096)
    p, g, m, v = f[:512], torch.zeros(512), torch.zeros(512), torch.zeros(512)
    q, r = torch.zeros(512).to(torch.float8_e4m3fn), torch.zeros(512).to(torch.float8_e4m3fn)
    sc = torch.zeros(8)
    make = lambda p=[p], g=[g], **kw: Bn.AdamW(p, g, lr=1e-3, **kw)
    make(), make(state=([m], [v])), make(state=([q], [r], [sc[:2]], [sc[2:4]])), make(p=[p, f[512:1024]], g=[g, g])
    for bad in (dict(state=([q], [r], [sc[:2]], [sc[:2]])), dict(state=([q], [r], [sc[:2]], [sc[1:3]])), dict(state=([m], [f[100:612]])), dict(g=[p]), dict(g=[f[511:1023]]),
                dict(p=[p, f[508:1020]], g=[g, g]), dict(state=([m], [v]), g=[v]), dict(p=[p.view(torch.bfloat16)[:512]], g=[g], master=[f[:512]]),
                dict(state=([q], [q.view(torch.uint8).view(torch.float8_e4m3fn)], [sc[:2]], [sc[2:4]])), dict(step_dev=p.view(torch.int32)[7:8]), dict(lr_dev=m[3:4], state=([m], [v]))):
        with pytest.raises(ValueError):
            make(**bad)


# ---- losses ------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
def test_policy_loss_is_finite_where_it_is_defined(dtype):
    """A KL term that is only watched, of a target that a mask has taken away since; no advantage at a ratio beyond fp32; both at once, and next to rows
    that hold neither."""
    say("policy finite", dtype)
    V, rows = 300, 6
    g0 = gen(41)
    l = randn(g0, rows, V, std=2.0, dtype=dtype)
    y = torch.randint(0, V, (rows,), generator=g0).to(DEV)
    at = torch.arange(rows, device=DEV)
    l[0, y[0]] = -200.0                     # lp about -206: exp(ref - lp) beyond fp32
    l[2, y[2]] = -torch.inf
    lp = torch.log_softmax(l.double(), 1)[at, y]
    ref = (lp + 0.1).float()
    ref[0], ref[2] = -3.0, -2.0
    old = (lp - 0.05).float()
    old[0], old[1], old[2], old[4] = -190.0, float(lp[1]) - 150.0, -1.0, float(lp[4]) - 100.0
    adv = torch.tensor([1.5, 0.0, -1.0, 0.7, -0.0, 0.0], device=DEV)
    kw = dict(old_logp=old, advantages=adv, clip=(0.2, 0.3), norm=float(rows))
    stats, got, dl = Bn.token_loss(l, y, ref_logp=ref, kl_coef=0.0, **kw)
    plain = Bn.token_loss(l, y, **kw)
    for a, b in ((stats[:2], plain[0][:2]), (got, plain[1]), (dl, plain[2])):
        assert torch.equal(a, b), "a KL term that does not count"
    assert math.isinf(float(stats[2])), "it is reported all the same"
    # row by row: ratios exp(lp - old), clipped where the clipped product is smaller, nothing where there is no advantage
    r = (lp - old.double()).exp().clamp(max=1e30)
    a = adv.double()
    slope = torch.where(torch.minimum(r * a, r.clamp(0.8, 1.3) * a) < r * a, 0.0, -r * a)
    first = -torch.minimum(r * a, r.clamp(0.8, 1.3) * a)
    p = torch.softmax(l.double(), 1)
    p.neg_()[at, y] += 1.0
    want = p * (slope / rows)[:, None]
    tol = (ops.EPS[dtype] + 2.0 ** -12) * want.abs() + 2.0 ** -12 * (slope.abs() / rows)[:, None] * 1e-3      # exp of lp - old: an lp of 206 is off by 2^-13 at most
    close(dl, want, tol, "dlogits")
    close(stats[0], first.sum() / rows, 2.0 ** -12 * first.abs().sum() / rows, "loss")
    # with a KL term that counts, the rows without an advantage have that term alone
    some = torch.tensor([1, 3, 4, 5], dtype=torch.int32, device=DEV)
    stats, _, dl = Bn.token_loss(l, y, ref_logp=ref, kl_coef=0.1, idx=some, **kw)
    i = some.long()
    q = ref.double()[i] - lp[i]
    want = p[i] * ((slope[i] + 0.1 * (1.0 - q.exp())) / rows)[:, None]
    close(dl, want, ops.EPS[dtype] * want.abs() + 2.0 ** -12 * ((slope[i].abs() + 0.1) / rows)[:, None] * (p[i].abs() + 1e-3), "dlogits with KL")
    close(stats[0], (first[i] + 0.1 * (q.exp() - 1.0 - q)).sum() / rows, 2.0 ** -12 * (first[i].abs() + 0.1).sum() / rows, "loss with KL")
    for bad in (float("nan"), float("inf")):        # what is not defined does not become so: a row of NaN keeps its NaN
        l[5, 7] = bad
        assert bool(Bn.token_loss(l, y, ref_logp=ref, kl_coef=0.0, **kw)[2][5].isnan().all())


def _loss_without_workspace(L, V, scale=0.0):
    """4, the workspace's refusal, where nothing before it is refused"""
    d = Bn.LossDesc(0, V, 0, scale, 0.0, 0.0, 0.0, 1.0)
    return L.cf_token_loss(C.byref(d), ops.FAKE, 0, ops.FAKE, None, None, None, None, None, None, 0, None, 0, ops.FAKE, None, None, 0, None)


def test_token_loss_refuses_a_vocabulary_that_its_index_does_not_hold(L):
    """Columns are counted in 32 bits, by a block's threads beyond the last one too."""
    assert [_loss_without_workspace(L, V) for V in (2 ** 31 - 1, 2 ** 30 + 1, 2 ** 30)] == [2, 2, 4]


def test_token_loss_refuses_a_scale_that_fp32_does_not_hold(L):
    """Logits are scaled by logit_scale * log2(e): infinite, it would be multiplied by the 0 of a row's maximum."""
    assert [_loss_without_workspace(L, 10, s) for s in (3e38, 2.4e38, 2.3e38, 1e-30)] == [2, 2, 4, 4]


# ---- query/key norm ----------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("n,Hq,Hkv", [(1, 1, 1), (301, 5, 2), (70, 64, 8), (2100, 3, 1)])
def test_qk_norm_of_the_smallest_heads(n, Hq, Hkv):
    """d = 8 in fp32: one lane a head, and one block sums the gains of both kinds."""
    ops.test_qk_norm_forward(F32, n, Hq, Hkv, 8, 64)
    for main in (False, True):
        ops.test_qk_norm_backward(F32, n, Hq, Hkv, 8, 64, main)


def test_qk_norm_refuses_outputs_that_lie_over_other_rows(L):
    """In place is row by row, queries over queries and keys over keys; anything else would be written before another wave has read it."""
    d = Bn.make_desc(B=2, S=64, H=256, Hq=4, Hkv=2, d=64, F=512, dtype="bf16")
    p = Bn.QkNorm(ops.FAKE, ops.FAKE, None, None, None)
    Q, K = 1 << 20, 1 << 21                # ten rows: 5120 and 2560 bytes of bf16

    def fwd(x, y, n=10):
        return L.cf_qk_norm_rope_fwd(C.byref(d), C.byref(p), C.byref(Bn.Qk(*x)), n, C.byref(Bn.Qk(*y)), None)

    def bwd(x, dy, dx, idx=None, n=10):
        return L.cf_qk_norm_rope_bwd(C.byref(d), C.byref(p), C.byref(Bn.Qk(*x)), C.byref(Bn.Qk(*dy)), idx, None, n, C.byref(Bn.Qk(*dx)), None, None, 0, None, 0, None)
    far = (1 << 22, 1 << 23, 0, 0)
    x = (Q, K, 0, 0)
    for y in ((Q + 512, K, 0, 0), (Q, K + 256, 0, 0), (Q + 16, 1 << 24, 0, 0), (1 << 24, Q + 512, 0, 0), (K, 1 << 24, 0, 0), (Q, K, 264, 0), (1 << 24, (1 << 24) + 256, 0, 0),
              (Q - 5104, 1 << 24, 0, 0), (1 << 24, K + 2544, 0, 0)):
        assert fwd(x, y) == 2 and bwd(far, x, y) == 2 and bwd(x, far, y) == 2 and bwd(x, far, y, idx=ops.FAKE) == 2, y
    assert bwd(x, far, x, idx=ops.FAKE) == 2           # compact rows over those that are read through the index
    # columns of one row: of equal strides, and not those of the other kind
    row = lambda q, k: (Q + 2 * q, Q + 2 * k, 512, 512)
    assert fwd(row(0, 256), row(256, 0)) == 2 and fwd(row(0, 256), row(0, 320)) == 2 and fwd(row(0, 256), row(8, 384)) == 2


def test_qk_norm_binding_refuses_compact_rows_over_full_ones(L):
    d = Bn.make_desc(B=2, S=64, H=256, Hq=4, Hkv=2, d=64, F=512, dtype="bf16")
    q, k, g, idx = torch.zeros(6, 256, dtype=BF), torch.zeros(6, 128, dtype=BF), torch.ones(64, dtype=BF), torch.arange(3, dtype=torch.int32)
    dq, dk = torch.zeros(3, 256, dtype=BF), torch.zeros(3, 128, dtype=BF)
    for out in ((q[:3], dk), (dq, k[3:]), (q[3:], k[3:])):
        with pytest.raises(ValueError, match="overlap"):
            Bn.qk_norm_rope_bwd(d, q, k, g, g, dq, dk, idx=idx, out=out)


@gpu
def test_qk_norm_over_columns_of_one_row():
    """Queries and keys side by side in one buffer, in place and into other columns of it, forward and backward."""
    say("qk columns")
    n, Hq, Hkv, d = 37, 4, 2, 64
    g0, q, k, gq, gk, cos, sin = ops._qk_case(61, BF, n, Hq, Hkv, d, 50)
    desc = Bn.make_desc(1, 50, 256, Hq, Hkv, d, 256, BF, rms_eps=EPS_N)
    dq, dk = randn(g0, n, Hq * d, dtype=BF), randn(g0, n, Hkv * d, dtype=BF)
    calls = (lambda a, b, **kw: Bn.qk_norm_rope_fwd(desc, a, b, gq, gk, cos, sin, **kw), lambda a, b, **kw: Bn.qk_norm_rope_bwd(desc, q, k, gq, gk, a, b, cos, sin, **kw),
             lambda a, b, **kw: Bn.qk_norm_rope_bwd(desc, a, b, gq, gk, dq, dk, cos, sin, **kw))
    for f in calls:
        a, b = (q, k) if f is not calls[1] else (dq, dk)
        want = f(a, b)
        wide = torch.full((n, 1000), 7.0, dtype=BF, device=DEV)
        fq, fk, oq, ok = wide[:, 8:264], wide[:, 264:392], wide[:, 400:656], wide[:, 656:784]
        fq.copy_(a), fk.copy_(b)
        f(fq, fk, out=(oq, ok))
        assert torch.equal(fq, a) and torch.equal(fk, b) and torch.equal(oq, want[0]) and torch.equal(ok, want[1])
        f(fq, fk, out=(fq, fk))
        assert torch.equal(fq, want[0]) and torch.equal(fk, want[1])
        assert all(bool((t == 7.0).all()) for t in (wide[:, :8], wide[:, 392:400], wide[:, 784:]))


def test_layer_workspaces_for_a_bound_of_zero(L):
    """0 stands for every token in the calls, so it does where their workspace is asked for."""
    for dtype in ("bf16", "f32"):
        d = Bn.make_desc(B=2, S=640, H=256, Hq=4, Hkv=2, d=64, F=512, dtype=dtype)
        for f in (L.cf_layer_workspace_bytes, L.cf_layer_qk_workspace_bytes, lambda d, n: L.cf_lora_workspace_bytes(d, 8, n), lambda d, n: L.cf_lora_qk_workspace_bytes(d, 8, n)):
            assert f(C.byref(d), 0) == f(C.byref(d), 1280) > f(C.byref(d), 640) > f(C.byref(d), 1) > 0


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("main", [False, True])
def test_dense_layer_call_whose_gains_lie_over_the_attention_output(dtype, main):
    """Outputs may lie over the attention output of a dense call; the gains' gradients come out earlier than most."""
    say("gains over attn_out", dtype, main)
    shape, W, sv, tabs, rng = ops._layer_qk_problem(dtype)
    dsv, dW = ops._layer_qk_device(shape, W, sv, tabs)
    dy = Hn.to_dev(Hn.quantize(rng.standard_normal((shape.T, shape.H)), shape.dtype), shape.dtype)
    desc = Bn.make_desc(shape.B, shape.S, shape.H, shape.Hq, shape.Hkv, shape.d, shape.F, shape.dtype)
    apart, over = (Bn.LayerBackward(desc, main_grad=main, qk_norm_eps=EPS_N) for _ in range(2))
    apart.dense(dsv, dW, dy)
    a = dsv["attn_out"].clone()
    flat = a.view(-1).view(F32) if main else a.view(-1)
    spots = [flat[k * 1024:k * 1024 + shape.d] for k in (1, 2)]
    if main:        # what lies there is added to: read the fp32 values as they are
        before = [t.clone() for t in spots]
    over.grads.update(dgq=spots[0], dgk=spots[1])
    over.dense({**dsv, "attn_out": a}, dW, dy)
    for k, g in apart.grads.items():
        if k in ("dgq", "dgk") and main:
            g = g + before[k == "dgk"]
        assert torch.equal(g, over.grads[k]), k


@gpu
def test_two_training_steps_with_cleared_gradients():
    """Main gradients are added to: a step clears them before the next backward pass, which then gives what a new plan gives."""
    say("two steps")
    shape, W, sv, tabs, rng = ops._layer_qk_problem(BF)
    dsv, dW = ops._layer_qk_device(shape, W, sv, tabs)
    desc = Bn.make_desc(shape.B, shape.S, shape.H, shape.Hq, shape.Hkv, shape.d, shape.F, shape.dtype)
    names = ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "g1", "g2", "gq", "gk")
    mask = torch.ones((shape.B, shape.S), dtype=torch.uint8, device=DEV)
    plan = Bn.LayerBackward(desc, main_grad=True, qk_norm_eps=EPS_N)
    grads = [plan.grads["d" + n] for n in names]
    opt = Bn.AdamW([dW[n] for n in names], grads, lr=1e-3, max_norm=1.0, master=True, state_bits=8)
    for _ in range(2):
        dy = Hn.to_dev(Hn.quantize(rng.standard_normal((shape.T, shape.H)), shape.dtype), shape.dtype)
        other = Bn.LayerBackward(desc, main_grad=True, qk_norm_eps=EPS_N)
        for p in (plan, other):
            p.filtered(dsv, dW, dy, mask)
        for n in names:
            assert torch.equal(plan.grads["d" + n], other.grads["d" + n]), n
        opt.step()
        norm = math.sqrt(sum(float(other.grads["d" + n].double().square().sum()) for n in names))
        assert abs(float(opt.grad_norm) - norm) <= 2 * U * norm
        for g in grads:
            g.zero_()


@gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("on_host", [True, False])
def test_head_gradients_of_a_partly_kept_batch(dtype, on_host):
    """Index, loss and head one after the other with the count on the host, and on the device with cleared operands, over memory that held NaN."""
    say("head", dtype, on_host)
    B, S, H, V = 2, 100, 64, 264
    g0 = gen(51)
    x, w = randn(g0, B * S, H, dtype=dtype), randn(g0, H, V, std=0.1, dtype=dtype)
    y = torch.randint(0, V, (B * S,), generator=g0).to(DEV)
    mask = (torch.rand((B, S), generator=g0) < 0.45).to(torch.uint8).to(DEV)
    logits = (x.float() @ w.float()).to(dtype)
    junk = [torch.full((B * S, V), float("nan"), dtype=dtype, device=DEV) for _ in range(4)]
    del junk
    if on_host:
        idx, _, _, n = Bn.build_keep_index(mask)
        stats, _, dl = Bn.token_loss(logits, y, idx=idx[:n])
        kept = Bn.gather_rows(x, idx, n)
    else:
        idx, _, nd, _ = Bn.build_keep_index(mask, sync=False)
        stats, _, dl = Bn.token_loss(logits, y, idx=idx, n_kept_dev=nd, out=torch.zeros((B * S, V), dtype=dtype, device=DEV))
        kept = Bn.gather_rows(x, idx, B * S, out=torch.zeros_like(x), n_kept_dev=nd)
        n = int(nd)
    dy, dw = Bn.linear_bwd_reduced(kept, dl, w)
    at = mask.view(-1).nonzero().squeeze(1)
    assert n == at.numel()
    p = torch.softmax(logits[at].double(), 1)
    p[torch.arange(n, device=DEV), y[at]] -= 1.0
    p /= n
    # dlogits are off by a rounding of their type (and 2^-18 of the largest in fp32), the products by one of theirs and fp32 sums
    e = ops.EPS[dtype] + 2.0 ** -18
    want = p @ w.double().t()
    close(dy[:n], want, e * want.abs() + (e + (V + 8) * U) * (p.abs() @ w.double().abs().t()) + 2.0 ** -18 / n, "dy")
    want = x[at].double().t() @ p
    close(dw, want, e * want.abs() + (e + (n + 8) * U) * (x[at].double().abs().t() @ p.abs()) + 2.0 ** -18 / n, "dw")
    assert on_host or not bool(dy[n:].any())


L = ops.L
