"""The operators around the optimizer step at the ends of their ranges (run with -m gpu): temperatures far from one, logits far
from zero, masked and infinite entries, thousands of rows, tensors that move or live on other streams.

Bounds are those of test_train_ops_gpu (`sum_err` and the formulas of `token_tols`), here evaluated in 64 bits on the GPU.  A
probability's bound does not grow with the logits' distance from zero: what the rounding of M / temperature leaves out of an
exponent has to be taken back, so the exponent's error is that of its difference from the maximum d and of ln S alone."""
import gc
import math
import weakref

import numpy as np
import pytest
import torch

from oracle import train_oracle as orc
from paper_2501_02379_b200 import binding as B
from paper_2501_02379_b200 import synth
from tests.parity import to_device
from tests.test_train_ops_gpu import DT, HALF_ULP, TINY, U, f64, gen, make_rows, sum_err, within

pytestmark = pytest.mark.gpu


class Exact:
    """64-bit values of rows of logits and the bounds on what fp32 arithmetic makes of them."""

    def __init__(self, z, y, tau):
        V = z.shape[1]
        self.live = y >= 0
        x = torch.where(self.live[:, None], z.double(), 0.0) / tau
        self.at = y.clamp(min=0)[:, None]
        self.top = x.amax(1, keepdim=True)
        self.q = x - self.top
        self.q -= self.q.exp().sum(1, keepdim=True).log()
        self.p = self.q.exp()
        d = torch.where(x > -math.inf, self.top - x, 0.0)
        self.logp = self.q.gather(1, self.at)[:, 0]
        self.lse = self.top[:, 0] - self.q.amax(1)
        self.qf = torch.where(self.p > 0, self.q, 0.0)                       # 0 log 0 = 0
        self.H = -(self.p * self.qf).sum(1)
        self.es = sum_err(V) + 2 * 3 * U * (self.p * d).sum(1) + 4 * U
        self.tl = self.es + 2 * 3 * U * (d.gather(1, self.at)[:, 0] + math.log(V) + 1)
        self.ts = self.es + 2 * 3 * U * (self.top[:, 0].abs() + math.log(V) + 1)
        self.tH = 2 * (self.es + 2 * 3 * U) * (1 + (self.p * d).sum(1) + math.log(V))
        self.rel = 2 * 4 * U * (d + math.log(V) + 1) + self.es[:, None]

    def near(self, got, want, tol, what):
        want = torch.where(self.live, want, 0.0)
        off = torch.where(self.live, (got.double() - want).abs() > tol, got != 0) | got.isnan()
        assert not bool(off.any()), f"{what}: {int(off.sum())} of {off.numel()} rows off, e.g. {got[off][:4].tolist()} for {want[off][:4].tolist()}"

    def near_grad(self, got, g, dg, dtype, scale_over_tau, what, rel=None):
        """got against scale / tau * g (1[target] - p), g off by dg."""
        s, rel = scale_over_tau, self.rel if rel is None else rel
        one = torch.zeros_like(self.p).scatter_(1, self.at, 1.0)
        want = torch.where(self.live[:, None], g[:, None] * (one - self.p), 0.0) * s
        tol = (self.p * g.abs()[:, None] * (rel + 8 * U) + self.p * dg[:, None] + one * (g.abs() * 4 * U + dg)[:, None]) * s
        tiny = TINY[dtype] + 2.0 ** -126 * g.abs()[:, None] * s                # a flushed result, a flushed probability times g
        off = ((got.double() - want).abs() > 2 * tol + 1.01 * HALF_ULP[dtype] * want.abs() + tiny) | got.isnan()
        assert not bool(off.any()), f"{what}: {int(off.sum())} entries off, e.g. {got[off][:4].tolist()} for {want[off][:4].tolist()}"


# ------------------------------------------------------------------------------------------------ far from one
FAR = [  # temperature, where the logits lie
    (1e-2, 0.0), (1e-3, 0.0), (1e-4, 0.0), (1e-6, 0.0), (1e-9, 0.0), (1e-20, 0.0), (1e-2, 600.0), (0.1, 1e4), (0.1, -1e4), (1.0, 3e3), (1.0, 6e4),
    (1.0, 1e5), (1.0, -1e5), (1.0, 1e8), (1.0, 1e12), (1e4, 0.0), (1e20, 1e5),
]


def far_rows(dtype, rows, V, tau, offset, seed=3):
    """Logits around `offset` (a few units or a few of the type's steps apart), their maximum in five places of each row of
    which the target is one, some entries masked, every seventh row ignored."""
    g = gen(seed)
    step = abs(offset) * 2 * HALF_ULP[dtype]
    z = torch.randn(rows, V, generator=g, device="cuda").mul_(max(2.0, 3 * step)).add_(offset).to(DT[dtype])
    z[:, 5] = -math.inf
    z[:, V - 70:V - 61] = -math.inf
    at = torch.randint(0, V, (rows, 4), generator=g, device="cuda")
    z.scatter_(1, at, z.amax(1, keepdim=True).expand(rows, 4))
    y = at[:, 0].clone()
    y[3::7] = -1
    z[3] = math.nan
    return z, y


def far_cases(dtype):
    return [c for c in FAR if dtype != "f16" or abs(c[1]) <= 6e4]


FAR_PARAMS = [pytest.param(d, t, o, id=f"{d}-{t:g}-{o:g}") for d in ("bf16", "f16", "f32") for t, o in far_cases(d)]


@pytest.mark.parametrize("dtype,tau,offset", FAR_PARAMS)
@pytest.mark.parametrize("rows,V", [(5, 40003), (1200, 20011), (5, 3001), (1200, 3001), (8, 140001)])
def test_sums_far_from_one(rows, V, dtype, tau, offset):
    """Log-probabilities, log-sum-exp and entropy of every kernel that forms them."""
    z, y = far_rows(dtype, rows, V, tau, offset)
    e = Exact(z, y, tau)
    logp, lse, H = B.token_logprob(z, y, temperature=tau)
    e.near(logp, e.logp, e.tl, "logp"); e.near(lse, e.lse, e.ts, "lse"); e.near(H, e.H, e.tH, "entropy")
    one = torch.ones(rows, device="cuda")
    for forward_only in (False, True):
        r = B.policy_loss(z, y, torch.where(y >= 0, e.logp, 0.0).float(), one, one / rows, temperature=tau, forward_only=forward_only)
        e.near(r.logp, e.logp, e.tl, "policy logp"); e.near(r.entropy, e.H, e.tH, "policy entropy")
        want = -float(e.live.sum()) / rows                                  # the ratio is one
        assert abs(float(r.stats[1]) - want) < 2 * float((e.tl + 8 * U + U * e.logp.abs()).max()) + 4 * U


@pytest.mark.parametrize("dtype,tau,offset", FAR_PARAMS)
@pytest.mark.parametrize("rows,V", [(5, 40003), (1200, 20011), (5, 3001), (1200, 3001)])
def test_gradients_far_from_one(rows, V, dtype, tau, offset):
    """The losses' gradients: the likeliest tokens' probabilities are as exact at a temperature of 1e-6 or around logits of 1e5
    as they are elsewhere, and a row's gradient sums to zero."""
    z, y = far_rows(dtype, rows, V, tau, offset)
    e = Exact(z, y, tau)
    r = torch.rand(rows, generator=gen(8), device="cuda")
    old, adv = torch.where(y >= 0, e.logp, 0.0).float() - 0.05, r + 0.5
    scale = tau                                                             # gradients of the size of the probabilities
    got = B.policy_loss(z, y, old, adv, torch.ones_like(adv), temperature=tau, grad_scale=scale)
    ratio = torch.where(e.live, (e.logp - old.double()).exp(), 0.0)
    g = -ratio * adv.double()
    dg = 2 * g.abs() * (e.tl + 8 * U + 4 * U * (old.abs() + 2).double()) + g.abs() * 4 * U
    e.near_grad(got.dlogits, g, dg, dtype, scale / tau, "policy")
    starts = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device="cuda")
    ref = torch.where(y >= 0, e.logp, 0.0).float()
    s = B.preference_loss(z, y, starts, ref, 0.5, 0.0, temperature=tau, grad_scale=scale)
    c = torch.where(torch.arange(rows, device="cuda") < rows // 2, -0.25, 0.25).double()     # at a margin of zero
    margin = 0.5 * (e.tl + U * (e.logp.abs() + 1))[e.live].sum()            # what the margin may be off by
    e.near_grad(s.dlogits, c, (0.5 * 0.25 * margin + 4 * U) * torch.ones_like(c), dtype, scale / tau, "pairs")


@pytest.mark.parametrize("V", [40003, 140001])
def test_one_logit_far_above_the_others(V):
    """One token has a logit of 1e32, and before it came the sums had grown relative to their reference: nothing but that token
    is left, and no infinity times zero."""
    z = torch.zeros(3, V, dtype=torch.bfloat16, device="cuda")
    z[:, V // 2:] = 27.0                   # 2^39 above the zeros that come first
    z[1, V - 100] = 1e32
    z[2, V - 1] = 1e32
    y = torch.tensor([V // 2, V - 100, 7], device="cuda")
    e = Exact(z, y, 1.0)
    one = torch.ones(3, device="cuda")
    for r in (B.policy_loss(z, y, one * 0, one, one), B.policy_loss(z, y, one * 0, one, one, forward_only=True)):
        e.near(r.logp, e.logp, e.tl, "logp"); e.near(r.entropy, e.H, e.tH, "entropy")
    many = [x.view(400, 3) for x in B.token_logprob(z.repeat(400, 1), y.repeat(400))]
    for i in range(400):                   # (the rows lie differently relative to 16 bytes)
        e.near(many[0][i], e.logp, e.tl, "logp"); e.near(many[1][i], e.lse, e.ts, "lse"); e.near(many[2][i], e.H, e.tH, "entropy")


# ------------------------------------------------------------------------------------------------ masked and infinite entries
@pytest.mark.parametrize("forward_only", [False, True])
@pytest.mark.parametrize("ent", [0.0, 0.02])
@pytest.mark.parametrize("dtype,V", [("bf16", 1003), ("f16", 9001), ("f32", 40003)])
def test_rows_of_weight_zero_add_nothing(V, dtype, ent, forward_only):
    """A mask in the weights: what stands beside a masked row (infinities, NaN, values whose ratio overflows) does not count."""
    z, y = make_rows(dtype, 12, V, 0, 5)
    w = torch.rand(12, generator=gen(1), device="cuda")
    w[2:9] = 0
    logp = B.token_logprob(z, y)[0]
    old, ref, adv = logp - 0.1, logp + 0.2, torch.linspace(-1, 1, 12, device="cuda")
    kw = dict(kl_coef=0.1, entropy_coef=ent, forward_only=forward_only)
    want = B.policy_loss(z, y, old, adv, w, ref_logp=ref, **kw)
    old, ref, adv = old.clone(), ref.clone(), adv.clone()
    old[2], old[3], old[4], ref[5], ref[6], adv[7], adv[8] = -math.inf, -500.0, math.nan, math.inf, math.nan, math.nan, -math.inf
    adv[2] = 0.0
    got = B.policy_loss(z, y, old, adv, w, ref_logp=ref, **kw)
    assert torch.equal(got.stats, want.stats) and torch.equal(got.logp, want.logp) and torch.equal(got.entropy, want.entropy)
    if not forward_only:
        assert torch.equal(got.dlogits, want.dlogits) and bool((got.dlogits[2:9] == 0).all())
    assert bool(torch.isfinite(got.stats).all())


@pytest.mark.parametrize("ent", [0.0, 0.02])
@pytest.mark.parametrize("dtype,rows,V", [("bf16", 12, 1003), ("f16", 12, 9001), ("f32", 12, 40003), ("bf16", 1300, 3001), ("bf16", 1300, 20011), ("f16", 12, 270001)])
def test_rows_without_a_part_in_the_loss_have_a_gradient_of_zero(rows, V, dtype, ent):
    """Whatever their logits are: rows of weight zero, rows outside every answer, coefficients of zero."""
    z, y = make_rows(dtype, rows, V, 0, 5)
    y[1::4] = -1
    out = torch.zeros(rows, dtype=torch.bool, device="cuda")
    out[2::5] = True
    out[:2] = out[-3:] = True
    zb = z.clone()
    zb[out] = math.nan
    zb[2], zb[-2] = math.inf, -math.inf
    w = torch.where(out, 0.0, torch.rand(rows, generator=gen(1), device="cuda"))
    logp, lse, H = B.token_logprob(z, y)
    for logits in (z, zb):
        for place in (None, logits.clone()):
            src = logits if place is None else place
            p = B.policy_loss(src, y, logp - 0.1, torch.ones_like(w), w, ref_logp=logp + 0.1, kl_coef=0.1, entropy_coef=ent, dlogits=place)
            if logits is z and place is None:
                want = p
            assert bool((p.dlogits[out] == 0).all()) and torch.equal(p.dlogits, want.dlogits) and torch.equal(p.stats, want.stats)
    lb, le, he = B.token_logprob(zb, y)
    h = w * 2 if ent else None
    a = B.token_logprob_backward(z, y, lse, w, entropy=H, grad_entropy=h)
    b = B.token_logprob_backward(zb, y, le, w, entropy=he, grad_entropy=h)
    assert torch.equal(a, b) and bool((b[out] == 0).all()) and bool((b[~out & (y >= 0)] != 0).any())
    zb = z.clone()
    zb[:2] = math.nan
    zb[-3:] = math.inf
    starts = torch.tensor([2, rows // 2, rows - 3], dtype=torch.int32, device="cuda")
    a, b = (B.preference_loss(x, y, starts, logp - 0.1) for x in (z, zb))
    assert torch.equal(a.dlogits, b.dlogits) and torch.equal(a.loss, b.loss) and bool((b.dlogits[:2] == 0).all()) and bool((b.dlogits[-3:] == 0).all())


@pytest.mark.parametrize("dtype,V", [("bf16", 1003), ("f32", 40003)])
def test_policy_loss_with_an_infinite_kl(V, dtype):
    """The reference forbids a token (-inf), or gives a token much that the policy forbids or almost does: the KL term is
    infinite, not NaN, and with a coefficient of zero, where it is only looked at, loss and gradient do not know of it."""
    z, y = make_rows(dtype, 6, V, 0, 9)
    y[:] = 3
    z[4, 3] = -math.inf                    # the policy forbids its own token
    one = torch.ones(6, device="cuda")
    logp = B.token_logprob(z, y)[0]
    old = torch.where(logp.isfinite(), logp, -5.0) - 0.1
    ref = torch.where(logp.isfinite(), logp, -5.0) + 0.1
    ref[1], ref[2] = -math.inf, logp[2] + 200.0
    plain = B.policy_loss(z, y, old, one, one / 6)
    assert bool(torch.isfinite(plain.stats).all()) and bool(torch.isfinite(plain.dlogits).all())
    for fwd in (False, True):
        got = B.policy_loss(z, y, old, one, one / 6, ref_logp=ref, forward_only=fwd)
        assert got.stats[2] == math.inf
        within(f64(got.stats[[0, 1, 3, 4]]), f64(plain.stats[[0, 1, 3, 4]]), 1e-4 if fwd else 0.0)      # forward only: another order of sums
        if not fwd:
            assert torch.equal(got.dlogits, plain.dlogits)
        got = B.policy_loss(z, y, old, one, one / 6, ref_logp=ref, kl_coef=0.1, forward_only=fwd)
        assert got.stats[0] == math.inf and got.stats[2] == math.inf
    ref[4], ref[2] = -5.0, logp[2]
    ref[1] = logp[1]
    assert B.policy_loss(z, y, old, one, one / 6, ref_logp=ref).stats[2] == math.inf


@pytest.mark.parametrize("dtype,V", [("bf16", 1003), ("f32", 40003)])
def test_an_advantage_of_zero_leaves_no_policy_term(dtype, V):
    """However far the policy has moved: a ratio that overflows times an advantage of zero is zero."""
    z, y = make_rows(dtype, 4, V, 0, 6)
    adv, w, old = torch.tensor([0.0, 0.0, 1.0, -1.0], device="cuda"), torch.ones(4, device="cuda") / 4, B.token_logprob(z, y)[0]
    want = B.policy_loss(z, y, old, adv, w)
    moved = old.clone()
    moved[0], moved[1] = -200.0, -math.inf
    got = B.policy_loss(z, y, moved, adv, w)
    assert torch.equal(got.stats, want.stats) and torch.equal(got.dlogits, want.dlogits) and bool((got.dlogits[:2] == 0).all())
    assert torch.equal(B.policy_loss(z, y, moved, adv, w, forward_only=True).stats, B.policy_loss(z, y, old, adv, w, forward_only=True).stats)


@pytest.mark.parametrize("dtype,V", [("bf16", 1003), ("f32", 40003)])
def test_pairs_with_a_forbidden_token(V, dtype):
    """An answer with a token of probability zero has a reward of -inf.  As the rejected one it leaves a loss of zero without
    smoothing and an infinite one with it, as the chosen one it is the other way round for a smoothing of one; both: NaN."""
    z, y = make_rows(dtype, 8, V, 0, 4)
    y[:] = 2
    z[3, 2] = -math.inf                    # the second answer's
    ref = torch.full((8,), -4.0, device="cuda")
    st = lambda *s: torch.tensor(s, dtype=torch.int32, device="cuda")  # noqa: E731
    r = B.preference_loss(z, y, st(0, 2, 4), ref)
    assert r.loss == 0 and r.rewards[1] == -math.inf and bool(torch.isfinite(r.rewards[0])) and bool((r.dlogits == 0).all())
    assert B.preference_loss(z, y, st(0, 2, 4), ref, label_smoothing=0.1).loss == math.inf
    r = B.preference_loss(z, y, st(2, 4, 6), ref, beta=0.1)
    assert r.loss == math.inf and r.rewards[0] == -math.inf
    one = torch.zeros(V, device="cuda").double()
    p = torch.softmax(z[2].double(), 0)
    one[2] = 1
    within(f64(r.dlogits[2]), f64(-0.1 * (one - p)), 2 * (0.1 * f64(p) * 2e-5 + 1.01 * HALF_ULP[dtype] * 0.1 * f64((one - p).abs())) + TINY[dtype])
    r = B.preference_loss(z, y, st(2, 4, 6), ref, label_smoothing=1.0)
    assert r.loss == 0 and bool((r.dlogits == 0).all())
    z[5, 2] = -math.inf                    # now the third answer's too
    assert math.isnan(B.preference_loss(z, y, st(2, 4, 6), ref).loss)


# ------------------------------------------------------------------------------------------------ waits that run out
@pytest.fixture
def copy_limit():
    yield B.set_copy_limit
    B.set_copy_limit()


def every_result(z, y):
    """{name: tensor with one row per row of logits} of all calls whose kernels wait, and the two losses."""
    rows = len(y)
    one, starts = torch.ones(rows, device="cuda"), torch.tensor([0, rows // 3, rows], dtype=torch.int32, device="cuda")
    logp, lse, H = B.token_logprob(z, y)
    p = B.policy_loss(z, y, one * -9, one, one / rows, entropy_coef=0.01)
    s = B.preference_loss(z, y, starts, one * -9, 0.01)
    d = B.token_logprob_backward(z, y, one * 9, one)
    out = {"logp": logp, "lse": lse, "H": H, "policy logp": p.logp, "policy H": p.entropy, "policy gradient": p.dlogits, "pairs logp": s.logp,
           "gradient": d}
    return {k: v if v.dim() == 2 else v[:, None] for k, v in out.items()}, torch.stack((p.stats[0], s.loss)), s.dlogits


@pytest.mark.parametrize("dtype,rows,V,copies", [
    ("bf16", 5, 40003, 0), ("bf16", 5, 40003, 1), ("f32", 500, 9001, 0), ("f32", 500, 9001, 1), ("bf16", 1250, 20011, 0), ("bf16", 1250, 20011, 2),
    ("f16", 200, 140001, 0), ("f16", 200, 140001, 2), ("f16", 200, 140001, 6), ("f16", 200, 140001, 10),      # sums, first and second reading
])
def test_waits_that_run_out_are_reported(copy_limit, dtype, rows, V, copies):
    """The copies stop before the first row or inside one.  The calls end, each row of a result is what it should be or NaN
    throughout, a loss is NaN where one of its rows is, and the next calls are as before."""
    z, y = make_rows(dtype, rows, V, 0, 4)
    y[::3] = -1
    want, losses, grad = every_result(z, y)
    assert all(bool(torch.isfinite(x).all()) for x in want.values())
    copy_limit(copies)
    got, lost, _ = every_result(z, y)
    copy_limit(-1)
    ring_forward = rows >= 8 * torch.cuda.get_device_properties(0).multi_processor_count      # fewer: clusters, without such waits
    for k, v in got.items():
        gone = v.isnan().all(1)
        assert torch.equal(torch.where(gone[:, None], want[k], v), want[k]), k
        if ring_forward or "policy" in k or "gradient" in k:
            assert bool(gone.any()) and (copies > 0 or bool(gone.all())), k
        else:
            assert not bool(gone.any()), k
    bad = torch.stack([got[k].isnan().any() for k in ("policy logp", "pairs logp")])      # also of an ignored row of an unfinished unit
    assert torch.equal(lost.isnan(), bad) and torch.equal(torch.where(bad, losses, lost), losses)
    again, l2, g2 = every_result(z, y)
    assert all(torch.equal(again[k], want[k]) for k in want) and torch.equal(l2, losses) and torch.equal(g2, grad)


# ------------------------------------------------------------------------------------------------ lists and tensors of the caller
def test_adamw_lets_go_of_plain_sequences():
    """Nothing of a call on plain sequences is kept, without the cycle collector's help; TensorLists keep their own tensors only."""
    gc.collect()
    gc.disable()
    try:
        w, m, v = ([torch.zeros(5, device="cuda")] for _ in range(3))
        dead = []
        for kept in (False, True):
            lists = [B.TensorList(x) for x in (w, m, v)] if kept else [w, m, v]
            for step in (1, 2, 3):
                g = torch.ones(5, device="cuda")
                dead.append(weakref.ref(g))
                B.adamw_step(lists[0], [g], lists[1], lists[2], step=step, lr=0.1)
                del g
        full = lists[:1] + [B.TensorList([torch.ones(5, device="cuda")])] + lists[1:]
        B.adamw_step(*full, step=4, lr=0.1)
        halves = [B.TensorList([torch.ones(5, device="cuda", dtype=torch.bfloat16)]) for _ in range(2)]
        master = B.TensorList([torch.ones(5, device="cuda")])
        B.adamw_step(*halves, *lists[1:], step=1, lr=0.1, masters=master)
        del master                                                          # the same lists without masters are another call
        before = halves[0].tensors[0].clone()
        B.adamw_step(*halves, *lists[1:], step=2, lr=0.1)
        assert not torch.equal(halves[0].tensors[0], before)
        dead += [weakref.ref(x) for x in full]
        del lists, full, halves
        assert [d() is None for d in dead] == [True] * 10
    finally:
        gc.enable()


def test_adamw_takes_any_strides_of_dimensions_of_one():
    p = torch.randn(7, 1, 5, device="cuda")
    g = torch.randn(7, 5, device="cuda")
    other = g.as_strided((7, 1, 5), (5, 35, 1))                             # the same places in memory
    m, v = torch.zeros(7, 1, 5, device="cuda").as_strided((7, 1, 5), (5, 3, 1)), torch.zeros_like(p)
    q, mq, vq = p.clone(), torch.zeros_like(p), torch.zeros_like(p)
    B.adamw_step([p], [other], [m], [v], step=1, lr=0.1)
    B.adamw_step([q], [g.view(7, 1, 5)], [mq], [vq], step=1, lr=0.1)
    assert torch.equal(p, q) and torch.equal(m, mq) and torch.equal(v, vq)


def test_results_in_place_count_as_changes():
    """autograd's own check of operands that were overwritten sees what the calls write."""
    def bumped(t, call):
        before = t._version
        call()
        return t._version > before

    w, g, m, v = (torch.ones(4, device="cuda") for _ in range(4))
    half, master = torch.ones(4, device="cuda", dtype=torch.bfloat16), torch.ones(4, device="cuda")
    step = lambda: B.adamw_step([w], [g], [m], [v], step=1, lr=0.1)  # noqa: E731
    assert bumped(w, step) and not bumped(g, step)
    lists = [B.TensorList([x]) for x in (w, g, m, v)]
    assert bumped(w, lambda: B.adamw_step(*lists, step=1, lr=0.1))
    with_master = lambda: B.adamw_step([half], [half.clone()], [m], [v], step=1, lr=0.1, masters=[master])  # noqa: E731
    assert bumped(half, with_master) and bumped(master, with_master)
    assert bumped(g, lambda: B.clip_grads([g], 0.5)) and not bumped(g, lambda: B.grad_norm([g], 0.5))
    z, y = make_rows("f32", 4, 10, 0, 0)
    one, starts = torch.ones(4, device="cuda"), torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    assert bumped(z, lambda: B.policy_loss(z, y, one, one, one, dlogits=z))
    assert bumped(z, lambda: B.preference_loss(z, y, starts, one, dlogits=z))
    assert bumped(z, lambda: B.token_logprob_backward(z, y, one, one, dlogits=z))
    assert not bumped(z, lambda: B.policy_loss(z, y, one, one, one))
    x = torch.ones(3, device="cuda", requires_grad=True)
    out = (x * 2).exp()                                                     # its backward needs its result
    B.clip_grads([out.detach()], 1e-3)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    with torch.inference_mode():
        t = torch.ones(4, device="cuda")
    B.clip_grads([t], 0.5)                                                  # has no version: as before
    within(f64(t), np.full(4, 0.25), 1e-6)


def test_a_list_keeps_its_memory():
    """What a list has laid out is its tensors' memory: a parameter that is given other memory (module.to(), p.data = ..) leaves
    the old one with the list, so that no call writes to memory that has become somebody else's."""
    n = 5 << 20
    p = torch.nn.Parameter(torch.ones(n, device="cuda"))
    g, m, v = (torch.full((n,), x, device="cuda") for x in (1.0, 0.0, 0.0))
    lists = [B.TensorList([x]) for x in (p, g, m, v)]
    B.adamw_step(*lists, step=1, lr=0.5)
    where, before = p.data_ptr(), torch.cuda.memory_allocated()
    p.data = torch.empty(0, device="cuda")
    assert torch.cuda.memory_allocated() == before
    others = [torch.full((n,), 7.0, device="cuda") for _ in range(4)]
    assert where not in [x.data_ptr() for x in others]
    B.adamw_step(*lists, step=2, lr=0.5)
    B.clip_grads(lists[0], 1e-3)
    assert all(bool((x == 7).all()) for x in others)
    late = [B.TensorList([x]) for x in (g, g, m, v)]
    g.data = torch.empty(0, device="cuda")
    with pytest.raises(ValueError):                                         # laid out for the step after it has moved
        B.adamw_step(*late, step=1, lr=0.5)
    del lists, late
    gc.collect()
    assert torch.cuda.memory_allocated() == before + (2 * n << 2)           # the old weights and gradients are free, the others are four


def test_inputs_outlive_a_call_on_another_stream():
    """Tensors that the caller lets go of after a call on another stream are not given to somebody else before it has run."""
    z, y = make_rows("bf16", 64, 10007, 0, 2)
    one = torch.ones(64, device="cuda")
    starts = torch.tensor([0, 20, 64], dtype=torch.int32, device="cuda")
    weights, moments = torch.ones(64, device="cuda"), [torch.zeros(64, device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()
    made = []

    def fresh(value, n=64):                                                 # a tensor that nobody keeps
        t = torch.full((n,), float(value), device="cuda")
        made.append(t.data_ptr())
        return t

    calls = {
        "policy": lambda s: B.policy_loss(z, y, fresh(-8), fresh(1), fresh(0.5), ref_logp=fresh(-9), kl_coef=0.1, stream=s).stats,
        "pairs": lambda s: B.preference_loss(z, y, starts.clone(), fresh(-8), stream=s).rewards,
        "logprob": lambda s: B.token_logprob(z.clone(), y.clone(), stream=s)[0],
        "gradient": lambda s: B.token_logprob_backward(z, y, fresh(10), fresh(2), stream=s),
        "norm": lambda s: B.grad_norm([fresh(3)], 1.0, stream=s),
        "list": lambda s: B.grad_norm(B.TensorList([fresh(3)]), 1.0, stream=s),
        "adamw": lambda s: B.adamw_step([weights], [fresh(2)], *([m] for m in moments), step=1, lr=0.1, grad_scale=fresh(0.5, 1), stream=s) or weights,
    }
    for name, call in calls.items():
        want = call(None).clone()
        if name == "adamw":
            for t, x in zip([weights] + moments, (1, 0, 0)):
                t.fill_(x)
        torch.cuda.synchronize()
        made.clear()
        with torch.cuda.stream(side):
            torch.cuda._sleep(int(4e8))
        # (the inputs are filled on the default stream, long before the other one is through with its sleep)
        got = call(side)
        others = [torch.full((n,), 99.0, device="cuda") for n in (64, 1) for _ in range(12)]
        others += [torch.full_like(z, 99.0), torch.full_like(y, 99), torch.full_like(starts, 99)]
        assert not side.query(), "the test has to come before the call has run"
        assert not set(made) & {x.data_ptr() for x in others}, name
        torch.cuda.synchronize()
        assert torch.equal(got, want), name


def test_a_scale_outlives_a_step_on_another_stream():
    wl = synth.WORKLOADS["small4"]
    src = synth.GradientSource(wl)
    side, results = torch.cuda.Stream(), []
    for batched in (False, True):
        for stream in (None, side):
            st = B.TgradState(B.make_config(wl.shape, wl.ranks, wl.k, wl.T))
            w, g = to_device(src.weight(), False), to_device(src.gradient(0), False)
            scale = torch.full((1,), 0.5, device="cuda")
            where = scale.data_ptr()
            torch.cuda.synchronize()
            if stream is not None:
                with torch.cuda.stream(side):
                    torch.cuda._sleep(int(4e8))
            if batched:
                B.step_batched([st], [w], [g], stream=stream, scale=scale)
            else:
                st.step_scaled(w, g, scale, stream=stream)
            del scale
            if stream is not None:
                others = [torch.full((1,), 99.0, device="cuda") for _ in range(12)]
                assert not side.query() and where not in [x.data_ptr() for x in others]
            torch.cuda.synchronize()
            results.append((w.clone(), st.export(B.WHAT_M_L)))
    assert all(torch.equal(a, results[0][0]) and np.array_equal(b, results[0][1]) for a, b in results)


@pytest.mark.parametrize("dtype,V,pad", [("bf16", 20011, 0), ("f16", 40000, 0), ("f32", 9001, 3), ("bf16", 3001, 1)])
def test_pairs_of_thousands_of_rows(dtype, V, pad):
    """Enough rows for the kernels that hand them out: rewards, loss and gradient against 64 bits.  What a sum over an answer's
    tokens is off by is the sum of the tokens' bounds."""
    lengths = [400, 1, 0, 777, 250, 250, 33, 500]
    rows = 7 + sum(lengths) + 5                                             # some belong to no answer
    z, y = make_rows(dtype, rows, V, pad, 12, std=3.0)
    y[::5] = -3
    z[5] = math.nan
    starts = torch.tensor(np.cumsum([7] + lengths), dtype=torch.int32, device="cuda")
    beta, eps, scale = 0.125, 0.25, 256.0                                   # exact in fp32
    ref = B.token_logprob(z, y)[0] + torch.randn(rows, generator=gen(2), device="cuda") * 0.1
    got = B.preference_loss(z, y, starts, ref, beta, eps, temperature=0.9, grad_scale=scale)
    gap, tol, part = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda"), 200
    for a in range(0, rows, part):
        c = slice(a, min(rows, a + part))
        e = Exact(z[c], y[c], 0.9)
        e.near(got.logp[c], e.logp, e.tl, "logp")
        gap[c] = torch.where(e.live, e.logp - ref[c].double(), 0.0)
        tol[c] = torch.where(e.live, e.tl, 0.0)
    at = starts.tolist()
    R, tR = (torch.stack([x[i:j].sum() for i, j in zip(at, at[1:])]) * beta for x in (gap, tol))
    tR = 2 * tR + 2 * U * R.abs() + 1e-30
    assert bool(((got.rewards.double() - R).abs() <= tR).all())
    h, th = R[0::2] - R[1::2], tR[0::2] + tR[1::2]
    loss = ((1 - eps) * torch.nn.functional.softplus(-h) + eps * torch.nn.functional.softplus(h)).mean()
    assert abs(float(got.loss) - float(loss)) <= float(th.mean()) + 4 * U * float(loss)
    d = beta * (torch.sigmoid(h) - (1 - eps)) / len(h)
    g, dg = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda")
    for s in range(len(lengths)):
        g[at[s]:at[s + 1]] = d[s // 2] * (1 if s % 2 == 0 else -1)
        dg[at[s]:at[s + 1]] = beta * th[s // 2] / len(h) + 8 * U * d[s // 2].abs()
    for a in range(0, rows, part):
        c = slice(a, min(rows, a + part))
        Exact(z[c], y[c], 0.9).near_grad(got.dlogits[c], g[c], dg[c], dtype, scale / 0.9, "gradient")
    assert bool((got.dlogits[:7] == 0).all()) and bool((got.dlogits[-5:] == 0).all())
    fwd = B.preference_loss(z, y, starts, ref, beta, eps, temperature=0.9, forward_only=True)
    assert torch.equal(fwd.loss, got.loss) and torch.equal(fwd.rewards, got.rewards)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tau,offset", [(1e-2, 0.0), (1e-3, 0.0), (1.0, 3e3), (1.0, -3e3), (1e4, 0.0)])
@pytest.mark.parametrize("rows,V", [(5, 40003), (1200, 3001), (300, 20011)])
def test_gradient_from_lse_is_as_exact_as_lse(rows, V, tau, offset, dtype):
    """token_logprob_backward has nothing but lse, rounded to fp32: what that leaves out is in every probability."""
    z, y = far_rows(dtype, rows, V, tau, offset)
    e = Exact(z, y, tau)
    g = torch.randn(rows, generator=gen(3), device="cuda")
    d = B.token_logprob_backward(z, y, B.token_logprob(z, y, temperature=tau)[1], g * tau, temperature=tau)
    rel = e.rel + 2 * 4 * U * e.top.abs()
    e.near_grad(d, g.double(), torch.zeros_like(e.logp), dtype, 1.0, "gradient", rel)


@pytest.mark.parametrize("tau", [1.0, 0.8, 0.7])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,V", [(1100, 2377), (1100, 10579), (600, 34057), (100, 131073), (6000, 2377), (4000, 10579), (2000, 34057), (2000, 131073)])
def test_log_probabilities_have_no_bias(rows, V, dtype, tau):
    """The sum over an answer's tokens shows what every token is off by in the same way.  Roundings to nearest have none, the
    exponential unit's mean error is corrected where it comes in; what is left on average is to be below half of an fp32
    rounding of one, plus four standard errors of the mean."""
    z, y = make_rows(dtype, rows, V, 0, 21)
    z.scatter_add_(1, y[:, None], (torch.randn(rows, 1, generator=gen(5), device="cuda") * 2 + 7).to(z.dtype))      # a likely token
    one = torch.ones(rows, device="cuda")
    got = {"logprob": B.token_logprob(z, y, temperature=tau)[0], "policy": B.policy_loss(z, y, -one, one, one, temperature=tau).logp}
    want = torch.cat([torch.log_softmax(a.double() / tau, 1).gather(1, b[:, None])[:, 0] for a, b in zip(z.split(200), y.split(200))])
    for name, x in got.items():
        err = x.double() - want
        bias, se = float(err.mean()), float(err.std()) / rows ** 0.5
        assert abs(bias) < U / 2 + 4 * se, f"{name}: {bias:.2e}, standard error {se:.1e}"
