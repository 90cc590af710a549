"""The operators around the optimizer step on a B200 against their 64-bit definitions (run with -m gpu).

Tolerances are bounds derived from the arithmetic, u = 2^-24 being half an fp32 ulp:
* a sum of squares adds at most 64 terms in fp32 and the rest in fp64, so a norm is off by at most (64 u) / 2 + 2 u;
* a probability 2^d / S: d has three roundings, |d| ln2 3 u; the exponential is good to 2 ulp; S is a sum of at most
  `chain` positive terms in sequence and 16 merges, each with a rescaling (4 u): see `sum_err`;
* a result stored in 16 bits is rounded once more: half an ulp of the stored value.
Each bound is taken with a factor of 2, because some of the roundings above were counted by their leading term only.
"""
import math

import numpy as np
import pytest
import torch

from oracle import train_oracle as orc
from paper_2501_02379_b200 import binding as B
from paper_2501_02379_b200 import synth
from tests.parity import to_device

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "c64": torch.complex64}
HALF_ULP = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}      # results below this may be flushed or rounded away


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def f64(t):
    return t.detach().cpu().to(torch.complex128 if t.is_complex() else torch.float64).numpy()


def within(got, want, tol, what=""):
    got, want = np.asarray(got, dtype=np.complex128 if np.iscomplexobj(want) else np.float64), np.asarray(want)
    assert got.shape == want.shape
    off = np.abs(got - want) > tol
    assert not off.any() and not np.isnan(got).any(), f"{what}: {off.sum()} of {off.size} off, worst {np.max(np.abs(got - want) / np.maximum(tol, 1e-300)):.3g} x the bound"


# ------------------------------------------------------------------------------------------------ lists
NORM_TOL = 2 * (32 * U + 2 * U)


def make_list(specs, seed, offset=0):
    """Views at an odd place of their own buffers: (kind, shape) -> tensor whose first entry is `offset` entries in."""
    out = []
    g = gen(seed)
    for i, (kind, shape) in enumerate(specs):
        n = math.prod(shape)
        buf = torch.full((n + offset + 9,), 3.0, dtype=DT[kind], device="cuda")      # what lies around must not count or change
        buf[offset:offset + n] = torch.randn(n, generator=g, device="cuda", dtype=DT[kind]) * 10.0 ** (i % 4 - 2)
        out.append(buf[offset:offset + n].view(shape))
    return out


LISTS = {
    "one": [("f32", (1,))],
    "edges": [("f32", (s,)) for s in (1, 2, 3, 4, 5, 7, 8, 9, 31, 33)] + [("bf16", (s,)) for s in (1, 2, 7, 8, 9, 15, 16, 17)] + [("f16", (5,)), ("c64", (1,)), ("c64", (3, 3))],
    "empty_ones": [("f32", (0,)), ("bf16", (17,)), ("f16", (0, 4)), ("c64", (5, 2)), ("f32", (0,))],
    "chunks": [("bf16", (16384 * 8,)), ("bf16", (16384 * 8 + 1,)), ("f32", (8192 * 3 - 1,)), ("c64", (4096 * 5 + 3,)), ("f16", (300001,))],
    "many": [("f32", (1 + i % 7,)) for i in range(300)],
    "slices": [(("f32", "bf16", "f16")[i % 3], (i % 5,)) for i in range(2500)],
    "large": [("f32", (1000, 1003)), ("c64", (64, 64, 32, 17)), ("bf16", (2999, 1001)), ("f32", (7,))],
}


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("name", sorted(LISTS))
def test_norm_and_clip(name, offset):
    grads = make_list(LISTS[name], 5, offset)
    keep = [g.clone() for g in grads]
    norm, c, norms = orc.grad_norm([f64(g) for g in grads], 0.5)
    out = B.grad_norm(grads, 0.5)
    assert out.shape == (2 + len(grads),)
    o = f64(out)
    within(o[0], norm, NORM_TOL * norm + 1e-45, "norm")
    within(o[1], c, (NORM_TOL + 4 * U) * c, "coefficient")
    within(o[2:], norms, NORM_TOL * np.array(norms) + 1e-45, "norms")
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    assert torch.equal(out, B.grad_norm(grads, 0.5))                         # the same bits again
    lst = B.TensorList(grads)
    assert torch.equal(B.clip_grads(lst, 0.5), out)
    for (kind, _), g, k in zip(LISTS[name], grads, keep):
        w = f64(k) * c
        h = HALF_ULP["f32" if kind == "c64" else kind]
        within(f64(g), w, (2 * NORM_TOL + 4 * U + 1.01 * h) * np.abs(w) + TINY["f32" if kind == "c64" else kind], kind)
        buf = g._base.view(-1) if g._base is not None else g
        n = g.numel()
        assert bool((buf[:offset] == 3).all()) and bool((buf[offset + n:] == 3).all())


def test_norm_of_nothing_and_without_clipping():
    o = B.grad_norm([])
    assert o.tolist() == [0.0, 1.0]
    g = [torch.randn(1000, device="cuda")]
    keep = g[0].clone()
    assert B.clip_grads(g, 1e9)[1] == 1.0 and torch.equal(g[0], keep)
    assert B.clip_grads(g, float("inf"))[1] == 1.0 and torch.equal(g[0], keep)


@pytest.mark.parametrize("kind,scale", [("f32", 1e-30), ("f32", 1e30), ("f32", 3e-42), ("bf16", 1e-35), ("bf16", 1e35), ("f16", 6e4)])
def test_norm_far_from_one(kind, scale):
    g = (torch.rand(70001, generator=gen(1), device="cuda") * 0.5 + 0.5).mul(scale).to(DT[kind])
    norm, _, _ = orc.grad_norm([f64(g)])
    within(f64(B.grad_norm([g]))[0], norm, NORM_TOL * norm + 2e-45)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_norm_of_nonfinite(bad):
    for kind in ("f32", "bf16", "f16"):
        g = [torch.ones(100, device="cuda", dtype=DT[kind]), torch.ones(5000, device="cuda", dtype=DT[kind])]
        g[1][4999] = bad
        o = B.grad_norm(g, 1.0).tolist()
        assert o[2] == 10.0 and o[0] != 10.0 and not math.isfinite(o[0]) and math.isnan(o[0]) == math.isnan(bad)
        assert math.isnan(o[1]) if math.isnan(bad) else o[1] == 0.0


def test_norm_takes_any_dense_order_and_refuses_gaps():
    x = torch.randn(40, 30, device="cuda")
    a = f64(B.grad_norm([x.t(), x.view(4, 10, 30).permute(2, 0, 1)]))
    within(a[2:], np.full(2, np.linalg.norm(f64(x))), NORM_TOL * np.linalg.norm(f64(x)))
    for bad in (x[:, :29], x.expand(2, 40, 30), x.double()):
        with pytest.raises(ValueError):
            B.grad_norm([bad])


def test_norm_past_32_bits():
    n = (1 << 31) + 12345
    g = torch.full((n,), 2.0, dtype=torch.bfloat16, device="cuda")
    g[-1] = 1024.0
    want = math.sqrt(4.0 * (n - 1) + 1024.0 ** 2)
    o = f64(B.clip_grads([g], 1.0))
    within(o[0], want, NORM_TOL * want)
    assert float(g[-1]) == float(torch.tensor(1024.0 * o[1]).bfloat16()) and bool((g[:-1] == g[0]).all()) and float(g[0]) < 1e-3


@pytest.mark.parametrize("offset", [0, 1, 2, 3])
@pytest.mark.parametrize("kind,master", [("f32", False), ("bf16", False), ("f16", False), ("bf16", True), ("f16", True), ("c64", False)])
def test_adamw(kind, master, offset):
    shapes = [(1,), (2,), (3,), (5,), (0,), (64, 33), (4096,), (4097,), (8200, 3), (513,)]
    lr, b1, b2, eps, wd, step, c = 0.02, 0.9, 0.95, 1e-6, 0.1, 7, 0.3
    mk = "c64" if kind == "c64" else "f32"
    specs = [(kind, s) for s in shapes]
    w, g = make_list(specs, 1, offset), make_list(specs, 2, offset)
    m, v = make_list([(mk, s) for s in shapes], 3, offset), make_list([("f32", s) for s in shapes], 4, offset)
    for x in v:
        x.abs_()
    ms = make_list([("f32", s) for s in shapes], 6, offset) if master else None
    scale = torch.tensor([c], device="cuda")
    c64 = float(scale.double())
    want, tol = [], []
    for i in range(len(shapes)):
        w0 = f64(ms[i] if master else w[i])
        W, M, V = orc.adamw(w0, f64(g[i]), f64(m[i]), f64(v[i]), step, lr, b1, b2, eps, wd, c64)
        tm = 2 * 4 * U * (np.abs(b1 * f64(m[i])) + (1 - b1) * np.abs(f64(g[i])) * c64) + 1e-44
        den = np.sqrt(V / (1 - b2 ** step)) + eps
        upd = lr / (1 - b1 ** step) / den
        tw = 2 * 4 * U * (np.abs(w0) + np.abs(upd * M)) + 2 * upd * tm + 1e-44
        want.append((W, M, V)); tol.append((tw, tm, 2 * 6 * U * V + 1e-44))
    others = [x._base.clone() for x in w + g + m + v]
    lists = [B.TensorList(x) for x in (w, g, m, v)]
    B.adamw_step(*lists, step=step, lr=lr, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, grad_scale=scale, masters=ms)
    for i, (W, M, V) in enumerate(want):
        tw, tm, tv = tol[i]
        within(f64(m[i]), M, tm, "m"); within(f64(v[i]), V, tv, "v")
        if master:
            within(f64(ms[i]), W, tw, "master")
            assert torch.equal(w[i], ms[i].to(w[i].dtype))
        else:
            h = HALF_ULP[mk if kind == "c64" else kind] if kind != "c64" else U
            within(f64(w[i]), W, tw + (1.01 * h * np.abs(W) + TINY.get(kind, 0.0) if kind not in ("f32", "c64") else 0.0), "w")
    for x, o in zip(w + g + m + v, others):
        n = x.numel()
        assert torch.equal(x._base[:offset], o[:offset]) and torch.equal(x._base[offset + n:], o[offset + n:])


def test_adamw_many_tensors_and_mixed_alignment():
    n = 700                                        # more than one launch takes
    w = [torch.randn(1 + i % 11, device="cuda") for i in range(n)]
    g = [torch.randn(x.numel() + 1, device="cuda")[1:] for x in w]        # aligned unlike the weights: no common vector
    m, v = [torch.zeros_like(x) for x in w], [torch.zeros_like(x) for x in w]
    want = [orc.adamw(f64(a), f64(b), 0 * f64(a), 0 * f64(a), 1, 0.1)[0] for a, b in zip(w, g)]
    B.adamw_step(w, g, m, v, step=1, lr=0.1)
    for a, b in zip(w, want):
        within(f64(a), b, 2 * 8 * U * (np.abs(b) + 0.2) + 1e-6 * 0.1)     # from zero moments the update is +-lr up to eps / |g|


def test_adamw_refuses_what_does_not_match():
    x = torch.zeros(4, 3, device="cuda")
    ok = [x], [x.clone()], [x.clone()], [x.clone()]
    for i, bad in ((1, x.bfloat16()), (2, x.bfloat16()), (3, torch.zeros(3, 4, device="cuda").t()), (1, torch.zeros(12, device="cuda"))):
        lists = list(ok)
        lists[i] = [bad]
        with pytest.raises(ValueError):
            B.adamw_step(*lists, step=1, lr=0.1)
    with pytest.raises(ValueError):
        B.adamw_step([x], [], [x], [x], step=1, lr=0.1)
    with pytest.raises(ValueError):
        B.adamw_step(*ok, step=1, lr=0.1, masters=[x])
    with pytest.raises(ValueError):
        B.adamw_step(*ok, step=1, lr=0.1, grad_scale=torch.zeros(2, device="cuda"))
    with pytest.raises(B.TgradError) as e:
        B.adamw_step(*ok, step=0, lr=0.1)
    assert e.value.status == B.ERR_INVALID_ARG


@pytest.mark.parametrize("composition", ["us_lr", "lr_us", "sum"])
@pytest.mark.parametrize("name", ["small4", "odd32", "lead300"])
def test_scaled_step_is_the_step_of_the_scaled_gradient(name, composition):
    # a power of two commutes with every rounding of the step, so the two agree to the last bit, refresh included
    wl = synth.WORKLOADS[name]
    src = synth.GradientSource(wl)
    out = []
    for scaled in (True, False):
        st = B.TgradState(B.make_config(wl.shape, wl.ranks, wl.k, wl.T, lr=wl.lr, composition=composition))
        w = to_device(src.weight(), False)
        for t in range(3):
            g = to_device(src.gradient(t), False)
            if scaled:
                st.step_scaled(w, g, torch.tensor([0.25], device="cuda"))
            else:
                st.step(w, g * 0.25)
        out.append((w.clone(), st.export(B.WHAT_M_L), st.export(B.WHAT_V_S)))
    assert torch.equal(out[0][0], out[1][0]) and np.array_equal(out[0][1], out[1][1]) and np.array_equal(out[0][2], out[1][2])


def test_scaled_step_without_a_scale_and_batched():
    wl = synth.WORKLOADS["small4"]
    src = synth.GradientSource(wl)
    g = to_device(src.gradient(0), False)
    ws = []
    for mode in range(4):
        sts = [B.TgradState(B.make_config(wl.shape, wl.ranks, wl.k, wl.T)) for _ in range(2)]
        w = [to_device(src.weight(), False) for _ in range(2)]
        half = torch.tensor([0.5], device="cuda")
        if mode == 0:
            [s.step(a, g.clone()) for s, a in zip(sts, w)]
        elif mode == 1:
            [s.step_scaled(a, g.clone(), None) for s, a in zip(sts, w)]
        elif mode == 2:
            B.step_batched(sts, w, [g.clone(), g.clone()], scale=half)
        else:
            [s.step_scaled(a, g.clone(), half) for s, a in zip(sts, w)]
        torch.cuda.synchronize()
        ws.append(w)
    assert torch.equal(ws[0][0], ws[1][0]) and torch.equal(ws[2][0], ws[3][0]) and torch.equal(ws[2][1], ws[3][1])


# ------------------------------------------------------------------------------------------------ rows of logits
def sum_err(V):
    """Relative error of S (and of T relative to sum 2^d |d|) without the exponents' own: the exponential, a chain of
    sequential additions per thread (the one-pass kernel adds 32 pairs, the streaming one V / 4096 batches more) and merges."""
    return 2 * U * (4 + 34 + V / 4096 + 16 * 4)


def make_rows(dtype, rows, V, pad, seed, lead=0, temperature=1.0, std=2.0):
    """Logits [rows, V] with row stride V + pad, `lead` entries into their buffer."""
    ld = V + pad
    buf = torch.randn(rows * ld + lead + 3, generator=gen(seed), device="cuda").mul_(std).to(DT[dtype])
    z = buf.as_strided((rows, V), (ld, 1), lead)
    y = torch.randint(0, V, (rows,), generator=gen(seed + 1), device="cuda")
    return z, y


def token_tols(z, y, tau):
    """Per row: absolute bounds on logp and lse, on the entropy, and the relative bound on a probability as a function of d."""
    x = f64(z) / tau
    rel, logp, lse, H = [], [], [], []
    for i in range(len(y)):
        if y[i] < 0:
            rel.append(np.zeros(x.shape[1])); logp.append(0.0); lse.append(0.0); H.append(0.0)
            continue
        d = np.abs(x[i] - x[i].max())
        d[~np.isfinite(d)] = 0.0
        p = np.exp(-d); p /= p.sum()
        es = sum_err(x.shape[1]) + 2 * 3 * U * float((p * d).sum()) + 4 * U
        rel.append(2 * 4 * U * (d + abs(x[i].max()) + np.log(x.shape[1])) + es)
        logp.append(es + 2 * 3 * U * (d[y[i]] + np.log(x.shape[1]) + 1))
        lse.append(es + 2 * 3 * U * (abs(x[i].max()) + np.log(x.shape[1]) + 1))
        H.append(2 * (es + 2 * 3 * U) * (1 + float((p * d).sum()) + np.log(x.shape[1])))
    return np.array(rel), np.array(logp), np.array(lse), np.array(H)


def grad_tol(z, y, tau, g, h, dg, rel, dtype, want, scale=1.0):
    """Bound on the gradient: probabilities off by `rel`, the row's factor g by `dg`."""
    _, _, H, = orc.token_logprob(f64(z), y, tau)
    tol = np.zeros(want.shape)
    for i in range(len(y)):
        if y[i] < 0:
            continue
        p = orc.token_row(f64(z)[i], y[i], tau)[3]
        lp = np.abs(np.log(np.where(p > 0, p, 1.0)))
        per = (abs(g[i]) + abs(h[i]) * (lp + H[i])) * scale / tau
        tol[i] = p * per * (rel[i] + 8 * U) + p * abs(h[i]) * (rel[i] * (1 + lp)) * scale / tau + p * dg[i] * scale / tau
        tol[i, y[i]] += (abs(g[i]) * 4 * U + dg[i]) * scale / tau
    return 2 * tol + 1.01 * HALF_ULP[dtype] * np.abs(want) + TINY[dtype]


SIZES = [  # rows, vocabulary, padding of a row, entries before the first row
    (1, 1, 0, 0), (3, 2, 0, 1), (5, 7, 0, 0), (4, 8, 0, 0), (4, 9, 3, 5), (2, 17, 7, 2), (6, 1000, 0, 0), (3, 4097, 1, 3), (5, 8191, 1, 0),
    (2, 16384, 0, 0), (2, 16385, 0, 7), (3, 40003, 5, 1), (2, 131072, 0, 0), (1, 131079, 0, 3), (2, 270001, 0, 1), (700, 129, 0, 0),
]


@pytest.mark.parametrize("tau", [1.0, 0.7])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,V,pad,lead", SIZES)
def test_token_logprob(rows, V, pad, lead, dtype, tau):
    z, y = make_rows(dtype, rows, V, pad, 10 + V % 7, lead)
    if rows > 2:
        y[1] = -100
        z[1] = float("nan")
    if V > 8:
        z[rows - 1, 5] = -math.inf
        y[rows - 1] = 3
    r = np.random.default_rng(0)
    g, h = r.standard_normal(rows).astype(np.float32), r.standard_normal(rows).astype(np.float32)
    yn = y.cpu().numpy()
    rel, tl, ts, tH = token_tols(z, yn, tau)
    logp, lse, H = B.token_logprob(z, y, temperature=tau)
    wl, ws, wH = orc.token_logprob(f64(z), yn, tau)
    within(f64(logp), wl, tl, "logp"); within(f64(lse), ws, ts, "lse"); within(f64(H), wH, tH, "entropy")
    for use_h in (False, True):
        d = B.token_logprob_backward(z, y, lse, torch.tensor(g).cuda(), entropy=H if use_h else None, grad_entropy=torch.tensor(h).cuda() if use_h else None, temperature=tau)
        hh = h * use_h
        want = orc.token_gradient(f64(z), yn, g, hh, tau)
        within(f64(d), want, grad_tol(z, yn, tau, g, hh, np.abs(hh) * tH, rel, dtype, want), "dlogits")
    assert torch.equal(logp, B.token_logprob(z, y, temperature=tau)[0])


def policy_inputs(z, y, tau, seed, clip=(0.2, 0.3)):
    r = np.random.default_rng(seed)
    n = len(y)
    logp = orc.token_logprob(f64(z), y, tau)[0]
    shift = r.standard_normal(n) * 0.4
    for b in (math.log(1 - clip[0]), math.log(1 + clip[1])):          # a ratio at a bound has no one-sided answer in fp32
        shift = np.where(np.abs(shift - b) < 1e-3, shift + 0.01, shift)
    old, ref = (logp - shift).astype(np.float32), (logp + r.standard_normal(n) * 0.3).astype(np.float32)
    return old, ref, r.standard_normal(n).astype(np.float32), (r.random(n) / n).astype(np.float32)


def check_policy(z, y, tau, dtype, seed, kl=0.1, ent=0.0, use_ref=True, grad_scale=1.0, dlogits=None, forward_only=False):
    yn = y.cpu().numpy()
    old, ref, adv, w = policy_inputs(z, yn, tau, seed)
    rel, tl, ts, tH = token_tols(z, yn, tau)
    want = orc.policy_loss(f64(z), yn, old, adv, w, ref if use_ref else None, np.float32(0.2), np.float32(0.3), np.float32(kl), np.float32(ent), tau, grad_scale)
    t = [torch.tensor(x).cuda() for x in (old, adv, w, ref)]
    zd = f64(z)
    got = B.policy_loss(z, y, t[0], t[1], t[2], ref_logp=t[3] if use_ref else None, clip_low=0.2, clip_high=0.3, kl_coef=kl, entropy_coef=ent,
                        temperature=tau, grad_scale=grad_scale, dlogits=dlogits, forward_only=forward_only)
    within(f64(got.logp), want["logp"], tl, "logp"); within(f64(got.entropy), want["entropy"], tH, "entropy")
    eu = np.exp(ref.astype(np.float64) - want["logp"]) if use_ref else np.zeros(len(yn))
    live = yn >= 0
    dl = np.where(live, tl + 4 * U * (np.abs(old) + np.abs(ref) + 2), 0.0)
    aw = np.abs(w) * live
    tpg = np.sum(aw * np.abs(adv) * want["ratio"] * (dl + 8 * U)) * 2
    tkl = np.sum(aw * (np.abs(eu - 1) * dl + (eu + 3) * 8 * U)) * 2
    tent = np.sum(aw * tH) * 2 + 8 * U * abs(want["stats"][3])
    tol = np.array([tpg + abs(kl) * tkl + abs(ent) * tent, tpg, tkl, tent, 4 * U]) + 4 * U * np.abs(want["stats"])
    within(f64(got.stats), want["stats"], tol, "stats")
    if forward_only:
        assert got.dlogits is None
        return got
    dg = 2 * aw * (np.abs(adv) * want["ratio"] * (dl + 8 * U) + abs(kl) * (eu * dl + (eu + 2) * 8 * U)) + abs(ent) * aw * tH
    h = -ent * w * live
    zz = torch.tensor(zd)      # the logits may have been overwritten
    within(f64(got.dlogits), want["dlogits"], grad_tol(zz, yn, tau, want["g"], h, dg, rel, dtype, want["dlogits"], grad_scale), "dlogits")
    return got


@pytest.mark.parametrize("ent", [0.0, 0.05])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,V,pad,lead", SIZES + [(2, 530001, 0, 0)])
def test_policy_loss(rows, V, pad, lead, dtype, ent):
    z, y = make_rows(dtype, rows, V, pad, 3 + V % 5, lead)
    if rows > 2:
        y[1] = -100
        z[1] = float("inf")
    if V > 8:
        z[rows - 1, 5] = -math.inf
        y[rows - 1] = V - 1
    scale = 256.0 if dtype == "f16" else 1.0
    got = check_policy(z, y, 0.9, dtype, V, ent=ent, grad_scale=scale)
    if rows > 2:
        assert bool((got.dlogits[1] == 0).all()) and got.logp[1] == 0
    if V > 8:
        assert got.dlogits[rows - 1, 5] == 0


@pytest.mark.parametrize("dtype,rows,V,pad,lead", [("bf16", 151, 9001, 0, 3), ("f16", 160, 33000, 1, 0), ("f32", 150, 16390, 0, 1), ("bf16", 150, 70001, 3, 0)])
def test_policy_loss_more_rows_than_sms(dtype, rows, V, pad, lead):
    z, y = make_rows(dtype, rows, V, pad, 8, lead)
    y[3::5] = -7
    check_policy(z, y, 1.1, dtype, V, ent=0.02, grad_scale=64.0)


@pytest.mark.parametrize("dtype,rows,V,pad", [("bf16", 6001, 9001, 0), ("bf16", 2600, 40001, 3), ("f16", 9473, 2051, 0), ("f32", 5003, 4099, 1), ("bf16", 1300, 131073, 0)])
def test_many_rows(dtype, rows, V, pad):
    """Thousands of rows, handed out in units, through the ring or a warp each, against 64-bit arithmetic on the GPU; the
    bounds are those of token_tols, grad_tol and check_policy."""
    z, y = make_rows(dtype, rows, V, pad, 3)
    y[::7] = -1
    z[7] = float("nan")
    g = gen(2)
    n = lambda: torch.randn(rows, generator=g, device="cuda")  # noqa: E731
    lp, lse, H = B.token_logprob(z, y)
    shift, adv, w, gap = n() * 0.05, n(), n(), n() * 0.1
    old, ref = lp - shift, lp + gap                                            # ratios far from the bounds 0.5 and 1.5
    kl, ent = (float(np.float32(v)) for v in (0.1, 0.01))
    got = B.policy_loss(z, y, old, adv, w, ref_logp=ref, clip_low=0.5, clip_high=0.5, kl_coef=kl, entropy_coef=ent)
    grad = B.token_logprob_backward(z, y, lse, adv, entropy=H, grad_entropy=w)
    sums, slack = torch.zeros(5, dtype=torch.float64, device="cuda"), 0.0
    for a in range(0, rows, 100):
        c = slice(a, min(rows, a + 100))
        live = (y[c] >= 0)[:, None]
        x = torch.where(live, z[c].double(), 0.0)
        at = y[c].clamp(min=0)[:, None]
        top = x.amax(1, keepdim=True)
        d, q = top - x, torch.log_softmax(x, 1)
        p = q.exp()
        want_lse, want_lp, want_H = torch.logsumexp(x, 1), q.gather(1, at)[:, 0], -(p * q).sum(1)
        es = sum_err(V) + 2 * 3 * U * (p * d).sum(1, keepdim=True) + 4 * U
        rel = 2 * 4 * U * (d + top.abs() + math.log(V)) + es
        tl = es[:, 0] + 2 * 3 * U * (d.gather(1, at)[:, 0] + math.log(V) + 1)
        tH = 2 * (es[:, 0] + 2 * 3 * U) * (1 + (p * d).sum(1) + math.log(V))
        m = live[:, 0]

        def near(got_, want_, tol_, what):
            off = ((got_.double() - torch.where(m, want_, 0.0)).abs() > tol_) & m | ~m & (got_ != 0)
            assert not bool(off.any()) and not bool(got_.isnan().any()), what

        near(lp[c], want_lp, tl, "logp"); near(got.logp[c], want_lp, tl, "policy logp"); near(got.entropy[c], want_H, tH, "policy entropy")
        near(lse[c], want_lse, es[:, 0] + 2 * 3 * U * (top.abs()[:, 0] + math.log(V) + 1), "lse"); near(H[c], want_H, tH, "entropy")

        def near_grad(got_, gg, hh, dg, what):
            one = torch.zeros_like(p).scatter_(1, at, 1.0)
            want_ = torch.where(live, gg[:, None] * (one - p) - hh[:, None] * p * (q + want_H[:, None]), 0.0)
            per = gg.abs()[:, None] + hh.abs()[:, None] * (q.abs() + want_H[:, None])
            tol = p * per * (rel + 8 * U) + p * hh.abs()[:, None] * rel * (1 + q.abs()) + p * dg[:, None] + one * (gg.abs() * 4 * U + dg)[:, None]
            off = (got_.double() - want_).abs() > 2 * tol + 1.01 * HALF_ULP[dtype] * want_.abs() + TINY[dtype]
            assert not bool(off.any()) and not bool(got_.isnan().any()), what

        A, W = adv[c].double(), w[c].double()
        near_grad(grad[c], A, W, W.abs() * tH, "gradient")
        r, u = (want_lp - old[c].double()).exp(), ref[c].double() - want_lp
        dl = tl + 4 * U * (old[c].abs() + ref[c].abs() + 2).double()
        gg = W * (-r * A - kl * torch.expm1(u))
        dg = 2 * W.abs() * (A.abs() * r * (dl + 8 * U) + kl * (u.exp() * dl + (u.exp() + 2) * 8 * U)) + ent * W.abs() * tH
        near_grad(got.dlogits[c], gg, -ent * W, dg, "policy gradient")
        terms = torch.stack([-r * A, torch.expm1(u) - u, want_H, torch.zeros_like(r)])
        part = (W * terms * m).sum(1)
        sums += torch.cat([(part[0] + kl * part[1] - ent * part[2]).reshape(1), part])
        slack += float((W.abs() * m * (A.abs() * r * (dl + 8 * U) + (u.exp() + 3) * (dl + 8 * U) + tH)).sum())
    assert float((got.stats.double() - sums).abs().max()) <= 2 * slack + 4 * U * float(sums.abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1003, 20000, 131072, 270001])
def test_policy_loss_in_place_elsewhere_and_forward_only(V, dtype):
    z, y = make_rows(dtype, 5, V, 1, 77)
    y[2] = -1
    zc = z.clone()
    a = check_policy(z, y, 1.0, dtype, 1)
    b = check_policy(z, y, 1.0, dtype, 1, forward_only=True)
    within(f64(a.stats), f64(b.stats), 1e-4 * np.abs(f64(b.stats)).max())
    other = torch.empty(5 * (V + 4) + 3, dtype=z.dtype, device="cuda").as_strided((5, V), (V + 4, 1), 3)     # lies differently than the logits
    c = check_policy(z, y, 1.0, dtype, 1, dlogits=other)
    assert torch.equal(c.dlogits, a.dlogits) and torch.equal(z, zc)
    d = check_policy(z, y, 1.0, dtype, 1, dlogits=z)
    assert d.dlogits.data_ptr() == z.data_ptr() and torch.equal(z, a.dlogits) and torch.equal(d.stats, a.stats)
    check_policy(zc, y, 1.0, dtype, 1, use_ref=False, kl=0.5)


def test_policy_ties_let_the_gradient_through():
    # ratio exactly 1 and bounds of 1: both terms are equal
    z = torch.zeros(2, 4, device="cuda")
    y = torch.tensor([1, 2], device="cuda")
    logp = B.token_logprob(z, y)[0]
    r = B.policy_loss(z, y, logp, torch.tensor([1.0, -1.0], device="cuda"), torch.ones(2, device="cuda"), clip_low=0.0, clip_high=0.0)
    assert r.stats.tolist() == [0.0, 0.0, 0.0, pytest.approx(2 * math.log(4), abs=1e-6), 0.0]
    within(f64(r.dlogits), [[0.25, -0.75, 0.25, 0.25], [-0.25, -0.25, 0.75, -0.25]], 4 * U)


def special_rows(dtype, V):
    z = torch.randn(9, V, generator=gen(1), device="cuda").to(DT[dtype])
    low = float(torch.finfo(DT[dtype]).min)
    z[0] = -math.inf                       # nothing is left: no distribution
    z[1] = low                             # the type's lowest value everywhere: uniform
    z[2, 3:] = low                         # and as a mask
    z[3, 1:] = -math.inf                   # one entry is left
    z[4, 2] = math.nan
    z[5, 2] = math.inf
    z[6] = float(torch.finfo(DT[dtype]).max)
    y = torch.tensor([1, 2, 1, 0, 1, 1, 4, V, V - 1], device="cuda")      # row 7: a target beyond the vocabulary
    return z, y


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [12, 3000, 40000, 600000])
def test_special_rows(V, dtype):
    z, y = special_rows(dtype, V)
    one = torch.ones(9, device="cuda")
    logp, lse, H = (f64(x) for x in B.token_logprob(z, y))
    nan = [0, 4, 5, 7]
    fine = [1, 2, 3, 6, 8]
    assert np.isnan(logp[nan]).all() and not np.isnan(logp[fine]).any() and not np.isnan(H[fine]).any()
    e = sum_err(V) + 1e-6 * math.log(V)
    assert abs(logp[1] + math.log(V)) < e and abs(logp[6] + math.log(V)) < e and abs(H[1] - math.log(V)) < 2 * e
    assert abs(logp[3]) < 1e-6 and abs(H[3]) < 1e-6
    r = B.policy_loss(z, y, torch.nan_to_num(B.token_logprob(z, y)[0]), one, one, entropy_coef=0.1)
    d = f64(r.dlogits)
    assert np.isnan(d[nan]).any(1).all() and not np.isnan(d[fine]).any() and np.isnan(f64(r.stats)[0])
    within(d[1], np.where(np.arange(V) == 2, 1.0 / V - 1.0, 1.0 / V), 1e-6 + HALF_ULP[dtype] * 1.0)
    assert (d[2, 3:] == 0).all() and (d[3] == 0).all()
    s = B.preference_loss(z[1:4], y[1:4], torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda"), torch.zeros(3, device="cuda"))
    assert not np.isnan(f64(s.dlogits)).any()
    # the pair's loss falls with the chosen row's log-probability: coefficient c < 0, gradient c (1[target] - 1 / V)
    lp = -math.log(V)
    hh = 0.1 * (lp - f64(s.logp)[1:].sum())
    c = -0.1 / (1 + math.exp(hh))
    row = c * ((np.arange(V) == 2) - 1.0 / V)
    within(f64(s.dlogits)[0], row, 2 * np.abs(c) * (np.where(np.arange(V) == 2, 1.0, 1.0 / V) * (e + 0.1 * 4 * e)) + 1.01 * HALF_ULP[dtype] * np.abs(row) + TINY[dtype])


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V,pad,lead,starts", [
    (50, 0, 0, [0, 3, 5]), (1003, 2, 1, [1, 4, 4, 9, 10, 15, 17]), (8192, 0, 0, [0, 40, 90, 130, 150]), (33001, 0, 5, [0, 4, 8, 12, 12]), (140001, 1, 0, [0, 2, 5]),
])
def test_preference_loss(V, pad, lead, starts, dtype, smoothing):
    rows = starts[-1] + 2                      # rows after the last answer belong to none
    z, y = make_rows(dtype, rows, V, pad, 5 + V % 3, lead)
    y[::4] = -100
    z[0] = float("nan")
    yn = y.cpu().numpy()
    tau, scale, beta = 0.8, 1024.0 if dtype == "f16" else 1.0, 0.3
    rel, tl, ts, tH = token_tols(z, yn, tau)
    ref = (orc.token_logprob(f64(z), yn, tau)[0] + np.random.default_rng(1).standard_normal(rows) * 0.5).astype(np.float32)
    want = orc.preference_loss(f64(z), yn, starts, ref, np.float32(beta), np.float32(smoothing), tau, scale)
    got = B.preference_loss(z, y, torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(ref).cuda(), beta, smoothing, tau, scale)
    within(f64(got.logp), want["logp"], tl, "logp")
    tR = np.array([2 * beta * (np.sum(tl[a:b]) + U) + 2 * U for a, b in zip(starts, starts[1:])]) + 2 * U * np.abs(want["rewards"])
    within(f64(got.rewards), want["rewards"], tR, "rewards")
    th = tR[0::2] + tR[1::2]
    within(f64(got.loss), want["loss"], th.mean() + 4 * U * want["loss"], "loss")
    dg = np.zeros(rows)
    for s in range(len(starts) - 1):
        dg[starts[s]:starts[s + 1]] = beta * th[s // 2] / len(th) + 8 * U * np.abs(want["g"][starts[s]:starts[s + 1]])
    within(f64(got.dlogits), want["dlogits"], grad_tol(z, yn, tau, want["g"], 0 * dg, dg, rel, dtype, want["dlogits"], scale), "dlogits")
    fwd = B.preference_loss(z, y, torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(ref).cuda(), beta, smoothing, tau, forward_only=True)
    assert torch.equal(fwd.rewards, got.rewards) and torch.equal(fwd.loss, got.loss) and fwd.dlogits is None
    whole = z._base.clone()                    # lies in memory like the logits: the order of the sums follows the alignment
    z2 = whole.as_strided(z.shape, z.stride(), z.storage_offset())
    same = B.preference_loss(z2, y, torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.tensor(ref).cuda(), beta, smoothing, tau, scale, dlogits=z2)
    assert torch.equal(same.dlogits, got.dlogits) and torch.equal(same.loss, got.loss)


def test_preference_starts_that_make_no_sense_stay_inside():
    z, y = make_rows("f32", 6, 40, 0, 1)
    ref = torch.zeros(6, device="cuda")
    r = B.preference_loss(z, y, torch.tensor([-5, 3, 1, 900, 2], dtype=torch.int32, device="cuda"), ref)
    assert bool(torch.isfinite(r.rewards).all())


def test_calls_without_rows():
    z, y, e = torch.zeros(0, 10, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda")
    assert B.token_logprob(z, y)[0].shape == (0,)
    r = B.policy_loss(z, y, e, e, e)
    assert r.stats.tolist() == [0.0] * 5 and r.dlogits.shape == (0, 10)
    s = B.preference_loss(z, y, torch.zeros(3, dtype=torch.int32, device="cuda"), e)
    assert s.loss.item() == pytest.approx(math.log(2), abs=1e-6) and s.rewards.tolist() == [0.0, 0.0]
    z, y = make_rows("f32", 3, 10, 0, 0)
    s = B.preference_loss(z, y, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(3, device="cuda"))
    assert s.loss.item() == 0.0 and bool((s.dlogits == 0).all())


def test_rows_past_32_bits():
    V, rows = 131072, 16500
    z = torch.zeros(rows, V, dtype=torch.bfloat16, device="cuda")
    y = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    tail = torch.randn(2, V, generator=gen(0), device="cuda").bfloat16()
    z[-2:] = tail
    y[-2:] = torch.tensor([5, V - 1], device="cuda")
    f = lambda a, b: B.policy_loss(a, b, *(torch.ones(len(b), device="cuda") * c for c in (-12.0, 1.0, 0.5)))  # noqa: E731
    big, small = f(z, y), f(tail, y[-2:].clone())
    assert torch.equal(big.dlogits[-2:], small.dlogits) and torch.equal(big.logp[-2:], small.logp) and torch.equal(big.stats, small.stats)
    assert bool((big.dlogits[:-2].abs().amax(1) == 0).all())
    lp = B.token_logprob(z, y)
    assert torch.equal(lp[0][-2:], B.token_logprob(tail, y[-2:].clone())[0])


@pytest.mark.parametrize("what", ["policy", "preference"])
def test_gradient_against_differences(what):
    """The loss along a direction, by central differences of the library's own loss.  With steps of 2^-6 the difference's
    own error is e^2 |third derivative| / 6 <= e^2 / 6 sum over the tokens, and the losses' roundings are 1e-6 / e."""
    z, y = make_rows("f32", 8, 500, 0, 4)
    y[3] = -1
    logp = B.token_logprob(z, y)[0]
    d = torch.zeros_like(z)
    d.scatter_(1, y.clamp(min=0)[:, None], 1.0)
    d += torch.randn(z.shape, generator=gen(9), device="cuda") * 0.1
    if what == "policy":
        w = torch.rand(8, generator=gen(5), device="cuda") / 8
        f = lambda x: B.policy_loss(x, y, logp - 0.05, torch.linspace(-1, 1, 8, device="cuda"), w, ref_logp=logp + 0.3, kl_coef=0.5, entropy_coef=0.1)  # noqa: E731
        value = lambda r: float(r.stats[0].double())  # noqa: E731
    else:
        f = lambda x: B.preference_loss(x, y, torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"), logp - 0.2, 0.5, 0.1)  # noqa: E731
        value = lambda r: float(r.loss.double())  # noqa: E731
    e = 2.0 ** -6
    d *= torch.where(torch.arange(8, device="cuda") < 4, 1.0, -1.0)[:, None]
    num = (value(f(z + e * d)) - value(f(z - e * d))) / (2 * e)
    ana = float((f(z).dlogits.double() * d.double()).sum())
    assert abs(num - ana) < e * e / 6 * 8 + 1e-6 * 8 / e and abs(ana) > 1e-2


def test_other_stream_graph_and_determinism():
    z, y = make_rows("bf16", 64, 10007, 0, 2)
    one = torch.ones(64, device="cuda")
    want = B.policy_loss(z, y, one * -8, one, one / 64)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    r = B.policy_loss(z, y, one * -8, one, one / 64, stream=side)
    n = B.grad_norm([z], 1.0, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(r.dlogits, want.dlogits) and torch.equal(r.stats, want.stats) and torch.equal(n, B.grad_norm([z], 1.0))
    starts = torch.tensor([0, 20, 64], dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p = B.preference_loss(z, y, starts, one * -8)
        q = B.policy_loss(z, y, one * -8, one, one / 64)
        c = B.clip_grads([q.dlogits.view(-1)], 1e-3)
    z.copy_(z.flip(0))
    y.copy_(y.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    again = B.policy_loss(z, y, one * -8, one, one / 64)
    cc = B.clip_grads([again.dlogits.view(-1)], 1e-3)
    assert torch.equal(q.dlogits, again.dlogits) and torch.equal(c, cc) and torch.equal(p.dlogits, B.preference_loss(z, y, starts, one * -8).dlogits)


def test_binding_refuses():
    z, y = make_rows("f32", 4, 10, 0, 0)
    f = torch.zeros(4, device="cuda")
    for bad in (lambda: B.token_logprob(z.t(), torch.zeros(10, dtype=torch.int64, device="cuda")), lambda: B.token_logprob(z, y.int()),
                lambda: B.token_logprob(z, y[:3]), lambda: B.token_logprob(z.double(), y), lambda: B.token_logprob(z, y.cpu()),
                lambda: B.token_logprob(z[None], y), lambda: B.policy_loss(z, y, f.double(), f, f), lambda: B.policy_loss(z, y, f, f[:3], f),
                lambda: B.policy_loss(z, y, f, f, f.cpu()), lambda: B.policy_loss(z, y, f, f, f, dlogits=z.bfloat16()),
                lambda: B.token_logprob_backward(z, y, f, f, grad_entropy=f), lambda: B.preference_loss(z, y, torch.zeros(4, dtype=torch.int32, device="cuda"), f),
                lambda: B.preference_loss(z, y, torch.zeros(3, dtype=torch.int64, device="cuda"), f)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.token_logprob(z, y, temperature=0.0), lambda: B.policy_loss(z, y, f, f, f, clip_low=2.0),
                lambda: B.preference_loss(z, y, torch.zeros(3, dtype=torch.int32, device="cuda"), f, label_smoothing=2.0), lambda: B.clip_grads([f], 0.0)):
        with pytest.raises(B.TgradError) as e:
            bad()
        assert e.value.status == B.ERR_INVALID_ARG
