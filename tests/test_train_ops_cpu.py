"""The 64-bit definitions of the operators around the step against autograd and differences, and what the library refuses
on the host.  No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import train_oracle as orc
from paper_2501_02379_b200 import binding as B
from paper_2501_02379_b200 import build as builder

rng = np.random.default_rng


@pytest.fixture(scope="module", autouse=True)
def _built():
    builder.build()


def _rows(seed, n=7, v=11):
    r = rng(seed)
    z = r.standard_normal((n, v)) * 2
    y = r.integers(0, v, n)
    y[2] = -100
    z[3, 4] = -np.inf if y[3] != 4 else z[3, 4]
    return r, z, y


# ---- the definitions ----
def test_adamw_is_torchs():
    r = rng(0)
    w, g = r.standard_normal(50), r.standard_normal(50)
    p = torch.nn.Parameter(torch.tensor(w))
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.95), eps=1e-7, weight_decay=0.1)
    m, v = np.zeros(50), np.zeros(50)
    for step in range(1, 4):
        p.grad = torch.tensor(g * step * 0.5)
        opt.step()
        w, m, v = orc.adamw(w, g * step, m, v, step, 1e-2, 0.9, 0.95, 1e-7, 0.1, scale=0.5)
    assert np.abs(w - p.detach().numpy()).max() < 1e-14


def test_grad_norm_is_torchs():
    r = rng(1)
    gs = [r.standard_normal(7), r.standard_normal((3, 4)) + 1j * r.standard_normal((3, 4)), np.zeros(0)]
    ps = [torch.nn.Parameter(torch.tensor(np.zeros_like(g))) for g in gs]
    for p, g in zip(ps, gs):
        p.grad = torch.tensor(g)
    norm, c, norms = orc.grad_norm(gs, 0.7)
    assert abs(float(torch.nn.utils.clip_grad_norm_(ps, 0.7)) - norm) < 1e-12
    assert np.allclose(ps[1].grad.numpy(), gs[1] * c, atol=1e-15) and norms[2] == 0.0


def _autograd(z, f):
    t = torch.tensor(z, requires_grad=True)
    out = f(t)
    out.backward()
    return float(out), t.grad.numpy()


@pytest.mark.parametrize("tau", [1.0, 0.6])
def test_token_gradient_is_autograds(tau):
    r, z, y = _rows(2)
    g, h = r.standard_normal(7), r.standard_normal(7)
    live = torch.tensor(y >= 0)

    def f(t):
        q = torch.log_softmax(t / tau, 1)
        lp = q.gather(1, torch.tensor(np.maximum(y, 0))[:, None])[:, 0]
        H = torch.special.entr(q.exp()).sum(1)
        return ((torch.tensor(g) * lp + torch.tensor(h) * H)[live]).sum()

    zf = np.where(np.isinf(z), -40.0, z)      # autograd of entr at -inf is NaN; the limit is what is wanted
    _, want = _autograd(zf, f)
    assert np.abs(orc.token_gradient(zf, y, g, h, tau) - want).max() < 1e-12
    got = orc.token_gradient(z, y, g, h, tau)
    assert np.abs(got - want).max() < 1e-12 and np.all(got[np.isinf(z)] == 0) and np.all(got[2] == 0)


def test_policy_loss_is_autograds_and_differences():
    r, z, y = _rows(3)
    z = np.where(np.isinf(z), -3.0, z)
    logp = orc.token_logprob(z, y)[0]
    old, ref, adv, w = logp + r.standard_normal(7) * 0.4, logp + r.standard_normal(7) * 0.3, r.standard_normal(7), r.random(7)
    kw = dict(ref=ref, clip_low=0.1, clip_high=0.3, kl_coef=0.2, entropy_coef=0.05, tau=1.0)
    out = orc.policy_loss(z, y, old, adv, w, **kw)
    live = torch.tensor(y >= 0)

    def f(t):
        q = torch.log_softmax(t, 1)
        lp = q.gather(1, torch.tensor(np.maximum(y, 0))[:, None])[:, 0]
        rr, A = (lp - torch.tensor(old)).exp(), torch.tensor(adv)
        u = torch.tensor(ref) - lp
        per = -torch.minimum(rr * A, rr.clamp(0.9, 1.3) * A) + 0.2 * (u.exp() - u - 1) + 0.05 * (q.exp() * q).sum(1)
        return (per * torch.tensor(w))[live].sum()

    loss, grad = _autograd(z, f)
    assert abs(loss - out["stats"][0]) < 1e-12 and np.abs(grad - out["dlogits"]).max() < 1e-12
    d = r.standard_normal(z.shape)
    e = 1e-6
    num = (orc.policy_loss(z + e * d, y, old, adv, w, **kw)["stats"][0] - orc.policy_loss(z - e * d, y, old, adv, w, **kw)["stats"][0]) / (2 * e)
    assert abs(num - np.sum(d * out["dlogits"])) < 1e-7


def test_preference_loss_is_autograds_and_differences():
    r, z, y = _rows(4, 9, 6)
    z = np.where(np.isinf(z), -3.0, z)
    starts = [1, 3, 5, 5, 8]                 # a row before and one after the answers, an empty answer
    ref = orc.token_logprob(z, y)[0] + r.standard_normal(9) * 0.5
    out = orc.preference_loss(z, y, starts, ref, 0.7, 0.1)
    live = torch.tensor((y >= 0).astype(float))

    def f(t):
        q = torch.log_softmax(t, 1).gather(1, torch.tensor(np.maximum(y, 0))[:, None])[:, 0]
        gap = (q - torch.tensor(ref)) * live
        R = torch.stack([0.7 * gap[a:b].sum() for a, b in zip(starts, starts[1:])])
        h = R[0::2] - R[1::2]
        return -(0.9 * torch.nn.functional.logsigmoid(h) + 0.1 * torch.nn.functional.logsigmoid(-h)).mean()

    loss, grad = _autograd(z, f)
    assert abs(loss - out["loss"]) < 1e-12 and np.abs(grad - out["dlogits"]).max() < 1e-12
    d, e = r.standard_normal(z.shape), 1e-6
    num = (orc.preference_loss(z + e * d, y, starts, ref, 0.7, 0.1)["loss"] - orc.preference_loss(z - e * d, y, starts, ref, 0.7, 0.1)["loss"]) / (2 * e)
    assert abs(num - np.sum(d * out["dlogits"])) < 1e-7


# ---- refusals of the C entry points: the pointers are plain numbers, so a call that got past its checks would launch ----
def _refused(call, status):
    n0 = B.launch_count()
    assert call() == status
    assert B.launch_count() == n0


def _tensor(data=0x10000, numel=8, dtype=B.R32):
    return (B.TgradTensor * 1)(B.TgradTensor(data, numel, dtype, 0))


@pytest.mark.parametrize("entry", ["tgrad_grad_norm", "tgrad_clip_grads"])
def test_list_calls_refuse(entry):
    f = getattr(B.lib(), entry)
    big = 1 << 20
    ok = _tensor()
    bad = B.ERR_INVALID_ARG
    for arr in (_tensor(data=0), _tensor(data=0x10002), _tensor(dtype=6), _tensor(dtype=-1), _tensor(numel=-1), _tensor(numel=1 << 48),
                _tensor(data=0x10001, dtype=B.R16B)):
        _refused(lambda: f(C.addressof(arr), 1, 1.0, 0x20000, 0x30000, big, None), bad)
    _refused(lambda: f(None, 1, 1.0, 0x20000, 0x30000, big, None), bad)
    _refused(lambda: f(C.addressof(ok), -1, 1.0, 0x20000, 0x30000, big, None), bad)
    for m in (0.0, -1.0, float("nan")):
        _refused(lambda: f(C.addressof(ok), 1, m, 0x20000, 0x30000, big, None), bad)
    _refused(lambda: f(C.addressof(ok), 1, 1.0, None, 0x30000, big, None), bad)
    _refused(lambda: f(C.addressof(ok), 1, 1.0, 0x20002, 0x30000, big, None), bad)
    _refused(lambda: f(C.addressof(ok), 1, 1.0, 0x20000, None, big, None), bad)
    _refused(lambda: f(C.addressof(ok), 1, 1.0, 0x20000, 0x30010, big, None), bad)
    _refused(lambda: f(C.addressof(ok), 1, 1.0, 0x20000, 0x30000, 64, None), B.ERR_BUFFER_TOO_SMALL)


def test_adamw_refuses():
    def call(cfg=None, **kw):
        t = B.TgradAdamwTensor(0x1000, 0x2000, 0x3000, 0x4000, None, 8, B.R32, 0)
        for k, v in kw.items():
            setattr(t, k, v)
        c = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, grad_scale=None)
        c.update(cfg or {})
        arr, cc = (B.TgradAdamwTensor * 1)(t), B.TgradAdamwConfig(**c)
        return B.lib().tgrad_adamw_step(C.addressof(arr), 1, C.addressof(cc), None)

    for kw in (dict(weight=0), dict(grad=0), dict(exp_avg=0), dict(exp_avg_sq=0), dict(weight=0x1002), dict(exp_avg=0x3002), dict(numel=-1),
               dict(dtype=9), dict(master=0x5000), dict(dtype=B.R16B, master=0x5002)):
        _refused(lambda: call(**kw), B.ERR_INVALID_ARG)
    for dt in (B.C32H, B.C32B):
        _refused(lambda: call(dtype=dt), B.ERR_UNSUPPORTED)
    for cfg in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(step=0), dict(lr=float("nan")), dict(weight_decay=float("inf")), dict(grad_scale=0x7001)):
        _refused(lambda: call(cfg), B.ERR_INVALID_ARG)
    assert B.lib().tgrad_adamw_step(None, 1, None, None) == B.ERR_INVALID_ARG


def _desc(**kw):
    d = B.TgradLogits(0x10000, 4, 100, 100, 0x20000, B.R16B, 1.0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


BAD_LOGITS = [dict(logits=None), dict(logits=0x10001), dict(rows=-1), dict(vocab=0), dict(vocab=1 << 31), dict(row_stride=99), dict(targets=None),
              dict(targets=0x20004), dict(dtype=B.C64), dict(dtype=B.C32H), dict(dtype=77), dict(temperature=0.0), dict(temperature=-1.0),
              dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-39)]


@pytest.mark.parametrize("bad", BAD_LOGITS)
def test_logits_calls_refuse(bad):
    l, d = B.lib(), _desc(**bad)
    a = C.addressof(d)
    _refused(lambda: l.tgrad_token_logprob(a, 0x3000, 0x4000, 0x5000, None), B.ERR_INVALID_ARG)
    _refused(lambda: l.tgrad_token_logprob_backward(a, 0x3000, 0x4000, 0x5000, 0x6000, 0x70000, 100, None), B.ERR_INVALID_ARG)
    p, q = _policy(), _preference()
    _refused(lambda: l.tgrad_policy_loss(a, C.addressof(p), 0x90000, 1 << 20, None), B.ERR_INVALID_ARG)
    _refused(lambda: l.tgrad_preference_loss(a, C.addressof(q), 0x90000, 1 << 20, None), B.ERR_INVALID_ARG)


def _policy(**kw):
    p = B.TgradPolicyArgs(0x1000, None, 0x2000, 0x3000, 0.2, 0.2, 0.1, 0.01, 1.0, 0.0, 0x4000, 0x5000, 0x6000, 0x70000, 100)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _preference(**kw):
    p = B.TgradPreferenceArgs(0x1000, 0x2000, 1, 0.1, 0.0, 1.0, 0x3000, 0x4000, 0x5000, 0x70000, 100)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("bad", [dict(old_logp=None), dict(advantages=None), dict(weights=0x3002), dict(ref_logp=0x1001), dict(stats=None), dict(logp=0x5001),
                                 dict(dlogits=0x70001), dict(dlogits_stride=99), dict(dlogits=0x10000, dlogits_stride=101), dict(clip_low=-0.1),
                                 dict(clip_low=1.1), dict(clip_high=-0.1), dict(kl_coef=float("nan")), dict(entropy_coef=float("inf")),
                                 dict(grad_scale=float("nan"))])
def test_policy_loss_refuses(bad):
    d, p = _desc(), _policy(**bad)
    _refused(lambda: B.lib().tgrad_policy_loss(C.addressof(d), C.addressof(p), 0x90000, 1 << 20, None), B.ERR_INVALID_ARG)


@pytest.mark.parametrize("bad", [dict(starts=None), dict(ref_logp=None), dict(pairs=-1), dict(beta=float("nan")), dict(label_smoothing=-0.1),
                                 dict(label_smoothing=1.1), dict(loss=None), dict(rewards=None), dict(logp=None), dict(dlogits=0x70001), dict(dlogits_stride=3)])
def test_preference_loss_refuses(bad):
    d, p = _desc(), _preference(**bad)
    _refused(lambda: B.lib().tgrad_preference_loss(C.addressof(d), C.addressof(p), 0x90000, 1 << 20, None), B.ERR_INVALID_ARG)


def test_workspaces_are_checked():
    l, d, p, q, b = B.lib(), _desc(), _policy(), _preference(), C.c_size_t(0)
    for ws in (None, 0x90010):
        _refused(lambda: l.tgrad_policy_loss(C.addressof(d), C.addressof(p), ws, 1 << 20, None), B.ERR_INVALID_ARG)
        _refused(lambda: l.tgrad_preference_loss(C.addressof(d), C.addressof(q), ws, 1 << 20, None), B.ERR_INVALID_ARG)
    _refused(lambda: l.tgrad_policy_loss(C.addressof(d), C.addressof(p), 0x90000, 16, None), B.ERR_BUFFER_TOO_SMALL)
    _refused(lambda: l.tgrad_preference_loss(C.addressof(d), C.addressof(q), 0x90000, 16, None), B.ERR_BUFFER_TOO_SMALL)
    assert l.tgrad_policy_loss_bytes(-1, C.byref(b)) == B.ERR_INVALID_ARG and l.tgrad_policy_loss_bytes(5, None) == B.ERR_INVALID_ARG
    assert l.tgrad_preference_loss_bytes(5, -1, C.byref(b)) == B.ERR_INVALID_ARG
    assert l.tgrad_grad_norm_bytes(-1, C.byref(b)) == B.ERR_INVALID_ARG
    assert l.tgrad_grad_norm_bytes(5000, C.byref(b)) == B.OK and b.value > 0


def test_scaled_step_refuses_a_misaligned_scale():
    assert B.lib().tgrad_step_scaled(None, 0x1000, 0x2000, 0x3000, None) == B.ERR_INVALID_ARG
    assert B.lib().tgrad_step_batched_scaled(None, None, None, 0, 0x3001, None) == B.ERR_INVALID_ARG
    assert B.lib().tgrad_step_batched_scaled(None, None, None, 0, 0x3000, None) == B.OK


def test_binding_refuses_tensors_it_cannot_describe():
    z = torch.zeros(4, 5)
    with pytest.raises(ValueError):
        B.TensorList([torch.zeros(3)])                      # not on a CUDA device
    with pytest.raises(ValueError):
        B.token_logprob(z, torch.zeros(4, dtype=torch.int64))
    assert B._dense(torch.zeros(3, 4).t()) and B._dense(torch.zeros(2, 3, 4).permute(2, 0, 1)) and B._dense(torch.zeros(1, 5)[:, :])
    assert not B._dense(torch.zeros(3, 4)[:, :2]) and not B._dense(torch.zeros(3).expand(2, 3)) and B._dense(torch.zeros(0, 4)[:, :2])
