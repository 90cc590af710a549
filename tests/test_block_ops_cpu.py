"""The 64-bit definitions of the operators of a trained block against autograd and differences, the format of the kept
activations, and what the library refuses on the host.  No GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import block_oracle as orc
from paper_2501_02379_b200 import binding as B
from paper_2501_02379_b200 import build as builder

rng = np.random.default_rng


@pytest.fixture(scope="module", autouse=True)
def _built():
    builder.build()


# ---- the definitions ----
def test_kept_entries_are_within_half_a_step():
    r = rng(0)
    x = r.standard_normal((9, 77)) * 10.0 ** r.integers(-9, 9, (9, 1))
    x[4, :40] = 0
    k = orc.kept(x)
    for at in range(0, 77, 32):
        top = np.abs(x[:, at:at + 32]).max(1, keepdims=True)
        step = np.where(top > 0, 2.0 ** (np.floor(np.log2(np.where(top > 0, top, 1))) - 6), 0)
        near = np.abs(x[:, at:at + 32]) > 127.5 * step          # codes that are clamped
        assert np.all(np.abs(k[:, at:at + 32] - x[:, at:at + 32]) <= np.where(near, step, step / 2))
    assert np.all(orc.kept(k) == k)                             # what was read back is kept as it is
    assert np.all(torch.tensor(k).bfloat16().double().numpy() == k)


@pytest.mark.parametrize("x,code,byte", [(1.0, 64, 121), (-127.4, -127, 127), (127.6, 127, 127), (128.0, 64, 128), (2.5 / 64, 80, 116), (0.0, 0, 0),
                                         (2.0 ** -126, 1, 1), (2.0 ** -127, 0, 1), (3.3895e38, 127, 248), (float("inf"), 0, 255), (float("nan"), 0, 255)])
def test_codes(x, code, byte):
    c, b = orc.packed(np.array([[x]]))
    assert c[0, 0] == code and b[0, 0] == byte


@pytest.mark.parametrize("act,torch_act", [("silu", torch.nn.functional.silu), ("gelu", torch.nn.functional.gelu),
                                           ("gelu_tanh", lambda v: torch.nn.functional.gelu(v, approximate="tanh"))])
def test_activation_is_torchs(act, torch_act):
    r = rng(1)
    a, u, dy = (r.standard_normal((5, 7)) * 2 for _ in range(3))
    ta, tu = (torch.tensor(v, requires_grad=True) for v in (a, u))
    y = torch_act(ta) * tu
    y.backward(torch.tensor(dy))
    assert np.abs(orc.gated(act, a, u) - y.detach().numpy()).max() < 1e-13
    for got, want in zip(orc.gated_gradient(act, a, u, dy), (ta.grad, tu.grad)):
        assert np.abs(got - want.numpy()).max() < 1e-13
    h = 1e-6
    d = (orc.gated(act, a + h) - orc.gated(act, a - h)) / (2 * h)
    assert np.abs(orc.gated_gradient(act, a, None, np.ones_like(a))[0] - d).max() < 1e-8


def _norm_case(seed, layer, post, gate, starts, rows=12, width=10):
    r = rng(seed)
    groups = {"none": 0, "one": 1, "equal": 3, "ragged": 4, "rows": rows}[gate]
    v = {k: r.standard_normal(width) for k in ("weight", "bias", "post_weight", "post_bias")}
    if not layer:
        v["bias"] = v["post_bias"] = np.zeros(width)
    return (r.standard_normal((rows, width)), r.standard_normal((rows, width)), v, r.standard_normal((groups, width)) if groups else None,
            [0, 0, 5, 9, 10] if gate == "ragged" else None, r.standard_normal((rows, width)), r.standard_normal((rows, width)))


@pytest.mark.parametrize("gate", ["none", "one", "equal", "ragged", "rows"])
@pytest.mark.parametrize("layer,post", [(False, True), (True, True), (False, False), (True, False)])
def test_norm_gradient_is_that_of_differences(layer, post, gate):
    x, f, v, gates, starts, dh, dx = _norm_case(2, layer, post, gate, None)
    scale, eps = 0.7, 1e-3

    def loss(x, f, v, gates):
        new, h, stats = orc.residual_norm(x, f, v["weight"], v["bias"], v["post_weight"], v["post_bias"], gates, starts, scale, layer, post, eps)
        return (new * dx).sum() + (h * dh).sum(), new, stats

    _, new, stats = loss(x, f, v, gates)
    got = orc.residual_norm_gradient(dh, dx, new, f, stats, v["weight"], v["post_weight"], v["post_bias"], gates, starts, scale, layer, post)
    args = {"x": x, "f": f, "gate": gates, **v}
    names = ["x", "f", "weight"] + (["gate"] if gates is not None else []) + (["bias"] if layer else []) + (["post_weight"] + (["post_bias"] if layer else []) if post else [])
    r = rng(3)
    for name in names:
        way = r.standard_normal(args[name].shape)
        h = 1e-5
        ends = []
        for s in (h, -h):
            moved = {**args, name: args[name] + s * way}
            ends.append(loss(moved["x"], moved["f"], moved, moved["gate"])[0])
        assert abs((ends[0] - ends[1]) / (2 * h) - (got[name] * way).sum()) < 1e-6 * (1 + np.abs(got[name] * way).sum()), name


def test_layer_norm_is_torchs():
    x, _, v, *_ = _norm_case(4, True, True, "none", None)
    n, _, _ = orc.norm(x, v["weight"], v["bias"], True, 1e-5)
    want = torch.nn.functional.layer_norm(torch.tensor(x), (10,), torch.tensor(v["weight"]), torch.tensor(v["bias"]), 1e-5)
    assert np.abs(n - want.numpy()).max() < 1e-13


# ---- what the library refuses ----
P = 4096      # an address that is aligned like device memory; nothing reads it


def rows(p=P, stride=64):
    return B._pack_rows(p, stride)


def test_packed_bytes():
    n = C.c_size_t(0)
    for r, w, want in [(0, 1, 0), (1, 1, 36), (3, 32, 108), (2, 33, 136), (5, 4096, 5 * (4096 + 128)), (7, 161, 7 * (192 + 8))]:
        assert B.lib().tgrad_packed_bytes(r, w, C.byref(n)) == B.OK and n.value == want == B._packed_bytes(r, w)
    for r, w in [(-1, 4), (4, 0), (4, (1 << 30) + 1), (1 << 40, 4), ((1 << 40) - 1, 1 << 30)]:
        assert B.lib().tgrad_packed_bytes(r, w, C.byref(n)) == B.ERR_INVALID_ARG
    assert B.lib().tgrad_packed_bytes(1, 1, None) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["tgrad_act_pack", "tgrad_act_unpack"])
def test_pack_refusals(name):
    call = getattr(B.lib(), name)

    def go(x=rows(), n=4, width=64, dtype=B.R16B, packed=P):
        return call(x, n, width, dtype, packed, None) if name == "tgrad_act_pack" else call(packed, n, width, dtype, x, None)

    assert go(n=0) == B.OK                                  # nothing to do, and nothing is looked at
    for bad in (dict(x=None), dict(x=rows(0)), dict(x=rows(P + 1)), dict(x=rows(stride=63)), dict(x=rows(P + 2), dtype=B.R32), dict(packed=None),
                dict(packed=P + 8), dict(width=0), dict(n=-1), dict(dtype=B.C64), dict(dtype=9)):
        assert go(**bad) == B.ERR_INVALID_ARG, bad


def gated(n=4, width=64, dtype=B.R16B, act=0, a=(P, 64), u=(P, 64), y=(P, 64), a8=P, u8=P, y8=0):
    return B._pack_gated(n, width, dtype, act, *a, *u, *y, a8, u8, y8)


def test_gated_refusals():
    fwd, bwd = B.lib().tgrad_gated_act, B.lib().tgrad_gated_act_backward
    assert fwd(gated(n=0), None) == B.OK and bwd(gated(n=0, y8=P), None) == B.OK
    for call in (fwd, bwd):
        assert call(None, None) == B.ERR_INVALID_ARG
        for bad in (dict(act=3), dict(act=-1), dict(dtype=B.C32H), dict(a=(0, 64)), dict(y=(0, 64)), dict(a=(P + 1, 64)), dict(y=(P, 63)), dict(u=(P, 5)),
                    dict(a8=P + 4), dict(u8=P + 4), dict(n=-1), dict(width=0)):
            assert call(gated(**bad), None) == B.ERR_INVALID_ARG, bad
    assert fwd(gated(a8=0), None) == B.ERR_INVALID_ARG              # u kept without a
    assert fwd(gated(u8=0), None) == B.ERR_INVALID_ARG              # a kept without u
    assert fwd(gated(u=(0, 64)), None) == B.ERR_INVALID_ARG         # nothing to keep as u
    assert fwd(gated(y8=P), None) == B.ERR_INVALID_ARG              # the backward call's
    assert bwd(gated(a8=0), None) == B.ERR_INVALID_ARG
    assert bwd(gated(u=(0, 64)), None) == B.ERR_INVALID_ARG         # no place for du
    assert bwd(gated(u8=0), None) == B.ERR_INVALID_ARG              # du without a kept u
    assert bwd(gated(y8=P + 2), None) == B.ERR_INVALID_ARG


def config(n=4, width=64, dtype=B.R16B, pd=B.R32, layer=0, post=1, scale=1.0, eps=1e-6, groups=0, starts=0, w=0, b=0, pw=0, pb=0, gate=0, gate_stride=64):
    return B._pack_norm(n, width, dtype, pd, layer, post, scale, eps, groups, 0, starts, w, b, pw, pb, gate, gate_stride)


BAD_NORMS = [dict(width=0), dict(n=-1), dict(dtype=B.C64), dict(pd=B.R16H), dict(pd=7), dict(scale=float("inf")), dict(eps=-1.0), dict(eps=float("nan")),
             dict(groups=-1), dict(groups=1), dict(gate=P), dict(starts=P), dict(groups=3, gate=P), dict(groups=2, gate=P, gate_stride=63),
             dict(groups=2, gate=P + 2), dict(groups=2, gate=P, starts=P + 2), dict(b=P), dict(pb=P), dict(w=P + 2), dict(post=0, pw=P), dict(layer=1, post=0, pb=P)]


def test_norm_refusals():
    call = B.lib().tgrad_residual_norm

    def io(x=(P, 64), f=(P, 64), ox=(P, 64), oh=(P, 64), x8=0, f8=0, h8=0, stats=P):
        return B._pack_norm_forward(*x, *f, *ox, *oh, x8, f8, h8, stats)

    assert call(config(n=0), io(), None) == B.OK
    assert call(None, io(), None) == B.ERR_INVALID_ARG and call(config(), None, None) == B.ERR_INVALID_ARG
    for bad in BAD_NORMS:
        assert call(config(**bad), io(), None) == B.ERR_INVALID_ARG, bad
    for bad in (dict(width=16385), dict(n=1 << 31)):
        assert call(config(**bad), io(), None) == B.ERR_UNSUPPORTED
    for bad in (dict(x=(0, 64)), dict(oh=(0, 64)), dict(x=(P, 63)), dict(f=(P + 1, 64)), dict(ox=(P, 5)), dict(x8=P + 8), dict(f8=P + 8), dict(h8=P + 8), dict(stats=P + 2)):
        assert call(config(), io(**bad), None) == B.ERR_INVALID_ARG, bad
    assert call(config(), io(f=(0, 0), f8=P), None) == B.ERR_INVALID_ARG              # nothing to keep
    assert call(config(pw=P), io(f=(0, 0)), None) == B.ERR_INVALID_ARG                # no block, but its norm
    assert call(config(groups=1, gate=P), io(f=(0, 0)), None) == B.ERR_INVALID_ARG


def test_norm_backward_refusals():
    call, size = B.lib().tgrad_residual_norm_backward, B.lib().tgrad_residual_norm_backward_bytes
    n = C.c_size_t(0)

    def io(dh=(P, 64), gx=(P, 64), x=(P, 64), f=(P, 64), x8=0, f8=0, stats=P, dx=(P, 64), df=(P, 64), dg=(0, 0), dw=0, db=0, dpw=0, dpb=0):
        return B._pack_norm_backward(*dh, *gx, *x, *f, x8, f8, stats, *dx, *df, *dg, dw, db, dpw, dpb)

    for bad in BAD_NORMS:
        assert call(config(**bad), io(), P, 1 << 30, None) == B.ERR_INVALID_ARG, bad
        assert size(config(**bad), C.byref(n)) == B.ERR_INVALID_ARG, bad
    assert size(config(), None) == B.ERR_INVALID_ARG
    for bad in (dict(dh=(0, 64)), dict(x=(0, 0)), dict(x8=P), dict(f8=P), dict(f=(0, 0), df=(P, 64), f8=P + 8), dict(stats=0), dict(stats=P + 2), dict(dx=(0, 64)), dict(df=(0, 64)),
                dict(dg=(P, 64)), dict(db=P), dict(dpb=P), dict(dw=P + 1), dict(gx=(P, 63)), dict(f=(0, 0), dpw=P)):
        assert call(config(), io(**bad), P, 1 << 30, None) == B.ERR_INVALID_ARG, bad
    assert call(config(post=0), io(dpw=P), P, 1 << 30, None) == B.ERR_INVALID_ARG
    assert call(config(), io(), None, 1 << 30, None) == B.ERR_INVALID_ARG
    assert call(config(), io(), P + 16, 1 << 30, None) == B.ERR_INVALID_ARG
    assert size(config(), C.byref(n)) == B.OK and n.value > 0
    assert call(config(), io(), P, n.value - 1, None) == B.ERR_BUFFER_TOO_SMALL


def test_weight_grad_refusals():
    call, size = B.lib().tgrad_weight_grad, B.lib().tgrad_weight_grad_bytes
    n = C.c_size_t(0)

    def args(rows=4, out=64, width=64, dtype=B.R16B, to=B.R16B, dy=(P, 64), packed=P, dw=(P, 64), add=0):
        return B._pack_weight_grad(rows, out, width, dtype, to, *dy, packed, *dw, add, 0)

    bad_ones = (dict(rows=-1), dict(out=0), dict(width=0), dict(dtype=B.C64), dict(to=B.R16H), dict(dtype=B.R32), dict(dy=(0, 64)), dict(dy=(P, 63)), dict(dy=(P + 1, 64)),
                dict(packed=0), dict(packed=P + 8), dict(dw=(0, 64)), dict(dw=(P, 63)), dict(dw=(P + 2, 64), to=B.R32))
    for bad in bad_ones:
        assert call(args(**bad), P, 1 << 40, None) == B.ERR_INVALID_ARG, bad
        assert size(args(**bad), C.byref(n)) == B.ERR_INVALID_ARG, bad
    for bad in (dict(rows=1 << 31), dict(out=(1 << 24) + 1), dict(width=(1 << 24) + 1, dw=(P, 1 << 25)), dict(out=1 << 20, width=1 << 20, dy=(P, 1 << 20), dw=(P, 1 << 20))):
        assert call(args(**bad), P, 1 << 40, None) == B.ERR_UNSUPPORTED, bad
    assert call(None, None, 0, None) == B.ERR_INVALID_ARG and size(args(), None) == B.ERR_INVALID_ARG
    assert size(args(), C.byref(n)) == B.OK and n.value == 0
    for odd in (dict(dy=(P + 2, 64)), dict(dy=(P, 65)), dict(dtype=B.R32, to=B.R32), dict(rows=65536)):      # a copy of dy, or splits
        assert size(args(**odd), C.byref(n)) == B.OK and n.value > 0
        assert call(args(**odd), None, n.value, None) == B.ERR_INVALID_ARG
        assert call(args(**odd), P, n.value - 1, None) == B.ERR_BUFFER_TOO_SMALL


def test_binding_refusals():
    x = torch.zeros(4, 64)
    for call in (lambda: B.act_pack(x), lambda: B.gated_act(x, x), lambda: B.residual_norm(x), lambda: B.weight_grad(x, None)):
        with pytest.raises(ValueError):
            call()                                            # not on a GPU
