"""The operators of a trained block on a B200 against their 64-bit definitions (run with -m gpu).

Tolerances are bounds derived from the arithmetic, u = 2^-24 being half an fp32 ulp:
* packing and unpacking have no rounding but the codes': equal to the bit;
* a logistic gate 1 / (1 + exp(-z)): the exponential is off by (4 + 2.4 |z|) u (its argument is rounded; 2 ulp), the division by 4 u, z of the
  tanh form by 4 u |z|; the normal distribution at a: 8 u, and (a^2 + 1) u from the rounding of its argument;
* a mean over a row: at most 16 terms in a thread and 11 merges, 32 u of the mean magnitude, so 1 / deviation is off by 24 u; what is
  formed from these is bounded by the sum of the magnitudes of its terms;
* a column sum: 256 rows in a thread, then at most 128 partial sums and 32 merges: 420 u of the sum of magnitudes;
* the tensor core cuts sums off at 2^-22 of the largest term per instruction of 16 tokens;
* a result stored in 16 bits is rounded once more: half an ulp of the stored value.
"""
import math

import numpy as np
import pytest
import torch

from oracle import block_oracle as orc
from paper_2501_02379_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def f64(t):
    return t.detach().cpu().double().numpy()


def within(got, want, tol, what=""):
    got, want = f64(got), np.asarray(want)
    assert got.shape == want.shape, what
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places"
    off = np.abs(got - want)[~nan] > np.broadcast_to(tol, want.shape)[~nan]
    if off.any():
        worst = np.max(np.abs(got - want)[~nan] / np.maximum(np.broadcast_to(tol, want.shape)[~nan], 1e-300))
        raise AssertionError(f"{what}: {off.sum()} of {off.size} off, worst {worst:.3g} x the bound")


def matrix(rows, width, dt, seed, pad=0, offset=0, size=1.0):
    """A matrix whose rows stand `pad` entries apart, the first one `offset` entries into its memory; 7 stands around them."""
    buf = torch.full((rows * (width + pad) + offset + 8,), 7.0, dtype=DT[dt], device="cuda")
    m = buf[offset:].as_strided((rows, width), (width + pad, 1))
    x = torch.randn(rows, width, generator=gen(seed), device="cuda") * size * torch.exp(torch.randn(width, generator=gen(seed + 1), device="cuda"))
    m.copy_(x)
    return m


SHAPES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 64), (7, 100), (13, 257), (4, 1000), (3, 4096), (2, 5001), (300, 96), (1, 16384)]
PLACES = [(0, 0), (1, 0), (3, 1), (8, 2), (0, 3)]


# ------------------------------------------------------------------------------------------------ 8 bits
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pad,offset", PLACES)
def test_pack_and_unpack(dt, pad, offset):
    for rows, width in SHAPES:
        x = matrix(rows, width, dt, rows + width, pad, offset)
        p = B.act_pack(x)
        codes, byte = orc.packed(f64(x))
        blocks = byte.shape[1]
        data = p.data.cpu().numpy()
        assert np.array_equal(data[:rows * 32 * blocks].view(np.int8).reshape(rows, -1), codes)
        assert np.array_equal(data[rows * 32 * blocks:].reshape(rows, -1)[:, :blocks], byte)
        want = orc.unpacked(codes, byte, width)
        assert np.array_equal(f64(B.act_unpack(p)), want)
        out = matrix(rows, width, dt, 5, pad, offset)
        around = out._base.clone()
        B.act_unpack(p, out=out)
        assert np.array_equal(f64(out), want)
        out.copy_(around.as_strided(out.shape, out.stride(), out.storage_offset()))
        assert torch.equal(out._base, around)               # nothing written beside the rows
        again = B.act_pack(x, out=B.Packed(torch.zeros_like(p.data), rows, width, x.dtype))
        assert torch.equal(again.data[:rows * 32 * blocks], p.data[:rows * 32 * blocks])


def test_pack_of_many_rows_and_wide_ones():
    for rows, width in ((20011, 96), (3, 100003), (1500, 4097)):
        x = matrix(rows, width, "bf16", 1)
        v = torch.zeros(rows, -(-width // 32) * 32, device="cuda", dtype=torch.float64)
        v[:, :width] = x
        v = v.view(rows, -1, 32)
        e = torch.frexp(v.abs().amax(2, keepdim=True)).exponent.long() - 7
        step = ((e + 1023) << 52).view(torch.float64)          # 2^e by its bits: pow is not exact
        want = (torch.round(v / step).clamp(-127, 127) * step).view(rows, -1)[:, :width]
        assert torch.equal(B.act_unpack(B.act_pack(x)).double(), want)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_pack_at_the_ends_of_the_range(dt):
    top, tiny = torch.finfo(DT[dt]).max, torch.finfo(DT[dt]).smallest_normal * torch.finfo(DT[dt]).eps
    rows = [[0.0] * 32, [-0.0] * 32, [top] * 32, [-top, top, 1.0] + [0.0] * 29, [tiny] * 32, [tiny, -3 * tiny] + [0.0] * 30, [math.inf] + [1.0] * 31,
            [1.0] * 31 + [math.nan], [-math.inf] * 32, [math.nan] * 32, [127.5] + [0.5] * 31, [-127.5, 126.5, 1.5, 2.5] + [0.0] * 28]
    x = torch.tensor(rows, dtype=DT[dt], device="cuda")
    x = torch.cat([x, torch.ones_like(x)], 1)               # a block beside: what stands in the first does not touch it
    back = B.act_unpack(B.act_pack(x))
    want = orc.kept(f64(x))
    got = f64(back)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])
    assert bool((back[:, 32:] == 1).all()) and bool(torch.isfinite(back[:6]).all())
    assert torch.equal(B.act_unpack(B.act_pack(back[:6])), back[:6])


# ------------------------------------------------------------------------------------------------ gated activation
def gate_tol(act, a):
    """Bounds on the relative error of p in act(a) = a p, and on the absolute error of act'."""
    p, slope = orc.gate_of(act, a)
    if act == "gelu":
        rel = (10 + 2 * (a * a + 1)) * U
        q, dz = np.exp(-a * a / 2) / math.sqrt(2 * math.pi), np.ones_like(a)
        return rel, p * rel + np.abs(a) * q * (10 + 2 * a * a) * U + U * np.abs(slope)
    k = 2 * math.sqrt(2 / math.pi)
    z, dz = (a, np.ones_like(a)) if act == "silu" else (k * (a + 0.044715 * a ** 3), k * (1 + 3 * 0.044715 * a * a))
    rel = (14 + 8 * np.abs(z)) * U
    return rel, p * rel + np.abs(a) * p * dz * ((1 - p) * (rel + 8 * U) + p * rel + U) + 4 * U * np.abs(slope)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [True, False])
def test_gated_act(act, dt, gated):
    h = HALF_ULP[dt] * 1.01
    for (rows, width), (pad, offset) in zip(SHAPES, PLACES + PLACES + PLACES):
        a, u = matrix(rows, width, dt, 1, pad, offset, 1.5), matrix(rows, width, dt, 3, pad + 1, offset) if gated else None
        dy = matrix(rows, width, dt, 5, pad, offset, 0.3)
        r = B.gated_act(a, u, act)
        av, uv, g = f64(a), f64(u) if gated else None, f64(dy)
        y = orc.gated(act, av, uv)
        rel, _ = gate_tol(act, av)
        within(r.y, y, np.abs(y) * (rel + 4 * U + h) + TINY[dt], "y")
        assert torch.equal(r.a8.data, B.act_pack(a).data) if width % 128 == 0 else torch.equal(B.act_unpack(r.a8), B.act_unpack(B.act_pack(a)))
        assert (r.u8 is None) == (not gated) and (not gated or torch.equal(B.act_unpack(r.u8), B.act_unpack(B.act_pack(u))))
        assert torch.equal(B.gated_act(a, u, act, keep=False).y, r.y)
        # the gradient at what was kept
        ak, uk = orc.kept(av), orc.kept(uv) if gated else None
        da, du = orc.gated_gradient(act, ak, uk, g)
        rel, slope = gate_tol(act, ak)
        out = B.gated_act_backward(r.a8, r.u8, dy, act, keep_y=True)
        scale = np.abs(g) * (np.abs(uk) if gated else 1)
        within(out.da, da, scale * (slope * 1.01 + 4 * U * np.abs(orc.gate_of(act, ak)[1])) + h * np.abs(da) + TINY[dt], "da")
        if gated:
            within(out.du, du, np.abs(du) * (rel + 4 * U + h) + TINY[dt], "du")
        else:
            assert out.du is None
        back = orc.gated(act, ak, uk)
        top = np.abs(np.pad(back, ((0, 0), (0, -width % 32)))).reshape(rows, -1, 32).max(2).repeat(32, 1)[:, :width]
        within(B.act_unpack(out.y8), back, top * (2.0 ** -6 + 2 * h) + TINY[dt], "y8")
        # into the halves of one tensor
        both = torch.full((rows, 2 * width + 1), 7.0, dtype=DT[dt], device="cuda")
        B.gated_act_backward(r.a8, r.u8, dy, act, da=both[:, :width], du=both[:, width:2 * width] if gated else None)
        assert torch.equal(both[:, :width], out.da) and bool((both[:, -1] == 7).all()) and (not gated or torch.equal(both[:, width:-1], out.du))


def test_gated_act_far_out():
    """Where exponentials overflow or vanish, and what is not finite."""
    for act in ("silu", "gelu", "gelu_tanh"):
        a = torch.tensor([[0.0, -0.0, 1e-30, -88.0, -104.0, -1000.0, 1e13, -1e13, 1e38, -1e38, 30.0, -30.0]], device="cuda")
        u = torch.ones_like(a)
        y = B.gated_act(a, u, act).y
        want = orc.gated(act, f64(a))
        within(y, np.where(f64(a) > 20, f64(a), want), np.abs(want) * 800 * U + 2e-37, act)
        for col in range(a.shape[1]):                        # a block of its own each, so that all are kept
            r = B.gated_act(a[:, col:col + 1], u[:, col:col + 1], act)
            g = B.gated_act_backward(r.a8, r.u8, u[:, col:col + 1], act)
            assert bool(torch.isfinite(g.da).all()) and bool(torch.isfinite(g.du).all())
            if abs(float(a[0, col])) > 50:                   # 1, or at most 88 exp(-88) = 5.3e-37
                assert abs(float(g.da) - (1.0 if float(a[0, col]) > 0 else 0.0)) < 1e-36
        bad = torch.tensor([[math.nan, 1.0], [math.inf, 1.0]], device="cuda")
        r = B.gated_act(bad, torch.ones_like(bad), act)
        assert bool(torch.isnan(r.y[0, 0])) and bool(torch.isfinite(r.y[:, 1]).all())
        assert bool(torch.isnan(B.gated_act_backward(r.a8, r.u8, torch.ones_like(bad), act).da).all())      # the whole block was lost


# ------------------------------------------------------------------------------------------------ norms around a block
def norm_case(rows, width, dt, pdt, layer, post, gate, seed, pad=0, offset=0):
    g = gen(seed)

    def vector(fill):
        return (fill + 0.3 * torch.randn(width, generator=g, device="cuda")).to(DT[pdt])

    how = {"weight": vector(1.0)}
    if post:
        how["post_weight"] = vector(1.0)
    if layer:
        how["bias"] = vector(0.0)
        if post:
            how["post_bias"] = vector(0.0)
    groups = {"none": 0, "one": 1, "equal": 3 if rows % 3 == 0 else 1, "ragged": 4, "rows": rows, "many": 40}[gate]
    starts = None
    if groups:
        how["gate"] = (0.5 + 0.5 * torch.randn(groups, width, generator=g, device="cuda")).to(DT[pdt])
    if gate in ("ragged", "many"):
        cuts = sorted(int(c) for c in torch.randint(0, rows + 1, (groups - 1,), generator=g, device="cuda").tolist())
        starts = [min(cuts + [rows // 9])] + cuts + [max(cuts + [rows - 1])]
        how["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    x, f = matrix(rows, width, dt, seed + 1, pad, offset, 2.0), matrix(rows, width, dt, seed + 3, pad + 1, offset)
    dh, dx = matrix(rows, width, dt, seed + 5, pad, offset, 0.3), matrix(rows, width, dt, seed + 7, pad, offset, 0.3)
    return x, f, dh, dx, how, starts


def oracle_params(how, width):
    one, zero = np.ones(width), np.zeros(width)
    return [f64(how[k]) if k in how else d for k, d in (("weight", one), ("bias", zero), ("post_weight", one), ("post_bias", zero))] + [f64(how["gate"]) if "gate" in how else None]


def check_norm(x, f, dh, dx, how, starts, dt, pdt, layer, post, scale=0.8, eps=1e-5, kept=(False, False)):
    rows, width = x.shape
    h = HALF_ULP[dt] * 1.01
    kind = "layer" if layer else "rms"
    w, b, pw, pb, gate = oracle_params(how, width)
    xv, fv = f64(x), f64(f) if f is not None else None
    r = B.residual_norm(x, f, scale=scale, kind=kind, post=post, eps=eps, keep_x=kept[0], keep_f=kept[1] and f is not None, keep_h=True, **how)
    new, hh, stats = orc.residual_norm(xv, fv, w, b, pw, pb, gate, starts, scale, layer, post, eps)
    mean = lambda v: np.abs(v).mean(1, keepdims=True)  # noqa: E731
    g = np.ones((1, width)) if gate is None else orc.row_gate(gate, rows, starts)[0]
    mag = np.abs(scale * xv)
    if f is not None:
        if post:
            r0 = stats[0][:, None]
            m0 = stats[2][:, None] if layer else 0
            mag = mag + np.abs(g) * (np.abs((fv - m0) * r0 * pw) + np.abs(pb) + r0 * np.abs(pw) * (mean(fv) if layer else 0))
        else:
            mag = mag + np.abs(g * fv)
    t32 = 64 * U * mag
    within(r.x, new, t32 + h * np.abs(new) + TINY[dt], "x'")
    r1, m1 = stats[1][:, None], stats[3][:, None] if layer else 0
    cut = (new - m1) * r1
    th = np.abs(w) * (r1 * (t32 + (t32.mean(1, keepdims=True) + 32 * U * mean(new) if layer else 0)) + np.abs(cut) * (64 * U + r1 * r1 * np.abs((new - m1) * t32).mean(1, keepdims=True)))
    th = th + 4 * U * (np.abs(cut * w) + np.abs(b))
    within(r.h, hh, th + h * np.abs(hh) + TINY[dt], "h")
    rel = 64 * U + (r1 * r1)[:, 0] * np.abs((new - m1) * t32).mean(1) * 2
    tol = np.stack([stats[0] * 64 * U, stats[1] * rel] + ([32 * U * (mean(fv)[:, 0] if f is not None else 0) + np.zeros(rows), 32 * U * mean(new)[:, 0] + t32.mean(1)] if layer else []))
    within(r.stats, stats, tol, "stats")
    for name, full in (("x8", r.x if kept[0] else None), ("f8", f if kept[1] else None), ("h8", r.h)):
        p = getattr(r, name)
        assert (p is None) == (full is None)
        if p is not None:
            assert torch.equal(B.act_unpack(p), B.act_unpack(B.act_pack(full))), name
    # backward, from what the forward call returned
    xb, fb = (r.x8 if kept[0] else r.x), (r.f8 if kept[1] and f is not None else f)
    back = {k: v for k, v in how.items() if k != "bias"}
    out = B.residual_norm_backward(dh, xb, r.stats, fb, grad_x=dx, scale=scale, kind=kind, post=post, **back)
    again = B.residual_norm_backward(dh, xb, r.stats, fb, grad_x=dx, scale=scale, kind=kind, post=post, **back)
    for k, v in out._asdict().items():
        assert v is None or torch.equal(v, getattr(again, k)), k                # the same bits again
    xk = orc.kept(f64(r.x)) if kept[0] else f64(r.x)
    fk = None if f is None else orc.kept(fv) if kept[1] else fv
    st = f64(r.stats)
    dhv, dxv = f64(dh), None if dx is None else f64(dx)
    want = orc.residual_norm_gradient(dhv, dxv, xk, fk, st, w, pw, pb, gate, starts, scale, layer, post)
    r1, m1 = st[1][:, None], st[3][:, None] if layer else 0
    xh, e = (xk - m1) * r1, dhv * w
    tmag = (0 if dxv is None else np.abs(dxv)) + r1 * (np.abs(e) + np.abs(xh) * np.abs(e * xh).mean(1, keepdims=True) + (mean(e) if layer else 0))
    t = np.abs(want["x"] / scale)
    within(out.x, want["x"], abs(scale) * 64 * U * tmag + h * np.abs(want["x"]) + TINY[dt], "dx")
    ph = HALF_ULP[pdt] * 1.01
    col = 420 * U

    def sums(name, got, mag):
        within(got, want[name], mag + ph * np.abs(want[name]) + TINY[pdt], name)

    sums("weight", out.weight, col * np.abs(dhv * xh).sum(0))
    if layer:
        sums("bias", out.bias, col * np.abs(dhv).sum(0))
    if f is None:
        assert out.f is None
        return r, out
    live = np.ones((rows, 1), bool) if gate is None else (orc.row_gate(gate, rows, starts)[1] >= 0)[:, None]
    fk = np.where(live, fk, 0)
    r0, m0 = (st[0][:, None], st[2][:, None] if layer else 0) if post else (1.0, 0.0)
    fh, d, dtol = (fk - m0) * r0, np.abs(g) * t, np.abs(g) * 64 * U * tmag
    if post:
        dp, dt_p = d * np.abs(pw), (dtol + 4 * U * d) * np.abs(pw)
        ftol = r0 * (dt_p + np.abs(fh) * np.abs(fh * dt_p).mean(1, keepdims=True) + (dt_p.mean(1, keepdims=True) if layer else 0)
                     + 64 * U * (dp + np.abs(fh) * np.abs(fh * dp).mean(1, keepdims=True) + (dp.mean(1, keepdims=True) if layer else 0)))
    else:
        ftol = dtol + 4 * U * d
    within(out.f, want["f"], np.where(live, ftol + h * np.abs(want["f"]), 0) + TINY[dt], "df")
    if post:
        sums("post_weight", out.post_weight, np.where(live, col * np.abs(fh) * d + np.abs(fh) * dtol, 0).sum(0))
        if layer:
            sums("post_bias", out.post_bias, (col * d + dtol).sum(0))
    if gate is not None:
        n = np.abs(fh * pw) + np.abs(pb) if post else np.abs(fh)
        part = np.where(live, (col * t + 64 * U * tmag) * n, 0)
        _, group = orc.row_gate(gate, rows, starts)
        sums("gate", out.gate, np.stack([part[group == k].sum(0) for k in range(len(gate))]))
    return r, out


@pytest.mark.parametrize("dt,pdt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("layer,post", [(False, True), (True, True), (False, False), (True, False)])
@pytest.mark.parametrize("gate", ["none", "one", "equal", "ragged", "many", "rows"])
def test_residual_norm(gate, layer, post, dt, pdt):
    for i, (rows, width) in enumerate([(1, 1), (3, 32), (2, 33), (9, 100), (13, 257), (6, 1000), (3, 4096), (150, 64), (333, 130), (12, 2050)]):
        pad, offset = PLACES[i % len(PLACES)]
        case = norm_case(rows, width, dt, pdt, layer, post, gate, 10 * i, pad, offset)
        check_norm(*case, dt, pdt, layer, post, kept=(i % 2 == 1, i % 3 == 1))


@pytest.mark.parametrize("rows,width,dt,layer,gate", [(5, 16384, "bf16", False, "one"), (3, 16384, "f32", True, "ragged"), (160, 16384, "bf16", True, "one"), (3, 8192, "f32", False, "rows"),
                                                      (600, 8192, "bf16", False, "one"), (170, 9001, "f16", False, "ragged"), (1200, 2048, "f32", True, "equal"),
                                                      (4001, 96, "bf16", True, "many"), (40000, 40, "f32", False, "one"), (2000, 512, "bf16", False, "none"), (160, 16384, "f32", False, "one"),
                                                      (5000, 64, "f32", True, "rows")])
def test_residual_norm_of_long_rows_and_many(rows, width, dt, layer, gate):
    case = norm_case(rows, width, dt, "f32", layer, True, gate, 3)
    check_norm(*case, dt, "f32", layer, True, kept=(False, dt != "f32"))


@pytest.mark.parametrize("layer", [False, True])
def test_norm_before_a_block_alone(layer):
    for rows, width in ((1, 64), (7, 1001), (400, 256)):
        x, _, dh, dx, how, _ = norm_case(rows, width, "bf16", "f32", layer, False, "none", 4)
        check_norm(x, None, dh, dx, how, None, "bf16", "f32", layer, False, scale=1.0)
        check_norm(x, None, dh, None, how, None, "bf16", "f32", layer, False, scale=-0.5, kept=(True, False))
    r = B.residual_norm(x)                                    # no parameters at all
    want = orc.norm(f64(x), np.ones(width), np.zeros(width), False, 1e-6)[0]
    within(r.h, want, (HALF_ULP["bf16"] + 80 * U) * np.abs(want), "h")
    g = B.residual_norm_backward(dh, r.x, r.stats)
    assert g.weight is None and g.gate is None and g.f is None


def test_rows_of_no_sequence_do_not_see_the_block():
    rows, width = 50, 300
    x, f, dh, dx, how, _ = norm_case(rows, width, "bf16", "f32", True, True, "ragged", 5)
    starts = [3, 3, 20, 21, 41]
    how["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    f[:3] = math.nan
    f[41:] = math.inf
    r = B.residual_norm(x, f, scale=0.5, kind="layer", **how)
    assert torch.equal(r.x[:3], (x[:3].float() * 0.5).bfloat16()) and torch.equal(r.x[41:], (x[41:].float() * 0.5).bfloat16())
    assert bool(torch.isfinite(r.h).all())
    back = {k: v for k, v in how.items() if k != "bias"}
    out = B.residual_norm_backward(dh, r.x, r.stats, f, grad_x=dx, scale=0.5, kind="layer", **back)
    assert all(bool(torch.isfinite(t).all()) for t in out) and bool((out.f[:3] == 0).all()) and bool((out.f[41:] == 0).all())
    assert bool((out.gate[0] == 0).all())                      # an empty sequence
    clean = f.clone()
    clean[:3] = 0
    clean[41:] = 0
    same = B.residual_norm_backward(dh, r.x, r.stats.nan_to_num(0), clean, grad_x=dx, scale=0.5, kind="layer", **back)
    assert all(torch.equal(a, b) for a, b in zip(out, same))


@pytest.mark.parametrize("keep_f", [False, True])
def test_rows_of_no_sequence_among_many(keep_f):
    """The same on the kernels for many aligned rows; a gate that is not finite stays with its own sequence."""
    rows, width = 2000, 512
    x, f, dh, dx, how, _ = norm_case(rows, width, "bf16", "f32", False, True, "ragged", 6)
    how["starts"] = torch.tensor([100, 500, 500, 900, 1900], dtype=torch.int32, device="cuda")
    how["gate"][0] = math.nan
    f[:100], f[1900:] = math.nan, math.inf
    r = B.residual_norm(x, f, scale=0.5, keep_f=keep_f, **how)
    none = torch.cat([torch.arange(100), torch.arange(1900, 2000)]).cuda()
    assert torch.equal(r.x[none], (x[none].float() * 0.5).bfloat16()) and bool(torch.isfinite(r.h[none]).all()) and bool(torch.isnan(r.x[100:500]).all())
    out = B.residual_norm_backward(dh, r.x.nan_to_num(1.0), r.stats.nan_to_num(1.0), r.f8 if keep_f else f, grad_x=dx, scale=0.5, **how)
    assert bool((out.f[none] == 0).all()) and bool(torch.isfinite(out.x).all()) and bool(torch.isnan(out.f[100:500]).all())
    assert bool(torch.isfinite(out.gate[1:]).all()) and bool(torch.isfinite(out.f[500:]).all())


def test_norm_calls_of_other_kinds():
    """One sequence with rows outside of it, more sequences than blocks on them, no gradient of x', everything kept, on either kernels."""
    for rows, width in ((70, 99), (900, 1024)):
        x, f, dh, dx, how, _ = norm_case(rows, width, "bf16", "f32", True, True, "one", 7)
        how["starts"] = torch.tensor([5, rows - 7], dtype=torch.int32, device="cuda")
        check_norm(x, f, dh, dx, how, [5, rows - 7], "bf16", "f32", True, True)
        x, f, dh, dx, how, _ = norm_case(rows, width, "f16", "f16", False, True, "one", 8)
        check_norm(x, f, dh, None, how, None, "f16", "f16", False, True, kept=(False, True))
        check_norm(x, f, dh, dx, how, None, "f16", "f16", False, True, kept=(True, True))
    rows, width, groups = 3000, 40, 1500
    x, f, dh, dx, how, _ = norm_case(rows, width, "f32", "f32", True, True, "none", 9)
    how["gate"] = torch.randn(groups, width, generator=gen(3), device="cuda")
    check_norm(x, f, dh, dx, how, None, "f32", "f32", True, True)
    starts = sorted([0, rows] + [int(k) for k in torch.randint(0, rows, (groups - 1,), generator=gen(4), device="cuda").tolist()])
    how["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    check_norm(x, f, dh, dx, how, starts, "f32", "f32", True, True)


def test_norm_of_rows_of_zeros_and_of_equal_entries():
    x = torch.zeros(4, 200, device="cuda")
    x[1] = 3.0
    for kind in ("rms", "layer"):
        r = B.residual_norm(x, x, kind=kind, eps=1e-5)
        assert bool((r.h[0] == 0).all()) and bool(torch.isfinite(r.h).all())
        g = B.residual_norm_backward(torch.ones_like(x), r.x, r.stats, x, kind=kind)
        assert bool(torch.isfinite(g.x).all()) and bool(torch.isfinite(g.f).all())
    r = B.residual_norm(x[:0], x[:0], weight=torch.ones(200, device="cuda"))
    assert r.h.shape == (0, 200)
    g = B.residual_norm_backward(x[:0], r.x, r.stats, x[:0], weight=torch.ones(200, device="cuda"))
    assert bool((g.weight == 0).all())


# ------------------------------------------------------------------------------------------------ weight gradient
def check_weight_grad(rows, n, width, dt, to, pad=0, offset=0, seed=0, add=False, dyscale=0.3):
    x, dy = matrix(rows, width, dt, seed + 1), matrix(rows, n, dt, seed + 3, pad, offset, dyscale)
    p = B.act_pack(x)
    xk = B.act_unpack(p).double()
    want, mag = (dy.double().T @ xk).cpu().numpy(), (dy.double().abs().T @ xk.abs()).cpu().numpy()
    out = None
    if add:
        out = torch.randn(n, width, generator=gen(9), device="cuda").to(DT[to])
        want, mag = want + f64(out), mag + np.abs(f64(out))
    got = B.weight_grad(dy, p, dtype=DT[to], out=out, accumulate=add)
    steps = -(-rows // 16) * (3 if dt == "f32" else 1)
    tol = mag * ((min(steps, 16) if to == "f32" else steps) * 2 * 2.0 ** -22 + (steps / 16 + 150) * U) + HALF_ULP[to] * 1.01 * np.abs(want) + TINY[to]
    within(got, want, tol, f"{rows} {n} {width}")
    if not add:
        assert torch.equal(got, B.weight_grad(dy, p, dtype=DT[to]))
    return got


@pytest.mark.parametrize("dt,to", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
def test_weight_grad(dt, to):
    for i, (rows, n, width) in enumerate([(1, 1, 1), (1, 128, 128), (64, 128, 128), (63, 64, 32), (65, 129, 127), (17, 8, 500), (130, 300, 40), (1000, 200, 257), (512, 16, 1024),
                                          (256, 1000, 130), (4096, 96, 100), (20000, 33, 65)]):
        pad, offset = PLACES[i % len(PLACES)]
        check_weight_grad(rows, n, width, dt, to, pad, offset, i)
        check_weight_grad(rows, n, width, dt, to, 0, 0, i, add=True)


def test_weight_grad_of_many_tiles():
    check_weight_grad(700, 2100, 1500, "bf16", "bf16")
    check_weight_grad(333, 1800, 2222, "f16", "f32", pad=1)


def test_weight_grad_of_full_rounds_and_a_rest():
    """More tiles than clusters, and tokens enough to split the tiles of the last round."""
    for n, width, dt, to in ((4096, 5120, "bf16", "bf16"), (2048, 2600, "f16", "f32")):
        rows = 1200
        x, dy = matrix(rows, width, dt, 1), matrix(rows, n, dt, 3, size=0.3)
        p = B.act_pack(x)
        xk = B.act_unpack(p).double()
        want, mag = dy.double().T @ xk, dy.double().abs().T @ xk.abs()
        steps = -(-rows // 16)
        tol = mag * ((min(steps, 16) if to == "f32" else steps) * 2 * 2.0 ** -22 + (steps / 16 + 150) * U) + HALF_ULP[to] * 1.01 * want.abs() + TINY[to]
        assert bool(((B.weight_grad(dy, p, dtype=DT[to]).double() - want).abs() <= tol).all())


def test_weight_grad_of_wide_ranges():
    """Parts of fp32 entries far apart in size, and what is not finite where it stands."""
    rows, n, width = 40, 70, 90
    x, dy = matrix(rows, width, "f32", 1), matrix(rows, n, "f32", 3)
    dy *= 10.0 ** torch.randint(-18, 18, (1, n), generator=gen(5), device="cuda").float()
    p = B.act_pack(x)
    xk = B.act_unpack(p).double()
    want, mag = (dy.double().T @ xk).cpu().numpy(), (dy.double().abs().T @ xk.abs()).cpu().numpy()
    within(B.weight_grad(dy, p), want, mag * (16 * 2.0 ** -22 + 160 * U) + 2.0 ** -120, "wide")
    dy[3, 5] = math.inf
    dy[4, 6] = math.nan
    got = B.weight_grad(dy, p)
    assert bool(torch.isnan(got[6]).all()) and not bool(torch.isfinite(got[5]).any())
    rest = [i for i in range(n) if i not in (5, 6)]
    within(got[rest], want[rest], (mag * (16 * 2.0 ** -22 + 160 * U) + 2.0 ** -120)[rest], "beside")
    x = matrix(rows, width, "bf16", 1)
    x[7, 40] = math.inf                                        # a block of 32 columns of one token
    got = B.weight_grad(dy.clamp(-1, 1).nan_to_num(0).bfloat16(), B.act_pack(x))
    assert bool(torch.isnan(got[:, 32:64]).all()) and bool(torch.isfinite(got[:, :32]).all()) and bool(torch.isfinite(got[:, 64:]).all())


def test_weight_grad_writes_its_own_place_only():
    x, dy = matrix(100, 70, "bf16", 1), matrix(100, 50, "bf16", 3)
    big = torch.full((52, 75), 7.0, device="cuda", dtype=torch.bfloat16)
    B.weight_grad(dy, B.act_pack(x), out=big[1:51, 2:72])
    assert torch.equal(big[1:51, 2:72], B.weight_grad(dy, B.act_pack(x)))
    big[1:51, 2:72] = 7
    assert bool((big == 7).all())
    z = B.weight_grad(dy[:0], B.act_pack(x[:0]), dtype=torch.float32)
    assert z.shape == (50, 70) and bool((z == 0).all())


# ------------------------------------------------------------------------------------------------ streams, graphs, refusals
def _chain(x, f, dh, w, gate):
    """A run of the operators as a block's two passes make it."""
    r = B.residual_norm(x, f, weight=w, post_weight=w, gate=gate, keep_f=True, keep_h=True)
    half = x.shape[1] // 2
    y, a8, u8 = B.gated_act(r.h[:, :half], r.h[:, half:])
    both = torch.empty_like(x)
    g = B.gated_act_backward(a8, u8, dh[:, :half], da=both[:, :half], du=both[:, half:], keep_y=True)
    d = B.residual_norm_backward(both, r.x, r.stats, r.f8, grad_x=dh, weight=w, post_weight=w, gate=gate)
    return [r.x, r.h, y, both, d.x, d.f, d.weight, d.post_weight, d.gate, B.weight_grad(dh, r.h8), B.weight_grad(dh, g.y8, dtype=torch.float32)]


def test_on_another_stream_and_captured():
    x, f, dh = (torch.randn(700, 512, generator=gen(i), device="cuda").bfloat16() for i in range(3))
    w, gate = torch.randn(512, generator=gen(4), device="cuda"), torch.randn(512, generator=gen(5), device="cuda")
    want = _chain(x, f, dh, w, gate)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    p = B.act_pack(x, stream=side)
    got = B.act_unpack(p, stream=side)
    dw = B.weight_grad(dh, p, stream=side)
    with torch.cuda.stream(side):
        there = _chain(x, f, dh, w, gate)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, B.act_unpack(B.act_pack(x))) and torch.equal(dw, B.weight_grad(dh, B.act_pack(x)))
    assert all(torch.equal(a, b) for a, b in zip(want, there))
    # captured, with other inputs at each replay
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _chain(x, f, dh, w, gate)
    for seed in (11, 12):
        for i, t in enumerate((x, f, dh)):
            t.copy_(torch.randn(700, 512, generator=gen(seed + i), device="cuda"))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, _chain(x, f, dh, w, gate)))


def test_rows_far_apart():
    """Rows whose distance passes 32 bits, in entries and in bytes."""
    far, rows, width = (1 << 31) + 8, 3, 200
    buf = torch.zeros(2 * far + 300, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, width), (far, 1))
    near = torch.randn(rows, width, generator=gen(1), device="cuda").bfloat16()
    x.copy_(near)
    p = B.act_pack(x)
    assert torch.equal(p.data, B.act_pack(near).data)
    r, q = B.gated_act(x, x), B.gated_act(near, near)
    assert torch.equal(r.y, q.y) and torch.equal(r.u8.data, q.u8.data)
    n, m = B.residual_norm(x, x, scale=0.5), B.residual_norm(near, near, scale=0.5)
    assert torch.equal(n.x, m.x) and torch.equal(n.h, m.h)
    assert all(torch.equal(a, b) for a, b in zip(B.residual_norm_backward(x, x, n.stats, x, grad_x=x)[:2], B.residual_norm_backward(near, near, n.stats, near, grad_x=near)[:2]))
    assert torch.equal(B.weight_grad(x, p), B.weight_grad(near, p))
    B.gated_act_backward(r.a8, r.u8, near, da=x)
    assert torch.equal(x, B.gated_act_backward(r.a8, r.u8, near).da)
    B.act_unpack(p, out=x)
    assert torch.equal(x, B.act_unpack(p)) and float(buf.abs().max()) == float(x.abs().max())
    del buf, x
    torch.cuda.empty_cache()


def test_waits_that_run_out_are_reported():
    """The copies stop early: what was not finished is NaN, the calls return, and the next ones are right."""
    x, f, dh, dx = (torch.randn(600, 8192, generator=gen(i), device="cuda").bfloat16() for i in range(4))
    w = torch.ones(8192, device="cuda")
    p = B.act_pack(x)
    forward = lambda: B.residual_norm(x, f, weight=w, post_weight=w)  # noqa: E731
    stats = forward().stats
    backward = lambda: B.residual_norm_backward(dh, x, stats, f, grad_x=dx, weight=w, post_weight=w)  # noqa: E731
    grads = [lambda: B.weight_grad(dh, p), lambda: B.weight_grad(dh, p, dtype=torch.float32)]
    want = [forward(), backward(), [c() for c in grads]]
    for limit in (0, 1, 2):
        B.set_copy_limit(limit)
        try:
            r, g, dw = forward(), backward(), [c() for c in grads]
            torch.cuda.synchronize()
        finally:
            B.set_copy_limit(-1)
        for got, right in ((r.x, want[0].x), (r.h, want[0].h), (g.x, want[1].x), (g.f, want[1].f)):
            bad = torch.isnan(got).all(1)
            assert bool((bad | (got == right).all(1)).all()) and bool(bad.any() if limit < 2 else True)      # whole rows, or right ones
        if limit == 0:
            assert bool(torch.isnan(r.h).all()) and bool(torch.isnan(g.x).all()) and all(bool(torch.isnan(t).all()) for t in dw)
        if bool(torch.isnan(g.x).any()):
            assert bool(torch.isnan(g.weight).all()) and bool(torch.isnan(g.post_weight).all())
        assert all(bool(torch.isnan(t).all()) or torch.equal(t, u) for t, u in zip(dw, want[2]))
    again = [forward(), backward(), [c() for c in grads]]
    assert all(a is b or torch.equal(a, b) for a, b in zip(again[0], want[0])) and all(a is b or torch.equal(a, b) for a, b in zip(again[1], want[1]))
    assert all(torch.equal(a, b) for a, b in zip(again[2], want[2]))


def test_two_streams_at_once():
    ins = [[torch.randn(3000, 512, generator=gen(10 * k + i), device="cuda").bfloat16() for i in range(3)] for k in range(2)]
    w, gate = torch.randn(512, generator=gen(4), device="cuda"), torch.randn(512, generator=gen(5), device="cuda")
    want = [_chain(*t, w, gate) for t in ins]
    streams = [torch.cuda.Stream() for _ in ins]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(3):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k] = _chain(*ins[k], w, gate)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k in range(2) for a, b in zip(want[k], got[k]))


def test_results_in_place_count_as_changes():
    x = torch.randn(4, 64, device="cuda")
    p = B.act_pack(x)
    t = torch.zeros(4, 64, device="cuda")
    for call in (lambda: B.act_unpack(p, out=t), lambda: B.gated_act_backward(p, p, x, da=t), lambda: B.gated_act_backward(p, p, x, du=t)):
        before = t._version
        call()
        assert t._version > before
    t = torch.zeros(64, 64, device="cuda")
    before = t._version
    B.weight_grad(x, p, out=t)
    assert t._version > before


def test_binding_refuses():
    x = torch.zeros(4, 64, device="cuda")
    p = B.act_pack(x)
    w = torch.ones(64, device="cuda")
    r = B.residual_norm(x, x, weight=w)
    bad = [lambda: B.act_pack(x[0]), lambda: B.act_pack(torch.complex(x, x).conj().imag), lambda: B.act_pack(x.T), lambda: B.act_pack(x.double()), lambda: B.act_pack(x[:, :0]), lambda: B.act_pack(x, out=B.act_pack(x[:2])),
           lambda: B.act_unpack(p._replace(rows=5)), lambda: B.act_unpack(p._replace(dtype=torch.float64)), lambda: B.act_unpack(p._replace(data=p.data[1:])), lambda: B.act_unpack(p, out=torch.zeros(4, 63, device="cuda")),
           lambda: B.act_unpack(p, out=x.half()), lambda: B.gated_act(x, x[:2]), lambda: B.gated_act(x, x.half()), lambda: B.gated_act_backward(p, None, x, du=x.clone()),
           lambda: B.gated_act_backward(p, p, x.half()), lambda: B.gated_act_backward(p, x, x), lambda: B.residual_norm(x, x, weight=w[:5]), lambda: B.residual_norm(x, x, weight=w.half()),
           lambda: B.residual_norm(x, x, weight=w, gate=w.bfloat16()), lambda: B.residual_norm(x, x, bias=w), lambda: B.residual_norm(x, gate=w), lambda: B.residual_norm(x, keep_f=True),
           lambda: B.residual_norm(x, x, gate=torch.ones(3, 64, device="cuda")), lambda: B.residual_norm(x, x, kind="batch"), lambda: B.residual_norm(x, x, gate=w, starts=torch.zeros(3, dtype=torch.int32, device="cuda")),
           lambda: B.residual_norm(x, x, starts=torch.zeros(2, dtype=torch.int32, device="cuda")), lambda: B.residual_norm(x, x, gate=w, starts=torch.zeros(2, device="cuda")),
           lambda: B.residual_norm_backward(x, x, r.stats, x, kind="layer"), lambda: B.residual_norm_backward(x, x[:2], r.stats, x), lambda: B.residual_norm_backward(x, x, r.stats, None, gate=w),
           lambda: B.weight_grad(x.half(), p), lambda: B.weight_grad(x[:3], p), lambda: B.weight_grad(x, p, accumulate=True), lambda: B.weight_grad(x, p, out=torch.zeros(4, 64, device="cuda")),
           lambda: B.weight_grad(x, p, dtype=torch.float16), lambda: B.weight_grad(x, p, dtype=torch.float64)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)
    with pytest.raises(KeyError):
        B.gated_act(x, x, act="relu")
    with pytest.raises(B.TgradError):
        B.residual_norm(x, x, weight=w, kind="rms", bias=w)
    with pytest.raises(B.TgradError):
        B.residual_norm(x, x, eps=-1.0)
    with pytest.raises(B.TgradError):
        B.act_pack(x[:1].expand(4, 64))                        # rows on top of one another
    with pytest.raises(B.TgradError):
        B.residual_norm(torch.zeros(1, 16385, device="cuda"))
