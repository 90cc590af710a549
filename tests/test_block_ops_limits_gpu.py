"""The operators of a trained block at the ends of their ranges (run with -m gpu): sums over many tokens, rows as the fast kernels
take them, sequences and batches without rows, waits that run out, arguments of other kinds.
u = 2^-24 is half an fp32 ulp, bounds are those of test_block_ops_gpu."""
import math

import pytest
import torch

from paper_2501_02379_b200 import binding as B
from tests.test_block_ops_gpu import DT, U, check_norm, gen, norm_case

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ weight gradient
@pytest.mark.parametrize("dt,digits", [("f16", 11), ("bf16", 8)])
def test_weight_grad_of_many_tokens_is_off_by_its_rounding(dt, digits):
    """Terms of one sign, whole tiles.  The tensor core cuts off at most 2^-22 of a sum per instruction, and 256 instructions
    of 16 tokens form a sum; these are added in fp32, u each; the stored result is off by half a step, 2^-digits of its power of two."""
    rows, clusters = 120000, torch.cuda.get_device_properties(0).multi_processor_count // 2
    n, width = 512, 256 * (clusters // 2)                     # two tiles by as many as make one full round
    dy = (0.125 + 0.125 * torch.rand(rows, n, generator=gen(1), device="cuda")).to(DT[dt])
    x8 = B.act_pack((0.5 + torch.rand(rows, width, generator=gen(2), device="cuda")).to(DT[dt]))
    got = B.weight_grad(dy, x8).double()
    want = dy.double().T @ B.act_unpack(x8).double()
    half = torch.exp2(torch.floor(torch.log2(want)) - digits)
    assert bool(((got - want).abs() <= half + want * (256 * 2.0 ** -22 + rows / 4096 * U)).all())


# ------------------------------------------------------------------------------------------------ norms of aligned rows
@pytest.mark.parametrize("dt,pdt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", ["none", "one", "equal", "ragged", "many"])
def test_residual_norm_of_aligned_rows(gate, layer, dt, pdt):
    """Every row at a multiple of 16 bytes, whole vectors, several rows a team: the kernels that copy rows ahead, in both directions."""
    shapes = [(603, 64), (3000, 40), (600, 512), (450, 1024), (303, 2008), (300, 4096), (300, 8192)]
    for i in range(len(gate) % 3, len(shapes), 3):
        x, f, dh, dx, how, starts = norm_case(*shapes[i], dt, pdt, layer, True, gate, 20 * i)
        check_norm(x, f.contiguous(), dh, dx, how, starts, dt, pdt, layer, True, kept=(False, i % 2 == 0))


@pytest.mark.parametrize("layer", [False, True])
def test_norm_before_a_block_of_aligned_rows(layer):
    for i, (rows, width, dt) in enumerate([(3000, 40, "bf16"), (450, 1024, "f32"), (300, 8192, "f16"), (300, 16384, "bf16")]):
        x, _, dh, dx, how, _ = norm_case(rows, width, dt, "f32", layer, False, "none", 30 * i)
        check_norm(x, None, dh, dx, how, None, dt, "f32", layer, False, scale=0.7, kept=(i % 2 == 0, False))


# ------------------------------------------------------------------------------------------------ norms: nothing there
def _dirty():
    """Memory that a workspace may be given holds NaN."""
    for n in (1 << 12, 1 << 16, 1 << 20, 1 << 24):
        torch.full((n,), math.nan, device="cuda")


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate", [(3, 64), (1, 64), (64,)])
def test_no_rows_give_gradients_of_zero(layer, gate):
    empty, one = torch.zeros(0, 64, device="cuda"), torch.ones(64, device="cuda")
    how = {"weight": one, "post_weight": one, "gate": torch.full(gate, 0.5, device="cuda"), "kind": "layer" if layer else "rms"}
    if layer:
        how["post_bias"] = one
    for starts in (None, [0] * (gate[0] + 1) if len(gate) == 2 else [0, 0]):
        if starts is not None:
            how["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        r = B.residual_norm(empty, empty, **how)
        assert r.x.shape == r.h.shape == (0, 64)
        for grad_x in (empty, None):
            _dirty()
            g = B.residual_norm_backward(empty, r.x, r.stats, empty, grad_x=grad_x, **how)
            assert g.x.shape == g.f.shape == (0, 64) and g.gate.shape == gate
            for name in ("weight", "bias", "post_weight", "post_bias", "gate"):
                t = getattr(g, name)
                assert t is None or bool((t == 0).all()), name


def test_no_rows_with_a_gate_for_each():
    empty, one = torch.zeros(0, 64, device="cuda"), torch.ones(64, device="cuda")
    for starts in (None, torch.zeros(1, dtype=torch.int32, device="cuda")):
        r = B.residual_norm(empty, empty, weight=one, post_weight=one, gate=empty, starts=starts, keep_f=True, keep_h=True)
        assert r.h.shape == (0, 64)
        _dirty()
        g = B.residual_norm_backward(empty, r.x, r.stats, r.f8, grad_x=empty, weight=one, post_weight=one, gate=empty, starts=starts)
        assert g.gate.shape == (0, 64) and bool((g.weight == 0).all()) and bool((g.post_weight == 0).all())
    with pytest.raises(ValueError):
        B.residual_norm(torch.zeros(2, 64, device="cuda"), torch.zeros(2, 64, device="cuda"), gate=empty)


@pytest.mark.parametrize("rows,width", [(90, 99), (2000, 512)])      # the general kernels; those for aligned rows
@pytest.mark.parametrize("layer", [False, True])
def test_gate_of_an_empty_sequence_has_no_part(rows, width, layer):
    x, f, dh, dx, how, _ = norm_case(rows, width, "bf16", "f32", layer, True, "ragged", 5)
    f = f.contiguous()
    kind = "layer" if layer else "rms"
    how.pop("bias", None)
    cases = [([3, 3, rows // 2, rows // 2, rows], (0, 2)), ([rows + 7, rows + 9, rows + 9, rows + 12, rows + 15], (0, 1, 2, 3)), ([0, 1, 2, rows, rows], (3,))]
    for starts, empty in cases:
        how["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        r = B.residual_norm(x, f, kind=kind, **how)
        out = []
        for fill in (0.0, math.nan, -math.inf):
            gate = how["gate"].clone()
            gate[list(empty)] = fill
            out.append(B.residual_norm_backward(dh, r.x, r.stats, f, grad_x=dx, kind=kind, **{**how, "gate": gate}))
        for got in out:
            assert all(t is None or (bool(torch.isfinite(t).all()) and torch.equal(t, u)) for t, u in zip(got, out[0]))
            assert bool((got.gate[list(empty)] == 0).all())
    # no post_weight that is not finite gets into the gradient of a gate without rows
    how["post_weight"][0] = math.inf
    assert bool((B.residual_norm_backward(dh, r.x, r.stats, f, grad_x=dx, kind=kind, **how).gate[3] == 0).all())
    how["post_weight"][0] = 1.0
    # one sequence, and it has no rows
    gate, starts = torch.full((1, width), math.nan, device="cuda"), torch.tensor([5, 5], dtype=torch.int32, device="cuda")
    got = B.residual_norm_backward(dh, r.x, r.stats, f, grad_x=dx, kind=kind, **{**how, "gate": gate, "starts": starts})
    assert bool((got.gate == 0).all()) and bool((got.post_weight == 0).all()) and (not layer or bool((got.post_bias == 0).all()))
    # no rows at all
    for gate in (gate, gate[0], gate.expand(3, width).contiguous()):
        got = B.residual_norm_backward(dh[:0], x[:0], r.stats[:, :0].contiguous(), f[:0], grad_x=dx[:0], kind=kind, **{**how, "gate": gate, "starts": None})
        assert bool((got.gate == 0).all()) and bool((got.post_weight == 0).all()) and (not layer or bool((got.post_bias == 0).all()))


# ------------------------------------------------------------------------------------------------ waits that run out
def _nan(t):
    return bool(torch.isnan(t).all())


@pytest.mark.parametrize("layer", [False, True])
def test_waits_that_run_out_leave_nothing_finite(layer):
    """No copy comes: all that was made from rows is NaN, kept copies, means and sums among them.  Some come: the same or right, entry by entry."""
    rows, width = 3000, 1024                                   # two rows a team and more
    x, f, dh, dx, how, _ = norm_case(rows, width, "bf16", "f32", layer, True, "one", 3)
    f = f.contiguous()                                         # rows that are copied ahead
    kind = "layer" if layer else "rms"
    alone = {k: how[k] for k in ("weight", "bias") if k in how}
    among = {**how, "gate": how["gate"].repeat(2, 1), "starts": torch.tensor([40, 300, rows - 60], dtype=torch.int32, device="cuda")}
    back = lambda h: {k: v for k, v in h.items() if k != "bias"}  # noqa: E731
    stats = B.residual_norm(x, f, kind=kind, **how).stats

    def calls():
        out = [B.residual_norm(x, f, kind=kind, keep_x=True, keep_f=True, keep_h=True, **h) for h in (how, among)]
        out.append(B.residual_norm(x, kind=kind, keep_x=True, keep_h=True, **alone))
        out += [B.residual_norm_backward(dh, x, stats, f, grad_x=dx, kind=kind, **back(h)) for h in (how, among)]
        flat = []
        for k, r in enumerate(out):
            for name, t in r._asdict().items():
                if t is not None:
                    flat.append((k, name, B.act_unpack(t) if isinstance(t, B.Packed) else t))
        return flat

    want = calls()
    for limit in (0, 1):
        B.set_copy_limit(limit)
        try:
            got = calls()
            torch.cuda.synchronize()
        finally:
            B.set_copy_limit(-1)
        outside = torch.cat([torch.arange(40), torch.arange(rows - 60, rows)]).cuda()
        for (k, name, t), (_, _, right) in zip(got, want):
            if limit == 0:
                if k == 2 and name == "stats":
                    t = t[[1, 3] if layer else [1]]           # (of a block that is not there: 1 and 0)
                if k == 4 and name == "f":
                    assert bool((t[outside] == 0).all())      # rows of no sequence: 0 whatever is there
                    t = t[40:rows - 60]
                assert _nan(t), (k, name)
            elif k < 3:
                bad = torch.isnan(t)
                assert bool((bad | (t == right)).all()) and (name == "stats" or bool(bad.any())), (k, name)
    assert all(torch.equal(t, right) for (_, _, t), (_, _, right) in zip(calls(), want))


def test_waits_that_run_out_within_long_sums():
    """A weight gradient whose sums leave the tensor core several times: tiles are NaN or right."""
    dy, x = (torch.randn(8192, n, generator=gen(n), device="cuda").bfloat16() for n in (2048, 2560))
    x8 = B.act_pack(x)
    want = B.weight_grad(dy, x8)
    for limit in (0, 70, 135):                                # of 139 steps of a block on 148 SMs: a tile of 128, which leaves twice, and a part of another
        B.set_copy_limit(limit)
        try:
            got = B.weight_grad(dy, x8)
            torch.cuda.synchronize()
        finally:
            B.set_copy_limit(-1)
        tiles = torch.isnan(got).view(8, 256, 10, 256).transpose(1, 2).flatten(2)
        assert bool((tiles.all(2) | ~tiles.any(2)).all()) and bool(tiles.any()) and (limit > 128 or bool(tiles.all()))
        assert bool((torch.isnan(got) | (got == want)).all())
    assert torch.equal(B.weight_grad(dy, x8), want)


# ------------------------------------------------------------------------------------------------ arguments
def test_packed_matrices_are_checked():
    x = torch.randn(4, 64, device="cuda")
    p = B.act_pack(x)
    host = p._replace(data=p.data.cpu())
    for call in (lambda: B.act_unpack(host), lambda: B.act_unpack(host, out=x),
                 lambda: B.act_unpack(x), lambda: B.act_unpack(p.data), lambda: B.weight_grad(x, None), lambda: B.weight_grad(x, x), lambda: B.weight_grad(x, host),
                 lambda: B.gated_act_backward(host, p, x)):
        with pytest.raises(ValueError):
            call()


def test_unknown_activations_are_refused():
    x = torch.randn(4, 64, device="cuda")
    p = B.act_pack(x)
    for call in (lambda: B.gated_act(x, x, act="relu"), lambda: B.gated_act(x, act=None), lambda: B.gated_act_backward(p, p, x, act="relu")):
        for kind in (ValueError, KeyError):
            with pytest.raises(kind):
                call()


def test_packing_in_place_counts_as_a_change():
    x = torch.randn(4, 64, device="cuda")
    p = B.act_pack(x)
    before = p.data._version
    assert B.act_pack(2 * x, out=p) is p and p.data._version > before
    assert torch.equal(B.act_unpack(p), 2 * B.act_unpack(B.act_pack(x)))


def test_parameters_that_stand_negated_are_refused():
    x, w = torch.randn(4, 64, device="cuda"), torch.rand(64, device="cuda")
    minus = torch._neg_view(w)
    r = B.residual_norm(x, x, weight=w, post_weight=w, gate=w)
    for name in ("weight", "post_weight", "gate"):
        how = {"weight": w, "post_weight": w, "gate": w, name: minus}
        for call in (lambda: B.residual_norm(x, x, **how), lambda: B.residual_norm_backward(x, r.x, r.stats, x, **how)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        B.residual_norm(x, x, weight=w, bias=minus, kind="layer")
    with pytest.raises(ValueError):
        B.residual_norm_backward(x, r.x, torch._neg_view(r.stats), x, weight=w)
