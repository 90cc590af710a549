"""The operators of a trained block at the ends of their ranges (run with -m gpu): sums over many tokens, batches without rows.
u = 2^-24 is half an fp32 ulp, bounds are those of test_block_ops_gpu."""
import math

import pytest
import torch

from paper_2501_02379_b200 import binding as B
from tests.test_block_ops_gpu import DT, U, gen

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
