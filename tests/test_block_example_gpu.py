"""The example's feed-forward blocks: a run of the operators as a model makes it (run with -m gpu)."""
import math

import numpy as np
import pytest
import torch

from examples import spectral_lm as ex
from oracle import block_oracle as orc

pytestmark = pytest.mark.gpu


def test_example_runs_with_blocks():
    pref, pol, flags = ex.main(steps=6, blocks=2)
    assert flags == 0 and bool(torch.isfinite(pref).all()) and bool(torch.isfinite(pol).all())
    assert abs(pref[0, 0] - math.log(2)) < 1e-5            # the model is its own reference at first


def _f64(t):
    return t.detach().cpu().double().numpy()


def test_block_gradients_are_the_formulas_at_what_is_kept():
    """fp32 products of 64 to 200 terms and what the operators add: 1e-5 of the largest entry is 160 roundings of 2^-24."""
    torch.manual_seed(1)
    rows, w = 200, ex.WIDTH
    model = ex.SpectralLM(blocks=1).cuda()
    b = model.blocks[0]
    for p in (b["post_weight"], b["weight"], b["gate"]):
        p.data += 0.3 * torch.randn_like(p)
    x = torch.randn(rows, w, device="cuda")
    first = ex.B.residual_norm(x, weight=model.norm, keep_h=True)
    leaves = [t.detach().clone().requires_grad_() for t in (x, first.h, b["w_in"], b["w_out"], b["post_weight"], b["gate"], b["weight"])]
    new, h, _ = ex.FeedForward.apply(leaves[0], leaves[1], first.h8.data, *leaves[2:])
    gx, gh = torch.randn_like(new), torch.randn_like(h)
    torch.autograd.backward([new, h], [gx, gh])
    wi, wo, pw, gate, wt = (_f64(t) for t in leaves[2:])
    au = first.h @ leaves[2].detach().T                     # what the block has kept
    a, u = (orc.kept(_f64(t)) for t in au.split(ex.HIDDEN, 1))
    y = ex.B.gated_act(*au.split(ex.HIDDEN, 1), keep=False).y
    f = _f64(y @ leaves[3].detach().T)
    zero = np.zeros(w)
    _, _, stats = orc.residual_norm(_f64(x), f, wt, zero, pw, zero, gate[None], None, 1.0, False, True, 1e-6)
    n = orc.residual_norm_gradient(_f64(gh), _f64(gx), _f64(new), orc.kept(f), stats, wt, pw, zero, gate[None], None, 1.0, False, True)
    dy = n["f"] @ wo
    d = np.concatenate(orc.gated_gradient("silu", a, u, dy), 1)
    want = [n["x"], d @ wi, orc.weight_grad(d, orc.kept(_f64(first.h))), orc.weight_grad(n["f"], orc.kept(orc.gated("silu", a, u))), n["post_weight"], n["gate"][0], n["weight"]]
    for i, (t, g) in enumerate(zip(leaves, want)):
        # (entry 3: the codes of y, computed here in 64 bits, may differ by a step where y lies between two: 2^-7 of a term in 200)
        tol = (1e-5 if i != 3 else 1e-4) * np.abs(g).max()
        assert np.abs(_f64(t.grad) - g).max() < tol, i


def test_model_gradients_are_near_those_without_packing():
    """Against autograd of the plain model in 64 bits: a kept entry is off by at most 2^-7 of its block's largest, about 2^-8 of the
    usual size of an entry; a gradient's terms have three such factors at most, whose errors average over rows."""
    torch.manual_seed(2)
    model = ex.SpectralLM(blocks=2).cuda()
    tokens = torch.randint(0, ex.VOCAB, (6, ex.LENGTH), device="cuda")
    logits = model(tokens)
    way = torch.randn_like(logits)
    logits.backward(way)
    got = {k: p.grad for k, p in model.named_parameters()}
    # (from the Fourier layer's output on: transforms back to real numbers treat the imaginary part of frequency 0 as they like)
    blocks, model.blocks = model.blocks, torch.nn.ModuleList()
    head, model.head = model.head, torch.nn.Parameter(torch.eye(ex.WIDTH, device="cuda"))
    x = model(tokens).detach().double()
    model.blocks, model.head = blocks, head
    params = {k: p.detach().double().requires_grad_() for k, p in model.named_parameters() if k.startswith(("blocks", "norm", "head"))}

    def norm(v, weight):
        return v * torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-6) * weight

    h = norm(x, params["norm"])
    for n in range(2):
        b = {k: params[f"blocks.{n}.{k}"] for k in ("w_in", "w_out", "post_weight", "gate", "weight")}
        a, u = (h @ b["w_in"].T).split(ex.HIDDEN, 1)
        f = (torch.nn.functional.silu(a) * u) @ b["w_out"].T
        x = x + b["gate"] * norm(f, b["post_weight"])
        h = norm(x, b["weight"])
    out = h @ params["head"]
    assert float((out - logits).detach().abs().max()) < 1e-4 * float(out.detach().abs().max())
    out.backward(way.double())
    for k, p in params.items():
        assert float((got[k] - p.grad).abs().pow(2).sum().sqrt()) < 3 * 2.0 ** -7 * float(p.grad.abs().pow(2).sum().sqrt()), k


def test_captured_beside_an_eager_graph():
    """A backward pass captured while an eager graph of other leaves lives."""
    torch.manual_seed(3)
    rows, w = 96, ex.WIDTH
    model = ex.SpectralLM(blocks=1).cuda()
    b = model.blocks[0]
    x, gx, gh = (torch.randn(rows, w, device="cuda") for _ in range(3))

    def passes(leaf):
        new, h, h8 = ex.FirstNorm.apply(leaf, model.norm)
        new, h, h8 = ex.FeedForward.apply(new, h, h8, b["w_in"], b["w_out"], b["post_weight"], b["gate"], b["weight"])
        return torch.autograd.grad([new, h], [leaf, b["w_in"], b["w_out"], b["gate"]], [gx, gh])

    leaf = x.clone().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            passes(leaf)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = passes(leaf)
    for seed in (5, 6):
        with torch.no_grad():
            leaf.copy_(torch.randn(rows, w, device="cuda", generator=torch.Generator("cuda").manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        want = passes(leaf.detach().clone().requires_grad_())
        assert all(torch.equal(p, q) for p, q in zip(out, want))
