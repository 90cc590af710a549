"""The example that runs the losses, the clipping and both optimizers together (run with -m gpu)."""
import math

import pytest
import torch

from examples import spectral_lm as ex

pytestmark = pytest.mark.gpu


def test_example_learns():
    pref, pol, flags = ex.main(steps=40)
    assert flags == 0 and bool(torch.isfinite(pref).all()) and bool(torch.isfinite(pol).all())
    assert abs(pref[0, 0] - math.log(2)) < 1e-5            # the model is its own reference at first
    assert pref[-1, 0] < 0.75 * pref[0, 0] and pref[-5:, 1].mean() > 0.9
    assert pol[-3:, 0].mean() > pol[:3, 0].mean() + 0.03


def test_clipped_step_is_the_step_of_clipped_gradients():
    """The coefficient read on the device against the same numbers scaled in place first (fp32: one rounding apart)."""
    results = []
    for in_place in (False, True):
        torch.manual_seed(0)
        model = ex.SpectralLM().cuda()
        tr = ex.Trainer(model, max_norm=1e-3)
        tokens, targets, starts = ex.pairs_batch(4, torch.Generator("cuda").manual_seed(3))
        logits = model(tokens)
        ref = ex.B.token_logprob(logits.detach(), targets)[0]
        r = ex.B.preference_loss(logits.detach(), targets, starts, ref, 0.1)
        if in_place:
            logits.backward(r.dlogits)
            ex.B.clip_grads(tr.grads, tr.max_norm)
            tr.state.step(model.spectral, model.spectral.grad)
            ex.B.adamw_step(*tr.dense, step=1, lr=tr.lr, weight_decay=0.01)
        else:
            tr.step(logits, r.dlogits)
        results.append([m.clone() for m in tr.dense[2].tensors] + [torch.from_numpy(tr.state.export(ex.B.WHAT_M_S))])
    for a, b in zip(*results):
        a, b = a.cpu(), b.cpu()
        assert float((a - b).abs().max()) <= 4 * 2.0 ** -24 * float(b.abs().max())
