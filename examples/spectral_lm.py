"""A small sequence model with a Fourier layer, trained on pairs of answers and then with a policy loss.

Everything between the logits and the updated weights is this package's: reference and sampling log-probabilities
(token_logprob), the two losses with their gradients, the global gradient norm over the complex and the dense tensors, and
the step: the spectral weight goes through the sparse + low-rank optimizer, the dense ones through AdamW, both scaled by the
clipping coefficient, which never leaves the device.

With --blocks n, n gated feed-forward blocks stand behind the Fourier layer.  They keep for their backward pass 8 bits an entry: the
normalised input, both halves of the first layer's output and the block's output; norms, gate, activation and weight
gradients are this package's.

    python examples/spectral_lm.py [--steps 60] [--blocks 2]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2501_02379_b200 import binding as B  # noqa: E402

VOCAB, WIDTH, LENGTH, PROMPT = 1000, 64, 64, 16
HIDDEN = 160


class FirstNorm(torch.autograd.Function):
    """x -> (x, h = norm(x), h packed)."""

    @staticmethod
    def forward(ctx, x, weight):
        r = B.residual_norm(x, weight=weight, keep_h=True)
        ctx.save_for_backward(r.x, r.stats, weight)
        ctx.mark_non_differentiable(r.h8.data)
        return r.x, r.h, r.h8.data

    @staticmethod
    def backward(ctx, grad_x, grad_h, _):
        x, stats, weight = ctx.saved_tensors
        g = B.residual_norm_backward(grad_h.contiguous(), x, stats, grad_x=grad_x.contiguous(), weight=weight)
        return g.x, g.weight


class FeedForward(torch.autograd.Function):
    """(x, h, h packed) -> (x' = x + gate * norm(f), h' = norm(x'), h' packed) with f = w_out (silu(a) u), (a, u) = w_in h."""

    @staticmethod
    def forward(ctx, x, h, h8, w_in, w_out, post_weight, gate, weight):
        a, u = (h @ w_in.T).split(HIDDEN, 1)
        y, a8, u8 = B.gated_act(a, u)
        r = B.residual_norm(x, y @ w_out.T, weight=weight, post_weight=post_weight, gate=gate, keep_f=True, keep_h=True)
        ctx.save_for_backward(h8, a8.data, u8.data, r.f8.data, r.x, r.stats, w_in, w_out, post_weight, gate, weight)
        ctx.mark_non_differentiable(r.h8.data)
        return r.x, r.h, r.h8.data

    @staticmethod
    def backward(ctx, grad_x, grad_h, _):
        h8, a8, u8, f8, x, stats, w_in, w_out, post_weight, gate, weight = ctx.saved_tensors
        rows, width = x.shape
        kept = lambda data, n: B.Packed(data, rows, n, x.dtype)  # noqa: E731
        n = B.residual_norm_backward(grad_h.contiguous(), x, stats, kept(f8, width), grad_x=grad_x.contiguous(), weight=weight, post_weight=post_weight, gate=gate)
        d = x.new_empty(rows, 2 * HIDDEN)
        g = B.gated_act_backward(kept(a8, HIDDEN), kept(u8, HIDDEN), n.f @ w_out, keep_y=True, da=d[:, :HIDDEN], du=d[:, HIDDEN:])
        return n.x, d @ w_in, None, B.weight_grad(d, kept(h8, width)), B.weight_grad(n.f, g.y8), n.post_weight, n.gate, n.weight


class SpectralLM(torch.nn.Module):
    """Embedding, one causal spectral convolution over the sequence (complex weight WIDTH x WIDTH x modes), feed-forward blocks, head."""

    def __init__(self, modes=32, blocks=0):
        super().__init__()
        self.embedding = torch.nn.Parameter(torch.randn(VOCAB, WIDTH) * 0.3)
        self.spectral = torch.nn.Parameter(torch.randn(WIDTH, WIDTH, modes, dtype=torch.complex64) * 0.02)
        self.bias = torch.nn.Parameter(torch.zeros(WIDTH))
        self.head = torch.nn.Parameter(torch.randn(WIDTH, VOCAB) * 0.05)
        self.blocks = torch.nn.ModuleList()
        if blocks:
            self.norm = torch.nn.Parameter(torch.ones(WIDTH))
        for _ in range(blocks):
            self.blocks.append(torch.nn.ParameterDict({"w_in": torch.randn(2 * HIDDEN, WIDTH) * WIDTH ** -0.5, "w_out": torch.randn(WIDTH, HIDDEN) * HIDDEN ** -0.5,
                                                       "post_weight": torch.ones(WIDTH), "gate": torch.full((WIDTH,), 0.1), "weight": torch.ones(WIDTH)}))

    def forward(self, tokens):
        x = self.embedding[tokens]                                              # [batch, length, width]
        n = 2 * tokens.shape[1]                                                 # zero padding: no wrap-around
        kernel = torch.fft.irfft(self.spectral, n=n)[..., :tokens.shape[1]]     # [width, width, length], causal
        spectrum = torch.einsum("bif,iof->bof", torch.fft.rfft(x.transpose(1, 2), n=n), torch.fft.rfft(kernel, n=n))
        mixed = torch.fft.irfft(spectrum, n=n)[..., :tokens.shape[1]].transpose(1, 2)
        x = x + torch.nn.functional.gelu(mixed + self.bias)
        if self.blocks:
            x, h, h8 = FirstNorm.apply(x.flatten(0, 1), self.norm)
            for b in self.blocks:
                x, h, h8 = FeedForward.apply(x, h, h8, b["w_in"], b["w_out"], b["post_weight"], b["gate"], b["weight"])
            return h @ self.head
        return (x @ self.head).flatten(0, 1)                                    # [batch * length, vocab]


class Trainer:
    def __init__(self, model, lr=3e-3, max_norm=1.0):
        self.model, self.lr, self.max_norm, self.t = model, lr, max_norm, 0
        dense = [p for p in model.parameters() if not p.is_complex()]
        for p in model.parameters():
            p.grad = torch.zeros_like(p)
        w = model.spectral
        ranks = [max(1, d // 4) for d in w.shape]
        self.state = B.TgradState(B.make_config(w.shape, ranks, k=w.numel() // 20, T=20, lr=lr, warm_refresh=True))
        # the tensors stay where they are, so their lists are laid out once
        self.grads = B.TensorList([p.grad for p in model.parameters()])
        self.dense = [B.TensorList(x) for x in ([p.data for p in dense], [p.grad for p in dense], [torch.zeros_like(p) for p in dense], [torch.zeros_like(p) for p in dense])]

    def step(self, logits, dlogits):
        """Backward from the logits' gradient, clipping, one optimizer step.  Returns the gradient norm (on the device)."""
        for p in self.model.parameters():
            p.grad.zero_()
        logits.backward(dlogits)
        norms = B.grad_norm(self.grads, self.max_norm)
        scale = norms[1:2]
        self.t += 1
        self.state.step_scaled(self.model.spectral, self.model.spectral.grad, scale)
        B.adamw_step(*self.dense, step=self.t, lr=self.lr, weight_decay=0.01, grad_scale=scale)
        return norms[0]


def pairs_batch(pairs, gen):
    """Prompts with two answers each: the chosen one counts on from the prompt's last token, the rejected one is random."""
    prompt = torch.randint(0, VOCAB, (pairs, 1, PROMPT), device="cuda", generator=gen).expand(pairs, 2, PROMPT)
    good = (prompt[:, :1, -1:] + torch.arange(1, LENGTH - PROMPT + 1, device="cuda")) % VOCAB
    bad = torch.randint(0, VOCAB, good.shape, device="cuda", generator=gen)
    tokens = torch.cat([prompt, torch.cat([good, bad], 1)], 2).flatten(0, 1)    # [2 * pairs, length]
    targets = torch.full_like(tokens, -100)
    targets[:, PROMPT - 1:-1] = tokens[:, PROMPT:]                              # row i predicts token i + 1; prompts are ignored
    starts = torch.arange(0, 2 * pairs + 1, device="cuda", dtype=torch.int32) * LENGTH
    return tokens, targets.flatten(), starts


def train_preference(model, trainer, steps, pairs=16, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    reference = SpectralLM(blocks=len(model.blocks)).cuda()
    reference.load_state_dict(model.state_dict())
    log = []
    for _ in range(steps):
        tokens, targets, starts = pairs_batch(pairs, gen)
        with torch.no_grad():
            ref_logp = B.token_logprob(reference(tokens), targets)[0]
        logits = model(tokens)
        r = B.preference_loss(logits.detach(), targets, starts, ref_logp, beta=0.1)
        norm = trainer.step(logits, r.dlogits)
        log.append(torch.stack([r.loss, (r.rewards[0::2] > r.rewards[1::2]).float().mean(), norm]))
    return torch.stack(log).cpu()


def train_policy(model, trainer, steps, batch=64, updates=2, seed=1):
    """Answers sampled from the model, rewarded for even tokens; each batch is used for `updates` steps."""
    gen = torch.Generator("cuda").manual_seed(seed)
    log = []
    for _ in range(steps):
        tokens = torch.randint(0, VOCAB, (batch, LENGTH), device="cuda", generator=gen)
        with torch.no_grad():
            logits = model(tokens)
            action = torch.multinomial(torch.softmax(logits, 1), 1, generator=gen)[:, 0]
            old_logp, _, _ = B.token_logprob(logits, action)
        reward = (action % 2 == 0).float()
        advantage = reward - reward.mean()
        weights = torch.full_like(reward, 1.0 / len(reward))
        for _ in range(updates):
            logits = model(tokens)
            r = B.policy_loss(logits.detach(), action, old_logp, advantage, weights, ref_logp=old_logp, kl_coef=0.01, entropy_coef=0.001)
            trainer.step(logits, r.dlogits)
        log.append(torch.stack([reward.mean(), r.stats[0], r.stats[2], r.stats[4]]))
    return torch.stack(log).cpu()


def main(steps=60, blocks=0):
    torch.manual_seed(0)
    model = SpectralLM(blocks=blocks).cuda()
    trainer = Trainer(model)
    pref = train_preference(model, trainer, steps)
    print("preference loss %.4f -> %.4f, chosen preferred %.2f -> %.2f" % (pref[0, 0], pref[-1, 0], pref[0, 1], pref[-5:, 1].mean()))
    pol = train_policy(model, trainer, steps)
    print("policy: mean reward %.3f -> %.3f (last KL %.4f, clipped %.3f)" % (pol[:3, 0].mean(), pol[-3:, 0].mean(), pol[-1, 2], pol[-1, 3]))
    flags, t, _ = trainer.state.query_status()
    print("steps", t, "flags", flags)
    return pref, pol, flags


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--blocks", type=int, default=0)
    args = ap.parse_args()
    main(args.steps, args.blocks)
