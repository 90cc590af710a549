"""Plain 64-bit definitions of the operators around the optimizer step (numpy only): gradient norm and clipping, AdamW,
token log-probabilities, the clipped policy loss and the loss on pairs of answers, with their gradients.

Shares no code with the library.  Loops over rows where that is the plainest way to write a definition down.
"""
import numpy as np


def grad_norm(grads, max_norm=np.inf):
    """(global norm, coefficient, norm of each tensor)."""
    norms = []
    for g in grads:
        g = np.asarray(g)
        a = np.abs(g.astype(np.complex128 if np.iscomplexobj(g) else np.float64)).reshape(-1)
        top = a.max() if a.size else 0.0
        norms.append(float(top * np.sqrt(np.sum((a / top) ** 2))) if 0 < top < np.inf else float(top))
    norm = float(np.sqrt(np.sum(np.square(norms)))) if norms else 0.0
    c = 1.0 if np.isinf(max_norm) else min(1.0, max_norm / (norm + 1e-6))
    return norm, c, norms


def adamw(w, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, scale=1.0):
    """Updated (w, m, v)."""
    kind = np.complex128 if np.iscomplexobj(w) else np.float64
    w, g, m, v = np.asarray(w, kind), np.asarray(g, kind) * scale, np.asarray(m, kind), np.asarray(v, np.float64)
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * np.abs(g) ** 2
    w = (1 - lr * weight_decay) * w - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return w, m, v


def token_row(z, y, tau=1.0):
    """(logp, lse, entropy, p) of one row with target y >= 0."""
    z = np.asarray(z, np.float64) / tau
    if y >= z.size or not np.any(z > -np.inf) or np.any(np.isnan(z)) or np.any(z == np.inf):
        return np.nan, np.nan, np.nan, np.full(z.size, np.nan)
    top = z.max()
    e = np.exp(z - top)
    lse = top + np.log(e.sum())
    p = e / e.sum()
    live = p > 0
    return z[y] - lse, lse, float(-np.sum(p[live] * np.log(p[live]))), p


def token_logprob(z, y, tau=1.0):
    """(logp, lse, entropy) of every row; 0 where y < 0."""
    out = np.zeros((3, len(y)))
    for i in range(len(y)):
        if y[i] >= 0:
            out[:, i] = token_row(z[i], y[i], tau)[:3]
    return out[0], out[1], out[2]


def token_gradient(z, y, g, h, tau=1.0):
    """Gradient of sum(g logp + h entropy) with respect to the logits."""
    d = np.zeros(np.shape(z))
    for i in range(len(y)):
        if y[i] < 0:
            continue
        _, _, H, p = token_row(z[i], y[i], tau)
        one = np.zeros(p.size)
        if y[i] < p.size:
            one[y[i]] = 1.0
        logp = np.log(np.where(p > 0, p, 1.0))
        d[i] = (g[i] * (one - p) - h[i] * p * (logp + H)) / tau
    return d


def policy_loss(z, y, old, adv, w, ref=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0, tau=1.0, grad_scale=1.0):
    """dict(stats, logp, entropy, dlogits, g, ratio)."""
    logp, _, H = token_logprob(z, y, tau)
    stats, g, h, ratio = np.zeros(5), np.zeros(len(y)), np.zeros(len(y)), np.ones(len(y))
    for i in range(len(y)):
        if y[i] < 0:
            continue
        r = ratio[i] = np.exp(logp[i] - old[i])
        free, bound = r * adv[i], min(max(r, 1 - clip_low), 1 + clip_high) * adv[i]
        cut = free > bound
        u = 0.0 if ref is None else ref[i] - logp[i]
        kl = np.expm1(u) - u
        terms = np.array([-min(free, bound), kl, H[i], float(cut)]) * w[i]
        stats[1:] += terms
        g[i] = w[i] * ((0.0 if cut else -free) - kl_coef * np.expm1(u))
        h[i] = -entropy_coef * w[i]
    stats[0] = stats[1] + kl_coef * stats[2] - entropy_coef * stats[3]
    return {"stats": stats, "logp": logp, "entropy": H, "dlogits": grad_scale * token_gradient(z, y, g, h, tau), "g": g, "ratio": ratio}


def preference_loss(z, y, starts, ref, beta=0.1, smoothing=0.0, tau=1.0, grad_scale=1.0):
    """dict(loss, rewards, logp, dlogits, g)."""
    logp, _, _ = token_logprob(z, y, tau)
    pairs = len(starts) // 2
    rewards, g, loss = np.zeros(2 * pairs), np.zeros(len(y)), 0.0
    for s in range(2 * pairs):
        for i in range(starts[s], starts[s + 1]):
            if y[i] >= 0:
                rewards[s] += beta * (logp[i] - ref[i])
    for b in range(pairs):
        x = rewards[2 * b] - rewards[2 * b + 1]
        loss += ((1 - smoothing) * np.logaddexp(0, -x) + smoothing * np.logaddexp(0, x)) / pairs
        d = beta * (1 / (1 + np.exp(-x)) - (1 - smoothing)) / pairs
        for s, sign in ((2 * b, 1), (2 * b + 1, -1)):
            g[starts[s]:starts[s + 1]] = sign * d
    return {"loss": loss, "rewards": rewards, "logp": logp, "dlogits": grad_scale * token_gradient(z, y, g, np.zeros(len(y)), tau), "g": g}
