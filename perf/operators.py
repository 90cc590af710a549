"""Cases of the operators around the optimizer step: what a training loop computes between a model's outputs and the
weights' update.

  norm       gradient norm over a list of tensors (per tensor and global) and the clipping coefficient
  clip       the same, and every gradient scaled in place
  adamw      AdamW over a list of dense tensors, the clipping coefficient applied on the way
  logprob    log-probability of one token per row of logits, its entropy, and the gradient of both
  policy     clipped policy loss with a KL term and an entropy bonus, with its gradient with respect to the logits
  preference loss on paired log-ratio sums of two answers, with its gradient with respect to the logits

`run` computes a case in its plain form (elementary torch operations in fp32), or, where `own` is true, with this
package's calls.  `exact` gives the same outputs from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "c64": torch.complex64}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "c64": 8}
BETA1, BETA2, EPS, DECAY, LR, STEP = 0.9, 0.999, 1e-8, 0.01, 1e-3, 12
LOSS_SCALE = {"f32": 1.0, "bf16": 1.0, "f16": 4096.0}  # gradients of a mean over tokens are too small for fp16 without it


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a small model with tiny layers: the norm is wanted every step and costs launches, not bytes
        {"name": "norm_small", "op": "norm", "max_norm": 1.0, "packed": False,
         "tensors": "8*f32:128x128;8*f32:128;4*f32:64x129;1*f32:1001x64"},
        # spectral layers' complex gradients beside dense 16-bit ones, as one optimizer step sees them
        {"name": "norm_large", "op": "norm", "max_norm": 1.0, "packed": False,
         "tensors": "4*c64:128x128x64x33;16*bf16:4096x4096;16*bf16:4096"},
        # views into a flat 16-bit gradient buffer, one after the other at odd offsets
        {"name": "clip_ragged", "op": "clip", "max_norm": 1.0, "packed": True,
         "tensors": "36*bf16:1023x1025;36*bf16:1025;36*bf16:33x64;36*bf16:1;1*bf16:2000003"},
        # a five-way spectral gradient beside dense fp32 ones, more than the caches hold
        {"name": "clip_large", "op": "clip", "max_norm": 1.0, "packed": False,
         "tensors": "1*c64:64x64x32x32x17;24*f32:2048x2048;24*f32:2048"},
        # biases, norms and small matrices in fp32
        {"name": "adamw_small", "op": "adamw", "master": False, "packed": False,
         "tensors": "16*f32:128x129;16*f32:128;8*f32:257x64"},
        # 16-bit weights with fp32 master weights, views into flat buffers
        {"name": "adamw_large", "op": "adamw", "master": True, "packed": True,
         "tensors": "32*bf16:2048x2049;32*bf16:2049;1*bf16:33x32001"},
        # scoring the tokens that four sequences have just sampled
        {"name": "logprob_step", "op": "logprob", "backward": False, "rows": 4, "vocab": 131072, "dtype": "bf16", "pad": 0,
         "ignored": 0.0, "masked": 0, "temperature": 0.7},
        # log-probabilities in training, with entropy, forward and backward; a vocabulary that is no multiple of anything
        {"name": "logprob_train", "op": "logprob", "backward": True, "rows": 6000, "vocab": 50257, "dtype": "bf16", "pad": 0,
         "ignored": 0.2, "masked": 0, "temperature": 1.0},
        # one micro-batch of a small model in fp32
        {"name": "policy_small", "op": "policy", "rows": 97, "vocab": 10007, "dtype": "f32", "pad": 5, "ignored": 0.25, "masked": 7,
         "temperature": 1.0, "kl": 0.05, "entropy": 0.01},
        # a full batch of answers over a large vocabulary
        {"name": "policy_large", "op": "policy", "rows": 8192, "vocab": 131072, "dtype": "bf16", "pad": 0, "ignored": 0.125, "masked": 64,
         "temperature": 0.9, "kl": 0.02, "entropy": 0.0},
        # three pairs of short answers, odd sizes
        {"name": "preference_small", "op": "preference", "pairs": 3, "longest": 61, "lengths": 5, "vocab": 8191, "dtype": "f16", "pad": 1,
         "ignored": 0.3, "masked": 3, "temperature": 1.0, "beta": 0.1, "smoothing": 0.0},
        # sixteen pairs of prompts with two answers each
        {"name": "preference_large", "op": "preference", "pairs": 16, "longest": 1024, "lengths": 9, "vocab": 32768, "dtype": "bf16", "pad": 0,
         "ignored": 0.3, "masked": 0, "temperature": 1.0, "beta": 0.1, "smoothing": 0.1},
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "clip", "adamw", "logprob", "policy", "preference"])
    if op in ("norm", "clip", "adamw"):
        count, most = _spread(rng, 1, 150), {"norm": 4e8, "clip": 2e8, "adamw": 1.2e8}[op]
        total = _spread(rng, 1e4, most)
        kinds = rng.choice(["f32", "bf16", "f16", "c64", "f32,bf16", "c64,f32", "c64,bf16,f16"]) if op != "adamw" else rng.choice(["f32", "bf16", "f16", "c64"])
        parts = [rng.paretovariate(0.8) for _ in range(count)]
        parts = ["%s:%d" % (rng.choice(kinds.split(",")), max(1, int(total * p / sum(parts)))) for p in parts]
        parts = [p if not p.startswith("c64") else "c64:%d" % max(1, int(p[4:]) // 2) for p in parts]
        case = {"op": op, "packed": rng.random() < 0.5, "tensors": ";".join(parts)}
        if op == "adamw":
            case["master"] = kinds in ("bf16", "f16") and rng.random() < 0.5
        else:
            case["max_norm"] = rng.choice([0.5, 1.0, 1e9])
        return case
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    vocab = _spread(rng, 1000, 200000)
    logits = {"vocab": vocab, "dtype": dtype, "pad": rng.choice([0, 0, -vocab % 64, 3]), "ignored": rng.choice([0.0, 0.3]),
              "masked": rng.choice([0, rng.randrange(1, 200)]), "temperature": rng.choice([1.0, 0.8])}
    rows = _spread(rng, 1, max(2, min(16384, 1.6e9 / BYTES[dtype] / vocab)))
    if op == "logprob":
        return {"op": op, "backward": rng.random() < 0.5, "rows": rows, **logits}
    if op == "policy":
        return {"op": op, "rows": rows, **logits, "kl": rng.choice([0.0, 0.04]), "entropy": rng.choice([0.0, 0.01])}
    pairs = _spread(rng, 1, 24)
    return {"op": op, "pairs": pairs, "longest": max(2, rows // (2 * pairs)), "lengths": rng.randrange(1 << 20), **logits,
            "beta": rng.choice([0.05, 0.1]), "smoothing": rng.choice([0.0, 0.1])}


def _tensors(case):
    """[(kind, entries)] of a list of tensors."""
    out = []
    for part in case["tensors"].split(";"):
        times, spec = part.split("*") if "*" in part else ("1", part)
        kind, dims = spec.split(":")
        out += [(kind, math.prod(int(d) for d in dims.split("x")))] * int(times)
    return out


def _lengths(case):
    """Lengths of the 2 * pairs answers, prompts included."""
    r = random.Random(case["lengths"])
    return [r.randint(max(1, case["longest"] // 4), case["longest"]) for _ in range(2 * case["pairs"])]


def _row_count(case):
    return sum(_lengths(case)) if case["op"] == "preference" else case["rows"]


def _ignored_rows(case, rows):
    """Rows without a target: prompts and padding."""
    r = random.Random(rows)
    if case["op"] != "preference":
        return [i for i in range(rows) if r.random() < case["ignored"]]
    out, at = [], 0
    for n in _lengths(case):
        out += range(at, at + int(n * case["ignored"]))
        at += n
    return out


# ---------------------------------------------------------------------------------------------- inputs
def _flat(specs, packed, make):
    """One flat buffer per dtype and the views into it, one after the other (packed) or each from a multiple of 16 bytes."""
    step = {k: 1 if packed else 16 // BYTES[k] for k, _ in specs}
    at, where = {}, []
    for kind, n in specs:
        start = -(-at.get(kind, 0) // step[kind]) * step[kind]
        where.append((kind, start, n))
        at[kind] = start + n
    flats = {kind: make(kind, n) for kind, n in at.items()}
    return flats, [flats[kind][start:start + n] for kind, start, n in where]


def _prepare_list(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    specs = _tensors(case)
    rnd = random.Random(seed)

    def normal(kind, n):
        return torch.randn(n, generator=gen, device="cuda", dtype=DTYPES[kind])

    flats, views = _flat(specs, case["packed"], normal)
    for v in views:  # layers differ in scale
        v.mul_(10 ** rnd.uniform(-3, -1))
    s = {"case": case, "flats": flats, "grads": views}
    if case["op"] == "adamw":
        real = {k: torch.float32 for k in DTYPES}
        s["p_flats"], s["params"] = _flat(specs, case["packed"], lambda k, n: normal(k, n).mul_(0.05))
        s["m_flats"], s["exp_avgs"] = _flat(specs, case["packed"], lambda k, n: torch.randn(n, generator=gen, device="cuda", dtype=torch.complex64 if k == "c64" else torch.float32).mul_(0.01))
        s["v_flats"], s["exp_avg_sqs"] = _flat(specs, case["packed"], lambda k, n: torch.rand(n, generator=gen, device="cuda", dtype=real[k]).mul_(1e-3).add_(1e-6))
        if case["master"]:
            s["w_flats"], s["masters"] = _flat(specs, case["packed"], lambda k, n: s["p_flats"][k].float())
        s["coefficient"] = torch.full((1,), 0.37, device="cuda")
    if own:
        from paper_2501_02379_b200 import binding as B
        s["lists"] = {k: B.TensorList(s[k]) for k in ("grads", "params", "exp_avgs", "exp_avg_sqs", "masters") if k in s}
    return s


def _prepare_logits(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rows, vocab = _row_count(case), case["vocab"]
    full = torch.randn(rows, vocab + case["pad"], generator=gen, device="cuda", dtype=DTYPES[case["dtype"]]).mul_(2.0)
    logits = full[:, :vocab]
    targets = torch.randint(0, vocab - case["masked"], (rows,), generator=gen, device="cuda")
    lift = torch.randn(rows, 1, generator=gen, device="cuda") * 2 + 7  # the sampled token is a likely one
    logits.scatter_add_(1, targets[:, None], lift.to(logits.dtype))
    if case["masked"]:
        logits[:, vocab - case["masked"]:] = -math.inf  # entries of the vocabulary that are never sampled
    s = {"case": case, "logits": logits, "targets": targets}
    logp = torch.cat([torch.log_softmax(x.float() / case["temperature"], 1).gather(1, t[:, None])[:, 0]
                      for x, t in zip(logits.split(256), targets.split(256))])
    off = _ignored_rows(case, rows)
    if off:
        off = torch.tensor(off, device="cuda")
        targets[off] = -100
        logits[off[0]] = math.nan  # what stands in an ignored row is never looked at
    live = targets >= 0

    def normal(std):
        return torch.randn(rows, generator=gen, device="cuda") * std

    if case["op"] == "logprob":
        s["grad_logp"], s["grad_entropy"] = normal(1.0), normal(0.01)
    elif case["op"] == "policy":
        # ratios of a policy that has moved since the tokens were sampled, not exactly at the clipping bounds
        shift = normal(0.3)
        for bound in (math.log(0.8), math.log(1.2)):
            shift = torch.where((shift - bound).abs() < 0.005, shift + 0.02, shift)
        s["old_logp"], s["ref_logp"] = logp - shift, logp + normal(0.2)
        s["advantages"] = normal(1.0)
        s["weights"] = live.float() / live.sum().clamp(min=1)  # mean over the tokens of the answers
    else:
        s["ref_logp"] = logp + normal(0.3)
        s["starts"] = torch.tensor([0] + torch.tensor(_lengths(case)).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    return _prepare_list(case, seed) if case["op"] in ("norm", "clip", "adamw") else _prepare_logits(case, seed)


# ---------------------------------------------------------------------------------------------- the package's calls
def _run_own(s):
    from paper_2501_02379_b200 import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "norm":
        return B.grad_norm(s["lists"]["grads"], case["max_norm"])
    if op == "clip":
        norms = B.clip_grads(s["lists"]["grads"], case["max_norm"])
        return {"norms": norms, "grads": s["flats"]}
    if op == "adamw":
        t = s["lists"]
        B.adamw_step(t["params"], t["grads"], t["exp_avgs"], t["exp_avg_sqs"], step=STEP, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                     weight_decay=DECAY, grad_scale=s["coefficient"], masters=t.get("masters"))
        return {k: s[k] for k in ("p_flats", "m_flats", "v_flats", "w_flats") if k in s}
    if op == "logprob":
        logp, lse, entropy = B.token_logprob(s["logits"], s["targets"], temperature=case["temperature"])
        out = {"logp": logp, "lse": lse, "entropy": entropy}
        if case["backward"]:
            out["dlogits"] = B.token_logprob_backward(s["logits"], s["targets"], lse, s["grad_logp"], entropy=entropy,
                                                      grad_entropy=s["grad_entropy"], temperature=case["temperature"])
        return out
    if op == "policy":
        r = B.policy_loss(s["logits"], s["targets"], s["old_logp"], s["advantages"], s["weights"], ref_logp=s["ref_logp"], clip_low=0.2,
                          clip_high=0.2, kl_coef=case["kl"], entropy_coef=case["entropy"], temperature=case["temperature"],
                          grad_scale=LOSS_SCALE[case["dtype"]])
        return {"stats": r.stats, "logp": r.logp, "entropy": r.entropy, "dlogits": r.dlogits}
    r = B.preference_loss(s["logits"], s["targets"], s["starts"], s["ref_logp"], beta=case["beta"], label_smoothing=case["smoothing"],
                          temperature=case["temperature"], grad_scale=LOSS_SCALE[case["dtype"]])
    return {"loss": r.loss, "rewards": r.rewards, "logp": r.logp, "dlogits": r.dlogits}


# ---------------------------------------------------------------------------------------------- the plain forms
def _reals(x):
    return torch.view_as_real(x) if x.is_complex() else x


def _plain_norm(case, grads):
    norms = torch.stack([_reals(g).float().square().sum().sqrt() for g in grads])
    norm = norms.square().sum().sqrt()
    coefficient = (case["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    return torch.cat([norm[None], coefficient[None], norms])


def _plain_adamw_one(p, g, m, v, w, c):
    g = g * c if g.is_complex() else g.float() * c
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(_reals(g).square().sum(-1) * (1 - BETA2) if g.is_complex() else g.square() * (1 - BETA2))
    update = m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
    at = p if w is None else w
    new = (at if at.is_complex() else at.float()) * (1 - LR * DECAY) - LR * update
    at.copy_(new)
    if w is not None:
        p.copy_(new)


def _plain_softmax(s):
    """Scaled logits, which rows count, their log-sum-exp, the targets' log-probability, probabilities and log-probabilities."""
    live = s["targets"] >= 0
    z = s["logits"].float() * (1.0 / s["case"]["temperature"])
    top = z.amax(1, keepdim=True)
    lse = (z - top).exp().sum(1, keepdim=True).log() + top
    logp = z.gather(1, s["targets"].clamp(min=0)[:, None])[:, 0] - lse[:, 0]
    z -= lse
    return live, torch.where(live, lse[:, 0], 0.0), torch.where(live, logp, 0.0), z


def _plain_entropy(live, logq):
    q = logq.exp()
    return torch.where(live, -torch.where(q > 0, q * logq, 0.0).sum(1), 0.0)


def _plain_dlogits(s, live, logq, entropy, d_logp, d_entropy):
    """Gradient of sum(d_logp * logp + d_entropy * entropy) with respect to the logits."""
    q = logq.exp()
    d = q * -d_logp[:, None]
    if d_entropy is not None:
        d -= torch.where(q > 0, q * (logq + entropy[:, None]), 0.0) * d_entropy[:, None]
    at = s["targets"].clamp(min=0)[:, None]
    d.scatter_add_(1, at, d_logp[:, None])
    d *= (1.0 if s["case"]["op"] == "logprob" else LOSS_SCALE[s["case"]["dtype"]]) / s["case"]["temperature"]
    return torch.where(live[:, None], d, 0.0).to(s["logits"].dtype)


def _plain_policy(s):
    case, w = s["case"], s["weights"]
    live, _, logp, logq = _plain_softmax(s)
    entropy = _plain_entropy(live, logq)
    ratio = (logp - s["old_logp"]).exp()
    free, bound = ratio * s["advantages"], ratio.clamp(0.8, 1.2) * s["advantages"]
    gap = s["ref_logp"] - logp
    kl = gap.exp() - gap - 1
    zero = torch.zeros_like(w)
    pg, kl, h, cut = (torch.where(live, x, zero) for x in (-torch.minimum(free, bound), kl, entropy, (free > bound).float()))
    sums = [(w * x).sum() for x in (pg, kl, h, cut)]
    stats = torch.stack([sums[0] + case["kl"] * sums[1] - case["entropy"] * sums[2]] + sums)
    d_logp = w * (torch.where(free <= bound, -free, zero) + case["kl"] * (1 - gap.exp()))
    d_entropy = -case["entropy"] * w if case["entropy"] else None
    return {"stats": stats, "logp": logp, "entropy": entropy, "dlogits": _plain_dlogits(s, live, logq, entropy, torch.where(live, d_logp, zero), d_entropy)}


def _plain_preference(s):
    case, starts = s["case"], s["starts"]
    live, _, logp, logq = _plain_softmax(s)
    gap = torch.where(live, logp - s["ref_logp"], 0.0)
    row = torch.arange(len(gap), device=gap.device)
    member = (row >= starts[:-1, None]) & (row < starts[1:, None])
    rewards = case["beta"] * torch.where(member, gap, 0.0).sum(1)
    h = rewards[0::2] - rewards[1::2]
    tail = (1 + (-h.abs()).exp()).log()
    e = case["smoothing"]
    loss = ((1 - e) * ((-h).clamp(min=0) + tail) + e * (h.clamp(min=0) + tail)).mean()
    right = 1 / (1 + (-h).exp())
    d_h = (-(1 - e) * (1 - right) + e * right) / case["pairs"] * case["beta"]
    d_seq = torch.stack([d_h, -d_h], 1).reshape(-1)
    d_logp = torch.where(live, torch.where(member, d_seq[:, None], 0.0).sum(0), 0.0)
    return {"loss": loss, "rewards": rewards, "logp": logp, "dlogits": _plain_dlogits(s, live, logq, None, d_logp, None)}


def _run_plain(s):
    case, op = s["case"], s["case"]["op"]
    if op in ("norm", "clip"):
        norms = _plain_norm(case, s["grads"])
        if op == "norm":
            return norms
        [g.copy_(g * norms[1] if g.is_complex() else g.float() * norms[1]) for g in s["grads"]]
        return {"norms": norms, "grads": s["flats"]}
    if op == "adamw":
        [_plain_adamw_one(p, g, m, v, w, s["coefficient"]) for p, g, m, v, w in
         zip(s["params"], s["grads"], s["exp_avgs"], s["exp_avg_sqs"], s.get("masters") or [None] * len(s["params"]))]
        return {k: s[k] for k in ("p_flats", "m_flats", "v_flats", "w_flats") if k in s}
    if op == "logprob":
        live, lse, logp, logq = _plain_softmax(s)
        out = {"logp": logp, "lse": lse, "entropy": _plain_entropy(live, logq)}
        if case["backward"]:
            out["dlogits"] = _plain_dlogits(s, live, logq, out["entropy"], s["grad_logp"], s["grad_entropy"])
        return out
    return _plain_policy(s) if op == "policy" else _plain_preference(s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    op = case["op"]
    if op in ("norm", "clip", "adamw"):
        nbytes = flops = 0
        for kind, n in _tensors(case):
            b, reals = BYTES[kind], n * (2 if kind == "c64" else 1)
            if op == "adamw":  # gradient read; weight, first and second moment read and written; with masters the weight is only written
                m = 8 if kind == "c64" else 4
                nbytes += n * (b + 2 * m + 2 * 4 + (8 + b if case["master"] else 2 * b))
                flops += 14 * reals
            else:
                nbytes += n * b * (2 if op == "clip" else 1)
                flops += reals * (3 if op == "clip" else 2)
        return {"bytes": nbytes, "flops": flops}
    rows = _row_count(case)
    live = rows - len(_ignored_rows(case, rows))
    vocab, b = case["vocab"], BYTES[case["dtype"]]
    back = op != "logprob" or case["backward"]
    return {"bytes": live * vocab * b + (rows * vocab * b if back else 0) + rows * 40, "flops": live * vocab * (10 if back else 5)}


# ---------------------------------------------------------------------------------------------- 64 bits
def _exact_list(case, seed):
    s = _prepare_list(case, seed)
    wide = [g.to(torch.complex128 if g.is_complex() else torch.float64) for g in s["grads"]]
    if case["op"] == "adamw":
        kept = {k: {d: f.to(torch.complex128 if f.is_complex() else torch.float64) for d, f in s[k].items()} for k in ("p_flats", "m_flats", "v_flats", "w_flats") if k in s}

        def views(name):  # the same places in the wide buffers
            return [kept[name][k].as_strided(v.shape, v.stride(), v.storage_offset()) for (k, _), v in zip(_tensors(case), s["grads"])]

        c = float(s["coefficient"].double()[0])
        to = views("w_flats") if case["master"] else views("p_flats")
        b1, b2, keep = BETA1, BETA2, 1 - LR * DECAY
        for g, p, m, v in zip(wide, to, views("m_flats"), views("v_flats")):
            g = g * c
            m.copy_(b1 * m + (1 - b1) * g)
            v.copy_(b2 * v + (1 - b2) * g.abs() ** 2)
            p.copy_(keep * p - LR * (m / (1 - b1 ** STEP)) / ((v / (1 - b2 ** STEP)).sqrt() + EPS))
        if case["master"]:
            for a, b in zip(views("p_flats"), to):
                a.copy_(b)
        return kept
    norms = torch.stack([torch.linalg.vector_norm(g) for g in wide])
    norm = torch.linalg.vector_norm(norms)
    c = torch.clamp(case["max_norm"] / (norm + 1e-6), max=1.0)
    out = torch.cat([norm.reshape(1), c.reshape(1), norms])
    if case["op"] == "norm":
        return out
    kept = {d: f.to(torch.complex128 if f.is_complex() else torch.float64) for d, f in s["flats"].items()}
    for (k, _), v, g in zip(_tensors(case), s["grads"], wide):
        kept[k].as_strided(v.shape, v.stride(), v.storage_offset()).copy_(g * c)
    return {"norms": out, "grads": kept}


def exact(case, seed):
    if case["op"] in ("norm", "clip", "adamw"):
        return _exact_list(case, seed)
    s = _prepare_logits(case, seed)
    z, y, tau = s["logits"], s["targets"], case["temperature"]
    rows, vocab = z.shape
    live = y >= 0
    pick = live.nonzero()[:, 0]
    part = max(1, (1 << 26) // vocab)
    scale = 1.0 if case["op"] == "logprob" else LOSS_SCALE[case["dtype"]]
    lse, logp, entropy = (torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(3))
    for at in pick.split(part):
        x = z[at].double() / tau
        lse[at] = torch.logsumexp(x, 1)
        logp[at] = torch.log_softmax(x, 1).gather(1, y[at][:, None])[:, 0]
        entropy[at] = torch.special.entr(torch.softmax(x, 1)).sum(1)
    out = {"logp": logp, "lse": lse, "entropy": entropy}
    if case["op"] == "logprob":
        d_logp, d_h = s["grad_logp"].double(), s["grad_entropy"].double()
    elif case["op"] == "policy":
        w, adv = s["weights"].double(), s["advantages"].double()
        r = torch.exp(logp - s["old_logp"].double())
        low, high = float(torch.tensor(0.8)), float(torch.tensor(1.2))
        a, b = r * adv, torch.clamp(r, low, high) * adv
        u = s["ref_logp"].double() - logp
        terms = [-torch.min(a, b), torch.expm1(u) - u, entropy, (a > b).double()]
        sums = [(w * t)[live].sum() for t in terms]
        out = {"stats": torch.stack([sums[0] + case["kl"] * sums[1] - case["entropy"] * sums[2]] + sums), "logp": logp, "entropy": entropy}
        d_logp = w * (torch.where(a > b, 0.0, -a) - case["kl"] * torch.expm1(u))
        d_h = -case["entropy"] * w
    else:
        n = [b - a for a, b in zip(s["starts"].tolist(), s["starts"].tolist()[1:])]
        gap = torch.where(live, logp - s["ref_logp"].double(), 0.0)
        rewards = case["beta"] * torch.stack([g.sum() for g in gap.split(n)])
        h, e = rewards[0::2] - rewards[1::2], case["smoothing"]
        loss = -((1 - e) * torch.nn.functional.logsigmoid(h) + e * torch.nn.functional.logsigmoid(-h)).mean()
        d = case["beta"] * (torch.sigmoid(h) - (1 - e)) / case["pairs"]
        d_logp = torch.cat([x.expand(k) for x, k in zip(torch.stack([d, -d], 1).reshape(-1), n)])
        d_h = torch.zeros_like(d_logp)
        out = {"loss": loss, "rewards": rewards, "logp": logp}
    if case["op"] != "logprob" or case["backward"]:
        dz = torch.zeros(rows, vocab, dtype=torch.float64, device="cuda")
        for at in pick.split(part):
            q = torch.log_softmax(z[at].double() / tau, 1)
            g = -torch.exp(q) * d_logp[at][:, None]
            g += (torch.special.entr(torch.exp(q)) - torch.exp(q) * entropy[at][:, None]) * d_h[at][:, None]
            g.scatter_add_(1, y[at][:, None], d_logp[at][:, None])
            dz[at] = g * scale / tau
        out["dlogits"] = dz
    return out
