"""Cases of the operators of a trained block: activations kept in 8 bits, and what computes from them.

  pack    activations to 8 bits, in blocks of 32 entries of a row that share a power of two, and back
  gated   gated activation act(a) * u that keeps its inputs in 8 bits, and its gradient from them
  norm    norms around a block: x' = scale x + gate * norm(f), h = norm(x'), forward
  dnorm   its gradient, with respect to the residual stream, the block's output, the norms' weights and the gate
  wgrad   weight gradient dy^T x of a linear layer whose input is kept in 8 bits

`run` computes a case in its plain form (elementary torch operations in fp32), or, where `own` is true, with this
package's calls.  `exact` gives the same outputs from the definitions in 64 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 32
EPS = 1e-6
SCALE = 0.9  # of the residual stream


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one layer's input of a short answer; a width that is no multiple of a block, rows at odd places
        {"name": "pack_small", "op": "pack", "rows": 13, "width": 1001, "dtype": "bf16", "pad": 2},
        # a layer's input over a full batch of tokens
        {"name": "pack_large", "op": "pack", "rows": 16384, "width": 8192, "dtype": "bf16", "pad": 0},
        # the feed-forward part of a small model on one short sequence
        {"name": "gated_small", "op": "gated", "rows": 24, "width": 1376, "dtype": "bf16", "act": "silu", "halves": False, "keep_y": False},
        # halves of one product's output, an odd number of tokens, the output wanted again for the next weight gradient
        {"name": "gated_ragged", "op": "gated", "rows": 3001, "width": 2730, "dtype": "f16", "act": "gelu_tanh", "halves": True, "keep_y": True},
        # a full batch of tokens of a large model
        {"name": "gated_large", "op": "gated", "rows": 16384, "width": 14336, "dtype": "bf16", "act": "silu", "halves": True, "keep_y": False},
        # one token of eight sequences: latency
        {"name": "norm_small", "op": "norm", "rows": 8, "width": 4096, "dtype": "bf16", "param": "bf16", "kind": "rms", "groups": 1, "ragged": False, "keep": False},
        # norms around a block over a full batch; the block's output is kept in 8 bits
        {"name": "norm_large", "op": "norm", "rows": 16384, "width": 8192, "dtype": "bf16", "param": "bf16", "kind": "rms", "groups": 1, "ragged": False, "keep": True},
        # layer norms and a gate for each of 17 sequences of different lengths, fp32
        {"name": "dnorm_ragged", "op": "dnorm", "rows": 4001, "width": 1000, "dtype": "f32", "param": "f32", "kind": "layer", "groups": 17, "ragged": True, "keep": False},
        # the gradient over a full batch, from the block's output in 8 bits
        {"name": "dnorm_large", "op": "dnorm", "rows": 16384, "width": 8192, "dtype": "bf16", "param": "f32", "kind": "rms", "groups": 1, "ragged": False, "keep": True},
        # a small model's layer in fp32, odd sizes
        {"name": "wgrad_small", "op": "wgrad", "rows": 500, "out": 131, "width": 257, "dtype": "f32", "to": "f32"},
        # a narrow layer over many tokens, gradient in fp32: the tokens have to be split to fill the GPU
        {"name": "wgrad_long", "op": "wgrad", "rows": 65536, "out": 512, "width": 512, "dtype": "bf16", "to": "f32"},
        # the output layer of a large feed-forward part over a full batch
        {"name": "wgrad_large", "op": "wgrad", "rows": 16384, "out": 4096, "width": 14336, "dtype": "bf16", "to": "bf16"},
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["pack", "gated", "norm", "dnorm", "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "wgrad":
        rows, out, width = _spread(rng, 1, 65536), _spread(rng, 16, 8192), _spread(rng, 16, 16384)
        if dtype == "f32":
            rows = max(1, rows // 4)
        while rows * out * width > 8e11:
            rows = max(1, rows // 2)
        return {"op": op, "rows": rows, "out": out, "width": width, "dtype": dtype, "to": rng.choice([dtype, "f32"])}
    width = _spread(rng, 32 if "norm" in op else 1, 16384)
    if rng.random() < 0.5:
        width = -(-width // 64) * 64
    rows = _spread(rng, 1, max(2, min(32768, 2.4e8 / BYTES[dtype] / width)))
    case = {"op": op, "rows": rows, "width": width, "dtype": dtype}
    if op == "pack":
        return {**case, "pad": rng.choice([0, 0, 3, 64])}
    if op == "gated":
        return {**case, "act": rng.choice(["silu", "gelu", "gelu_tanh"]), "halves": rng.random() < 0.5, "keep_y": rng.random() < 0.3}
    groups = rng.choice([1, 1, rng.randrange(1, 33)])
    return {**case, "param": rng.choice([dtype, "f32"]), "kind": rng.choice(["rms", "layer"]), "groups": groups, "ragged": groups > 1, "keep": rng.random() < 0.5}


def _starts(case):
    """First rows of the sequences, the end of the last one behind them; rows after that belong to none."""
    r = random.Random(case["rows"] * 64 + case["groups"])
    cuts = sorted(r.randint(0, case["rows"]) for _ in range(case["groups"] - 1))
    return [0] + cuts + [case["rows"] if case["groups"] % 2 else max(cuts + [case["rows"] - 5])]


# ---------------------------------------------------------------------------------------------- inputs
def _activations(case, gen, size=1.0, pad=0, width=None):
    """Rows as they stand in a model: channels of different size, a few of them far above the rest."""
    rows, width = case["rows"], width or case["width"]
    x = torch.empty(rows, width + pad, device="cuda", dtype=DTYPES[case["dtype"]])
    channel = torch.exp(0.5 * torch.randn(width + pad, generator=gen, device="cuda")) * size
    channel[torch.rand(width + pad, generator=gen, device="cuda") < 0.002] *= 15
    for part in x.split(2048):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * channel)
    return x[:, :width]


def _inputs(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    op, rows, width, kind = case["op"], case["rows"], case["width"], DTYPES[case["dtype"]]

    def gradient(n, size):
        return (torch.randn(rows, n, generator=gen, device="cuda", dtype=kind) * size).to(kind)

    s = {"case": case}
    if op == "pack":
        s["x"] = _activations(case, gen, 1.0, case["pad"])
    elif op == "gated":
        if case["halves"]:
            both = _activations(case, gen, 0.7, 0, 2 * width)
            s["a"], s["u"] = both[:, :width], both[:, width:]
        else:
            s["a"], s["u"] = _activations(case, gen, 0.7), _activations(case, gen, 0.7)
        s["dy"] = gradient(width, 0.1)
    elif op == "wgrad":
        s["x"], s["dy"] = _activations(case, gen), gradient(case["out"], 0.1)
    else:
        param = DTYPES[case["param"]]
        s["x"], s["f"] = _activations(case, gen, 2.0), _activations(case, gen, 0.5)
        for name in ("weight", "post_weight"):
            s[name] = (1 + 0.1 * torch.randn(width, generator=gen, device="cuda")).to(param)
        if case["kind"] == "layer":
            for name in ("bias", "post_bias"):
                s[name] = (0.1 * torch.randn(width, generator=gen, device="cuda")).to(param)
        s["gate"] = (0.5 + 0.2 * torch.randn(case["groups"], width, generator=gen, device="cuda")).to(param)
        s["starts"] = torch.tensor(_starts(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        if op == "dnorm":
            s["dh"], s["dx"] = gradient(width, 0.1), gradient(width, 0.1)
            stats = []
            for v in (s["f"], s["x"]):
                v = v.float()
                mean = v.mean(1) if case["kind"] == "layer" else torch.zeros(rows, device="cuda")
                stats += [1 / ((v - mean[:, None]).square().mean(1) + EPS).sqrt(), mean]
            s["stats"] = torch.stack([stats[0], stats[2]] + ([stats[1], stats[3]] if case["kind"] == "layer" else []))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    kept = {"wgrad": "x", "dnorm": "f" if case.get("keep") else ""}.get(case["op"])
    if kept:  # what the forward pass has kept
        if own:
            from paper_2501_02379_b200 import binding as B
            s[kept + "8"] = B.act_pack(s[kept])
        else:
            s[kept + "8"] = _plain_pack(s[kept])
        if case["op"] == "wgrad":
            s.pop(kept)
    return s


# ---------------------------------------------------------------------------------------------- the package's calls
def _run_own(s):
    from paper_2501_02379_b200 import binding as B
    case, op = s["case"], s["case"]["op"]
    if op == "pack":
        return B.act_unpack(B.act_pack(s["x"]))
    if op == "wgrad":
        return B.weight_grad(s["dy"], s["x8"], dtype=DTYPES[case["to"]])
    if op == "gated":
        y, a8, u8 = B.gated_act(s["a"], s["u"], act=case["act"])
        rows, width = case["rows"], case["width"]
        both = s["dy"].new_empty(rows, 2 * width) if case["halves"] else None
        g = B.gated_act_backward(a8, u8, s["dy"], act=case["act"], keep_y=case["keep_y"],
                                 da=both[:, :width] if case["halves"] else None, du=both[:, width:] if case["halves"] else None)
        out = {"y": y, "d": both} if case["halves"] else {"y": y, "da": g.da, "du": g.du}
        if case["keep_y"]:
            out["y8"] = B.act_unpack(g.y8)
        return out
    how = {"weight": s["weight"], "post_weight": s["post_weight"], "post_bias": s.get("post_bias"), "gate": s["gate"], "starts": s["starts"],
           "scale": SCALE, "kind": case["kind"]}
    if op == "norm":
        r = B.residual_norm(s["x"], s["f"], bias=s.get("bias"), eps=EPS, keep_f=case["keep"], **how)
        out = {"x": r.x, "h": r.h, "stats": r.stats}
        if case["keep"]:
            out["f8"] = B.act_unpack(r.f8)
        return out
    r = B.residual_norm_backward(s["dh"], s["x"], s["stats"], s["f8"] if case["keep"] else s["f"], grad_x=s["dx"], **how)
    return {k: v for k, v in r._asdict().items() if v is not None}


# ---------------------------------------------------------------------------------------------- the plain forms
def _plain_pack(x):
    """Codes, the power of two of each block, width and type."""
    rows, width = x.shape
    v = torch.zeros(rows, -(-width // BLOCK) * BLOCK, device=x.device)
    v[:, :width] = x
    v = v.view(rows, -1, BLOCK)
    top = v.abs().amax(2, keepdim=True)
    e = (torch.frexp(top).exponent - 1 - 6).clamp(min=-126)  # a power of two times codes of 64 to 127 for the largest entry
    step = ((e + 127) << 23).view(torch.float32)  # 2^e by its bits: exp2 is not exact
    codes = torch.round(v / step).clamp(-127, 127).to(torch.int8)
    return codes, step, width, x.dtype


def _plain_unpack(packed):
    codes, step, width, dtype = packed
    return (codes.float() * step).view(codes.shape[0], -1)[:, :width].to(dtype)


def _plain_act(act, a):
    """act(a) and its derivative."""
    if act == "gelu":
        p = 0.5 * torch.erfc(a * -math.sqrt(0.5))
        return a * p, p + a * (a.square() * -0.5).exp() * (1 / math.sqrt(2 * math.pi))
    k = 2 * math.sqrt(2 / math.pi)
    z, dz = (a, 1.0) if act == "silu" else (k * (a + 0.044715 * a * a * a), k * (1 + 3 * 0.044715 * a * a))
    p = 1 / (1 + (-z).exp())
    return a * p, p + a * p * (1 - p) * dz


def _plain_gated(s):
    case, dtype = s["case"], s["a"].dtype
    y = (_plain_act(case["act"], s["a"].float())[0] * s["u"].float()).to(dtype)
    a, u, dy = _plain_unpack(_plain_pack(s["a"])).float(), _plain_unpack(_plain_pack(s["u"])).float(), s["dy"].float()
    f, df = _plain_act(case["act"], a)
    da, du = (dy * u * df).to(dtype), (dy * f).to(dtype)
    out = {"y": y, "d": torch.cat([da, du], 1)} if case["halves"] else {"y": y, "da": da, "du": du}
    if case["keep_y"]:
        out["y8"] = _plain_unpack(_plain_pack((f * u).to(dtype)))
    return out


def _plain_gate(s):
    """The gate of each row: 0 behind the last sequence."""
    gate, starts = s["gate"].float(), s["starts"]
    if starts is None:
        return gate.expand(s["case"]["rows"], -1), None
    row = torch.arange(s["case"]["rows"], device=gate.device)
    member = ((row >= starts[:-1, None]) & (row < starts[1:, None])).float()  # [groups, rows]
    return member.T @ gate, member


def _plain_norm(s):
    case = s["case"]
    x, f = s["x"].float(), s["f"].float()
    layer = case["kind"] == "layer"

    def norm(v, w, b):
        mean = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
        r = ((v - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
        n = (v - mean) * r * w.float()
        return n + b.float() if layer else n, r[:, 0], mean[:, 0]

    n, r0, m0 = norm(f, s["post_weight"], s.get("post_bias"))
    new = SCALE * x + _plain_gate(s)[0] * n
    h, r1, m1 = norm(new, s["weight"], s.get("bias"))
    out = {"x": new.to(s["x"].dtype), "h": h.to(s["x"].dtype), "stats": torch.stack([r0, r1] + ([m0, m1] if layer else []))}
    if case["keep"]:
        out["f8"] = _plain_unpack(_plain_pack(s["f"]))
    return out


def _plain_dnorm(s):
    case, stats = s["case"], s["stats"]
    layer = case["kind"] == "layer"
    f = (_plain_unpack(s["f8"]) if case["keep"] else s["f"]).float()
    gate, member = _plain_gate(s)
    r0, r1 = stats[0][:, None], stats[1][:, None]
    fh, xh = (f - stats[2][:, None], s["x"].float() - stats[3][:, None]) if layer else (f, s["x"].float())
    fh, xh = fh * r0, xh * r1

    def back(d, unit, r):
        d = d - unit * (d * unit).mean(1, keepdim=True)
        return r * (d - (d.mean(1, keepdim=True) if layer else 0))

    dh, dtype = s["dh"].float(), s["x"].dtype
    t = s["dx"].float() + back(dh * s["weight"].float(), xh, r1)
    n = fh * s["post_weight"].float() + (s["post_bias"].float() if layer else 0)
    d = gate * t
    param = DTYPES[case["param"]]
    out = {"x": (SCALE * t).to(dtype), "f": back(d * s["post_weight"].float(), fh, r0).to(dtype),
           "weight": (dh * xh).sum(0).to(param), "post_weight": (d * fh).sum(0).to(param),
           "gate": ((t * n).sum(0, keepdim=True) if member is None else member @ (t * n)).to(param)}
    if layer:
        out["bias"], out["post_bias"] = dh.sum(0).to(param), d.sum(0).to(param)
    return out


def _run_plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "pack":
        return _plain_unpack(_plain_pack(s["x"]))
    if op == "wgrad":
        return (s["dy"].float().T @ _plain_unpack(s["x8"]).float()).to(DTYPES[case["to"]])
    return {"gated": _plain_gated, "norm": _plain_norm, "dnorm": _plain_dnorm}[op](s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    op, n, b = case["op"], case["rows"] * case["width"], BYTES[case["dtype"]]
    kept = 1 + 1 / BLOCK
    if op == "pack":  # written once, read once
        return {"bytes": n * (2 * b + 2 * kept), "flops": 4 * n}
    if op == "gated":  # a, u, dy read, y, da, du written, a and u kept and read
        return {"bytes": n * (6 * b + 4 * kept + (2 * kept + b if case["keep_y"] else 0)), "flops": 30 * n}
    if op == "norm":
        return {"bytes": n * (4 * b + (2 * kept + b if case["keep"] else 0)), "flops": 12 * n}
    if op == "dnorm":
        return {"bytes": n * (5 * b + (kept if case["keep"] else b)), "flops": 25 * n}
    return {"bytes": n * kept + case["rows"] * case["out"] * b + case["out"] * case["width"] * BYTES[case["to"]], "flops": 2 * n * case["out"]}


# ---------------------------------------------------------------------------------------------- 64 bits
def _exact_kept(x):
    """What 8 bits keep of x, in 64 bits."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for at in range(0, x.shape[1], BLOCK * 64):
        part = x[:, at:at + BLOCK * 64].double()
        for b, block in enumerate(part.split(BLOCK, 1)):
            top = block.abs().amax(1, keepdim=True)
            e = torch.clamp((top.view(torch.int64) >> 52) - 1029, min=-126)
            step = ((e + 1023) << 52).view(torch.float64)
            out[:, at + b * BLOCK:at + b * BLOCK + block.shape[1]] = torch.clamp(torch.round(block / step), -127, 127) * step
    return out


def _exact_act(act, a):
    if act == "silu":
        p = torch.sigmoid(a)
        return a * p, p * (1 + a * (1 - p))
    if act == "gelu":
        p = torch.special.ndtr(a)
        return a * p, p + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    th = torch.tanh(c * (a + 0.044715 * a ** 3))
    return 0.5 * a * (1 + th), 0.5 * (1 + th) + 0.5 * a * (1 - th * th) * c * (1 + 3 * 0.044715 * a * a)


def _exact_norms(s):
    case = s["case"]
    layer, rows = case["kind"] == "layer", case["rows"]
    spans = list(zip(_starts(case), _starts(case)[1:])) if case["ragged"] else [(0, rows)]
    gate = torch.zeros(rows, case["width"], dtype=torch.float64, device="cuda")
    for (a, b), g in zip(spans, s["gate"].double()):
        gate[a:b] = g
    w, pw = s["weight"].double(), s["post_weight"].double()
    if case["op"] == "norm":
        def norm(v, w, b):
            m = torch.mean(v, 1, keepdim=True) if layer else 0.0 * v[:, :1]
            r = 1 / torch.sqrt(torch.mean((v - m) ** 2, 1, keepdim=True) + EPS)
            return torch.addcmul(b.double() if layer else torch.zeros_like(w), (v - m) * r, w), r[:, 0], m[:, 0]

        n, r0, m0 = norm(s["f"].double(), pw, s.get("post_bias"))
        new = torch.addcmul(SCALE * s["x"].double(), gate, n)
        h, r1, m1 = norm(new, w, s.get("bias"))
        out = {"x": new, "h": h, "stats": torch.stack([r0, r1] + ([m0, m1] if layer else []))}
        if case["keep"]:
            out["f8"] = _exact_kept(s["f"])
        return out
    st = s["stats"].double()
    f = _exact_kept(s["f"]) if case["keep"] else s["f"].double()
    mf, mx = (st[2], st[3]) if layer else (0 * st[0], 0 * st[1])
    f = (f - mf[:, None]) * st[0][:, None]
    x = (s["x"].double() - mx[:, None]) * st[1][:, None]

    def back(d, u, r):  # the Jacobian of (v - mean) / deviation, transposed
        g = d - u * torch.mean(d * u, 1, keepdim=True)
        if layer:
            g = g - torch.mean(g, 1, keepdim=True)
        return g * r[:, None]

    dh = s["dh"].double()
    t = s["dx"].double() + back(dh * w, x, st[1])
    part = torch.addcmul(s["post_bias"].double() if layer else 0 * pw, f, pw) * t
    out = {"x": SCALE * t, "f": back(t * gate * pw, f, st[0]), "weight": torch.einsum("rc,rc->c", dh, x),
           "post_weight": torch.einsum("rc,rc->c", t * gate, f), "gate": torch.stack([part[a:b].sum(0) for a, b in spans])}
    if layer:
        out["bias"], out["post_bias"] = dh.sum(0), (t * gate).sum(0)
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "pack":
        return _exact_kept(s["x"])
    if op == "wgrad":
        return torch.einsum("mn,mk->nk", s["dy"].double(), _exact_kept(s["x"]))
    if op != "gated":
        return _exact_norms(s)
    y = _exact_act(case["act"], s["a"].double())[0].mul_(s["u"].double())
    a, u = _exact_kept(s["a"]), _exact_kept(s["u"])
    f, df = _exact_act(case["act"], a)
    dy = s["dy"].double()
    da, du = df.mul_(u).mul_(dy), dy * f
    out = {"y": y, "d": torch.cat([da, du], 1)} if case["halves"] else {"y": y, "da": da, "du": du}
    if case["keep_y"]:
        out["y8"] = _exact_kept((f * u).to(s["a"].dtype))
    return out
