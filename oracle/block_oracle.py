"""Plain 64-bit definitions of the operators of a trained block (numpy only): activations kept in 8 bits, the gated activation
and the norms around a block with their gradients, and the weight gradient of a linear layer.

Shares no code with the library.
"""
import math

import numpy as np

BLOCK = 32


def packed(x):
    """(codes [rows, 32 * blocks], bytes [rows, blocks]) of a matrix: blocks of 32 entries of a row share a power of two."""
    x = np.asarray(x, np.float64)
    rows, width = x.shape
    blocks = -(-width // BLOCK)
    v = np.zeros((rows, blocks * BLOCK))
    v[:, :width] = x
    v = v.reshape(rows, blocks, BLOCK)
    codes, byte = np.zeros((rows, blocks, BLOCK), np.int8), np.zeros((rows, blocks), np.uint8)
    for r in range(rows):
        for b in range(blocks):
            if not np.all(np.isfinite(v[r, b])):
                byte[r, b] = 255
                continue
            top = np.abs(v[r, b]).max()
            if top == 0:
                continue
            e = max(math.frexp(top)[1] - 1 - 6, -126)
            byte[r, b] = e + 127
            codes[r, b] = np.clip(np.rint(np.ldexp(v[r, b], -e)), -127, 127)      # rint: halves to even
    return codes.reshape(rows, -1), byte


def unpacked(codes, byte, width):
    e = byte.astype(np.int64) - 127
    v = np.ldexp(codes.astype(np.float64).reshape(len(codes), -1, BLOCK), e[:, :, None].astype(np.int32))
    v[byte == 255] = np.nan
    return v.reshape(len(codes), -1)[:, :width]


def kept(x):
    """What a matrix reads back as."""
    x = np.asarray(x)
    return unpacked(*packed(x), x.shape[1])


def gate_of(act, a):
    """p in act(a) = a p, and act'(a)."""
    a = np.asarray(a, np.float64)
    if act == "gelu":
        p = np.vectorize(lambda v: 0.5 * math.erfc(-v / math.sqrt(2)))(a) if a.size else a
        return p, p + a * np.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    k = 2 * math.sqrt(2 / math.pi)
    z, dz = (a, 1.0) if act == "silu" else (k * (a + 0.044715 * a ** 3), k * (1 + 3 * 0.044715 * a * a))
    with np.errstate(over="ignore"):
        p, q = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))
    slope = np.where(p * q == 0, 0.0, a * p * q * dz)
    return p, p + slope


def gated(act, a, u=None):
    y = a * gate_of(act, a)[0]
    return y if u is None else y * u


def gated_gradient(act, a, u, dy):
    """(da, du) at the inputs a, u."""
    p, slope = gate_of(act, a)
    return (dy * slope, None) if u is None else (dy * u * slope, dy * a * p)


def row_gate(gate, rows, starts=None):
    """(gate of each row [rows, width], group of each row; -1: none, gate 0)."""
    gate = np.asarray(gate, np.float64)
    group = np.full(rows, -1)
    if starts is None:
        group[:] = np.arange(rows) // max(rows // len(gate), 1)
    else:
        for g in range(len(gate)):
            group[starts[g]:starts[g + 1]] = g
    return np.where(group[:, None] >= 0, gate[np.maximum(group, 0)], 0.0), group


def norm(v, weight, bias, layer, eps):
    """(normalised, 1 / deviation, mean)."""
    mean = v.mean(1) if layer else np.zeros(len(v))
    c = v - mean[:, None]
    r = 1 / np.sqrt((c * c).mean(1) + eps)
    n = c * r[:, None] * weight
    return n + bias, r, mean


def residual_norm(x, f, weight, bias, post_weight, post_bias, gate, starts, scale, layer, post, eps):
    """(x', h, stats).  gate None: 1."""
    rows, width = x.shape
    new, r0, m0 = scale * x, np.ones(rows), np.zeros(rows)
    if f is not None:
        n = f
        if post:
            n, r0, m0 = norm(f, post_weight, post_bias, layer, eps)
        if gate is None:
            new = new + n
        else:
            g, group = row_gate(gate, rows, starts)
            new = np.where(group[:, None] >= 0, new + g * n, new)
    h, r1, m1 = norm(new, weight, bias, layer, eps)
    return new, h, np.stack([r0, r1] + ([m0, m1] if layer else []))


def _back(d, unit, r, layer):
    out = d - unit * (d * unit).mean(1, keepdims=True)
    if layer:
        out = out - d.mean(1, keepdims=True)
    return out * r[:, None]


def residual_norm_gradient(dh, dx, x, f, stats, weight, post_weight, post_bias, gate, starts, scale, layer, post):
    """Gradients by name, from x', f and the forward call's statistics as they are given."""
    rows, width = x.shape
    r0, r1 = stats[0], stats[1]
    m0, m1 = (stats[2], stats[3]) if layer else (np.zeros(rows), np.zeros(rows))
    xh = (x - m1[:, None]) * r1[:, None]
    t = _back(dh * weight, xh, r1, layer) + (0 if dx is None else dx)
    out = {"x": scale * t, "weight": (dh * xh).sum(0), "bias": dh.sum(0)}
    if f is None:
        return out
    g, group = row_gate(np.ones((1, width)) if gate is None else gate, rows, starts)
    live = (group >= 0)[:, None]
    f = np.where(live, f, 0.0)
    fh = (f - m0[:, None]) * r0[:, None] if post else f
    n = fh * post_weight + post_bias if post else fh
    d = g * t
    out["f"] = np.where(live, _back(d * post_weight, fh, r0, layer) if post else d, 0.0)
    out["post_weight"], out["post_bias"] = np.where(live, d * fh, 0.0).sum(0), d.sum(0)
    if gate is not None:
        part = np.where(live, t * n, 0.0)
        out["gate"] = np.stack([part[group == k].sum(0) for k in range(len(gate))])
    return out


def weight_grad(dy, x):
    return dy.T @ x
