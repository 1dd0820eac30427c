"""Plain CPU oracle of the operators at the ends of a training step, in 64 bits, written from the formulas in
include/okt.h: AdamW and its 8-bit averages, norms and rotation of heads, cross entropy over a vocabulary.  numpy only, no thought of speed; shares
nothing with the GPU path."""
from __future__ import annotations

import numpy as np

from oracle.okt_operators import philox, values

# ------------------------------------------------------------------ AdamW

BLOCK = 256


def adamw(p, g, m, v, *, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, rate_scale=1.0, grad_scale=1.0):
    """(p, m, v) after a step, of arrays in 64 bits."""
    t, rate = max(int(step), 1), lr * rate_scale
    g = grad_scale * g
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    with np.errstate(divide="ignore", invalid="ignore"):
        change = m / (1.0 - beta1 ** t) / (np.sqrt(v / (1.0 - beta2 ** t)) + eps)
    return p - rate * weight_decay * p - rate * change, m, v


def averages32(g, m, v, beta1, beta2, grad_scale=1.0):
    """The averages as fp32 arithmetic has them, each operation rounded: what 8-bit codes are made of."""
    f = np.float32
    g = g.astype(f) * f(grad_scale)
    with np.errstate(over="ignore", invalid="ignore"):
        return f(beta1) * m + f(1.0 - beta1) * g, f(beta2) * v + f(1.0 - beta2) * g * g


def e4m3_values():
    """The 127 values from 0 to 448: four bits of exponent, three of mantissa, the last code is no number."""
    code = np.arange(127)
    e, f = code // 8, code % 8
    return np.where(e == 0, f * 2.0 ** -9, (1.0 + f / 8.0) * 2.0 ** (e - 7.0))


def element_halves(n, tensor, seed, site=0):
    """The 16-bit values of n elements for m and for v; the middle without a seed."""
    if seed is None:
        return np.full(n, 0x8000), np.full(n, 0x8000)
    four = np.arange(-(-n // 4), dtype=np.uint64)
    r = values(philox(four & np.uint64(0xFFFFFFFF), four >> np.uint64(32), tensor, site, seed)).astype(np.int64)
    return r[:, :4].reshape(-1)[:n], r[:, 4:].reshape(-1)[:n]


def _blocks(x):
    for first in range(0, x.size, BLOCK):
        yield first, x[first:first + BLOCK]


def block_scale(x):
    """The power of two by which a block's largest magnitude lies above 224 and at most at 448, at least 2^-126; NaN
    where that is not finite."""
    top = float(np.max(np.abs(x)))
    if not np.isfinite(top):
        return np.nan
    e = -126
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def to_e4m3(x, halves):
    """Codes (sign in bit 7) and scales of an array of fp32 values."""
    table, codes, scales = e4m3_values(), np.zeros(x.size, np.uint8), []
    for first, block in _blocks(x):
        scale = block_scale(block)
        scales.append(scale)
        if np.isnan(scale):
            continue
        y = np.abs(block.astype(np.float64)) / scale
        at = np.searchsorted(table, y, side="right") - 1
        a, b = table[at], table[np.minimum(at + 1, 126)]
        frac = np.where(at < 126, (y - a) / np.where(at < 126, b - a, 1.0), 0.0)
        up = np.rint(frac * 2.0 ** 20) / 2.0 ** 20 + halves[first:first + BLOCK] / 65536.0 >= 1.0
        codes[first:first + BLOCK] = at + up + 128 * np.signbit(block)
    return codes, np.array(scales, np.float32)


def to_e4m3_root(v, halves):
    """Codes and scales of the roots of an array of fp32 values."""
    table, codes, scales = e4m3_values(), np.zeros(v.size, np.uint8), []
    root = np.sqrt(v.astype(np.float32))
    f = np.float32
    for first, block in _blocks(root):
        scale = block_scale(block)
        scales.append(scale)
        if np.isnan(scale):
            continue
        y = f(block / f(scale)) if scale > 2.0 ** -126 else (block.astype(np.float64) / scale).astype(f)
        at = np.searchsorted(table, y.astype(np.float64), side="right") - 1
        a, b = table[at].astype(f), table[np.minimum(at + 1, 126)].astype(f)
        share = halves[first:first + BLOCK].astype(f) * f(2.0 ** -16)
        up = (y * y - a * a > share * (b * b - a * a)) & (at < 126)      # in fp32: a border is where fp32 has it
        code = at + up
        codes[first:first + BLOCK] = np.where((code == 0) & (block > 0), 1, code)
    return codes, np.array(scales, np.float32)


def from_e4m3(codes, scales):
    table = np.append(e4m3_values(), np.nan)
    with np.errstate(invalid="ignore"):
        return np.where(codes & 128, -1.0, 1.0) * table[codes & 127] * np.repeat(scales.astype(np.float64), BLOCK)[:codes.size]


# ------------------------------------------------------------------ norms and rotation of heads

def _pairs(dim, rot, adjacent):
    j = np.arange(rot // 2)
    return (2 * j, 2 * j + 1) if adjacent else (j, j + rot // 2)


def angles(batch, length, inv_freq, positions=None, axis_of_pair=None):
    """[batch, length, 1, pairs]; positions [batch, length, axes]."""
    pairs = 0 if inv_freq is None else len(inv_freq)
    if positions is None:
        positions = np.broadcast_to(np.arange(length)[None, :, None], (batch, length, 1))
    axis = np.zeros(pairs, int) if axis_of_pair is None else np.asarray(axis_of_pair, int)
    freq = np.zeros(0) if inv_freq is None else np.asarray(inv_freq, np.float64)
    # positions are whole and frequencies have 24 bits: the product is exact in the long double that it is reduced in
    turns = positions[:, :, axis].astype(np.longdouble) * freq.astype(np.longdouble)
    return np.mod(turns, 2 * np.longdouble(np.pi) + np.longdouble(1.2246467991473532e-16) * 2).astype(np.float64)[:, :, None]


def turned(x, angle, adjacent, back=False):
    a, b = _pairs(x.shape[-1], 2 * angle.shape[-1], adjacent)
    c, s = np.cos(angle), np.sin(angle) * (-1.0 if back else 1.0)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def head_statistics(x, kind, eps):
    mean = x.mean(-1, keepdims=True) if kind == "layer" else np.zeros(x.shape[:-1] + (1,))
    return mean, 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)


def norm_rotary(x, angle, *, weight=None, kind="rms", eps=1e-6, adjacent=False):
    if weight is not None:
        mean, r = head_statistics(x, kind, eps)
        x = (x - mean) * r * weight
    return turned(x, angle, adjacent)


def norm_rotary_backward(x, dy, angle, *, weight=None, kind="rms", eps=1e-6, adjacent=False):
    """(dx, dweight), dweight None without a weight."""
    d = turned(dy, angle, adjacent, back=True)
    if weight is None:
        return d, None
    mean, r = head_statistics(x, kind, eps)
    h = (x - mean) * r
    w = d * weight
    dx = w - h * (w * h).mean(-1, keepdims=True)
    if kind == "layer":
        dx = dx - w.mean(-1, keepdims=True)
    return r * dx, (d * h).sum((0, 1, 2))


# ------------------------------------------------------------------ cross entropy over a vocabulary

def logits(h, weight, bias=None):
    s = h @ weight.T
    return s if bias is None else s + bias


def cross_entropy(h, weight, labels, bias=None):
    """(loss, lse) of every row; 0 where the label is not in the vocabulary."""
    rows = np.flatnonzero((labels >= 0) & (labels < weight.shape[0]))
    loss, lse = np.zeros(len(labels)), np.zeros(len(labels))
    s = logits(h[rows], weight, bias)
    top = s.max(1, keepdims=True)
    lse[rows] = np.log(np.exp(s - top).sum(1)) + top[:, 0]
    loss[rows] = lse[rows] - s[np.arange(len(rows)), labels[rows]]
    return loss, lse


def cross_entropy_backward(h, weight, labels, g, bias=None):
    """(dh, dweight, dbias)."""
    rows = np.flatnonzero((labels >= 0) & (labels < weight.shape[0]))
    s = logits(h[rows], weight, bias)
    p = np.exp(s - s.max(1, keepdims=True))
    d = p / p.sum(1, keepdims=True)
    d[np.arange(len(rows)), labels[rows]] -= 1.0
    d *= g[rows, None]
    dh = np.zeros(h.shape)
    dh[rows] = d @ weight
    return dh, d.T @ h[rows], d.sum(0)
