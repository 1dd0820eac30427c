"""Plain CPU oracle of the operators of a layer's training step: the random field, dropout,
the residual norm and attention, forward and backward, in 64 bits, written from the formulas
in include/okt.h.  numpy only, no thought of speed; shares nothing with the GPU path."""
from __future__ import annotations

import math

import numpy as np

MASK32 = 0xFFFFFFFF


def philox(c0, c1, c2, c3, seed: int, rounds: int = 7) -> np.ndarray:
    """Philox4x32 output words, [..., 4] uint32, of arrays of counters."""
    word = np.uint64(MASK32)
    x = [np.array(c, dtype=np.uint64) for c in np.broadcast_arrays(c0, c1, c2, c3)]
    k0, k1 = seed & MASK32, (seed >> 32) & MASK32
    for _ in range(rounds):
        p0, p1 = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(p1 >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), p1 & word,
             (p0 >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), p0 & word]
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    return np.stack(x, axis=-1).astype(np.uint32)


def values(words: np.ndarray) -> np.ndarray:
    """The eight 16-bit values of each block: value 2w + h is half h of word w."""
    return np.stack([words & np.uint32(0xFFFF), words >> np.uint32(16)], axis=-1).reshape(*words.shape[:-1], 8)


def bar_of(p: float) -> int:
    return int(math.floor((1.0 - p) * 65536.0 + 0.5))


def scale_of(p: float) -> float:
    return 65536.0 / bar_of(p) if bar_of(p) else 0.0


def kept_flat(n: int, p: float, seed: int, site: int = 0, first: int = 0) -> np.ndarray:
    """Elements first .. first + n - 1 of a flat vector; `first` a multiple of 8."""
    group = np.arange(-(-n // 8), dtype=np.uint64) + np.uint64(first // 8)
    v = values(philox(group & np.uint64(MASK32), group >> np.uint64(32), 0, site, seed))
    return v.reshape(-1)[:n] < bar_of(p)


def kept_rows(rows: int, width: int, p: float, seed: int, site: int = 0) -> np.ndarray:
    v = values(philox(np.arange(-(-width // 8))[None, :], np.arange(rows)[:, None], 0, site, seed))
    return v.reshape(rows, -1)[:, :width] < bar_of(p)


def kept_pairs(plane: int, q_len: int, k_len: int, p: float, seed: int, site: int = 0) -> np.ndarray:
    """[q_len, k_len] of one plane b * heads + h: a block is two queries by four keys."""
    nq, nk = -(-q_len // 2), -(-k_len // 4)
    v = values(philox(np.arange(nk)[None, :], np.arange(nq)[:, None], plane, site, seed))
    v = v.reshape(nq, nk, 4, 2).transpose(0, 3, 1, 2).reshape(2 * nq, 4 * nk)
    return v[:q_len, :k_len] < bar_of(p)


def dropout(x, p: float, seed: int, site: int = 0) -> np.ndarray:
    return np.where(kept_flat(x.size, p, seed, site), np.asarray(x, np.float64) * scale_of(p), 0.0)


# ------------------------------------------------------------------ residual norm

def statistics(v, kind: str, eps: float):
    mean = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((v.shape[0], 1))
    return mean, 1.0 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)


def _norm(v, stats, weight, bias):
    out = (v - stats[0]) * stats[1] * weight
    return out if bias is None else out + bias


def norm_factor(rows: int, width: int, p: float, seed: int, site: int = 0):
    return kept_rows(rows, width, p, seed, site) * scale_of(p) if p > 0 else 1.0


def dropped(v, factor):
    """v times its factor, 0 where that is 0 whatever v holds."""
    return np.where(np.equal(factor, 0), 0.0, factor * v)


def residual_norm(u, x, *, kind="layer", eps=1e-5, residual_scale=1.0, post_weight=None, post_bias=None,
                  gate=None, rows_per_gate=0, pre_weight=None, pre_bias=None, factor=1.0, store=lambda h: h):
    """(h, y or None, stats [rows, 4]); `factor` is what dropout multiplies by, `store` rounds h as
    it is stored."""
    rows, width = u.shape
    stats = np.zeros((rows, 4))
    a = u
    if post_weight is not None:
        m, r = statistics(u, kind, eps)
        stats[:, 0:1], stats[:, 1:2] = m, r
        a = _norm(u, (m, r), post_weight, post_bias)
    a = dropped(a, factor)
    if gate is not None:
        a = a * gate[np.arange(rows) // (rows_per_gate or max(rows, 1))]
    h = residual_scale * x + a
    y = None
    if pre_weight is not None:
        held = store(h)
        m, r = statistics(held, kind, eps)
        stats[:, 2:3], stats[:, 3:4] = m, r
        y = _norm(held, (m, r), pre_weight, pre_bias)
    return h, y, stats


def _norm_backward(d, v, m, r, weight, kind):
    xhat = (v - m) * r
    w = d * weight
    dv = w - xhat * (w * xhat).mean(1, keepdims=True)
    if kind == "layer":
        dv = dv - w.mean(1, keepdims=True)
    return dv * r, (d * xhat).sum(0), d.sum(0)


def residual_norm_backward(u, h, stats, dh, dy, *, kind="layer", residual_scale=1.0, post_weight=None,
                           post_bias=None, gate=None, rows_per_gate=0, pre_weight=None, factor=1.0):
    """Gradients by name: dx, du and those of the parameters there are."""
    rows = stats.shape[0]
    out = {}
    total = np.zeros_like(u) if dh is None else dh
    if pre_weight is not None:
        d, out["dpre_weight"], out["dpre_bias"] = _norm_backward(dy, h, stats[:, 2:3], stats[:, 3:4], pre_weight, kind)
        total = total + d
    out["dx"] = residual_scale * total
    da = dropped(total, factor)
    if gate is not None:
        group = np.arange(rows) // (rows_per_gate or max(rows, 1))
        a = u if post_weight is None else _norm(u, (stats[:, 0:1], stats[:, 1:2]), post_weight, post_bias)
        out["dgate"] = np.zeros_like(gate)
        np.add.at(out["dgate"], group, total * dropped(a, factor))
        da = da * gate[group]
    if post_weight is not None:
        da, out["dpost_weight"], out["dpost_bias"] = _norm_backward(da, u, stats[:, 0:1], stats[:, 1:2], post_weight, kind)
    out["du"] = da
    return out


# ------------------------------------------------------------------ attention

def visible(ql: int, kl: int, causal: bool) -> np.ndarray:
    i, j = np.arange(ql)[:, None], np.arange(kl)[None, :]
    return (j <= i + kl - ql) if causal else np.ones((ql, kl), bool)


def _plane(q, k, scale, seen):
    """(scores, probabilities, log-sum-exp) of one plane."""
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    top = s.max(1, initial=-np.inf, keepdims=True)
    e = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    total = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = np.log(total) + np.where(np.isfinite(top), top, 0.0)
    return s, np.divide(e, total, out=np.zeros_like(e), where=total > 0), lse[:, 0]


def _lengths(lens, batch, most):
    return [most] * batch if lens is None else [min(max(int(n), 0), most) for n in lens]


def attention(q, k, v, *, causal=False, scale=None, q_lens=None, k_lens=None, dropout_p=0.0, seed=0, site=0):
    """(o, lse) of [batch, length, heads, dim] arrays; lse is [batch, heads, q_len]."""
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1:3]
    scale = D ** -0.5 if scale is None else scale
    o, lse = np.zeros(q.shape), np.full((B, H, Sq), -np.inf)
    for b, (ql, kl) in enumerate(zip(_lengths(q_lens, B, Sq), _lengths(k_lens, B, Sk))):
        for h in range(H):
            g = h // (H // G)
            _, p, lse[b, h, :ql] = _plane(q[b, :ql, h], k[b, :kl, g], scale, visible(ql, kl, causal))
            if dropout_p > 0:
                p = p * kept_pairs(b * H + h, ql, kl, dropout_p, seed, site) * scale_of(dropout_p)
            o[b, :ql, h] = p @ v[b, :kl, g]
    return o, lse


def attention_backward(q, k, v, do, *, causal=False, scale=None, q_lens=None, k_lens=None, dropout_p=0.0,
                       seed=0, site=0):
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1:3]
    scale = D ** -0.5 if scale is None else scale
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b, (ql, kl) in enumerate(zip(_lengths(q_lens, B, Sq), _lengths(k_lens, B, Sk))):
        for h in range(H):
            g = h // (H // G)
            qq, kk, vv, dd = q[b, :ql, h], k[b, :kl, g], v[b, :kl, g], do[b, :ql, h]
            seen = visible(ql, kl, causal)
            dd = np.where(seen.any(1, keepdims=True), dd, 0.0)          # a row that sees nothing is constant
            _, p, _ = _plane(qq, kk, scale, seen)
            f = 1.0
            if dropout_p > 0:
                f = kept_pairs(b * H + h, ql, kl, dropout_p, seed, site) * scale_of(dropout_p)
            dp = f * (dd @ vv.T)
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            dq[b, :ql, h] = scale * (ds @ kk)
            dk[b, :kl, g] += scale * (ds.T @ qq)
            dv[b, :kl, g] += (f * p).T @ dd
    return dq, dk, dv
