"""Helpers of the GPU tests of the layer's operators: inputs, calls, and how far an output may be
from the 64-bit oracle.

The bounds are sums of what each rounding can do, worked out before any run:
  u    rounding to the tensors' type, relative: 2^-8 bf16, 2^-11 fp16 (and half of its
       smallest step, 2^-25), 2^-24 fp32
  E    2^-24, one fp32 operation
  K E  a sum of fp32 terms, relative to the sum of their magnitudes: no term passes through more than
       K additions (8 in a lane, 6 across a wave, 8 across waves, twice that with two groups: below 64)
"""
from __future__ import annotations

import numpy as np
import torch

from oracle import okt_operators as ops

DEV = "cuda:0"
E = 2.0 ** -24
K = 64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def step(kind):
    """Half of the smallest step of a type."""
    return {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}[kind]


def wide(t):
    return None if t is None else t.detach().double().cpu().numpy()


def rand(shape, kind, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(TYPES[kind]).to(DEV)


def seed_tensor(seed):
    return torch.tensor([seed], dtype=torch.int64, device=DEV)


def within(got, want, bound, what):
    got, bound = wide(got), np.broadcast_to(bound, want.shape)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), what + ": not finite elsewhere"
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), what
    over = np.full(want.shape, -1.0)
    over[fine] = np.abs(got[fine] - want[fine]) - bound[fine]
    assert over.size == 0 or over.max() <= 0, f"{what}: {over.max():.3g} over the bound, at {np.unravel_index(np.argmax(over), over.shape)}"


# ------------------------------------------------------------------ residual norm

def statistics_error(v, mean, r, kind):
    """What mean and (relative) reciprocal deviation of rows v may be off by."""
    dm = K * E * np.abs(v).mean(1, keepdims=True) if kind == "layer" else np.zeros_like(mean)
    off = np.abs(v - mean)
    variance = (K + 4) * E * (off ** 2).mean(1, keepdims=True) + 2 * dm * off.mean(1, keepdims=True) + dm ** 2
    return dm, 0.5 * variance * r * r + 4 * E


def norm_error(v, mean, r, weight, bias, kind):
    dm, dr = statistics_error(v, mean, r, kind)
    off, out = np.abs(v - mean), np.abs((v - mean) * r * weight)
    b = 0.0 if bias is None else np.abs(bias)
    return np.abs(weight) * r * (dm + 3 * E * off) + out * (dr + 4 * E) + 2 * E * b


def norm_backward_error(d, derr, v, mean, r, weight):
    """Errors of a norm's input gradient (before it is rounded) and of its weight's and bias's, when
    the gradient d of its output is off by derr."""
    xhat = np.abs((v - mean) * r)
    w, werr = np.abs(d * weight), derr * np.abs(weight)
    plain, along = w.mean(1, keepdims=True), (w * xhat).mean(1, keepdims=True)
    own = K * E * plain + xhat * K * E * along + 8 * E * (w + plain + xhat * along)
    carried = werr + werr.mean(1, keepdims=True) + xhat * (werr * xhat).mean(1, keepdims=True)
    # rows of a workgroup, four waves, and up to 16 + 32 partial sums: below 128 additions for 5,000 rows
    dw = 130 * E * (np.abs(d) * xhat).sum(0) + (derr * xhat).sum(0)
    return r * (own + carried), dw, 130 * E * np.abs(d).sum(0) + derr.sum(0)


# ------------------------------------------------------------------ attention

def pair_errors(q, k, scale, seen, factor):
    """Probabilities of a plane and what their relative error can be: scores are sums of
    head_dim products, taken from log-sum-exps that are off by as much."""
    D = q.shape[1]
    _, p, lse = ops._plane(q, k, scale, seen)
    size = scale * (np.abs(q) @ np.abs(k).T)
    one = (D + 8) * E * size
    many = (np.where(seen, one, 0.0)).max(1, initial=0.0, keepdims=True)
    return p, lse, 2 * (one + many) + 2.0 ** -19


def attention_bounds(q, k, v, o_kind, *, causal, scale, q_lens, k_lens, dropout_p, seed, site, do=None, o=None):
    """Bounds of o and lse, or with do and o (as stored) of dq, dk and dv."""
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1:3]
    u, least = UNIT[o_kind], step(o_kind)
    bo, blse = np.zeros(q.shape), np.zeros((B, H, Sq))
    bq, bk, bv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b, (ql, kl) in enumerate(zip(ops._lengths(q_lens, B, Sq), ops._lengths(k_lens, B, Sk))):
        for h in range(H):
            g = h // (H // G)
            qq, kk, vv = q[b, :ql, h], k[b, :kl, g], v[b, :kl, g]
            seen = ops.visible(ql, kl, causal)
            f = 1.0
            if dropout_p > 0:
                f = ops.kept_pairs(b * H + h, ql, kl, dropout_p, seed, site) * ops.scale_of(dropout_p)
            p, lse, rel = pair_errors(qq, kk, scale, seen, f)
            if do is None:
                # each probability rounded once (kept to 2^8 of the row's largest before), then fp32 sums over keys
                bo[b, :ql, h] = (f * p * (rel + u + (kl + 8) * E) + f * least) @ np.abs(vv) + rel.max(1, initial=0.0, keepdims=True) * np.abs(f * p @ np.abs(vv))
                blse[b, h, :ql] = rel.max(1, initial=0.0) + (kl + 8) * E + 4 * E * np.abs(np.where(np.isfinite(lse), lse, 0.0))
                continue
            dd = np.where(seen.any(1, keepdims=True), do[b, :ql, h], 0.0)
            dp = f * (dd @ vv.T)
            d = (p * dp).sum(1, keepdims=True)
            e_dp = f * (D + 8) * E * (np.abs(dd) @ np.abs(vv).T)
            # D = do . o, o being off by its rounding and by its own bound; few keys are exact to the same order
            e_d = (np.abs(dd) * o[b, :ql, h]).sum(1, keepdims=True) + (D + 8) * E * (np.abs(dd) * np.abs(p @ np.abs(vv))).sum(1, keepdims=True) + (
                p * (e_dp + 40 * E * np.abs(dp))).sum(1, keepdims=True)
            ds = p * np.abs(dp - d)
            e_ds = ds * (rel + u + 4 * E) + p * (e_dp + e_d + 4 * E * (np.abs(dp) + np.abs(d))) + least * max(ops.scale_of(dropout_p), 1.0)
            bq[b, :ql, h] = scale * ((e_ds + (kl + 8) * E * ds) @ np.abs(kk))
            bk[b, :kl, g] += scale * ((e_ds + (H // G * ql + 40) * E * ds).T @ np.abs(qq))
            bv[b, :kl, g] += (f * p * (rel + u + (H // G * ql + 40) * E) + f * least).T @ np.abs(dd)
    return (bo, blse) if do is None else (bq, bk, bv)
