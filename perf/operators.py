"""What the speed of this library's operators for a layer's training step is measured on.

Three operators, which meet between the matrix products of a transformer layer and draw
from one counter-based random field:

  dropout    y = x / keep where kept, else 0; its backward is the same call on the gradient
  norm       h = alpha x + gate * dropout(norm(u)), y = norm(h), each norm optional, and
             the gradient of that
  attention  softmax(scale q k') with dropout, times v, over padded batches and causal
             masks, with grouped heads; and its gradient, which recomputes the
             probabilities from q, k and the log-sum-exp

A case is one pass of one direction.  The plain form (own = False) is the operators'
formulas in elementary torch operations in 32 bits; own = True makes the calls of this
library's Python binding.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
MASK32 = 0xFFFFFFFF


def listed():
    return [
        # one token's hidden vector: what a call costs beside its work
        {"name": "dropout_token", "op": "dropout", "n": 768, "type": "bf16", "p": 0.1},
        # the inner activations of a layer: 32 sequences of 512 tokens, 4096 wide
        {"name": "dropout_inner", "op": "dropout", "n": 67_108_864, "type": "bf16", "p": 0.1},
        # a short sequence of a small layer in full precision, norm after the sum
        {"name": "norm_short", "op": "norm", "grad": False, "rows": 128, "width": 768, "type": "f32",
         "kind": "layer", "post": False, "pre": True, "gates": 0, "alpha": 1.0, "p": 0.1},
        # a batch of 32 sequences of 512 tokens of a large layer, norm after the sum
        {"name": "norm_batch", "op": "norm", "grad": False, "rows": 16_384, "width": 1024,
         "type": "bf16", "kind": "layer", "post": False, "pre": True, "gates": 0, "alpha": 1.0,
         "p": 0.1},
        # its gradient
        {"name": "norm_batch_grad", "op": "norm", "grad": True, "rows": 16_384, "width": 1024,
         "type": "bf16", "kind": "layer", "post": False, "pre": True, "gates": 0, "alpha": 1.0,
         "p": 0.1},
        # norms on both sides of a gated block, a width whose rows are not aligned, odd rows
        {"name": "norm_gated_grad", "op": "norm", "grad": True, "rows": 4099, "width": 2500,
         "type": "f16", "kind": "rms", "post": True, "pre": True, "gates": 1, "alpha": 0.81,
         "p": 0.0},
        # a short sequence of a small layer: latency
        {"name": "attention_short", "op": "attention", "grad": False, "batch": 1, "heads": 12,
         "kv_heads": 12, "q_len": 128, "k_len": 128, "dim": 64, "type": "bf16", "causal": False,
         "padded": False, "p": 0.0},
        # a padded batch of 32 sequences of up to 512 tokens, sixteen heads, dropout
        {"name": "attention_padded", "op": "attention", "grad": False, "batch": 32, "heads": 16,
         "kv_heads": 16, "q_len": 512, "k_len": 512, "dim": 64, "type": "bf16", "causal": False,
         "padded": True, "p": 0.1},
        # its gradient
        {"name": "attention_padded_grad", "op": "attention", "grad": True, "batch": 32, "heads": 16,
         "kv_heads": 16, "q_len": 512, "k_len": 512, "dim": 64, "type": "bf16", "causal": False,
         "padded": True, "p": 0.1},
        # odd lengths on both axes, two key heads for six query heads, a narrow head
        {"name": "attention_odd_grad", "op": "attention", "grad": True, "batch": 3, "heads": 6,
         "kv_heads": 2, "q_len": 197, "k_len": 333, "dim": 40, "type": "f16", "causal": True,
         "padded": False, "p": 0.0},
        # long causal sequences, four query heads to a key head
        {"name": "attention_long", "op": "attention", "grad": False, "batch": 2, "heads": 16,
         "kv_heads": 4, "q_len": 4096, "k_len": 4096, "dim": 128, "type": "bf16", "causal": True,
         "padded": False, "p": 0.0},
        # their gradient
        {"name": "attention_long_grad", "op": "attention", "grad": True, "batch": 2, "heads": 16,
         "kv_heads": 4, "q_len": 4096, "k_len": 4096, "dim": 128, "type": "bf16", "causal": True,
         "padded": False, "p": 0.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: lengths from one to the listed ones' largest, any of the types, masks
    and norms."""
    op = rng.choice(["dropout", "norm", "norm", "attention", "attention", "attention"])
    if op == "dropout":
        return {"op": op, "n": _log_int(rng, 1, 67_108_864), "type": rng.choice(list(TYPES)),
                "p": rng.choice([0.05, 0.1, 0.25, 0.5])}
    if op == "norm":
        width = _log_int(rng, 32, 8192)
        if rng.random() < 0.6:
            width = -(-width // 64) * 64
        rows = _log_int(rng, 1, max(1, min(16_384, 16_777_216 // width)))
        post = rng.random() < 0.5
        return {"op": op, "grad": rng.random() < 0.5, "rows": rows, "width": width,
                "type": rng.choice(list(TYPES)), "kind": rng.choice(["layer", "rms"]), "post": post,
                "pre": not post or rng.random() < 0.7, "gates": rng.choice([0, 1, 1 + rng.randrange(min(rows, 8))]),
                "alpha": rng.choice([1.0, 1.0, 0.81]), "p": rng.choice([0.0, 0.1, 0.3])}
    q_len = _log_int(rng, 1, 4096)
    k_len = q_len if rng.random() < 0.7 else _log_int(rng, 1, 4096)
    group = rng.choice([1, 1, 2, 4])
    dim = rng.choice([64, 64, 128, 128, 8 * rng.randint(2, 16)])
    cost = 32 * 4096 * 4096 // 2                  # visible pairs of the largest listed case
    most = max(1, min(64, cost // (q_len * k_len * group)))
    kv_heads = rng.randint(1, min(16, most))
    batch = rng.randint(1, max(1, min(32, most // kv_heads)))
    return {"op": op, "grad": rng.random() < 0.6, "batch": batch, "heads": kv_heads * group,
            "kv_heads": kv_heads, "q_len": q_len, "k_len": k_len, "dim": dim,
            "type": rng.choice(["bf16", "bf16", "f16"]), "causal": rng.random() < 0.5,
            "padded": rng.random() < 0.4, "p": rng.choice([0.0, 0.0, 0.1])}


def _lengths(case, most):
    """The lengths of a padded batch: every sequence another one, the longest whole."""
    if not case["padded"]:
        return [most] * case["batch"]
    return [max(1, most - (b * 5 % case["batch"]) * (3 * most // 4) // case["batch"])
            for b in range(case["batch"])]


def _gate_rows(case):
    """Rows that share a gate (the last group may be shorter)."""
    return -(-case["rows"] // case["gates"]) if case["gates"] else 0


def _gate_count(case):
    return -(-case["rows"] // _gate_rows(case)) if case["gates"] else 0


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device=DEV) * scale).to(dtype)

    s = {"case": case, "seed": torch.randint(-(1 << 62), 1 << 62, (1,), generator=gen, device=DEV)}
    t = TYPES[case["type"]]
    if case["op"] == "dropout":
        s["x"] = normal(case["n"], dtype=t)
        s["y"] = torch.empty_like(s["x"])
    elif case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        s["u"] = normal(rows, width, scale=0.8, dtype=t)
        s["x"] = normal(rows, width, dtype=t)
        for name in ("post", "pre"):
            s[name + "_weight"] = 1.0 + normal(width, scale=0.1) if case[name] else None
            s[name + "_bias"] = normal(width, scale=0.1) if case[name] and case["kind"] == "layer" else None
        s["gate"] = 0.5 + normal(_gate_count(case), width, scale=0.2) if case["gates"] else None
        s["h"] = torch.empty_like(s["u"])
        s["y"] = torch.empty_like(s["u"]) if case["pre"] else None
        s["stats"] = torch.empty(rows, 4, device=DEV)
        if case["grad"]:
            plain = _norm_forward(s)
            s["h"], s["stats"] = plain["h"], plain["stats"]
            s["dh"] = normal(rows, width, scale=0.1, dtype=t)
            s["dy"] = normal(rows, width, scale=0.1, dtype=t) if case["pre"] else None
            s["dx"], s["du"] = torch.empty_like(s["u"]), torch.empty_like(s["u"])
            for name in ("post_weight", "post_bias", "pre_weight", "pre_bias", "gate"):
                s["d" + name] = torch.empty_like(s[name]) if s[name] is not None else None
    else:
        B, H, G, D = case["batch"], case["heads"], case["kv_heads"], case["dim"]
        Sq, Sk = case["q_len"], case["k_len"]
        if Sq == Sk:                              # one projection gives all three
            qkv = normal(B, Sq, H + 2 * G, D, dtype=t)
            s["q"], s["k"], s["v"] = qkv.split([H, G, G], 2)
        else:                                     # queries and keys of two sequences
            s["q"] = normal(B, Sq, H, D, dtype=t)
            s["k"], s["v"] = normal(B, Sk, 2 * G, D, dtype=t).split([G, G], 2)
        s["q_lens"] = s["k_lens"] = None
        if case["padded"]:
            s["q_lens"] = torch.tensor(_lengths(case, Sq), dtype=torch.int32).to(DEV)
            s["k_lens"] = torch.tensor(_lengths(case, Sk), dtype=torch.int32).to(DEV)
        s["o"] = torch.empty(B, Sq, H, D, dtype=t, device=DEV)
        s["lse"] = torch.empty(B, H, Sq, device=DEV)
        if case["grad"]:
            plain = _attention_forward(s)
            s["o"], s["lse"] = plain["o"], plain["lse"]
            s["do"] = normal(B, Sq, H, D, dtype=t)
            s["dq"] = torch.empty(B, Sq, H, D, dtype=t, device=DEV)
            s["dk"] = torch.empty(B, Sk, G, D, dtype=t, device=DEV)
            s["dv"] = torch.empty(B, Sk, G, D, dtype=t, device=DEV)
    return s


# ------------------------------------------------------------------ the plain form

def _random_words(c0, c1, c2, seed, site=0):
    """Philox4x32 with seven rounds: four 32-bit words (in int64) for each counter."""
    c0, c1, c2 = torch.broadcast_tensors(c0, c1, c2)
    c3 = torch.full_like(c0, site)
    k0, k1 = seed & MASK32, (seed >> 32) & MASK32
    for _ in range(7):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57    # products of 32 bits fill 64: no bit is lost
        c0, c1, c2, c3 = (((b >> 32) & MASK32) ^ c1 ^ k0, b & MASK32,
                          ((a >> 32) & MASK32) ^ c3 ^ k1, a & MASK32)
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    return torch.stack([c0, c1, c2, c3], -1)


def _halves(words):
    """The eight 16-bit values of each block, along the last axis."""
    return torch.stack([words & 0xFFFF, words >> 16], -1).flatten(-2)


def _bar(p):
    """Values below it are kept."""
    return int(math.floor((1.0 - p) * 65536.0 + 0.5))


def _index(n):
    return torch.arange(n, device=DEV)


def _keep_flat(n, p, seed):
    block = _index(-(-n // 8))
    return _halves(_random_words(block & MASK32, block >> 32, torch.zeros_like(block), seed)).flatten()[:n] < _bar(p)


def _keep_rows(rows, width, p, seed):
    words = _random_words(_index(-(-width // 8))[None, :], _index(rows)[:, None],
                          torch.zeros(1, 1, dtype=torch.int64, device=DEV), seed)
    return _halves(words).flatten(-2)[:, :width] < _bar(p)


def _keep_attention(planes, q_len, k_len, p, seed):
    """A block is two queries by four keys: word = key, half = query."""
    nq, nk = -(-q_len // 2), -(-k_len // 4)
    words = _random_words(_index(nk)[None, None, :], _index(nq)[None, :, None], _index(planes)[:, None, None], seed)
    kept = torch.stack([words & 0xFFFF, words >> 16], 2)          # planes, nq, 2, nk, 4
    return kept.reshape(planes, 2 * nq, 4 * nk)[:, :q_len, :k_len] < _bar(p)


def _dropped(x, keep, p):
    return torch.where(keep, x * (65536.0 / _bar(p)), torch.zeros_like(x))


def _statistics(a, kind):
    mean = a.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(a[:, :1])
    return mean, torch.rsqrt(((a - mean) * (a - mean)).mean(-1, keepdim=True) + EPS)


def _norm_forward(s):
    case = s["case"]
    rows, width, t = case["rows"], case["width"], TYPES[case["type"]]
    a = s["u"].float()
    none = torch.zeros(rows, 1, device=DEV)
    post = pre = (none, none)
    if case["post"]:
        post = _statistics(a, case["kind"])
        a = (a - post[0]) * post[1] * s["post_weight"]
        if s["post_bias"] is not None:
            a = a + s["post_bias"]
    if case["p"] > 0:
        a = _dropped(a, _keep_rows(rows, width, case["p"], s["seed"]), case["p"])
    if case["gates"]:
        a = a * s["gate"][_index(rows) // _gate_rows(case)]
    h = case["alpha"] * s["x"].float() + a
    out = {"h": h.to(t)}
    if case["pre"]:
        # the norm reads what was stored, as the backward pass does
        h = out["h"].float()
        pre = _statistics(h, case["kind"])
        y = (h - pre[0]) * pre[1] * s["pre_weight"]
        out["y"] = (y + s["pre_bias"] if s["pre_bias"] is not None else y).to(t)
    out["stats"] = torch.cat([*post, *pre], 1)
    return out


def _norm_input_gradient(dout, x, weight, mean, rstd, kind):
    xhat = (x - mean) * rstd
    w = dout * weight
    d = w - xhat * (w * xhat).mean(-1, keepdim=True)
    if kind == "layer":
        d = d - w.mean(-1, keepdim=True)
    return d * rstd, (dout * xhat).sum(0), dout.sum(0)


def _norm_backward(s):
    case = s["case"]
    rows, width, t = case["rows"], case["width"], TYPES[case["type"]]
    m0, r0, m1, r1 = s["stats"].split(1, 1)
    out = {}
    dh = s["dh"].float()
    if case["pre"]:
        d, dw, db = _norm_input_gradient(s["dy"].float(), s["h"].float(), s["pre_weight"], m1, r1, case["kind"])
        dh = dh + d
        out["dpre_weight"] = dw
        if s["pre_bias"] is not None:
            out["dpre_bias"] = db
    out["dx"] = (case["alpha"] * dh).to(t)
    keep = _keep_rows(rows, width, case["p"], s["seed"]) if case["p"] > 0 else None
    da = dh
    if case["gates"]:
        a = s["u"].float()
        if case["post"]:
            a = (a - m0) * r0 * s["post_weight"]
            if s["post_bias"] is not None:
                a = a + s["post_bias"]
        if keep is not None:
            a = _dropped(a, keep, case["p"])
        share, count = _gate_rows(case), _gate_count(case)
        each = torch.zeros(count * share, width, device=DEV)
        each[:rows] = dh * a
        out["dgate"] = each.view(count, share, width).sum(1)
        da = dh * s["gate"][_index(rows) // share]
    if keep is not None:
        da = _dropped(da, keep, case["p"])
    if case["post"]:
        da, dw, db = _norm_input_gradient(da, s["u"].float(), s["post_weight"], m0, r0, case["kind"])
        out["dpost_weight"] = dw
        if s["post_bias"] is not None:
            out["dpost_bias"] = db
    out["du"] = da.to(t)
    return out


def _planes(x, group=1):
    """[batch, length, heads, dim] as [batch * heads, length, dim] in 32 bits, each head
    repeated for its group."""
    x = x.float().permute(0, 2, 1, 3)
    return x.repeat_interleave(group, 1).flatten(0, 1).contiguous()


def _rows_of(x, case, heads):
    """The reverse of _planes, in the case's type."""
    return x.view(case["batch"], heads, *x.shape[1:]).permute(0, 2, 1, 3).to(TYPES[case["type"]]).contiguous()


def _probabilities(s):
    """(queries, keys, probabilities, log-sum-exp, kept or None), one plane for each batch
    and query head."""
    case = s["case"]
    B, H, Sq, Sk = case["batch"], case["heads"], case["q_len"], case["k_len"]
    q, k = _planes(s["q"]), _planes(s["k"], H // case["kv_heads"])
    scores = torch.matmul(q, k.transpose(1, 2).contiguous()) * case["dim"] ** -0.5
    i, j = _index(Sq)[:, None], _index(Sk)[None, :]
    if s["q_lens"] is not None:
        ql, kl = (s[n].long().repeat_interleave(H)[:, None, None] for n in ("q_lens", "k_lens"))
    else:
        ql, kl = Sq, Sk
    visible = (i < ql) & (j < kl)
    if case["causal"]:
        visible = visible & (j <= i + (kl - ql))
    scores = torch.where(visible, scores, torch.full_like(scores, -math.inf))
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = torch.exp(scores - top)
    total = e.sum(-1, keepdim=True)
    p = torch.where(total > 0, e / total, torch.zeros_like(e))
    lse = (torch.log(total) + top).view(B, H, Sq)
    kept = _keep_attention(B * H, Sq, Sk, case["p"], s["seed"]) if case["p"] > 0 else None
    return q, k, p, lse, kept


def _attention_forward(s):
    case = s["case"]
    _, _, p, lse, kept = _probabilities(s)
    if kept is not None:
        p = _dropped(p, kept, case["p"])
    v = _planes(s["v"], case["heads"] // case["kv_heads"])
    return {"o": _rows_of(torch.matmul(p, v), case, case["heads"]), "lse": lse}


def _attention_backward(s):
    case = s["case"]
    H, G = case["heads"], case["kv_heads"]
    scale = case["dim"] ** -0.5
    q, k, p, _, kept = _probabilities(s)
    v, do = _planes(s["v"], H // G), _planes(s["do"])
    dp = torch.matmul(do, v.transpose(1, 2).contiguous())
    dropped = p
    if kept is not None:
        dp = _dropped(dp, kept, case["p"])
        dropped = _dropped(p, kept, case["p"])
    dv = torch.matmul(dropped.transpose(1, 2).contiguous(), do)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(1, 2).contiguous(), q) * scale

    def summed(x):
        return x.view(case["batch"] * G, H // G, *x.shape[1:]).sum(1)

    return {"dq": _rows_of(dq, case, H), "dk": _rows_of(summed(dk), case, G), "dv": _rows_of(summed(dv), case, G)}


# ------------------------------------------------------------------ the library's calls

def _workspace(s, nbytes):
    """What a training program allocates once and keeps."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _own_dropout(s, okt):
    okt.okt_dropout(s["x"], s["y"], s["case"]["p"], s["seed"])
    return {"y": s["y"]}


def _own_norm(s, okt):
    case = s["case"]
    options = {"kind": case["kind"], "eps": EPS, "residual_scale": case["alpha"], "dropout_p": case["p"],
               "seed": s["seed"], "post_weight": s["post_weight"], "post_bias": s["post_bias"],
               "gate": s["gate"], "rows_per_gate": _gate_rows(case), "pre_weight": s["pre_weight"],
               "pre_bias": s["pre_bias"]}
    if not case["grad"]:
        okt.okt_residual_norm_forward(s["u"], s["x"], s["h"], s["y"], s["stats"], **options)
        return {k: s[k] for k in ("h", "y", "stats") if s[k] is not None}
    ws = s["ws"] if "ws" in s else _workspace(
        s, okt.okt_residual_norm_workspace_bytes(case["rows"], case["width"], _gate_rows(case)))
    okt.okt_residual_norm_backward(s["u"], s["h"], s["stats"], s["dh"], s["dy"], s["dx"], s["du"], ws,
                                   dpost_weight=s["dpost_weight"], dpost_bias=s["dpost_bias"],
                                   dgate=s["dgate"], dpre_weight=s["dpre_weight"],
                                   dpre_bias=s["dpre_bias"], **options)
    names = ("dx", "du", "dpost_weight", "dpost_bias", "dgate", "dpre_weight", "dpre_bias")
    return {k: s[k] for k in names if s[k] is not None}


def _own_attention(s, okt):
    case = s["case"]
    options = {"causal": case["causal"], "q_lens": s["q_lens"], "k_lens": s["k_lens"],
               "dropout_p": case["p"], "seed": s["seed"]}
    ws = s["ws"] if "ws" in s else _workspace(s, okt.okt_attention_workspace_bytes(
        case["batch"], case["heads"], case["kv_heads"], case["q_len"], case["k_len"], case["dim"]))
    if not case["grad"]:
        okt.okt_attention_forward(s["q"], s["k"], s["v"], s["o"], s["lse"], ws, **options)
        return {"o": s["o"], "lse": s["lse"]}
    okt.okt_attention_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"],
                               ws, **options)
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def run(state):
    case = state["case"]
    if own:
        import paper_2201_07598_amd as okt
        call = {"dropout": _own_dropout, "norm": _own_norm, "attention": _own_attention}[case["op"]]
        return call(state, okt)
    if case["op"] == "dropout":
        return {"y": _dropped(state["x"].float(), _keep_flat(case["n"], case["p"], state["seed"]),
                              case["p"]).to(state["x"].dtype)}
    if case["op"] == "norm":
        return _norm_backward(state) if case["grad"] else _norm_forward(state)
    return _attention_backward(state) if case["grad"] else _attention_forward(state)


# ------------------------------------------------------------------ floors and 64 bits

def _pairs(case):
    """Visible pairs of a query and a key, over batch and query heads."""
    total = 0
    for ql, kl in zip(_lengths(case, case["q_len"]), _lengths(case, case["k_len"])):
        if not case["causal"]:
            total += ql * kl
        else:                                     # row i sees min(kl, max(0, i + kl - ql + 1)) keys
            first = max(0, ql - kl)
            least, rows = first + kl - ql + 1, ql - first
            total += rows * (least + kl) // 2 if rows > 0 else 0
    return total * case["heads"]


def work(case):
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "dropout":
        return {"bytes": 2 * size * case["n"], "flops": case["n"]}
    if case["op"] == "norm":
        places = case["rows"] * case["width"]
        parameters = 4 * case["width"] * (
            (case["post"] + case["pre"]) * (2 if case["kind"] == "layer" else 1) + _gate_count(case))
        if not case["grad"]:
            return {"bytes": (3 + case["pre"]) * size * places + 16 * case["rows"] + parameters,
                    "flops": (3 + 8 * (case["post"] + case["pre"])) * places}
        reads = 1 + 2 * case["pre"] + (1 if case["post"] or case["gates"] else 0)
        return {"bytes": (reads + 2) * size * places + 16 * case["rows"] + 2 * parameters,
                "flops": (4 + 14 * (case["post"] + case["pre"])) * places}
    D = case["dim"]
    queries = sum(_lengths(case, case["q_len"])) * case["heads"]
    keys = sum(_lengths(case, case["k_len"])) * case["kv_heads"]
    written = case["batch"] * case["q_len"] * case["heads"]
    if not case["grad"]:
        return {"bytes": size * D * (queries + 2 * keys + written) + 4 * written,
                "flops": 4 * D * _pairs(case)}
    keys_written = case["batch"] * case["k_len"] * case["kv_heads"]
    return {"bytes": size * D * (3 * queries + 2 * keys + written + 2 * keys_written) + 4 * queries,
            "flops": 10 * D * _pairs(case)}


def _kept_64(c0, c1, c2, seed, p):
    """Truth values of whole blocks, [..., word, half], by numpy's unsigned arithmetic."""
    word = np.uint64(MASK32)
    x = [np.asarray(c, np.uint64) for c in np.broadcast_arrays(c0, c1, c2)] + [np.uint64(0)]
    key = [seed & MASK32, seed >> 32]
    for step in range(7):
        first, second = np.uint64(0xD2511F53) * x[0], np.uint64(0xCD9E8D57) * x[2]
        ka, kb = (np.uint64((key[n] + step * w) & MASK32) for n, w in ((0, 0x9E3779B9), (1, 0xBB67AE85)))
        x = [(second >> np.uint64(32)) ^ x[1] ^ ka, second & word, (first >> np.uint64(32)) ^ x[3] ^ kb, first & word]
    limit = np.uint32(math.floor((1.0 - p) * 65536.0 + 0.5))
    return np.stack([np.stack([(v.astype(np.uint32) & np.uint32(0xFFFF)) < limit,
                               (v.astype(np.uint32) >> np.uint32(16)) < limit], -1) for v in x], -2)


def _factor_64(kept, p):
    """0 or one over the share that is kept, on the GPU."""
    return torch.from_numpy(np.ascontiguousarray(kept)).to(DEV).double() * (
        65536.0 / math.floor((1.0 - p) * 65536.0 + 0.5))


def _exact_norm(s, seed):
    case, (rows, width) = s["case"], (s["case"]["rows"], s["case"]["width"])
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    factor = 1.0
    if case["p"] > 0:
        kept = _kept_64(np.arange(-(-width // 8))[None, :], np.arange(rows)[:, None], 0, seed, case["p"])
        factor = _factor_64(kept.reshape(rows, -1)[:, :width], case["p"])
    group = torch.arange(rows, device=DEV) // max(1, _gate_rows(case))
    gate = wide["gate"][group] if case["gates"] else 1.0
    layer = case["kind"] == "layer"

    def normal(x):
        m = x.mean(1, keepdim=True) if layer else torch.zeros(rows, 1, dtype=torch.float64, device=DEV)
        return m, 1.0 / torch.sqrt((x - m).square().mean(1, keepdim=True) + EPS)

    def scaled(x, m, r, name):
        return (x - m) * r * wide[name + "_weight"] + wide.get(name + "_bias", 0.0)

    zero = torch.zeros(rows, 1, dtype=torch.float64, device=DEV)
    if not case["grad"]:
        first = normal(wide["u"]) if case["post"] else (zero, zero)
        a = scaled(wide["u"], *first, "post") if case["post"] else wide["u"]
        h = case["alpha"] * wide["x"] + gate * (factor * a)
        held = h.to(s["u"].dtype).double()       # the second norm is defined on the stored sum
        second = normal(held) if case["pre"] else (zero, zero)
        out = {"h": h, "stats": torch.cat([*first, *second], 1)}
        if case["pre"]:
            out["y"] = scaled(held, *second, "pre")
        return out
    m0, r0, m1, r1 = (wide["stats"][:, c:c + 1] for c in range(4))
    out = {}

    def back(d, x, m, r, name):
        hat = (x - m) * r
        out["d" + name + "_weight"] = (d * hat).sum(0)
        if name + "_bias" in wide:
            out["d" + name + "_bias"] = d.sum(0)
        d = d * wide[name + "_weight"]
        return r * (d - (d.mean(1, keepdim=True) if layer else 0.0) - hat * (d * hat).mean(1, keepdim=True))

    dh = wide["dh"] + (back(wide["dy"], wide["h"], m1, r1, "pre") if case["pre"] else 0.0)
    out["dx"] = case["alpha"] * dh
    if case["gates"]:
        a = scaled(wide["u"], m0, r0, "post") if case["post"] else wide["u"]
        out["dgate"] = torch.zeros_like(wide["gate"]).index_add_(0, group, dh * factor * a)
    da = factor * (gate * dh)
    out["du"] = back(da, wide["u"], m0, r0, "post") if case["post"] else da
    return out


def _exact_attention(s, seed):
    case = s["case"]
    B, H, G, Sq, Sk = (case[n] for n in ("batch", "heads", "kv_heads", "q_len", "k_len"))
    scale = 1.0 / math.sqrt(case["dim"])
    names = ("q", "k", "v", "do") if case["grad"] else ("q", "k", "v")
    wide = {n: s[n].double().permute(0, 2, 1, 3).contiguous() for n in names}
    o = torch.zeros_like(wide["q"])
    lse = torch.full((B, H, Sq), -math.inf, dtype=torch.float64, device=DEV)
    dq, dk, dv = torch.zeros_like(wide["q"]), torch.zeros_like(wide["k"]), torch.zeros_like(wide["v"])
    for b, (ql, kl) in enumerate(zip(_lengths(case, Sq), _lengths(case, Sk))):
        hidden = torch.ones(ql, kl, dtype=torch.bool, device=DEV).triu(kl - ql + 1) if case["causal"] else None
        for h in range(H):
            g = h // (H // G)
            q, k, v = wide["q"][b, h, :ql], wide["k"][b, g, :kl], wide["v"][b, g, :kl]
            a = scale * (q @ k.t().contiguous())
            if hidden is not None:
                a = a.masked_fill(hidden, -math.inf)
            lse[b, h, :ql] = torch.logsumexp(a, 1)
            p = torch.exp(a - lse[b, h, :ql, None]).nan_to_num(0.0)
            f = 1.0
            if case["p"] > 0:
                kept = _kept_64(np.arange(-(-kl // 4))[None, :], np.arange(-(-ql // 2))[:, None], b * H + h, seed, case["p"])
                f = _factor_64(kept.transpose(0, 3, 1, 2).reshape(2 * kept.shape[0], -1)[:ql, :kl], case["p"])
            if not case["grad"]:
                o[b, h, :ql] = (f * p) @ v
                continue
            do = wide["do"][b, h, :ql]
            dp = f * (do @ v.t().contiguous())
            ds = p * (dp - (dp * p).sum(1, keepdim=True))
            dq[b, h, :ql] = scale * (ds @ k)
            dk[b, g, :kl] += scale * (ds.t().contiguous() @ q)
            dv[b, g, :kl] += (f * p).t().contiguous() @ do
    if not case["grad"]:
        return {"o": o.permute(0, 2, 1, 3).contiguous(), "lse": lse}
    return {n: x.permute(0, 2, 1, 3).contiguous() for n, x in (("dq", dq), ("dk", dk), ("dv", dv))}


def exact(case, seed):
    s = prepare(case, seed)
    key = int(s["seed"].cpu()[0]) & 0xFFFFFFFFFFFFFFFF
    if case["op"] == "dropout":
        kept = _kept_64(np.arange(-(-case["n"] // 8)), 0, 0, key, case["p"])
        return {"y": s["x"].double() * _factor_64(kept.reshape(-1)[:case["n"]], case["p"])}
    return _exact_norm(s, key) if case["op"] == "norm" else _exact_attention(s, key)
