"""okt_norm_rotary_forward / _backward against the 64-bit oracle: heads of every width, parts of a common projection, several
axes, places far away, one token and many, with bounds that add up the roundings."""
import numpy as np
import pytest
import torch

import paper_2201_07598_amd as okt
from operators_harness import DEV, E, TYPES, UNIT, rand, step as least, wide, within
from oracle import okt_training as ref

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, batch=2, length=5, heads=4, kv_heads=2, dim=64, rot=None, kind="bf16", norm="rms", adjacent=False, axes=1,
                 positions=True, far=1000, seed=0, layout="projection"):
        self.kind, self.norm = kind, norm
        shape = lambda n: (batch, length, n, dim)  # noqa: E731
        if layout == "projection":                       # queries, keys, values side by side
            self.q, self.k, _ = rand(shape(heads + 2 * kv_heads), kind, seed).split([heads, kv_heads, kv_heads], 2)
        elif layout == "heads first":                    # [batch, heads, length, dim], odd strides
            room = rand((batch, heads + kv_heads, length, dim + 3), kind, seed)[..., 1:dim + 1].transpose(1, 2)
            self.q, self.k = room.split([heads, kv_heads], 2)
        else:                                            # [batch, length, dim] of each head by itself, each head's own q, k, v
            room = rand((batch, length, max(heads, kv_heads), 3, dim), kind, seed)
            self.q, self.k = room[:, :, :heads, 0], room[:, :, :kv_heads, 1]
        rot = dim if rot is None else rot
        gen = torch.Generator().manual_seed(seed + 1)
        self.inv_freq = (100.0 ** (-torch.arange(0, rot, 2) / max(rot, 1))).float().to(DEV) if rot else None
        self.positions = torch.randint(-far, far, (batch, length, axes), generator=gen).to(torch.int32).to(DEV) if positions else None
        self.axis_of_pair = [j % axes for j in range(rot // 2)] if axes > 1 else None
        self.weights = [None, None] if norm is None else [1.0 + rand((dim,), "f32", seed + 2, 0.3), 1.0 + rand((dim,), "f32", seed + 3, 0.3)]
        self.options = {"positions": self.positions, "axis_of_pair": self.axis_of_pair, "adjacent": adjacent, "kind": norm or "rms", "eps": 1e-5,
                        "q_weight": self.weights[0], "k_weight": self.weights[1]}
        freq = None if self.inv_freq is None else self.inv_freq.cpu().numpy()
        self.angle = ref.angles(batch, length, freq, None if self.positions is None else self.positions.cpu().numpy(), self.axis_of_pair)
        self.adjacent, self.seed = adjacent, seed

    def oracle(self, n):
        w = self.weights[n]
        return dict(weight=None if w is None else wide(w), kind=self.norm or "rms", eps=float(np.float32(1e-5)), adjacent=self.adjacent)


def forward_error(x, c, n):
    """What the output may be off by before it is rounded.  A norm: sums of up to 256 elements, none through more than 8 + 6 additions, the product with
    the reciprocal and the weight; the turn: two products and a sum of values whose cosines and sines are off by 4 E (the angle in
    turns rounded to fp32, pi E, and the function's ulp)."""
    o = c.oracle(n)
    size = np.abs(x)
    off = 0.0 * size
    if o["weight"] is not None:
        mean, r = ref.head_statistics(x, o["kind"], o["eps"])
        e_mean = (16 * E * size.mean(-1, keepdims=True)) if o["kind"] == "layer" else 0.0
        centred = np.abs(x - mean)
        var = (centred ** 2).mean(-1, keepdims=True)
        e_r = 0.5 * r * r * (20 * E * var + 2 * e_mean * centred.mean(-1, keepdims=True) + e_mean ** 2) + 4 * E     # relative
        size = centred * r * np.abs(o["weight"])
        off = size * (e_r + 4 * E) + r * np.abs(o["weight"]) * (e_mean + E * (np.abs(x) + np.abs(mean)))
    a, b = ref._pairs(x.shape[-1], 2 * c.angle.shape[-1], c.adjacent)
    both = size[..., a] + size[..., b]
    turned = off.copy()
    turned[..., a] = turned[..., b] = off[..., a] + off[..., b] + 8 * E * both
    return turned


def rounded(bound, want, kind):
    return bound + UNIT[kind] * (np.abs(want) + bound) + least(kind)


def run_forward(c, q_out=None, k_out=None):
    q_out = torch.full(c.q.shape, 7.0, dtype=c.q.dtype, device=DEV) if q_out is None else q_out
    k_out = torch.full(c.k.shape, 7.0, dtype=c.q.dtype, device=DEV) if k_out is None else k_out
    okt.okt_norm_rotary_forward(c.q, c.k, q_out, k_out, c.inv_freq, **c.options)
    return q_out, k_out


def check_forward(c, outs, inputs):
    for n, (x, got) in enumerate(zip(inputs, outs)):
        want = ref.norm_rotary(x, c.angle, **c.oracle(n))
        within(got, want, rounded(forward_error(x, c, n), want, c.kind), "qk"[n])


CASES = [
    dict(), dict(kind="f32", norm="layer"), dict(kind="f16", dim=128, adjacent=True), dict(dim=80, rot=64, axes=3, adjacent=True, norm="layer"),
    dict(dim=256, kind="f32"), dict(dim=8, heads=3, kv_heads=1), dict(dim=24, rot=8, kind="f16"), dict(dim=136, rot=128, heads=5, kv_heads=5),
    dict(dim=72, rot=0, kind="f32"), dict(norm=None, kind="f32", dim=40), dict(norm=None, dim=128, axes=2), dict(batch=1, length=1),
    dict(batch=300, length=1, far=10 ** 9, kind="f32"), dict(batch=3, length=700, dim=64, heads=12, kv_heads=12, positions=False),
    dict(batch=1, length=2049, heads=16, kv_heads=4, dim=128, far=2 ** 31 - 1), dict(layout="heads first", length=33, kind="f16"),
    dict(layout="each head", length=9, heads=4, kv_heads=4, adjacent=True), dict(heads=1, kv_heads=40, dim=32, length=17), dict(axes=8, dim=64, kind="f32")]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_forward(n):
    c = Case(**CASES[n], seed=n)
    check_forward(c, run_forward(c), [wide(c.q), wide(c.k)])


@pytest.mark.parametrize("layout", ["projection", "heads first", "each head"])
def test_forward_in_place(layout):
    c = Case(layout=layout, length=21, seed=50)
    inputs, rest = [wide(c.q), wide(c.k)], c.q._base.clone()
    run_forward(c, c.q, c.k)
    check_forward(c, (c.q, c.k), inputs)
    touched = torch.zeros_like(rest)                     # values, gaps and everything else are as they were
    for view in (c.q, c.k):
        touched.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(1.0)
    assert torch.equal(torch.where(touched > 0, rest, c.q._base), rest)


def backward_error(x, dy, c, n):
    """Of dx before it is rounded, and of dweight."""
    o = c.oracle(n)
    a, b = ref._pairs(x.shape[-1], 2 * c.angle.shape[-1], c.adjacent)
    d, ed = ref.turned(dy, c.angle, c.adjacent, back=True), 0.0 * dy
    ed[..., a] = ed[..., b] = 8 * E * (np.abs(dy[..., a]) + np.abs(dy[..., b]))
    if o["weight"] is None:
        return ed, None
    mean, r = ref.head_statistics(x, o["kind"], o["eps"])
    e_mean = (16 * E * np.abs(x).mean(-1, keepdims=True)) if o["kind"] == "layer" else 0.0
    centred = np.abs(x - mean)
    var = (centred ** 2).mean(-1, keepdims=True)
    e_r = 0.5 * r * r * (20 * E * var + 2 * e_mean * centred.mean(-1, keepdims=True) + e_mean ** 2) + 4 * E
    h = centred * r
    eh = h * (e_r + 2 * E) + r * (e_mean + E * (np.abs(x) + np.abs(mean)))
    w = np.abs(d * o["weight"])
    ew = ed * np.abs(o["weight"]) + E * w
    along = (w * h).mean(-1, keepdims=True)
    e_along = (ew * h + w * eh).mean(-1, keepdims=True) + 20 * E * along
    level = w.mean(-1, keepdims=True)
    e_level = ew.mean(-1, keepdims=True) + 20 * E * level
    inner = w + h * along + level
    dx = r * (ew + eh * along + h * e_along + e_level + inner * (e_r + 6 * E))
    # a lane's additions one after the other (all tokens of a workgroup: up to 2^24 / 1024), 3 + 4 across, then 64 + 16
    steps = 8 + 4 + 80 + x.shape[0] * x.shape[1] * x.shape[2] // (8 * min(1024, max(1, x.shape[0] * x.shape[1] // 32)))
    dw = (ed * h + np.abs(d) * eh).sum((0, 1, 2)) + steps * E * (np.abs(d) * h).sum((0, 1, 2))
    return dx, dw


def run_backward(c, in_place=False):
    dq, dk = rand(c.q.shape, c.kind, c.seed + 7, 0.5), rand(c.k.shape, c.kind, c.seed + 8, 0.5)
    given = [wide(dq), wide(dk)]
    outs = (dq, dk) if in_place else tuple(torch.full(t.shape, 7.0, dtype=t.dtype, device=DEV) for t in (dq, dk))
    dws = [None if w is None else torch.full_like(w, 7.0) for w in c.weights]
    ws = torch.full((okt.okt_norm_rotary_workspace_bytes(*c.q.shape[:3], c.k.shape[2], c.q.shape[3]),), 255, dtype=torch.uint8, device=DEV)
    okt.okt_norm_rotary_backward(c.q, c.k, dq, dk, *outs, c.inv_freq, ws, dq_weight_out=dws[0], dk_weight_out=dws[1], **c.options)
    return given, outs, dws


def check_backward(c, given, outs, dws):
    for n, x in enumerate((wide(c.q), wide(c.k))):
        want, want_w = ref.norm_rotary_backward(x, given[n], c.angle, **c.oracle(n))
        e_x, e_w = backward_error(x, given[n], c, n)
        within(outs[n], want, rounded(e_x, want, c.kind), "d" + "qk"[n])
        if want_w is not None:
            within(dws[n], want_w, e_w + E * np.abs(want_w), "d" + "qk"[n] + "_weight")


@pytest.mark.parametrize("n", range(len(CASES)))
def test_backward(n):
    c = Case(**CASES[n], seed=n)
    check_backward(c, *run_backward(c))


def test_backward_in_place_and_again():
    c = Case(batch=3, length=333, heads=6, kv_heads=2, dim=96, seed=70)
    first, second = run_backward(c), run_backward(c, True)
    check_backward(c, *second)
    for a, b in zip((*first[1], *first[2]), (*second[1], *second[2])):
        assert torch.equal(a, b)                         # the same bits


def test_one_of_the_two():
    c = Case(seed=80)
    both = run_forward(c)
    alone = torch.empty(c.k.shape, dtype=c.k.dtype, device=DEV)
    okt.okt_norm_rotary_forward(c.k, None, alone, None, c.inv_freq, **{**c.options, "q_weight": c.weights[1], "k_weight": None})
    assert torch.equal(alone, both[1])
    (gq, gk), outs, dws = run_backward(c)
    dk, dw = rand(c.k.shape, c.kind, c.seed + 8, 0.5), torch.empty_like(dws[1])
    ws = torch.empty(okt.okt_norm_rotary_workspace_bytes(*c.k.shape[:3], 0, c.k.shape[3]), dtype=torch.uint8, device=DEV)
    okt.okt_norm_rotary_backward(c.k, None, dk, None, alone, None, c.inv_freq, ws, dq_weight_out=dw,
                                 **{**c.options, "q_weight": c.weights[1], "k_weight": None})
    assert torch.equal(alone, outs[1])
    # a norm for queries alone: keys are turned only
    c.options["k_weight"] = c.weights[1] = None
    check_forward(c, run_forward(c), [wide(c.q), wide(c.k)])
    check_backward(c, *run_backward(c))


def test_broadcast_inputs_and_shared_positions():
    """A key head that all heads read, and one row of positions for all sequences."""
    c = Case(heads=4, kv_heads=4, length=6, positions=False, seed=90)
    c.k = rand((2, 6, 1, 64), "bf16", 91).expand(2, 6, 4, 64)
    row = torch.arange(6, dtype=torch.int32, device=DEV) * 3 + 5
    c.options["positions"] = row
    c.angle = ref.angles(2, 6, c.inv_freq.cpu().numpy(), np.broadcast_to(row.cpu().numpy()[None, :, None], (2, 6, 1)))
    check_forward(c, run_forward(c), [wide(c.q), wide(c.k)])
    c.options["positions"] = row.view(1, 6).expand(2, 6)
    check_forward(c, run_forward(c), [wide(c.q), wide(c.k)])


def test_not_finite_stays_in_its_head():
    c = Case(length=40, heads=5, kv_heads=3, seed=95)
    clean = run_forward(c)
    c.q[1, 7, 2, 3], c.k[0, 39, 0, 63] = float("nan"), float("inf")
    outs = run_forward(c)
    for a, b, place in ((outs[0], clean[0], (1, 7, 2)), (outs[1], clean[1], (0, 39, 0))):
        assert not torch.isfinite(a[place]).all()
        a[place], b[place] = 0.0, 0.0
        assert torch.equal(a, b)


def test_no_tokens():
    c = Case(batch=2, length=0, seed=1)
    run_forward(c)
    given, outs, dws = run_backward(c)
    assert all(not w.any() for w in dws)


def test_replayed_and_on_another_stream():
    c = Case(batch=2, length=100, heads=8, kv_heads=2, dim=128, seed=99)
    dq, dk = rand(c.q.shape, c.kind, 1), rand(c.k.shape, c.kind, 2)
    make = lambda: [torch.zeros(t.shape, dtype=t.dtype, device=DEV) for t in (c.q, c.k, c.q, c.k, c.weights[0], c.weights[1])]  # noqa: E731
    ws = [torch.empty(okt.okt_norm_rotary_workspace_bytes(2, 100, 8, 2, 128), dtype=torch.uint8, device=DEV) for _ in range(2)]

    def both(o, ws):
        okt.okt_norm_rotary_forward(c.q, c.k, o[0], o[1], c.inv_freq, **c.options)
        okt.okt_norm_rotary_backward(c.q, c.k, dq, dk, o[2], o[3], c.inv_freq, ws, dq_weight_out=o[4], dk_weight_out=o[5], **c.options)

    captured, eager = make(), make()
    both(captured, ws[0])
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        both(captured, ws[0])
    for n in range(3):
        for t in (c.q, c.k, dq, dk):
            t.mul_(0.75)
        c.positions.add_(1000)
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            both(eager, ws[1])
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager)), n
