"""The operators at the ends of a training step at sizes that take forms of their kernels of which smaller calls see nothing: three pieces of a vocabulary, products
of several large tiles, narrow products for few rows, accesses around the caches.  tests/test_training_forms.py holds these sizes to the forms."""
import numpy as np
import pytest
import torch

import paper_2201_07598_amd as okt
from operators_harness import DEV, E, TYPES, rand, seed_tensor, wide
from test_gpu_adamw import cut, int64
from test_gpu_cross_entropy import Case, check

pytestmark = pytest.mark.gpu

# ------------------------------------------------------------------ cross entropy

LARGE, NARROW = "ProductShapeILi4ELi2ELi2ELi4ELi2EE", "ProductShapeILi2ELi2ELi2ELi2ELi2EE"
# sizes, pieces of the vocabulary, products
LOSSES = [
    (dict(rows=65_000, width=264, vocab=16_500, labelled=0.012, bias=True), 3, LARGE),                 # dh of several tiles over pieces
    (dict(rows=65_000, width=264, vocab=16_500, labelled=0.003, kind="f16", wide_dw=True), 3, LARGE),  # the same of few rows, in two parts
    (dict(rows=131_000, width=72, vocab=8449, labelled=0.004, kind="f16", bias=True), 3, LARGE),
    (dict(rows=16_384, width=520, vocab=40_000, labelled=0.05, one_g=True), 2, LARGE),
    (dict(rows=10, width=256, vocab=70_000, bias=True), 1, NARROW), (dict(rows=10, width=256, vocab=70_000, kind="f16", wide_dw=True), 1, NARROW),
    (dict(rows=200, width=1032, vocab=16_400, kind="f16", bias=True), 1, NARROW), (dict(rows=200, width=1032, vocab=16_400, wide_dw=True, pad=8), 1, NARROW),
    (dict(rows=256, width=520, vocab=30_011, labelled=0.7), 1, NARROW)]


@pytest.mark.parametrize("n", range(len(LOSSES)))
def test_loss_and_gradients(n):
    c = Case(**LOSSES[n][0], seed=200 + 10 * n)
    loss, lse = c.forward()
    grads = c.backward(lse)
    check(c, loss, lse, grads)
    assert not grads[0][(c.labels < 0) | (c.labels >= c.vocab)].any()
    for a, b in zip(grads, c.backward(lse)):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("rows,width,vocab,labelled", [(2, 8, 3, 1.0), (125, 776, 10_007, 1.0), (120, 40_000 // 64 * 8, 9000, 0.5), (300, 64, 777, 1.0), (2049, 64, 700, 1.0),
                                                     (2600, 64, 5001, 0.9), (10, 256, 70_000, 1.0), (16_384, 64, 4000, 1.0), (65_000, 64, 16_500, 0.02)])
def test_nothing_is_written_behind_the_workspace(rows, width, vocab, labelled):
    c = Case(rows, width, vocab, labelled=labelled, bias=True, seed=250)
    room, c.ws = c.ws, None
    guard = torch.full((room.numel() + (1 << 22),), 171, dtype=torch.uint8, device=DEV)
    c.ws = guard[:room.numel()]
    loss, lse = c.forward()
    c.backward(lse)
    assert bool((guard[room.numel():] == 171).all())
    c.ws = room
    again = c.forward()
    assert torch.equal(loss, again[0]) and torch.equal(lse, again[1])


# ------------------------------------------------------------------ rotation

# one call moves more than 256 MiB, a sequence of it less
ROTATIONS = [dict(batch=3, length=7501, heads=16, kv_heads=8, dim=128, rot=128, kind="bf16", adjacent=False, norm="rms"),
             dict(batch=4, length=5003, heads=12, kv_heads=12, dim=72, rot=64, kind="f32", adjacent=True, norm="layer"),
             dict(batch=5, length=3001, heads=9, kv_heads=9, dim=256, rot=64, kind="f16", adjacent=False, norm="rms"),
             dict(batch=3, length=30_001, heads=6, kv_heads=2, dim=104, rot=104, kind="bf16", adjacent=True, norm="layer")]


@pytest.mark.parametrize("n", range(len(ROTATIONS)))
def test_rotation_around_the_caches(n):
    """All tokens at once against the same in slices."""
    c = ROTATIONS[n]
    B, S, H, G, D, t = c["batch"], c["length"], c["heads"], c["kv_heads"], c["dim"], TYPES[c["kind"]]
    gen = torch.Generator(device=DEV).manual_seed(300 + n)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)  # noqa: E731
    x, dy = (normal(B, S, H + 2 * G, D + 1).to(t)[..., 1:] for _ in range(2))          # rows at odd elements
    (q, k, _), (dq, dk, _) = x.split([H, G, G], 2), dy.split([H, G, G], 2)
    inv_freq = 100.0 ** (-torch.arange(0, c["rot"], 2, device=DEV) / c["rot"])
    positions = torch.randint(0, 10 ** 6, (B, S), generator=gen, device=DEV).to(torch.int32)
    weights = [1 + 0.2 * normal(D) for _ in range(2)]
    options = dict(adjacent=c["adjacent"], kind=c["norm"], q_weight=weights[0], k_weight=weights[1])
    ws = torch.empty(okt.okt_norm_rotary_workspace_bytes(B, S, H, G, D), dtype=torch.uint8, device=DEV)

    def run(s):
        outs = [torch.empty_like(a[s], memory_format=torch.contiguous_format) for a in (q, k, dq, dk)]
        dws = [torch.empty(D, device=DEV) for _ in range(2)]
        okt.okt_norm_rotary_forward(q[s], k[s], outs[0], outs[1], inv_freq, positions=positions[s], **options)
        okt.okt_norm_rotary_backward(q[s], k[s], dq[s], dk[s], outs[2], outs[3], inv_freq, ws, dq_weight_out=dws[0], dk_weight_out=dws[1],
                                     positions=positions[s], **options)
        return outs, dws

    whole, sums = run(slice(0, B))
    parts = [run(slice(b, b + 1)) for b in range(B)]
    for b, (outs, _) in enumerate(parts):
        for a, p in zip(whole, outs):
            assert torch.equal(a[b:b + 1], p)
    for got, name in zip(range(2), "qk"):
        # Each term is the same number in both.  |h| <= D^0.5 and the turned dy is 2^0.5 max |dy| at most, the mean of their product's magnitude far
        # below; it is at most the root of the product of mean squares (of h: 1), times the number of terms.  One sum has fewer additions than
        # terms of a lane (all over 1024 workgroups of 8 lanes of a kind, at worst) and 12 + 80 behind them.
        d = (dq, dk)[got].double()
        heads = B * S * (H, G)[got]
        size = heads * d.square().mean((0, 1, 2)).max().sqrt().item() * 2 ** 0.5 * 1.5
        steps = heads // (8 * 700) + 92
        want = sum(p[1][got].double() for p in parts)
        assert bool(((sums[got].double() - want).abs() <= 2 * steps * E * size).all()), name


# ------------------------------------------------------------------ AdamW

# a step that moves more than 640 MiB, of tensors of which each moves less
STEPS = [(0, "f32", "f32", None, None, [1, 8_400_001, 3, 9_000_002, 255, 4097, 8_100_003, 257]),
         (0, "bf16", "f16", "f16", None, [8_999_999, 0, 9_000_001, 5, 9_000_003]),
         (1, "f32", "bf16", "bf16", 77, [3, 10_000_001, 1, 11_000_002, 257, 12_000_003, 4097, 13_000_255]),
         (1, "f16", "f32", None, None, [15_000_001, 15_000_002, 15_000_003, 2])]


@pytest.mark.parametrize("n", range(len(STEPS)))
def test_steps_around_the_caches(n):
    """All tensors in one plan against a plan for each, in which the others are empty: the same numbers of tensors, the same random bits."""
    eight, p_kind, g_kind, copy, seed, lengths = STEPS[n]
    gen = torch.Generator(device=DEV).manual_seed(400 + n)
    total = sum(lengths) + 7 * (len(lengths) + 1)
    blocks = [-(-x // 256) for x in lengths]
    normal = lambda scale: torch.randn(total, generator=gen, device=DEV) * scale  # noqa: E731
    all_of = {"p": normal(0.05).to(TYPES[p_kind]), "g": normal(0.01).to(TYPES[g_kind])}
    if eight:
        codes = lambda signs: torch.randint(0, 127, (total,), generator=gen, device=DEV) + signs * 128 * torch.randint(0, 2, (total,), generator=gen, device=DEV)  # noqa: E731
        all_of["m"], all_of["v"] = (codes(s).to(torch.uint8).view(torch.float8_e4m3fn) for s in (1, 0))
        scales = sum(blocks) + 7 * (len(lengths) + 1)
        for name, size in (("m_scale", 1e-5), ("v_scale", 1e-5)):
            all_of[name] = size * torch.rand(scales, generator=gen, device=DEV)
    else:
        all_of["m"], all_of["v"] = normal(3e-3), normal(3e-3).square()
    if copy:
        all_of["copy"] = normal(1.0).to(TYPES[copy])
    again = {name: t.clone() for name, t in all_of.items()}

    def step(buffers, only=None):
        sizes = {name: blocks if name.endswith("scale") else lengths for name in buffers}
        t = {name: [x if only in (None, i) else x[:0] for i, x in enumerate(cut(b, sizes[name]))] for name, b in buffers.items()}
        plan = okt.okt_adamw_plan(t["p"], t["g"], t["m"], t["v"], m_scales=t.get("m_scale"), v_scales=t.get("v_scale"), copies=t.get("copy"), weight_decay=0.01)
        okt.okt_adamw_step(plan, int64(5), lr=0.01, seed=None if seed is None else seed_tensor(seed), site=3)

    step(all_of)
    for i in range(len(lengths)):
        step(again, i)
    for name, t in all_of.items():                       # and between the tensors nothing is written
        assert torch.equal(t.view(torch.uint8), again[name].view(torch.uint8)), name
