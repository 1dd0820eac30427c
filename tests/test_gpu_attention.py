"""okt_attention_forward / _backward on the GPU against the 64-bit oracle: masks, lengths, head
layouts, strides, types, the split over the long axis, within bounds that add up the
roundings (operators_harness)."""
import numpy as np
import pytest
import torch

import paper_2201_07598_amd as okt
from oracle import okt_operators as ops
from tests.operators_harness import DEV, TYPES, UNIT, attention_bounds, rand, seed_tensor, step, wide, within

pytestmark = pytest.mark.gpu

SEED = (1 << 63) + 12345 - (1 << 64)          # as the int64 that carries the uint64


def make(B, H, G, Sq, Sk, D, kind="bf16", scale=1.0):
    if Sq == Sk:
        q, k, v = rand((B, Sq, H + 2 * G, D), kind, Sq * 7 + D, scale).split([H, G, G], 2)
    else:
        q = rand((B, Sq, H, D), kind, Sq + D, scale)
        k, v = rand((B, Sk, 2 * G, D), kind, Sk + D, scale).split([G, G], 2)
    return q, k, v, rand((B, Sq, H, D), kind, 5)


def workspace(q, k, fill=0xA5):
    n = okt.okt_attention_workspace_bytes(q.shape[0], q.shape[2], k.shape[2], q.shape[1], k.shape[1], q.shape[3])
    return torch.full((n,), fill, dtype=torch.uint8, device=DEV)


def forward(q, k, v, **options):
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), 7.0, device=DEV)
    okt.okt_attention_forward(q, k, v, o, lse, workspace(q, k), **options)
    return o, lse


def backward(q, k, v, o, lse, do, **options):
    dq, dk, dv = (torch.full(t.shape, 7.0, dtype=q.dtype, device=DEV) for t in (q, k, v))
    okt.okt_attention_backward(q, k, v, o, lse, do, dq, dk, dv, workspace(q, k), **options)
    return dq, dk, dv


def norm_of(x):
    return float(np.linalg.norm(x))


def check(q, k, v, do, kind, *, causal=False, scale=None, lens=None, p=0.0, site=2):
    options = dict(causal=causal, scale=scale, dropout_p=p, site=site, seed=seed_tensor(SEED) if p else None)
    for name, n in zip(("q_lens", "k_lens"), lens or (None, None)):
        options[name] = None if n is None else torch.tensor(n, dtype=torch.int32, device=DEV)
    plain = dict(causal=causal, scale=scale, q_lens=lens and lens[0], k_lens=lens and lens[1], dropout_p=p,
                 seed=SEED & ((1 << 64) - 1), site=site)
    Q, KK, V, DO = (wide(t) for t in (q, k, v, do))
    u, least = UNIT[kind], step(kind)
    o, lse = forward(q, k, v, **options)
    want_o, want_lse = ops.attention(Q, KK, V, **plain)
    plain["scale"] = q.shape[-1] ** -0.5 if scale is None else scale
    bo, blse = attention_bounds(Q, KK, V, kind, **plain)
    within(o, want_o, bo * (1 + u) + u * np.abs(want_o) + least, "o")
    within(lse, want_lse, blse, "lse")
    # independent roundings add up in squares: each is at most u / sqrt 3 of what it rounds
    assert norm_of(wide(o) - want_o) <= u * norm_of(want_o) + 1e-30
    got = backward(q, k, v, o, lse, do, **options)
    want = ops.attention_backward(Q, KK, V, DO, **plain)
    stored = bo * (1 + u) + u * np.abs(want_o) + least
    for name, g, w, b in zip(("dq", "dk", "dv"), got, want, attention_bounds(Q, KK, V, kind, do=DO, o=stored, **plain)):
        within(g, w, b * (1 + u) + u * np.abs(w) + least, name)
    again = backward(q, k, v, o, lse, do, **options)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "runs differ"
    return o, lse, got


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Sq,Sk", [(1, 1), (2, 2), (1, 70), (70, 1), (31, 33), (32, 32), (64, 64), (65, 129), (129, 65),
                                   (128, 128), (200, 200), (257, 300), (300, 257)])
@pytest.mark.parametrize("D", [64, 128])
def test_lengths(Sq, Sk, D, causal, kind):
    check(*make(2, 2, 1, Sq, Sk, D, kind), kind, causal=causal)


@pytest.mark.parametrize("D", [8, 16, 24, 32, 40, 56, 72, 80, 96, 104, 120])
def test_head_sizes(D):
    check(*make(2, 3, 3, 100, 100, D), "bf16", causal=True, p=0.1)


@pytest.mark.parametrize("H,G", [(1, 1), (5, 5), (6, 2), (8, 1), (7, 7)])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_head_groups(H, G, p):
    check(*make(3, H, G, 90, 150, 64, "f16"), "f16", causal=True, p=p)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_padded_batches(D, causal, p):
    """Lengths of nothing, of one, whole, and such that the causal mask leaves rows empty."""
    lens = ([140, 0, 1, 77, 140, 100, 33], [140, 140, 0, 1, 33, 140, 64])
    check(*make(7, 2, 2, 140, 140, D), "bf16", causal=causal, lens=lens, p=p)


def test_lengths_out_of_range_are_held_to_the_tensors():
    q, k, v, do = make(3, 2, 1, 50, 50, 64)
    o, lse, g = check(q, k, v, do, "bf16", lens=([50, 0, 50], [50, 50, 0]))
    options = dict(q_lens=torch.tensor([1 << 30, -5, 51], dtype=torch.int32, device=DEV),
                   k_lens=torch.tensor([50, 99, -1], dtype=torch.int32, device=DEV))
    o2, lse2 = forward(q, k, v, **options)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert all(torch.equal(a, b) for a, b in zip(g, backward(q, k, v, o2, lse2, do, **options)))


@pytest.mark.parametrize("D", [40, 64, 128])
def test_what_lies_past_the_lengths_is_not_looked_at(D):
    """Infinities and NaN in the padding, and in rows that the causal mask leaves empty."""
    B, H, G, S = 2, 2, 1, 150
    lens = ([100, 150], [37, 90])
    q, k, v, do = (t.contiguous() for t in make(B, H, G, S, S, D))
    options = dict(causal=True, q_lens=torch.tensor(lens[0], dtype=torch.int32, device=DEV),
                   k_lens=torch.tensor(lens[1], dtype=torch.int32, device=DEV))
    o, lse = forward(q, k, v, **options)
    clean = backward(q, k, v, o, lse, do, **options)
    for b in range(B):
        ql, kl = lens[0][b], lens[1][b]
        for t, n in ((q, ql), (do, ql), (k, kl), (v, kl)):
            t[b, n:] = float("nan")
            t[b, n::3] = float("inf")
        q[b, :ql - kl] = float("nan")                              # these see no key
        do[b, :ql - kl] = float("nan")
    o2, lse2 = forward(q, k, v, **options)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert all(torch.equal(a, b) for a, b in zip(clean, backward(q, k, v, o2, lse2, do, **options)))


@pytest.mark.parametrize("D", [24, 40, 72, 104])
def test_what_lies_between_heads_is_not_looked_at(D):
    """Narrow heads in wide places: the columns past head_dim belong to somebody else."""
    B, H, S, room = 2, 2, 70, 128
    wide_ones = [torch.full((B, S, H, room), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    views = [w[..., :D] for w in wide_ones]
    for n, t in enumerate(views):
        t.copy_(rand((B, S, H, D), "bf16", 20 + n))
    check(*views, "bf16", causal=True)


def test_strides_of_every_kind():
    """Length before batch, heads before length, and gradients written into one packed buffer."""
    S, B, H, D = 90, 3, 2, 64
    q, k, v, do = (rand((S, B, H, D), "bf16", n).transpose(0, 1) for n in range(4))
    o, lse, g = check(q, k, v, do, "bf16", causal=True)
    swapped = [t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (q, k, v, do)]
    o2, lse2 = forward(*swapped[:3], causal=True)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    packed = torch.full((B, S, 3 * H, D), 5.0, dtype=torch.bfloat16, device=DEV)
    dq, dk, dv = packed.split([H, H, H], 2)
    okt.okt_attention_backward(q, k, v, o, lse, do, dq, dk, dv, workspace(q, k), causal=True)
    assert all(torch.equal(a, b) for a, b in zip(g, (dq, dk, dv)))


def test_offsets_beyond_32_bits():
    """Sequences that lie more than 2^32 bytes, and 2^31 elements, apart."""
    B, S, H, D = 2, 70, 1, 64
    apart = (1 << 31) + (1 << 12)
    store = torch.empty(apart + S * H * D, dtype=torch.bfloat16, device=DEV)
    k = store.as_strided((B, S, H, D), (apart, H * D, D, 1))
    q, _, v, do = make(B, H, H, S, S, D)
    k.copy_(rand((B, S, H, D), "bf16", 99))
    check(q, k, v, do, "bf16")
    del store, k
    torch.cuda.empty_cache()


@pytest.mark.parametrize("Sq,Sk,H,G,D,causal,p", [(1, 3000, 2, 1, 64, False, 0.0), (40, 2500, 2, 2, 128, True, 0.2),
                                                  (2500, 3, 4, 1, 128, False, 0.1), (1500, 40, 2, 2, 64, True, 0.0),
                                                  (700, 700, 3, 1, 64, True, 0.1), (3, 2049, 8, 2, 40, True, 0.0)])
def test_work_split_over_the_long_axis(Sq, Sk, H, G, D, causal, p):
    lens = ([Sq, max(1, Sq // 2)], [Sk, max(1, Sk // 3)])
    check(*make(2, H, G, Sq, Sk, D), "bf16", causal=causal, p=p, lens=lens)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("Sq,Sk,H,G,D", [(1, 1, 8, 2, 64), (1, 700, 8, 2, 128), (1, 3000, 6, 1, 64), (7, 500, 6, 2, 40),
                                         (33, 100, 9, 3, 64), (64, 64, 10, 2, 128), (64, 200, 5, 1, 8), (64, 40, 4, 1, 64)])
def test_few_queries_of_a_group_s_heads(Sq, Sk, H, G, D, causal):
    """Heads that share a block of rows: blocks that end inside one, lengths of their own, sequences of none."""
    lens = ([Sq, max(1, Sq // 2), 0, Sq, 1], [Sk, max(1, Sk // 3), Sk, 0, 1])
    q, k, v, do = make(5, H, G, Sq, Sk, D)
    check(q, k, v, do, "bf16", causal=causal, lens=lens)
    check(q, k, v, do, "bf16", causal=causal)


@pytest.mark.parametrize("p", [0.0, 0.1])
def test_scores_of_every_size(p):
    """A softmax that is all but one key, and one that is nearly even; a maximum that grows along the keys."""
    q, k, v, do = make(1, 2, 2, 130, 260, 64, "bf16", scale=4.0)
    check(q, k, v, do, "bf16", p=p)
    check(q, k, v, do, "bf16", scale=1e-3, p=p)
    ramp = torch.linspace(0, 1, 260, device=DEV).to(torch.bfloat16)[None, :, None, None]
    check(q, k * ramp, v, do, "bf16", p=p)


def test_one_key_has_no_gradient_but_its_value():
    q, k, v, do = make(2, 4, 2, 33, 1, 64)
    _, _, (dq, dk, _) = check(q, k, v, do, "bf16")
    assert bool((dq == 0).all()) and bool((dk == 0).all())


def test_everything_dropped_and_nothing_there():
    q, k, v, do = make(2, 2, 2, 40, 40, 64)
    seed = seed_tensor(3)
    o, lse = forward(q, k, v, dropout_p=1.0, seed=seed)
    assert bool((o == 0).all()) and bool(torch.isfinite(lse).all())
    assert all(bool((g == 0).all()) for g in backward(q, k, v, o, lse, do, dropout_p=1.0, seed=seed))
    none = torch.empty(2, 0, 2, 64, dtype=torch.bfloat16, device=DEV)
    o, lse = forward(q, none, none)
    assert bool((o == 0).all()) and bool(torch.isneginf(lse).all())
    dq, _, _ = backward(q, none, none, o, lse, do)
    assert bool((dq == 0).all())
    o, lse = forward(none, k, v)
    _, dk, dv = backward(none, k, v, o, lse, none)
    assert bool((dk == 0).all()) and bool((dv == 0).all())


def test_another_stream():
    q, k, v, do = make(2, 2, 1, 100, 100, 64)
    o, lse = forward(q, k, v, causal=True)
    side = torch.cuda.Stream()
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    ws = workspace(q, k)
    torch.cuda.synchronize()
    okt.okt_attention_forward(q, k, v, o2, lse2, ws, causal=True, stream=side)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_a_graph_replays_with_new_inputs_and_seeds():
    q, k, v, do = (t.contiguous() for t in make(2, 4, 2, 150, 700, 64))
    seed, ws = seed_tensor(1), workspace(q, k)
    o, lse = torch.empty_like(q), torch.empty(2, 4, 150, device=DEV)
    grads = [torch.empty_like(t) for t in (q, k, v)]
    options = dict(dropout_p=0.1, seed=seed)

    def step_():
        okt.okt_attention_forward(q, k, v, o, lse, ws, **options)
        okt.okt_attention_backward(q, k, v, o, lse, do, *grads, ws, **options)

    step_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step_()
    for n in range(3):
        seed.fill_(40 + n)
        q.copy_(rand(q.shape, "bf16", 60 + n))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (o, lse, *grads)]
        step_()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (o, lse, *grads))), n


@pytest.mark.parametrize("D", [64, 128])
def test_backward_on_another_stream(D):
    q, k, v, do = make(2, 4, 2, 100, 700, D)
    o, lse = forward(q, k, v, causal=True)
    want = backward(q, k, v, o, lse, do, causal=True)
    side = torch.cuda.Stream()
    got = [torch.full(t.shape, 7.0, dtype=q.dtype, device=DEV) for t in (q, k, v)]
    ws = workspace(q, k)
    torch.cuda.synchronize()
    okt.okt_attention_backward(q, k, v, o, lse, do, *got, ws, causal=True, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def one_key_above_the_rest(H, K, above, kind, seen=1):
    """Keys of score 0 but for the first, whose score is `above`; values 1, that key's 0."""
    q = torch.zeros(1, seen, H, 64, dtype=TYPES[kind], device=DEV)
    q[..., 0] = 1.0
    k = torch.zeros(1, K, 1, 64, dtype=TYPES[kind], device=DEV)
    k[:, 0, :, 0] = above
    v = torch.ones_like(k)
    v[:, 0] = 0.0
    return q, k, v


@pytest.mark.parametrize("H,seen", [(300, 1), (2, 1), (3, 100)])
def test_small_probabilities_add_up_in_fp16(H, seen):
    """4095 keys 2^-25.6 of the largest: each is below the smallest fp16 number beside a 1.  o and dv are sums over
    them; each probability is at least 2^7 and 2^12 times that in the products, so it is off by 2^-32 and
    2^-37 at the most."""
    K, above = 4096, 17.75
    q, k, v = one_key_above_the_rest(H, K, above, "f16", seen)
    v *= 1000.0
    rest = np.exp(-above)
    total = 1 + (K - 1) * rest
    keys = [t.expand(1, K, H, 64).contiguous() for t in (k, v)]
    for ks, vs in ((k, v), keys):                              # shared by the heads, and one each
        o, lse = forward(q, ks, vs, scale=1.0)
        want = 1000.0 * (K - 1) * rest / total
        assert np.abs(wide(o) - want).max() <= 1000.0 * (K - 1) * 2.0 ** -32 + 2 * UNIT["f16"] * want
        assert np.abs(wide(lse) - (above + np.log(total))).max() <= 2.0 ** -24 * (16 + 8 * above)
        do = torch.full_like(q, 1000.0)
        _, _, dv = backward(q, ks, vs, o, lse, do, scale=1.0)
        rows = seen * (H if ks is k else 1)
        want = 1000.0 * rows * rest / total
        assert np.abs(wide(dv)[:, 1:] - want).max() <= 1000.0 * rows * 2.0 ** -37 + 2 * UNIT["f16"] * want + step("f16")
    # differences of the forward pass in the direction of v agree with dv where only v changes (o is linear in it)
    o2, _ = forward(q, keys[0], keys[1] * 2, scale=1.0)
    o1, _ = forward(q, keys[0], keys[1], scale=1.0)
    assert torch.equal(o2, o1 * 2)


@pytest.mark.parametrize("H", [300, 2])
def test_the_sum_of_very_many_probabilities(H):
    """A million keys of 0.3 of the largest: lse by the formula, within the roundings of one exponential, of a
    tile's sums, of the compensated sum over tiles and of the logarithm; on workgroups of their own and in parts."""
    K, above = 1 << 20, 1.2
    q, k, v = one_key_above_the_rest(H, K, above, "bf16")
    above = float(k[0, 0, 0, 0])
    ks, vs = (t.expand(1, K, H, 64) for t in (k, v))
    o, lse = forward(q, ks, vs, scale=1.0)
    rest = np.exp(-above)
    total = 1 + (K - 1) * rest
    want = above + np.log(total)
    assert np.abs(wide(lse) - want).max() <= 2.0 ** -24 * (24 + 8 * want)
    assert np.abs(wide(o) - (K - 1) * rest / total).max() <= 2 * UNIT["bf16"]


@pytest.mark.parametrize("kind,p", [("bf16", 0.0), ("f16", 0.1)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_many_tiles_a_workgroup(D, causal, kind, p):
    """More blocks than are split: fifteen tiles of keys and as many of queries pass by a workgroup, four heads a group."""
    lens = ([900, 700, 900, 1, 333], [900, 900, 451, 900, 1])
    q, k, v, do = make(5, 8, 2, 900, 900, D, kind)
    check(q, k, v, do, kind, causal=causal, p=p)
    check(q, k, v, do, kind, causal=causal, p=p, lens=lens)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,H,G,Sq,Sk,D", [(4, 6, 6, 2, 2, 128), (3, 2, 2, 6, 6, 64), (5, 4, 2, 1, 45, 64), (1, 8, 4, 10, 44, 128),
                                           (2, 13, 13, 27, 27, 16), (1, 2, 1, 180, 180, 64), (1, 4, 4, 2, 5000, 40), (1, 2, 2, 3000, 7, 128)])
def test_few_pairs_are_rounded_once(monkeypatch, B, H, G, Sq, Sk, D, causal, p, kind):
    """Up to 2^16 pairs p and ds go into the products in two parts: what is left of their rounding is twice the square of
    one, and the outputs are off by little more than their own."""
    q, k, v, do = make(B, H, G, Sq, Sk, D, kind)
    options = dict(causal=causal, dropout_p=p, site=2, seed=seed_tensor(SEED) if p else None)
    plain = dict(causal=causal, scale=D ** -0.5, q_lens=None, k_lens=None, dropout_p=p, seed=SEED & ((1 << 64) - 1), site=2)
    Q, KK, V, DO = (wide(t) for t in (q, k, v, do))
    u, least = UNIT[kind], step(kind)
    o, lse = forward(q, k, v, **options)
    want_o, _ = ops.attention(Q, KK, V, **plain)
    got, want = backward(q, k, v, o, lse, do, **options), ops.attention_backward(Q, KK, V, DO, **plain)
    monkeypatch.setitem(UNIT, kind, 2 * u * u)
    bo, _ = attention_bounds(Q, KK, V, kind, **plain)
    stored = bo * (1 + u) + u * np.abs(want_o) + least
    within(o, want_o, stored, "o")
    for name, g, w, b in zip(("dq", "dk", "dv"), got, want, attention_bounds(Q, KK, V, kind, do=DO, o=stored, **plain)):
        within(g, w, b * (1 + u) + u * np.abs(w) + least, name)
