"""The oracle of the layer's operators against published values of its generator, against
differences of its own forward passes, and against the properties its formulas have."""
import numpy as np
import pytest

from oracle import okt_operators as ops


def test_generator_gives_the_published_values():
    # known answers of Philox4x32 at all-zero and all-one counters and keys
    assert [hex(w) for w in ops.philox(0, 0, 0, 0, 0, rounds=7)] == ["0x5f6fb709", "0xd893f64", "0x4f121f81", "0x4f730a48"]
    assert [hex(w) for w in ops.philox(0, 0, 0, 0, 0, rounds=10)] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    ones = 0xFFFFFFFF
    assert [hex(w) for w in ops.philox(ones, ones, ones, ones, (1 << 64) - 1, rounds=10)] == [
        "0x408f276d", "0x41c83b0e", "0xa20bc7c6", "0x6d5451fd"]


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_share_that_is_kept(p):
    n = 400_000
    kept = ops.kept_flat(n, p, seed=7, site=3)
    want = ops.bar_of(p) / 65536
    assert abs(kept.mean() - want) <= 5 * np.sqrt(max(want * (1 - want), 1e-12) / n)
    # neighbours, and two sites, agree as often as independent draws do
    for a, b in ((kept[:-1], kept[1:]), (kept, ops.kept_flat(n, p, seed=7, site=4))):
        both = want * want
        assert abs((a & b).mean() - both) <= 6 * np.sqrt(max(both * (1 - both), 1e-12) / n)
    assert abs(ops.bar_of(p) / 65536 * ops.scale_of(p) - (1 if p < 1 else 0)) < 1e-12


def test_the_three_numberings_read_the_same_field():
    words = ops.values(ops.philox(5, 3, 2, 9, seed=11))
    assert np.array_equal(ops.kept_pairs(2, 8, 24, 0.3, 11, 9)[6:8, 20:24].T.reshape(-1), words < ops.bar_of(0.3))
    rows = ops.values(ops.philox(5, 3, 0, 9, seed=11))
    assert np.array_equal(ops.kept_rows(4, 48, 0.3, 11, 9)[3, 40:48], rows < ops.bar_of(0.3))
    flat = ops.values(ops.philox(1, 1, 0, 9, seed=11))
    assert np.array_equal(ops.kept_flat(8, 0.3, 11, 9, first=8 * ((1 << 32) + 1)), flat < ops.bar_of(0.3))


def difference(f, x, d, step=1e-6):
    """Directional derivative of f at x along d."""
    return (f(x + step * d) - f(x - step * d)) / (2 * step)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("post,pre,gates", [(False, True, 0), (True, True, 1), (True, False, 3), (False, True, 2),
                                            (False, False, 1), (True, True, 7)])
def test_norm_gradients_match_differences(kind, post, pre, gates):
    rng = np.random.default_rng(5)
    rows, width = 7, 19
    share = -(-rows // gates) if gates else 0
    arg = {"u": rng.standard_normal((rows, width)), "x": rng.standard_normal((rows, width))}
    for name, there in (("post", post), ("pre", pre)):
        if there:
            arg[name + "_weight"] = 1 + 0.2 * rng.standard_normal(width)
            arg[name + "_bias"] = rng.standard_normal(width)
    if gates:
        arg["gate"] = rng.standard_normal((-(-rows // share), width))
    factor = ops.norm_factor(rows, width, 0.3, 99, 2)
    dh, dy = rng.standard_normal((rows, width)), rng.standard_normal((rows, width))
    fixed = dict(kind=kind, residual_scale=0.7, rows_per_gate=share, factor=factor)

    def loss(values):
        h, y, _ = ops.residual_norm(**values, **fixed)
        return (h * dh).sum() + ((y * dy).sum() if pre else 0.0)

    h, _, stats = ops.residual_norm(**arg, **fixed)
    given = {k: v for k, v in arg.items() if k not in ("x", "u", "pre_bias")}
    got = ops.residual_norm_backward(arg["u"], h, stats, dh, dy if pre else None, **given, **fixed)
    for name in arg:
        d = rng.standard_normal(arg[name].shape)
        want = difference(lambda v: loss({**arg, name: v}), arg[name], d)
        # central differences at step 1e-6: truncation ~1e-12, rounding of the losses ~1e-9 of their size
        assert abs((got["d" + name] * d).sum() - want) <= 1e-6 * (1 + abs(want)), name


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("sq,sk,lens", [(6, 6, None), (5, 9, None), (9, 5, None), (7, 8, ([7, 3, 0], [0, 8, 5])),
                                        (1, 1, None)])
@pytest.mark.parametrize("p", [0.0, 0.4])
def test_attention_gradients_match_differences(causal, sq, sk, lens, p):
    rng = np.random.default_rng(6)
    B, H, G, D = 3, 4, 2, 8
    arg = {"q": rng.standard_normal((B, sq, H, D)), "k": rng.standard_normal((B, sk, G, D)),
           "v": rng.standard_normal((B, sk, G, D))}
    do = rng.standard_normal((B, sq, H, D))
    fixed = dict(causal=causal, dropout_p=p, seed=12345678901, site=4,
                 q_lens=lens and lens[0], k_lens=lens and lens[1])
    got = dict(zip("qkv", ops.attention_backward(**arg, do=do, **fixed)))
    for name in arg:
        d = rng.standard_normal(arg[name].shape)
        want = difference(lambda x: (ops.attention(**{**arg, name: x}, **fixed)[0] * do).sum(), arg[name], d)
        assert abs((got[name] * d).sum() - want) <= 1e-6 * (1 + abs(want)), name


def test_rows_that_see_nothing():
    rng = np.random.default_rng(8)
    q, k, v = (rng.standard_normal((1, n, 1, 8)) for n in (5, 3, 3))
    o, lse = ops.attention(q, k, v, causal=True)                    # the first two queries see no key
    assert np.all(o[0, :2] == 0) and np.all(np.isneginf(lse[0, 0, :2])) and np.all(np.isfinite(lse[0, 0, 2:]))
    dq, dk, dv = ops.attention_backward(q, k, v, np.ones_like(q), causal=True)
    assert np.all(dq[0, :3] == 0)                                   # the third sees one key: constant
    # every row's values add up to what its queries sent
    assert np.allclose(dv.sum(), 8 * 3)


def test_what_is_dropped_does_not_matter():
    rng = np.random.default_rng(9)
    rows, width = 6, 24
    u, x, dh = (rng.standard_normal((rows, width)) for _ in range(3))
    gate = rng.standard_normal((2, width))
    factor = ops.norm_factor(rows, width, 0.4, 99, 2)
    fixed = dict(gate=gate, rows_per_gate=3, factor=factor)
    clean = ops.residual_norm(u, x, **fixed)[0], ops.residual_norm_backward(u, None, np.zeros((rows, 4)), dh, None, **fixed)
    u[factor == 0] = np.inf
    with np.errstate(invalid="ignore"):
        h, back = ops.residual_norm(u, x, **fixed)[0], ops.residual_norm_backward(u, None, np.zeros((rows, 4)), dh, None, **fixed)
    assert np.array_equal(h, clean[0])
    assert all(np.array_equal(back[n], clean[1][n]) for n in ("dx", "du", "dgate"))
