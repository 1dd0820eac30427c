"""The oracle of the operators at the ends of a training step, pinned by loops over single numbers, by differences and by the
type's own conversions."""
import math

import numpy as np
import pytest
import torch

from oracle import okt_training as ref


def difference(f, x, way, eps=1e-6):
    return (f(x + eps * way) - f(x - eps * way)) / (2 * eps)


def test_e4m3_values_are_the_type():
    codes = torch.arange(127, dtype=torch.uint8)
    assert np.array_equal(ref.e4m3_values(), codes.view(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(float(torch.tensor([127], dtype=torch.uint8).view(torch.float8_e4m3fn).double()))
    assert ref.from_e4m3(np.array([0, 1, 129, 126], np.uint8), np.array([0.5], np.float32)).tolist() == [0.0, 2.0 ** -10, -2.0 ** -10, 224.0]


def test_block_scales():
    for top in (1.0, 1.75, 1.7500001, 2.0, 448.0, 448.0001, 3e38, 1e-30):
        s = ref.block_scale(np.array([0.0, -np.float32(top)]))
        assert 224.0 < abs(float(np.float32(top))) / s <= 448.0 and math.log2(s) == int(math.log2(s))
    assert ref.block_scale(np.zeros(3)) == 2.0 ** -126 and np.isnan(ref.block_scale(np.array([np.nan, 1.0]))) and np.isnan(ref.block_scale(np.array([np.inf])))


def test_rounding_to_e4m3():
    """Without random bits the nearest value; with all of them the value (or its square) on average."""
    x = np.random.default_rng(0).standard_normal(256).astype(np.float32)
    table = ref.e4m3_values()
    codes, scale = ref.to_e4m3(x, np.full(256, 0x8000))
    for v, got in zip(x, ref.from_e4m3(codes, scale)):
        assert abs(abs(v) - abs(got)) <= np.abs(table * scale[0] - abs(v)).min() * (1 + 1e-6) and np.sign(v) * got >= 0
    x[:5] = [0.0, 1e-6, 3.0, -2.5e-3, 1.9]
    mean, square = 0.0, 0.0
    for r in range(0, 65536, 64):
        mean = mean + ref.from_e4m3(*ref.to_e4m3(x, np.full(256, r))) / 1024
        square = square + ref.from_e4m3(*ref.to_e4m3_root(x * x, np.full(256, r))) ** 2 / 1024
    step = np.abs(np.diff(table)).max() * scale[0]
    assert np.abs(mean - x).max() <= step / 1024 * 2
    above = np.abs(x) >= 2.0 ** -9 * scale[0]                        # below that a root becomes the least value, not 0
    assert np.abs(square - x.astype(np.float64) ** 2)[above].max() <= 2 * 448.0 * scale[0] * step / 1024 * 2
    assert (ref.to_e4m3_root(x * x, np.zeros(256, int))[0][1:5] > 0).all() and ref.to_e4m3_root(x * x, np.zeros(256, int))[0][0] == 0


def test_adamw_one_number_at_a_time():
    rng = np.random.default_rng(1)
    p, m, v = rng.standard_normal(7), np.zeros(7), np.zeros(7)
    for t in range(1, 5):
        g = rng.standard_normal(7)
        want = []
        for i in range(7):
            mi, vi = 0.8 * m[i] + 0.2 * (0.5 * g[i]), 0.9 * v[i] + 0.1 * (0.5 * g[i]) ** 2
            want.append((p[i] * (1 - 0.02 * 0.3) - 0.02 * (mi / (1 - 0.8 ** t)) / (math.sqrt(vi / (1 - 0.9 ** t)) + 1e-3), mi, vi))
        p, m, v = ref.adamw(p, g, m, v, step=t, lr=0.01, beta1=0.8, beta2=0.9, eps=1e-3, weight_decay=0.3, rate_scale=2.0, grad_scale=0.5)
        assert np.allclose(np.array(want).T, [p, m, v], rtol=1e-13, atol=0)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("kind,normed", [("rms", True), ("layer", True), ("rms", False)])
def test_norm_rotary(adjacent, kind, normed):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((2, 3, 2, 8)), rng.standard_normal((2, 3, 2, 8))
    weight = rng.standard_normal(8) if normed else None
    positions, axes = rng.integers(-50, 50, (2, 3, 2)), [0, 1, 1]
    freq = np.array([1.0, 0.25, 0.01])
    angle = ref.angles(2, 3, freq, positions, axes)
    options = dict(kind=kind, eps=1e-3, adjacent=adjacent)
    y = ref.norm_rotary(x, angle, weight=weight, **options)
    for b, i, h in np.ndindex(2, 3, 2):
        v = x[b, i, h]
        if normed:
            c = v - (v.mean() if kind == "layer" else 0.0)
            v = c / math.sqrt((c * c).mean() + 1e-3) * weight
        want = v.copy()
        for j in range(3):
            p, q = (2 * j, 2 * j + 1) if adjacent else (j, j + 3)
            t = positions[b, i, axes[j]] * freq[j]
            want[p], want[q] = v[p] * math.cos(t) - v[q] * math.sin(t), v[p] * math.sin(t) + v[q] * math.cos(t)
        assert np.allclose(y[b, i, h], want, atol=1e-12)
    dx, dw = ref.norm_rotary_backward(x, dy, angle, weight=weight, **options)
    way = rng.standard_normal(x.shape)
    assert np.isclose((dx * way).sum(), difference(lambda z: (ref.norm_rotary(z, angle, weight=weight, **options) * dy).sum(), x, way), atol=1e-7)
    if normed:
        way = rng.standard_normal(8)
        assert np.isclose((dw * way).sum(), difference(lambda z: (ref.norm_rotary(x, angle, weight=z, **options) * dy).sum(), weight, way), atol=1e-7)


def test_angles_of_far_places():
    angle = ref.angles(1, 1, np.array([1.0]), np.array([[[10 ** 9]]]))[0, 0, 0, 0]
    # 10^9 mod 2 pi, from pi to 40 digits in whole numbers
    two_pi = 2 * 3141592653589793238462643383279502884197
    want = (10 ** 9 * 10 ** 39 % two_pi) / 10 ** 39
    assert abs(angle - want) < 1e-9


def test_cross_entropy():
    rng = np.random.default_rng(3)
    h, w, b = rng.standard_normal((6, 4)), rng.standard_normal((5, 4)), rng.standard_normal(5)
    y, g = np.array([0, 4, -100, 2, 5, 1 << 40]), rng.standard_normal(6)
    loss, lse = ref.cross_entropy(h, w, y, b)
    for n in range(6):
        s = [float(h[n] @ w[v] + b[v]) for v in range(5)]
        whole = math.log(sum(math.exp(x) for x in s))
        there = 0 <= y[n] < 5
        assert math.isclose(loss[n], whole - s[y[n]] if there else 0.0, abs_tol=1e-12) and math.isclose(lse[n], whole if there else 0.0, abs_tol=1e-12)
    got = ref.cross_entropy_backward(h, w, y, g, b)
    for n, x in enumerate((h, w, b)):
        way = rng.standard_normal(x.shape)
        assert np.isclose((got[n] * way).sum(), difference(
            lambda z: (ref.cross_entropy(*[z if k == n else o for k, o in enumerate((h, w))], y, z if n == 2 else b)[0] * g).sum(), x, way), atol=1e-7)
    assert not got[0][[2, 4, 5]].any()
