"""okt_cross_entropy_forward / _backward against the 64-bit oracle: tiles of both sizes, ragged rows, widths and vocabularies, several
pieces, rows without a label, with bounds that add up the roundings."""
import numpy as np
import pytest
import torch

import paper_2201_07598_amd as okt
from operators_harness import DEV, E, TYPES, UNIT, rand, step as least, wide, within
from oracle import okt_training as ref

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, rows=5, width=64, vocab=50, kind="bf16", labelled=1.0, bias=False, scale=2.0, seed=0, one_g=False, pad=0, wide_dw=False):
        self.rows, self.width, self.vocab, self.kind = rows, width, vocab, kind
        self.h = rand((rows, width + pad), kind, seed)[:, :width]
        self.weight = rand((vocab, width + 2 * pad), kind, seed + 1, scale * width ** -0.5)[:, :width]
        self.bias = rand((vocab,), "f32", seed + 2, 0.5) if bias else None
        gen = torch.Generator().manual_seed(seed + 3)
        y = torch.randint(vocab, (rows,), generator=gen)
        out = torch.tensor([-100, -1, vocab, 1 << 40])[torch.randint(4, (rows,), generator=gen)]
        self.y = torch.where(torch.rand(rows, generator=gen) < labelled, y, out)
        self.labels = self.y.to(DEV)
        g = torch.randn(rows, generator=gen) / rows
        self.g = torch.full((1,), 1.0 / rows, device=DEV) if one_g else g.to(DEV)
        self.pad, self.wide_dw = pad, wide_dw
        self.ws = torch.full((okt.okt_cross_entropy_workspace_bytes(rows, width, vocab),), 255, dtype=torch.uint8, device=DEV)

    def numbers(self):
        return wide(self.h), wide(self.weight), self.y.numpy(), None if self.bias is None else wide(self.bias)

    def forward(self, lse=True):
        loss = torch.full((self.rows,), 7.0, device=DEV)
        lse = torch.full((self.rows,), 7.0, device=DEV) if lse else None
        okt.okt_cross_entropy_forward(self.h, self.weight, self.labels, loss, lse, self.ws, bias=self.bias)
        return loss, lse

    def backward(self, lse, dh=True, dw=True, db=True):
        room = lambda n, by, t: torch.full((n, self.width + by), 7.0, dtype=t, device=DEV)  # noqa: E731
        t = TYPES[self.kind]
        dh = room(self.rows, self.pad, t)[:, :self.width] if dh else None
        dw = room(self.vocab, 3 * self.pad, torch.float32 if self.wide_dw else t)[:, :self.width] if dw else None
        db = torch.full((self.vocab,), 7.0, device=DEV) if db and self.bias is not None else None
        okt.okt_cross_entropy_backward(self.h, self.weight, self.labels, lse, self.g, dh, dw, self.ws, bias=self.bias, dbias_out=db)
        return dh, dw, db


def logit_errors(h, w, b):
    """A logit: products of 16-bit values are exact, their fp32 sum has width + 8 additions; the bias's."""
    one = (h.shape[1] + 8) * E * (np.abs(h) @ np.abs(w).T)
    s = ref.logits(h, w, b)
    return s, one + E * np.abs(np.where(np.isfinite(s), s, 0.0))


def lse_error(s, one):
    """The largest logit's error moves lse by as much; exponents are rounded at the size of a logit (thrice: product, scaled
    largest, and when parts are joined), exponentials and 80 additions (64 in a lane, then parts in sixteen by sixteen)."""
    size = np.abs(np.where(np.isfinite(s), s, 0.0)).max(1)
    parts = s.shape[1] // 64 // 16 + 16
    return one.max(1) + 6 * E * size + (64 + 8 + 3 * parts) * E


def check(c, loss, lse, grads=None):
    h, w, y, b = c.numbers()
    rows = np.flatnonzero((y >= 0) & (y < c.vocab))
    want_loss, want_lse = ref.cross_entropy(h, w, y, b)
    s, one = logit_errors(h[rows], w, b)
    e_lse = np.zeros(c.rows)
    e_lse[rows] = lse_error(s, one)
    said = np.zeros(c.rows)
    said[rows] = one[np.arange(len(rows)), y[rows]]
    if lse is not None:
        within(lse, want_lse, e_lse + 4 * E * np.abs(want_lse), "lse")
    within(loss, want_loss, e_lse + said + 4 * E * (np.abs(want_lse) + np.abs(want_loss)), "loss")
    if grads is None:
        return
    g = np.broadcast_to(wide(c.g), (c.rows,))
    u, tiny = UNIT[c.kind], 0.0
    if c.kind == "f16" and len(rows):
        tiny = 2.0 ** -25 * np.abs(g[rows]).max() * 2.0 ** -14
    p = np.exp(s - want_lse[rows, None])
    d = np.abs(g[rows, None]) * np.abs(p - (np.arange(c.vocab) == y[rows, None]))
    size = np.abs(np.where(np.isfinite(s), s, 0.0))
    e_p = p * (one + e_lse[rows, None] + E * (8 + 3 * size + 4 * np.abs(want_lse[rows, None])))
    e_d = np.abs(g[rows, None]) * (e_p + 2.0 ** -126) + 2 * E * d         # an exponential below 2^-126 may be 0
    e_r = e_d + u * (d + e_d) + tiny                     # as the second products read it
    dh, dw, db = ref.cross_entropy_backward(h, w, y, g, b)
    full = np.zeros(h.shape)
    # additions: over the piece's k in the unit, then pieces or parts
    full[rows] = (e_r + (c.vocab + 600) * E * d) @ np.abs(w)
    if grads[0] is not None:
        within(grads[0], dh, full + u * (np.abs(dh) + full) + least(c.kind), "dh")
    if grads[1] is not None:
        bound = (e_r + (len(rows) + 8) * E * d).T @ np.abs(h[rows])
        within(grads[1], dw, bound + E * np.abs(dw) if c.wide_dw else bound + u * (np.abs(dw) + bound) + least(c.kind), "dweight")
    if grads[2] is not None:
        within(grads[2], db, (e_d + (len(rows) + 40) * E * d).sum(0), "dbias")


CASES = [
    dict(rows=1, width=8, vocab=1), dict(rows=1, width=8, vocab=2, bias=True), dict(rows=3, width=8, vocab=5, kind="f16", bias=True),
    dict(rows=125, width=776, vocab=1003, kind="f16"), dict(rows=128, width=64, vocab=256, bias=True), dict(rows=129, width=72, vocab=257, one_g=True),
    dict(rows=260, width=136, vocab=520, labelled=0.5, bias=True), dict(rows=513, width=200, vocab=300, labelled=0.15, kind="f16", bias=True),
    dict(rows=40, width=120, vocab=130, pad=8, labelled=0.7), dict(rows=300, width=320, vocab=1000, scale=12.0, bias=True),
    dict(rows=300, width=64, vocab=777, labelled=0.6, wide_dw=True, pad=8, bias=True, kind="f16"),
    dict(rows=2600, width=64, vocab=5001, bias=True, labelled=0.8),               # logits in large tiles
    dict(rows=2600, width=88, vocab=5100, kind="f16", labelled=0.97),
    dict(rows=140, width=1112, vocab=10_300, bias=True),                            # dweight in large tiles
    dict(rows=140, width=1112, vocab=10_300, kind="f16", wide_dw=True),
    dict(rows=1300, width=328, vocab=200, bias=True), dict(rows=2500, width=136, vocab=130, kind="f16", wide_dw=True, labelled=0.9, pad=8),   # dweight in parts
    dict(rows=300, width=520, vocab=6000, bias=True, one_g=True),                   # dh in parts
    dict(rows=257, width=64, vocab=600), dict(rows=256, width=64, vocab=600, kind="f16"),
    dict(rows=65_000, width=64, vocab=9001, labelled=0.006, bias=True),             # three pieces, few rows among many
    dict(rows=131_000, width=72, vocab=4300, labelled=0.03, bias=True),             # two pieces, the last one's dweight in parts
    dict(rows=65_000, width=40, vocab=4097, labelled=0.02, kind="f16", one_g=True)]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_loss_and_gradients(n):
    c = Case(**CASES[n], seed=10 * n)
    loss, lse = c.forward()
    grads = c.backward(lse)
    check(c, loss, lse, grads)
    # where nothing is labelled the gradient is 0, and between rows nothing is written
    out = torch.from_numpy((c.y.numpy() < 0) | (c.y.numpy() >= c.vocab)).to(DEV)
    assert not grads[0][out].any() and not loss[out].any() and not lse[out].any()
    if c.pad:
        for g in grads[:2]:
            base = g._base.clone()
            base[:, :c.width] = 7.0
            assert (base == 7.0).all()


def test_no_row_has_a_label():
    c = Case(rows=300, width=64, vocab=500, labelled=0.0, bias=True)
    loss, lse = c.forward()
    grads = c.backward(lse)
    assert not loss.any() and not lse.any() and all(not g.any() for g in grads)


def test_no_rows():
    c = Case(rows=0, width=64, vocab=500, bias=True)
    loss, lse = c.forward()
    dh, dw, db = c.backward(lse)
    assert not dw.any() and not db.any()


def test_rows_without_a_label_may_hold_anything():
    c = Case(rows=400, width=128, vocab=600, labelled=0.5, bias=True, seed=3)
    clean = [*c.forward(), *c.backward(c.forward()[1])]
    out = (c.labels < 0) | (c.labels >= c.vocab)
    c.h[out] = float("nan")
    c.g[out] = float("inf")
    loss, lse = c.forward()
    for a, b in zip(clean, [loss, lse, *c.backward(lse)]):
        assert torch.equal(a, b)                         # the same bits, and the same from run to run


def test_not_finite_stays_in_its_row():
    c = Case(rows=300, width=64, vocab=500, seed=4)
    clean_loss, clean = c.forward()
    clean_dh = c.backward(clean)[0]
    c.h[7, 3], c.h[200, 5] = float("nan"), float("inf")
    loss, lse = c.forward()
    dh = c.backward(lse)[0]
    assert torch.isnan(loss[7]) and not torch.isfinite(loss[200])
    rest = torch.ones(300, dtype=torch.bool, device=DEV)
    rest[7] = rest[200] = False
    assert torch.equal(loss[rest], clean_loss[rest]) and torch.equal(dh[rest], clean_dh[rest])


def test_entries_taken_out_by_the_bias():
    c = Case(rows=200, width=64, vocab=700, bias=True, seed=5)
    kept = torch.zeros(700, dtype=torch.bool)
    kept[c.y] = True
    kept[::3] = True
    kept[256:512] = False                                # a whole tile without any
    kept[c.y] = True
    c.bias[~kept.to(DEV)] = -float("inf")
    loss, lse = c.forward()
    dh, dw, db = c.backward(lse)
    check(c, loss, lse, (dh, dw, db))
    assert not dw[~kept.to(DEV)].any() and not db[~kept.to(DEV)].any()


def test_gradients_of_differences():
    """Along a direction in each input, by central differences of the sum of losses in 64 bits at the inputs as they are."""
    c = Case(rows=60, width=48, vocab=90, bias=True, kind="f16", seed=6, labelled=0.8)
    loss, lse = c.forward()
    grads = c.backward(lse)
    h, w, y, b = c.numbers()
    g, rng, eps = wide(c.g), np.random.default_rng(0), 1e-5
    for n, x in enumerate((h, w, b)):
        way = rng.standard_normal(x.shape)
        at = [[h, w, b], [h, w, b]]
        at[0][n], at[1][n] = x + eps * way, x - eps * way
        up, down = ((ref.cross_entropy(a[0], a[1], y, a[2])[0] * g).sum() for a in at)
        got = (wide(grads[n]) * way).sum()
        size = (np.abs(wide(grads[n])) * np.abs(way)).sum()
        assert abs((up - down) / (2 * eps) - got) <= 4 * UNIT["f16"] * size + 1e-7, n


def test_some_gradients_alone():
    c = Case(rows=300, width=64, vocab=500, labelled=0.5, bias=True, seed=7)
    _, lse = c.forward()
    all_three = c.backward(lse)
    for which in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        for want, got, there in zip(all_three, c.backward(lse, *which), which):
            assert (got is not None) == there and (got is None or torch.equal(got, want))
    loss = c.forward()[0]
    assert torch.equal(c.forward(lse=False)[0], loss)


def test_replayed_and_on_another_stream():
    one, two = (Case(rows=500, width=96, vocab=1500, labelled=0.3, bias=True, seed=8) for _ in range(2))

    def both(c):
        loss, lse = c.out[:2]
        okt.okt_cross_entropy_forward(c.h, c.weight, c.labels, loss, lse, c.ws, bias=c.bias)
        okt.okt_cross_entropy_backward(c.h, c.weight, c.labels, lse, c.g, c.out[2], c.out[3], c.ws, bias=c.bias, dbias_out=c.out[4])

    for c in (one, two):
        c.out = [torch.zeros(500, device=DEV), torch.zeros(500, device=DEV), torch.zeros_like(c.h), torch.zeros_like(c.weight), torch.zeros_like(c.bias)]
    both(one)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        both(one)
    for n in range(3):
        gen = torch.Generator().manual_seed(n)
        y = torch.randint(-1500 * n, 1500, (500,), generator=gen).to(DEV)            # another number of rows with a label
        for c in (one, two):
            c.h.mul_(0.75)
            c.labels.copy_(y)
            for t in c.out:
                t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            both(two)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(one.out, two.out)), n


def test_a_large_bias():
    """Rows behind the last one see the bias alone, whose exponential need not be finite."""
    c = Case(rows=130, width=64, vocab=300, bias=True, seed=9)
    c.bias[5], c.bias[7] = 150.0, 149.0
    loss, lse = c.forward()
    check(c, loss, lse, c.backward(lse))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,one_g", [(300, True), (300, False), (2600, True), (7, False)])
def test_a_gradient_that_all_rows_share_is_not_rounded(rows, one_g, kind):
    """A mean's gradient stands half a step between two values of the type; it is every row's, so rounding it would move the whole result
    one way.  With W = 0 all p are 2^-10, and of the entries of d only 1 - 2^-10 is rounded, to 1 in bfloat16."""
    vocab, g = 1024, (1.0 + UNIT[kind]) * 2.0 ** -11
    c = Case(rows, 64, vocab, kind, bias=True, wide_dw=True, seed=90 + rows)
    c.weight.zero_()
    c.bias.zero_()
    c.g = torch.full((1 if one_g else rows,), g, device=DEV)
    loss, lse = c.forward()
    dh, dw, db = c.backward(lse)
    h, w, y, b = c.numbers()
    _, want, want_db = ref.cross_entropy_backward(h, w, y, np.full(rows, g), b)
    said = (np.arange(vocab)[:, None] == y) * 1.0
    rounded = 0.0 if kind == "f16" or rows <= 256 else 2.0 ** -10
    # p: lse's seven and the exponent's units of fp32 at the size 10, thus 2^-16 of p; an entry of d eight units, a sum's additions
    one = g * (2.0 ** -10 * 2.0 ** -16 + (8 + rows) * E * (2.0 ** -10 + said))
    within(dw, want, (g * rounded * said + one) @ np.abs(h), "dweight")
    within(db, want_db, one.sum(1), "dbias")
    assert (dh == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("labelled", [1.0, 0.4, 0.004, 0.0])
@pytest.mark.parametrize("rows,vocab", [(2048, 700), (2049, 700), (2048, 1030), (1, 16_385), (129, 8193), (120, 40_000)])
def test_rows_as_they_lie_and_side_by_side(rows, vocab, labelled, kind):
    """Up to 2048 rows are read as they lie where tiles are few, from 2049 on they are laid side by side; tiles of 64 columns, one too many of them for the
    CUs, more tiles than one a CU.  Between the rows there is NaN, as in those without a label."""
    c = Case(rows, 136, vocab, kind, labelled, bias=True, seed=95, pad=8)
    c.h._base[:, 136:] = float("nan")
    c.h[(c.labels < 0) | (c.labels >= vocab)] = float("nan")
    loss, lse = c.forward()
    c.h[(c.labels < 0) | (c.labels >= vocab)] = 0.0
    check(c, loss, lse)
    again = c.forward()
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)


@pytest.mark.parametrize("rows", [1024, 1025])
def test_rows_far_apart(rows):
    """The last one begins just below 2^31 bytes behind the first, and at it, where 32-bit offsets from the first row end."""
    c = Case(rows, 64, 300, labelled=0.9, seed=96)
    far = torch.full((rows, 1 << 20), float("nan"), dtype=torch.bfloat16, device=DEV)
    far[:, :64] = c.h
    c.h = far[:, :64]
    check(c, *c.forward())
