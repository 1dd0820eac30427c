"""The operators at the ends of a training step where numbers end: infinities and NaN beside finite values, losses of nothing,
denominators near nothing."""
import pytest
import torch

import paper_2201_07598_amd as okt
from operators_harness import DEV, rand
from test_gpu_adamw import State, int64
from test_gpu_cross_entropy import Case as Loss
from test_gpu_norm_rotary import Case, run_forward

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), nan=1e30, posinf=2e30, neginf=-2e30), torch.nan_to_num(b.float(), nan=1e30, posinf=2e30, neginf=-2e30))


# ------------------------------------------------------------------ rotation

UNROTATED = [(kind, dim, rot, adjacent) for kind in ("f32", "bf16", "f16") for dim, rot in ((64, 32), (80, 0), (128, 120), (256, 8)) for adjacent in (False, True)]


def spoil(t, clean, rot):
    """Every element from `rot` on in a token of its own, in heads 0 to 2; where `clean` is what comes of it, it goes there as well."""
    for i, e in enumerate(range(rot, t.shape[-1])):
        for head, value in enumerate((INF, -INF, NAN)):
            t[0, i, head, e] = value
            clean[0, i, head, e] = value


@pytest.mark.parametrize("kind,dim,rot,adjacent", UNROTATED)
def test_what_is_not_rotated_stays_beside_anything(kind, dim, rot, adjacent):
    c = Case(batch=1, length=dim - rot, heads=4, kv_heads=3, dim=dim, rot=rot, kind=kind, norm=None, adjacent=adjacent, seed=20)
    clean = run_forward(c)
    spoil(c.q, clean[0], rot)
    spoil(c.k, clean[1], rot)
    for got, want in zip(run_forward(c), clean):
        assert same(got, want)


@pytest.mark.parametrize("kind,dim,rot,adjacent", UNROTATED)
def test_gradients_of_what_is_not_rotated_stay_beside_anything(kind, dim, rot, adjacent):
    c = Case(batch=1, length=dim - rot, heads=4, kv_heads=3, dim=dim, rot=rot, kind=kind, norm=None, adjacent=adjacent, seed=21)
    grads = [rand(c.q.shape, kind, 1), rand(c.k.shape, kind, 2)]
    outs = [[torch.zeros_like(t) for t in grads] for _ in range(2)]
    okt.okt_norm_rotary_backward(c.q, c.k, *grads, *outs[0], c.inv_freq, **c.options)
    for g, clean in zip(grads, outs[0]):
        spoil(g, clean, rot)
    okt.okt_norm_rotary_backward(c.q, c.k, *grads, *outs[1], c.inv_freq, **c.options)
    for got, want in zip(outs[1], outs[0]):
        assert same(got, want)


@pytest.mark.parametrize("kind,dim,rot,adjacent", UNROTATED)
def test_normed_heads_with_an_infinity(kind, dim, rot, adjacent):
    """The mean square is infinite and its root's reciprocal 0, so what is finite becomes 0 and the infinity itself NaN."""
    c = Case(batch=1, length=dim - rot, heads=4, kv_heads=3, dim=dim, rot=rot, kind=kind, adjacent=adjacent, seed=22)
    clean = run_forward(c)
    for t, want in zip((c.q, c.k), clean):
        want[0, :, 0] = 0.0
        for i, e in enumerate(range(rot, dim)):
            t[0, i, 0, e] = INF
            want[0, i, 0, e] = NAN
    for got, want in zip(run_forward(c), clean):
        assert same(got + 0.0, want)


@pytest.mark.parametrize("places", ["one row for all", "a row a sequence"])
def test_positions_of_several_axes_turned_by_the_first(places):
    """Without axis_of_pair the first axis turns all pairs, however many the positions have."""
    c = Case(batch=2, length=6, seed=23)
    room = torch.randint(0, 1000, (6, 3) if places == "one row for all" else (2, 6, 3), generator=torch.Generator().manual_seed(1)).to(torch.int32).to(DEV)
    first = room[..., 0].contiguous().expand(2, 6).unsqueeze(-1)
    c.options["positions"] = first
    want = run_forward(c)
    c.options["positions"] = room
    for got, plain in zip(run_forward(c), want):
        assert torch.equal(got, plain)


# ------------------------------------------------------------------ cross entropy

@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,bias", [(3, 1, False), (300, 1, True), (2100, 1, False), (300, 700, False), (130, 9000, True), (2600, 5001, True)])
def test_a_sure_row_has_no_loss_and_no_gradient(rows, vocab, bias, kind):
    """One logit, of 10 to 300, is 140 or more above all others (or the only one): its exponential is the whole sum, to the last bit."""
    c = Loss(rows, 64, vocab, kind, bias=bias, seed=30)
    c.weight.zero_()
    c.weight[:, 0] = -1.0
    c.weight[0, 0] = 1.0
    c.labels.zero_()
    c.y = c.labels.cpu()
    c.h[:, 0] = torch.linspace(10.0 if vocab == 1 else 100.0, 300.0, rows, device=DEV).to(c.h.dtype)
    loss, lse = c.forward()
    dh, dw, db = c.backward(lse)
    assert bool((lse > 9.0).all())
    for t in (loss, dh, dw) + ((db,) if bias else ()):
        assert not t.any()


@pytest.mark.parametrize("rows,vocab", [(500, 40), (300, 1500), (2600, 5001)])
def test_no_loss_is_below_nothing(rows, vocab):
    """The sum has the largest entry's exponential, 1, and others that are not negative; so lse is the label's logit at least."""
    c = Loss(rows, 96, vocab, bias=True, scale=40.0, seed=31)
    logits = c.h.float() @ c.weight.float().t() + c.bias
    c.labels.copy_(logits.argmax(1))
    loss, _ = c.forward()
    assert bool((loss >= 0).all()) and bool((loss == 0).any()) and bool((loss > 0).any())


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("rows", [300, 3000])
def test_a_gradient_that_is_not_finite_stays_in_its_row(rows, value, kind):
    """The largest finite one is what all others are rounded as multiples of."""
    c = Loss(rows, 64, 900, kind, seed=32)
    _, lse = c.forward()
    clean = c.backward(lse)[0]
    order = c.g.abs().argsort()
    at = int(order[rows // 2])
    c.g[at] = value
    dh = c.backward(lse)[0]
    rest = torch.arange(rows, device=DEV) != at
    assert torch.equal(dh[rest], clean[rest]) and not bool(torch.isfinite(dh[at]).any())


# ------------------------------------------------------------------ AdamW

@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("eps", [1e-8, 1e-38, 3e-39, 1e-45, 1e-60, 2.0 ** -1074])
def test_any_eps_above_zero_divides_nothing_by_something(eps, eight):
    """Averages and gradients of 0 change no parameter, as 0 over eps is 0."""
    s = State([300], seed=33, eight=eight)
    for t in (s.g_all, s.m_all, s.v_all):
        t.view(torch.uint8).zero_()
    p = s.p[0].clone()
    okt.okt_adamw_step(s.plan(), int64(3), lr=0.1, eps=eps)
    assert torch.equal(s.p[0], p)
