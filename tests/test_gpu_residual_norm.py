"""okt_residual_norm_forward / _backward on the GPU against the 64-bit oracle, at widths of every
layout, ragged and unaligned rows, with and without each part, within bounds that add up
the roundings (operators_harness)."""
import numpy as np
import pytest
import torch

import paper_2201_07598_amd as okt
from oracle import okt_operators as ops
from tests.operators_harness import (DEV, E, UNIT, norm_backward_error, norm_error, rand, seed_tensor, statistics_error,
                                     step, wide, within)

pytestmark = pytest.mark.gpu

SEED = 987654321987
ALPHA = 0.81


class Case:
    def __init__(self, rows, width, kind="bf16", norm="layer", post=False, pre=True, gates=0, p=0.0, bias=True, stride=None):
        self.rows, self.width, self.kind, self.norm, self.p = rows, width, kind, norm, p
        self.share = -(-rows // gates) if gates else 0
        stride = stride or width

        def rows_of(seed, scale=1.0):
            return rand((rows, stride), kind, seed, scale)[:, :width]

        self.u, self.x = rows_of(1), rows_of(2)
        self.h, self.y = rows_of(3), rows_of(4) if pre else None
        self.dh, self.dy = rows_of(5), rows_of(6) if pre else None
        self.dx, self.du = rows_of(7), rows_of(8)
        self.stats = torch.full((rows, 4), 3.0, device=DEV)
        self.par = {}
        for name, there, seed in (("post", post, 9), ("pre", pre, 11)):
            if there:
                self.par[name + "_weight"] = 1 + rand((width,), "f32", seed, 0.2)
                if bias:
                    self.par[name + "_bias"] = rand((width,), "f32", seed + 1, 0.3)
        if gates:
            self.par["gate"] = rand((-(-rows // self.share), width), "f32", 13)
        self.options = dict(kind=norm, residual_scale=ALPHA, rows_per_gate=self.share, dropout_p=p, seed=seed_tensor(SEED),
                            site=3, **self.par)

    def forward(self):
        okt.okt_residual_norm_forward(self.u, self.x, self.h, self.y, self.stats, **self.options)

    def check_forward(self):
        par = {k: wide(v) for k, v in self.par.items()}
        factor = ops.norm_factor(self.rows, self.width, self.p, SEED, 3)
        held = wide(self.h)
        h, y, stats = ops.residual_norm(wide(self.u), wide(self.x), kind=self.norm, residual_scale=float(np.float32(ALPHA)),
                                        rows_per_gate=self.share, factor=factor, store=lambda _: held, **par)
        u = UNIT[self.kind]
        u_in, a_err = wide(self.u), 0.0
        a = u_in
        bounds = np.zeros_like(stats)
        if "post_weight" in par:
            m, r = stats[:, 0:1], stats[:, 1:2]
            a = ops._norm(u_in, (m, r), par["post_weight"], par.get("post_bias"))
            a_err = norm_error(u_in, m, r, par["post_weight"], par.get("post_bias"), self.norm)
            dm, dr = statistics_error(u_in, m, r, self.norm)
            bounds[:, 0:1], bounds[:, 1:2] = dm, r * dr
        g = par["gate"][np.arange(self.rows) // self.share] if "gate" in par else 1.0
        size = np.abs(ALPHA * wide(self.x)) + np.abs(factor * g * a)
        within(self.h, h, np.abs(factor * g) * a_err + 5 * E * size + u * np.abs(h) + step(self.kind), "h")
        if y is not None:
            m, r = stats[:, 2:3], stats[:, 3:4]
            err = norm_error(held, m, r, par["pre_weight"], par.get("pre_bias"), self.norm)
            within(self.y, y, err * (1 + u) + u * np.abs(y) + step(self.kind), "y")
            dm, dr = statistics_error(held, m, r, self.norm)
            bounds[:, 2:3], bounds[:, 3:4] = dm, r * dr
        within(self.stats, stats, bounds + 2 * E * np.abs(stats), "stats")

    def backward(self, with_dh=True):
        self.ws = torch.full((okt.okt_residual_norm_workspace_bytes(self.rows, self.width, self.share),), 0xA5,
                             dtype=torch.uint8, device=DEV)
        self.grads = {"d" + n: torch.full_like(t, 7.0) for n, t in self.par.items()}
        okt.okt_residual_norm_backward(self.u, self.h, self.stats, self.dh if with_dh else None, self.dy, self.dx, self.du,
                                       self.ws, **self.grads, **self.options)
        self.with_dh = with_dh

    def check_backward(self):
        par = {k: wide(v) for k, v in self.par.items()}
        factor = ops.norm_factor(self.rows, self.width, self.p, SEED, 3)
        alpha, u = float(np.float32(ALPHA)), UNIT[self.kind]
        uu, h, stats = wide(self.u), wide(self.h), wide(self.stats)
        dh, dy = wide(self.dh) if self.with_dh else None, wide(self.dy)
        want = ops.residual_norm_backward(uu, h, stats, dh, dy, kind=self.norm, residual_scale=alpha, factor=factor,
                                          rows_per_gate=self.share, **{k: v for k, v in par.items() if k != "pre_bias"})
        total_err, bounds = np.zeros_like(uu), {}
        total = want["dx"] / alpha
        if "pre_weight" in par:
            total_err, bounds["dpre_weight"], bounds["dpre_bias"] = norm_backward_error(
                dy, np.zeros_like(dy), h, stats[:, 2:3], stats[:, 3:4], par["pre_weight"])
        total_err = total_err + 2 * E * (np.abs(total) + (0 if dh is None else np.abs(dh)))
        bounds["dx"] = alpha * total_err + E * np.abs(want["dx"]) + u * np.abs(want["dx"]) + step(self.kind)
        da, err = factor * total, factor * total_err + 2 * E * np.abs(factor * total)
        if "gate" in par:
            m, r = stats[:, 0:1], stats[:, 1:2]
            group = np.arange(self.rows) // self.share
            a = uu if "post_weight" not in par else ops._norm(uu, (m, r), par["post_weight"], par.get("post_bias"))
            size = np.abs(uu)
            if "post_weight" in par:                       # the statistics are inputs here: a few operations each
                size = np.abs((uu - m) * r * par["post_weight"]) + np.abs(m * r * par["post_weight"]) + np.abs(par.get("post_bias", 0.0))
            bounds["dgate"] = np.zeros_like(par["gate"])
            np.add.at(bounds["dgate"], group, err * np.abs(a) + np.abs(da) * 5 * E * size + 130 * E * np.abs(da * a))
            da, err = da * par["gate"][group], err * np.abs(par["gate"][group]) + 2 * E * np.abs(da * par["gate"][group])
        if "post_weight" in par:
            err, bounds["dpost_weight"], bounds["dpost_bias"] = norm_backward_error(
                da, err, uu, stats[:, 0:1], stats[:, 1:2], par["post_weight"])
        bounds["du"] = err + u * np.abs(want["du"]) + step(self.kind)
        within(self.dx, want["dx"], bounds["dx"], "dx")
        within(self.du, want["du"], bounds["du"], "du")
        for name, got in self.grads.items():
            within(got, want[name], bounds[name] + 2 * E * np.abs(want[name]), name)


FORMS = [dict(), dict(p=0.1), dict(norm="rms", bias=False), dict(post=True, pre=False), dict(post=True, gates=1, p=0.2),
         dict(gates=3, bias=False, norm="rms"), dict(pre=False, gates=2, p=0.3), dict(post=True, gates=4, norm="rms")]


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("rows,width,kind", [
    (1, 8, "f32"), (5, 37, "bf16"), (130, 512, "f16"), (67, 768, "f32"), (33, 1000, "bf16"), (9, 1024, "bf16"), (21, 1025, "f16"),
    (40, 2500, "f16"), (17, 4096, "f32"), (6, 4104, "bf16"), (7, 8191, "f16"), (3, 8192, "f32")])
def test_against_the_oracle(rows, width, kind, form):
    c = Case(rows, width, kind, **form)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("form", [dict(p=0.1), dict(post=True, gates=5, norm="rms", p=0.1), dict(post=True, gates=700)], ids=str)
def test_many_rows(form):
    """More rows than workgroups, gates that lie within a workgroup's rows and across several."""
    c = Case(4099, 264, "bf16", **form)
    c.forward()
    c.check_forward()
    c.backward(with_dh=False)
    c.check_backward()


@pytest.mark.parametrize("form", [dict(post=True, gates=3, norm="rms", bias=False, p=0.1), dict(post=True, gates=1), dict(pre=False, gates=9000)], ids=str)
def test_many_rows_of_two_groups_a_lane(form):
    c = Case(9001, 532, "f16", **form)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


def test_rows_apart_and_unaligned():
    c = Case(50, 333, "f16", post=True, gates=2, p=0.1, stride=339)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


def test_what_lies_between_rows_is_not_touched():
    c = Case(20, 100, "bf16", stride=107)
    whole = c.h._base if c.h._base is not None else c.h
    before = whole.clone()
    c.forward()
    gap = torch.ones_like(whole, dtype=torch.bool)
    gap[:, :100] = False
    assert torch.equal(whole[gap], before[gap])


def test_outputs_in_the_place_of_inputs():
    a, b = Case(65, 700, "bf16", post=True, gates=1, p=0.1), Case(65, 700, "bf16", post=True, gates=1, p=0.1)
    a.forward()
    okt.okt_residual_norm_forward(b.u, b.x, b.x, b.y, b.stats, **b.options)         # h over x
    assert torch.equal(a.h, b.x) and torch.equal(a.y, b.y) and torch.equal(a.stats, b.stats)
    a.backward()
    b.h, b.dx, b.du = b.x, b.dh, b.dy                                               # dx over dh, du over dy
    b.backward()
    assert torch.equal(a.dx, b.dx) and torch.equal(a.du, b.du)
    for n in a.grads:
        assert torch.equal(a.grads[n], b.grads[n]), n


@pytest.mark.parametrize("form", [dict(), dict(pre=False, gates=1), dict(pre=False, gates=2, post=True, p=0.1)], ids=str)
@pytest.mark.parametrize("width", [516, 1028, 4100])
def test_in_place_at_widths_that_end_inside_a_group(width, form):
    """The row's last group reads columns that another wave stores, and drops them."""
    a, b = Case(1500, width, "bf16", **form), Case(1500, width, "bf16", **form)
    a.forward()
    okt.okt_residual_norm_forward(b.u, b.x, b.x, b.y, b.stats, **b.options)
    assert torch.equal(a.h, b.x) and (a.y is None or torch.equal(a.y, b.y)) and torch.equal(a.stats, b.stats)
    a.backward()
    b.h, b.dx = b.x, b.dh
    b.backward()
    assert torch.equal(a.dx, b.dx) and torch.equal(a.du, b.du)
    b.dh, b.dx, b.du = a.dh, a.dx.clone(), b.u                                      # du over u
    if form:
        b.backward()
        assert torch.equal(a.dx, b.dx) and torch.equal(a.du, b.u)


def test_results_do_not_change_from_run_to_run():
    c = Case(3001, 520, "bf16", post=True, gates=3, p=0.2)
    c.forward()
    c.backward()
    first = [c.dx.clone(), c.du.clone(), *(t.clone() for t in c.grads.values())]
    c.backward()
    assert all(torch.equal(a, b) for a, b in zip(first, [c.dx, c.du, *c.grads.values()]))


def test_no_rows_and_everything_dropped():
    c = Case(0, 64, "bf16", post=True, gates=0, p=0.1)
    c.forward()
    c.backward()
    assert all(bool((t == 0).all()) for t in c.grads.values())
    c = Case(9, 64, "f32", gates=1, p=1.0)
    c.forward()
    assert torch.allclose(c.h, ALPHA * c.x)
    c.backward()
    assert bool((c.du == 0).all()) and bool((c.grads["dgate"] == 0).all())


def test_a_graph_replays_with_new_inputs_and_seeds():
    c = Case(257, 1024, "bf16", p=0.1)
    seed = c.options["seed"]
    c.forward()
    c.backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        okt.okt_residual_norm_forward(c.u, c.x, c.h, c.y, c.stats, **c.options)
        okt.okt_residual_norm_backward(c.u, c.h, c.stats, c.dh, c.dy, c.dx, c.du, c.ws, **c.grads, **c.options)
    for n in range(3):
        seed.fill_(1000 + n)
        c.u.copy_(rand((257, 1024), "bf16", 50 + n))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (c.h, c.y, c.dx, c.du, *c.grads.values())]
        okt.okt_residual_norm_forward(c.u, c.x, c.h, c.y, c.stats, **c.options)
        okt.okt_residual_norm_backward(c.u, c.h, c.stats, c.dh, c.dy, c.dx, c.du, c.ws, **c.grads, **c.options)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (c.h, c.y, c.dx, c.du, *c.grads.values()))), n


@pytest.mark.parametrize("rows,width,kind,gates", [(40, 100, "bf16", 1), (9000, 536, "f16", 3), (700, 1028, "f16", 700),
                                                   (600, 2500, "f16", 2), (520, 4104, "f32", 1)])
def test_what_is_dropped_does_not_reach_the_gradient_of_a_gate(rows, width, kind, gates):
    """dg sums dh * dropout(a): a place that is dropped adds 0, whatever u holds there."""
    c = Case(rows, width, kind, pre=False, gates=gates, p=0.3)
    dropped = torch.from_numpy(~ops.kept_rows(rows, width, 0.3, SEED, 3)).to(DEV)
    c.u = c.u.masked_fill(dropped, 0.0)
    c.forward()
    c.backward()
    clean = [t.clone() for t in (c.h, c.dx, c.du, c.grads["dgate"])]
    c.u = c.u.masked_fill(dropped, float("inf"))
    c.u[:, ::3] = c.u[:, ::3].masked_fill(dropped[:, ::3], float("nan"))
    c.forward()
    c.backward()
    assert all(torch.equal(a, b) for a, b in zip(clean, (c.h, c.dx, c.du, c.grads["dgate"])))


WIDE_FORMS = [dict(p=0.1), dict(post=True, gates=3, p=0.1), dict(post=True, gates=700), dict(post=True, norm="rms", bias=False, p=0.2),
              dict(pre=False, gates=7), dict(post=True, pre=False, gates=1, p=0.1)]


@pytest.mark.parametrize("form", WIDE_FORMS, ids=str)
@pytest.mark.parametrize("rows,width,kind", [(1500, 1028, "bf16"), (1600, 760, "f32"), (1300, 2500, "f16"), (1100, 4104, "f16"),
                                             (1100, 4104, "f32"), (1031, 8192, "bf16")])
def test_many_rows_of_a_workgroup_each(rows, width, kind, form):
    """Sums over rows that a workgroup takes one after the other, in registers and in LDS, and gates that
    end inside its rows."""
    c = Case(rows, width, kind, **form)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("width", [200, 1000, 2500, 5000])
def test_another_stream(width):
    c = Case(300, width, "bf16", post=True, gates=2, p=0.1)
    c.forward()
    c.backward()
    want = [t.clone() for t in (c.h, c.y, c.stats, c.dx, c.du, *c.grads.values())]
    side = torch.cuda.Stream()
    for t in (c.h, c.y, c.stats, c.dx, c.du, *c.grads.values()):
        t.fill_(7.0)
    torch.cuda.synchronize()
    okt.okt_residual_norm_forward(c.u, c.x, c.h, c.y, c.stats, stream=side, **c.options)
    okt.okt_residual_norm_backward(c.u, c.h, c.stats, c.dh, c.dy, c.dx, c.du, c.ws, stream=side, **c.grads, **c.options)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (c.h, c.y, c.stats, c.dx, c.du, *c.grads.values())))


@pytest.mark.parametrize("width", [300, 700, 1028, 4100])
def test_both_outputs_in_the_place_of_inputs(width):
    """h over one of u and x and y over the other."""
    for swap in (False, True):
        a, b = (Case(1500, width, "bf16", post=True, gates=1, p=0.1) for _ in range(2))
        a.forward()
        h, y = (b.u, b.x) if swap else (b.x, b.u)
        okt.okt_residual_norm_forward(b.u, b.x, h, y, b.stats, **b.options)
        assert torch.equal(a.h, h) and torch.equal(a.y, y) and torch.equal(a.stats, b.stats)


@pytest.mark.parametrize("width,gates", [(100, 1), (2500, 3)])
def test_nothing_is_hidden_from_the_gradient_of_a_gate_where_nothing_is_dropped(width, gates):
    """Without dropout a place with an infinite u and a gradient of 0 makes its gate's gradient NaN, as the formula does."""
    c = Case(90, width, "bf16", pre=False, gates=gates)
    c.u = c.u.clone()
    c.u[7, 5] = float("inf")
    c.dh = c.dh.clone()
    c.dh[7, 5] = 0.0
    c.backward()
    nan = torch.isnan(c.grads["dgate"])
    assert bool(nan[0, 5]) and int(nan.sum()) == 1
