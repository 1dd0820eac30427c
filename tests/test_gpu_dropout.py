"""okt_dropout on the GPU: bit for bit the oracle's field, at every length, type and probability."""
import numpy as np
import pytest
import torch

import paper_2201_07598_amd as okt
from oracle import okt_operators as ops
from tests.operators_harness import DEV, TYPES, rand, seed_tensor

pytestmark = pytest.mark.gpu

SEED = -0x123456789ABCDEF


def expected(x, p, seed, site=0, first=0):
    """fp32 product, rounded once to the type."""
    kept = torch.from_numpy(ops.kept_flat(x.numel(), p, seed & ((1 << 64) - 1), site, first))
    scaled = x.cpu().float() * np.float32(ops.scale_of(p)).item()
    return torch.where(kept, scaled, torch.zeros(())).to(x.dtype)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [1, 7, 8, 9, 15, 768, 2047, 8191, 8192, 8193, 100_003])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_matches_the_field(kind, n, p):
    x = rand((n,), kind, n)
    y = torch.full_like(x, 7.0)
    okt.okt_dropout(x, y, p, seed_tensor(SEED), site=5)
    assert torch.equal(y.cpu(), expected(x, p, SEED, 5))
    okt.okt_dropout(x, x, p, seed_tensor(SEED), site=5)              # in place
    assert torch.equal(x, y)


def test_what_is_dropped_does_not_matter():
    x = torch.full((4096,), float("nan"), device=DEV)
    kept = torch.from_numpy(ops.kept_flat(4096, 0.5, 3)).to(DEV)
    x[kept] = 2.0
    okt.okt_dropout(x, x, 0.5, seed_tensor(3))
    assert torch.equal(x, torch.where(kept, torch.full((), 4.0, device=DEV), torch.zeros((), device=DEV)))


def test_backward_is_the_same_call():
    x, dy = rand((5000,), "f32", 1), rand((5000,), "f32", 2)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    okt.okt_dropout(x, y, 0.3, seed_tensor(9), site=1)
    okt.okt_dropout(dy, dx, 0.3, seed_tensor(9), site=1)
    # <dy, f x> = <f dy, x> for a mask f that is the same in both
    assert abs(float((dy.double() * y.double()).sum() - (dx.double() * x.double()).sum())) < 1e-3


def test_offsets_beyond_32_bits():
    n = (1 << 32) + 4099
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    okt.okt_dropout(x, x, 0.5, seed_tensor(77))
    for first, count in ((0, 4096), ((1 << 31) - 64, 4096), ((1 << 32) - 2048, 6147)):
        kept = ops.kept_flat(count, 0.5, 77, first=first)
        assert np.array_equal(x[first:first + count].float().cpu().numpy(), np.where(kept, 2.0, 0.0)), first
    del x
    torch.cuda.empty_cache()


def test_another_stream_and_a_graph_with_a_new_seed():
    side = torch.cuda.Stream()
    x, seed = rand((70_001,), "bf16", 4), seed_tensor(5)
    y = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        okt.okt_dropout(x, y, 0.2, seed)
    side.synchronize()
    assert torch.equal(y.cpu(), expected(x, 0.2, 5))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        okt.okt_dropout(x, y, 0.2, seed)
    for s in (6, 7, 8):
        seed.fill_(s)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.cpu(), expected(x, 0.2, s)), s
