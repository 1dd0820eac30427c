"""The example that runs the layer's operators together with the gradient's sparsification."""
import pytest

pytestmark = pytest.mark.gpu


def test_encoder_learns():
    from examples import train_encoder
    losses = train_encoder.train(60)
    first, last = sum(losses[:10]) / 10, sum(losses[-10:]) / 10
    assert all(x == x for x in losses)
    assert last < 0.5 * first, (first, last)


def test_norm_gradients_are_written_into_the_flat_vector(monkeypatch):
    """The library's calls get places of the flat gradient for the norms' weights and biases, and after the backward
    pass the places hold what a call writes: nothing is added to it or put elsewhere."""
    import torch
    from examples import train_encoder as ex
    model = ex.Encoder()
    written, call = [], ex.okt.okt_residual_norm_backward

    def watch(*args, **options):
        apart = {n: torch.full_like(options[n], 7.0) for n in ("dpre_weight", "dpre_bias")}
        call(*args, **{**options, **apart})
        written.extend((options[n].data_ptr(), apart[n]) for n in apart)
        call(*args, **options)

    monkeypatch.setattr(ex.okt, "okt_residual_norm_backward", watch)
    gen = torch.Generator().manual_seed(3)
    names = torch.randint(ex.VOCAB, (ex.BATCH,), generator=gen).to(ex.DEV)
    tokens = torch.randint(ex.VOCAB, (ex.BATCH, ex.LENGTH), generator=gen).to(ex.DEV)
    lens = torch.full((ex.BATCH,), ex.LENGTH, dtype=torch.int32, device=ex.DEV)
    seed = torch.tensor([5], dtype=torch.int64, device=ex.DEV)
    model.loss(tokens, names, lens, seed).backward()
    assert len(written) == 4 * ex.LAYERS
    for address, want in written:
        at = (address - model.grad.data_ptr()) // 4
        assert 0 <= at <= model.grad.numel() - ex.WIDTH
        assert torch.equal(model.grad[at:at + ex.WIDTH], want) and bool(want.any())
    names = [f"{n}.{norm}_{part}" for n in range(ex.LAYERS) for norm in ("mid", "end") for part in ("weight", "bias")]
    assert {a for a, _ in written} == {model.par[name].grad.data_ptr() for name in names}
