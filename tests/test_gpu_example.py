"""The example that runs the layer's operators together with the gradient's sparsification."""
import pytest

pytestmark = pytest.mark.gpu


def test_encoder_learns():
    from examples import train_encoder
    losses = train_encoder.train(60)
    first, last = sum(losses[:10]) / 10, sum(losses[-10:]) / 10
    assert all(x == x for x in losses)
    assert last < 0.5 * first, (first, last)
