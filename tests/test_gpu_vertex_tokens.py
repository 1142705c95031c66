"""The token network of examples/vertex_tokens.py: its training brings the
loss down, and a token run alone gives what it gives in the batch."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_09388_gb300 import build, hc
    build.build()
    hc.load_library()
    assert hc.hc_get_device_status() == hc.HC_OK


def test_training_and_serving():
    import vertex_tokens
    losses, worst = vertex_tokens.main(say=None)
    assert all(b == b and b < 10 for b in losses)
    # Gradient descent with a small rate on a smooth loss: falling throughout.
    # Gradients and outputs pass through 8 bits (a relative step of 1/16), which
    # leaves a floor well below a quarter of the start.
    assert losses[-1] < 0.25 * losses[0]
    # alone and in the batch a row is normalised and quantised alike; only the
    # order of the fp32 sums over 2 blocks and 128 products may differ: 256
    # additions of terms below 4 in all
    assert worst <= 256 * 2 ** -24 * 16
