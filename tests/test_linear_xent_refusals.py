"""What the cross entropy refuses, on the host."""
import ctypes

import pytest

from paper_2608_09388_gb300 import build, hc

torch = pytest.importorskip("torch")

FAKE = ctypes.c_void_p(0x1000)
OTHER = ctypes.c_void_p(0x2000)
ODD = ctypes.c_void_p(0x1001)
TWO = ctypes.c_void_p(0x1002)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hc.load_library()


def refuses(call, cases):
    for kw in cases:
        assert call(**kw) == hc.HC_ERR_INVALID_ARG, kw
        assert hc.hc_last_error_string()


BAD = (dict(dt=2), dict(cap=-1), dict(C=0), dict(C=2 ** 31 - 1), dict(V=0), dict(V=-3),
       dict(V=2 ** 31 - 1), dict(x=None), dict(W=None), dict(t=None), dict(x=ODD), dict(W=ODD),
       dict(dt=0, x=TWO), dict(dt=0, W=TWO), dict(b=TWO), dict(t=TWO), dict(count=ODD))


def test_forward(lib):
    def call(x=FAKE, W=OTHER, dt=1, b=None, t=FAKE, count=None, cap=4, C=8, V=9, loss=FAKE, lse=FAKE):
        return lib.hc_linear_cross_entropy_fwd(x, W, dt, b, t, count, cap, C, V, loss, lse, None)

    refuses(call, BAD + (dict(loss=None, lse=None), dict(loss=TWO), dict(lse=ODD)))
    assert call(cap=0, x=None, t=None) == hc.HC_OK


def test_backward(lib):
    def call(x=FAKE, W=OTHER, dt=1, b=None, t=FAKE, lse=FAKE, dl=FAKE, count=None, cap=4, C=8, V=9,
             dx=FAKE, dW=FAKE, db=None):
        return lib.hc_linear_cross_entropy_bwd(x, W, dt, b, t, lse, dl, count, cap, C, V, dx, dW, db,
                                               None)

    refuses(call, BAD + (dict(dx=None, dW=None), dict(lse=None), dict(dl=None), dict(lse=TWO),
                         dict(dl=ODD), dict(dx=ODD), dict(dW=ODD), dict(db=TWO), dict(dW=OTHER)))
    assert call(cap=0, x=None, t=None, dW=None) == hc.HC_OK


def test_binding_checks_shapes_and_types(lib):
    z = torch.zeros
    x, W, t = z(6, 8), z(5, 8), z(6, dtype=torch.int32)
    for bad in (dict(W=z(5, 9)), dict(W=z(5, 8, dtype=torch.bfloat16)), dict(bias=z(6)),
                dict(targets=t.long()), dict(targets=t[:5]), dict(loss=z(5)),
                dict(lse=z(6, dtype=torch.float64)), dict()):
        kw = dict(W=W, bias=None, targets=t, loss=z(6))
        kw.update(bad)
        with pytest.raises((ValueError, TypeError)):
            hc.hc_linear_cross_entropy_fwd(x, **kw)
    for bad in (dict(lse=z(5)), dict(dloss=z(6, 1)), dict(dx=z(6, 9)), dict(dW=z(8, 5)),
                dict(dbias=z(6)), dict(dW=z(5, 8, dtype=torch.bfloat16)), dict()):
        kw = dict(W=W, bias=None, targets=t, lse=z(6), dloss=z(6), dx=x)
        kw.update(bad)
        with pytest.raises((ValueError, TypeError)):
            hc.hc_linear_cross_entropy_bwd(x, **kw)
