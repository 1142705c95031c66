"""What the root-mean-square norm refuses, on the host."""
import ctypes

import pytest

from paper_2608_09388_gb300 import build, hc

torch = pytest.importorskip("torch")

FAKE = ctypes.c_void_p(0x1000)
OTHER = ctypes.c_void_p(0x2000)
ODD = ctypes.c_void_p(0x1001)
TWO = ctypes.c_void_p(0x1002)
F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hc.load_library()


def refuses(call, cases):
    for kw in cases:
        assert call(**kw) == hc.HC_ERR_INVALID_ARG, kw
        assert hc.hc_last_error_string()


def test_forward(lib):
    def call(x=FAKE, res=None, dt=1, count=None, cap=4, C=8, eps=1e-5, ga=None, h=None, y=OTHER,
             r=None, q=None, s=None):
        return lib.hc_rms_norm_fwd(x, res, dt, count, cap, C, F(eps), ga, h, y, r, q, s, None)

    refuses(call, (dict(dt=2), dict(cap=-1), dict(C=0), dict(C=2 ** 31 - 1), dict(eps=-1.0),
                   dict(eps=float("nan")), dict(x=None), dict(y=None), dict(q=FAKE), dict(s=FAKE),
                   dict(x=ODD), dict(res=ODD), dict(h=ODD), dict(dt=0, y=TWO), dict(ga=TWO),
                   dict(r=TWO), dict(count=ODD), dict(q=ctypes.c_void_p(0x1008), s=FAKE),
                   dict(q=FAKE, s=TWO), dict(h=OTHER)))
    assert call(cap=0, x=None, y=None) == hc.HC_OK


def test_backward(lib):
    def call(h=FAKE, dy=FAKE, dres=None, dt=1, count=None, cap=4, C=8, ga=None, r=FAKE, dx=FAKE,
             dg=None):
        return lib.hc_rms_norm_bwd(h, dy, dres, dt, count, cap, C, ga, r, dx, dg, None)

    refuses(call, (dict(dt=-1), dict(cap=-1), dict(C=0), dict(dx=None), dict(h=None),
                   dict(dy=None), dict(r=None), dict(dy=ODD), dict(dres=ODD), dict(dx=ODD),
                   dict(dg=TWO), dict(r=TWO), dict(ga=ODD), dict(count=TWO)))
    assert call(cap=0) == hc.HC_OK


def test_binding_checks_shapes_and_types(lib):
    z = torch.zeros
    x, y = z(6, 8), z(6, 8)
    u8 = torch.uint8
    for bad in (dict(y=z(6, 9)), dict(y=z(6, 8, dtype=torch.bfloat16)), dict(res=z(5, 8)),
                dict(h=z(6, 7)), dict(rstd=z(5)), dict(q=z(6, 8, dtype=u8), scales=z(1, 6)),
                dict(q=z(6, 16, dtype=u8), scales=z(6, 1)), dict(count=z(1)), dict()):
        kw = dict(y=y)
        kw.update(bad)
        with pytest.raises((ValueError, TypeError)):
            hc.hc_rms_norm_fwd(x, 1e-5, None, **kw)
    for bad in (dict(dres=z(6, 9)), dict(dx=z(5, 8)), dict(dgamma=z(9)), dict()):
        kw = dict(dx=z(6, 8))
        kw.update(bad)
        with pytest.raises((ValueError, TypeError)):
            hc.hc_rms_norm_bwd(x, y, None, z(6), **kw)
    with pytest.raises((ValueError, TypeError)):
        hc.hc_rms_norm_bwd(x, y, z(7), z(6), dx=x)


def test_tensors_of_another_device_are_refused(monkeypatch):
    class Far:
        def get_device(self):
            return 1

    class Near:
        def get_device(self):
            return 0

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(hc, "_devices", 2)
    hc._on_current_device(Near(), None, Near())
    with pytest.raises(ValueError, match="device 1"):
        hc._on_current_device(Near(), Far())
