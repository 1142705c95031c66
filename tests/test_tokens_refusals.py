"""What the token operators refuse, on the host: argument checks of the C ABI
and of the binding, before anything reaches a GPU."""
import ctypes

import pytest

from paper_2608_09388_gb300 import build, hc

torch = pytest.importorskip("torch")

FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1001)
TWO = ctypes.c_void_p(0x1002)
F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hc.load_library()


def refuses(call, cases, status=None):
    for kw in cases:
        assert call(**kw) == (hc.HC_ERR_INVALID_ARG if status is None else status), kw
        assert hc.hc_last_error_string()


def test_layer_norm_fwd(lib):
    def call(x=FAKE, dt=1, count=None, cap=4, C=8, eps=1e-5, ga=None, be=None, y=FAKE, m=None,
             r=None):
        return lib.hc_layer_norm_fwd(x, dt, count, cap, C, F(eps), ga, be, y, m, r, None)

    refuses(call, (dict(dt=2), dict(cap=-1), dict(C=0), dict(eps=-1.0), dict(eps=float("nan")),
                   dict(x=None), dict(y=None), dict(x=ODD), dict(dt=0, y=TWO), dict(ga=TWO),
                   dict(be=TWO), dict(m=TWO), dict(r=ODD), dict(count=ODD)))
    assert call(cap=0, x=None, y=None) == hc.HC_OK


def test_layer_norm_bwd(lib):
    def call(x=FAKE, dy=FAKE, dt=1, count=None, cap=4, C=8, ga=None, m=FAKE, r=FAKE, dx=FAKE,
             dg=None, db=None):
        return lib.hc_layer_norm_bwd(x, dy, dt, count, cap, C, ga, m, r, dx, dg, db, None)

    refuses(call, (dict(dt=-1), dict(cap=-1), dict(C=0), dict(dx=None), dict(x=None),
                   dict(dy=None), dict(m=None), dict(r=None), dict(dy=ODD), dict(dg=TWO),
                   dict(db=ODD), dict(m=TWO)))
    assert call(cap=0) == hc.HC_OK


def test_embedding(lib):
    def fwd(t=FAKE, dt=0, V=9, C=8, ids=FAKE, st=1, count=None, cap=4, y=FAKE):
        return lib.hc_embedding_fwd(t, dt, V, C, ids, st, count, cap, F(1.0), y, None)

    refuses(fwd, (dict(dt=3), dict(V=-1), dict(V=2 ** 31 - 1), dict(C=0), dict(ids=None),
                  dict(st=0), dict(cap=-2), dict(t=None), dict(y=None), dict(t=TWO), dict(ids=TWO)))
    assert fwd(cap=0) == hc.HC_OK

    def sort(ids=FAKE, st=1, count=None, cap=4, V=9, rp=FAKE, od=FAKE):
        return lib.hc_embedding_sort(ids, st, count, cap, V, rp, od, None)

    refuses(sort, (dict(ids=None), dict(st=-1), dict(cap=-1), dict(V=-1), dict(rp=None),
                   dict(od=None), dict(rp=TWO), dict(ids=ODD)))

    def bwd(dy=FAKE, dt=0, rp=FAKE, od=FAKE, cap=4, V=9, C=8, dt_=FAKE):
        return lib.hc_embedding_bwd(dy, dt, rp, od, cap, V, C, F(1.0), dt_, None)

    refuses(bwd, (dict(dt=3), dict(V=-1), dict(C=0), dict(cap=-1), dict(dy=None), dict(rp=None),
                  dict(od=None), dict(dt_=None), dict(dy=TWO), dict(dt_=TWO)))
    assert bwd(V=0) == hc.HC_OK


def test_quantize(lib):
    def rows(x=FAKE, dt=0, count=None, cap=4, C=8, q=FAKE, s=FAKE):
        return lib.hc_quantize_fp8_rows(x, dt, count, cap, C, q, s, None)

    refuses(rows, (dict(dt=2), dict(cap=-1), dict(C=0), dict(C=2 ** 31 - 1), dict(x=None),
                   dict(q=None), dict(s=None), dict(q=ctypes.c_void_p(0x1008)), dict(s=TWO),
                   dict(x=TWO)))
    assert rows(cap=0) == hc.HC_OK

    def weight(W=FAKE, dt=0, ci=8, co=8, q=FAKE, s=FAKE):
        return lib.hc_quantize_fp8_weight(W, dt, ci, co, q, s, None)

    refuses(weight, (dict(dt=2), dict(ci=0), dict(co=0), dict(W=None), dict(q=None), dict(s=None),
                     dict(q=ctypes.c_void_p(0x1008)), dict(W=TWO)))


def test_fp8_linear(lib):
    def call(xq=FAKE, xs=FAKE, count=None, cap=4, ci=8, co=8, wq=FAKE, ws=FAKE, b=None, act=0,
             dt=1, y=FAKE):
        return lib.hc_fp8_linear_fwd(xq, xs, count, cap, ci, co, wq, ws, b, act, dt, y, None)

    refuses(call, (dict(cap=-1), dict(ci=0), dict(co=0), dict(act=3), dict(dt=2), dict(xq=None),
                   dict(xs=None), dict(wq=None), dict(ws=None), dict(y=None), dict(y=ODD),
                   dict(xq=ctypes.c_void_p(0x1008)), dict(wq=ctypes.c_void_p(0x1004)),
                   dict(b=TWO)))
    assert call(cap=0) == hc.HC_OK


def test_binding_checks_shapes_and_types(lib):
    """Shapes and dtypes that do not fit each other, and host tensors, are
    refused before any library call."""
    z = torch.zeros
    x = z(6, 8)
    i = z(6, dtype=torch.int32)
    for bad in (dict(y=z(6, 9)), dict(y=z(6, 8, dtype=torch.bfloat16)), dict(gamma=z(7)),
                dict(mean=z(5)), dict(count=z(2, dtype=torch.int32)), dict(count=z(1)), dict()):
        kw = dict(eps=1e-5, gamma=None, beta=None, y=z(6, 8))
        kw.update(bad)
        with pytest.raises((ValueError, TypeError)):
            hc.hc_layer_norm_fwd(x, **kw)
    for bad in (dict(dy=z(6, 9)), dict(dx=z(5, 8)), dict(dgamma=z(9)), dict(rstd=z(6, 1)), dict()):
        kw = dict(dy=z(6, 8), gamma=None, mean=z(6), rstd=z(6), dx=z(6, 8))
        kw.update(bad)
        with pytest.raises((ValueError, TypeError)):
            hc.hc_layer_norm_bwd(x, **kw)
    for ids, y in ((i.long(), z(6, 8)), (i, z(7, 8)), (i[:5], z(6, 8)), (i, z(6, 8))):
        with pytest.raises((ValueError, TypeError)):
            hc.hc_embedding_fwd(z(3, 8), ids, 1.0, y)
    for rp, od in ((z(3, dtype=torch.int32), i), (z(4, dtype=torch.int32), i[:4]),
                   (z(4, dtype=torch.int32), i)):
        with pytest.raises((ValueError, TypeError)):
            hc.hc_embedding_sort(i, 3, rp, od)
        with pytest.raises((ValueError, TypeError)):
            hc.hc_embedding_bwd(x, rp, od, 1.0, z(3, 8))
    u8 = torch.uint8
    for q, s in ((z(6, 8, dtype=u8), z(1, 6)), (z(6, 16), z(1, 6)), (z(6, 16, dtype=u8), z(6, 1)),
                 (z(6, 16, dtype=u8), z(1, 6))):
        with pytest.raises((ValueError, TypeError)):
            hc.hc_quantize_fp8_rows(x, q, s)
    with pytest.raises((ValueError, TypeError)):
        hc.hc_quantize_fp8_weight(z(8, 4), z(4, 16, dtype=u8), z(1, 2))
    q, s = z(6, 16, dtype=u8), z(1, 6)
    for wq, ws, y in ((z(4, 32, dtype=u8), z(1, 1), z(6, 4)), (z(4, 16, dtype=u8), z(2, 1), z(6, 4)),
                      (z(4, 16, dtype=u8), z(1, 1), z(6, 5)), (z(4, 16, dtype=u8), z(1, 1), z(6, 4))):
        with pytest.raises((ValueError, TypeError)):
            hc.hc_fp8_linear_fwd(q, s, wq, ws, None, 0, y)
