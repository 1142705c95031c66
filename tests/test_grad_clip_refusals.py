"""What a list of tensors, the gradient norm and the clipping refuse, on the
host; the table itself, which is written without a GPU call."""
import ctypes

import pytest

from paper_2608_09388_gb300 import build, hc

torch = pytest.importorskip("torch")

P = ctypes.c_void_p
UNIT = 4096  # fp32 elements, 8192 bf16: 16 KiB


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hc.load_library()


def fill(lib, tensors, in_place=False, n=None, host=None, device=0x5000, drop=(), outs=None):
    """tensors: (address in, address out, elements, dtype) each."""
    k = len(tensors)
    ins, out = (P * k)(*[t[0] for t in tensors]), (P * k)(*[t[1] for t in tensors])
    numel, dt = (ctypes.c_longlong * k)(*[t[2] for t in tensors]), (ctypes.c_int * k)(*[t[3] for t in tensors])
    table = ctypes.create_string_buffer(max(1, lib.hc_tensor_list_bytes(k)) + 8)
    at = (ctypes.addressof(table) + 7) // 8 * 8 if host is None else host
    desc = hc.hc_tensor_list.__new__(hc.hc_tensor_list)
    args = dict(ins=ins, out=None if in_place else out, numel=numel, dt=dt, host=at, device=device,
                desc=ctypes.byref(desc))
    for name in drop:
        args[name] = None
    st = lib.hc_tensor_list_fill(args["ins"], args["out"], args["numel"], args["dt"],
                                 k if n is None else n, args["host"], args["device"], args["desc"])
    return st, desc


def test_units(lib):
    """A tensor's units count from the 16-byte boundary at or below it."""
    for numel, dt, at, units in ((0, 0, 0, 0), (1, 0, 0x1000, 1), (UNIT, 0, 0x1000, 1),
                                 (2 * UNIT + 1, 1, 0x1000, 2), (2 * UNIT, 1, 0x1002, 2),
                                 (UNIT - 3, 0, 0x100c, 1), (UNIT - 2, 0, 0x100c, 2),
                                 (2 ** 40, 1, 0x1000, 2 ** 27)):
        st, d = fill(lib, [(at, at, numel, dt)])
        assert st == hc.HC_OK and (d.units, d.tensors, d.table) == (units, 1, 0x5000)
    st, d = fill(lib, [(0x1000, 0x9000, 5, 0), (0, 0, 0, 1), (0x2000, 0xa000, 2 * UNIT, 1)])
    assert st == hc.HC_OK and d.units == 2 and d.tensors == 3
    st, d = fill(lib, [])
    assert st == hc.HC_OK and d.units == 0


def test_fill_refuses(lib):
    ok = [(0x1000, 0x9000, 16, 0), (0x2000, 0xa000, 16, 1)]
    assert fill(lib, ok)[0] == hc.HC_OK
    for kw in (dict(n=-1), dict(n=2 ** 31 - 1), dict(host=0x5004), dict(device=0x5004),
               dict(device=None), dict(drop=("ins",)), dict(drop=("numel",)), dict(drop=("dt",)),
               dict(drop=("desc",)), dict(drop=("host",))):
        assert fill(lib, ok, **kw)[0] == hc.HC_ERR_INVALID_ARG, kw
        assert hc.hc_last_error_string()
    for t in ((0x1000, 0x9000, 16, 2), (0x1000, 0x9000, -1, 0), (0x1000, 0x9000, 2 ** 48, 0),
              (0, 0x9000, 16, 0), (0x1000, 0, 16, 0), (0x1002, 0x9000, 16, 0),
              (0x1000, 0x9001, 16, 1)):
        assert fill(lib, [ok[1], t])[0] == hc.HC_ERR_INVALID_ARG, t
    assert fill(lib, [(0x1000, 0, 16, 0)], in_place=True)[0] == hc.HC_OK


def test_overlaps_are_refused(lib):
    a = (0x1000, 0x9000, 16, 0)  # 64 bytes
    for b in ((0x2000, 0x9000, 16, 0),   # the same output
              (0x2000, 0x903c, 16, 0),   # outputs that share an element
              (0x9020, 0xa000, 16, 0),   # an input that another output writes
              (0x2000, 0x1010, 16, 1),   # an output on another input
              (0x2000, 0x2004, 16, 0),   # its own input, shifted
              (0x9000, 0x9000, 16, 0)):  # in place, on another's output
        for pair in ([a, b], [b, a]):
            assert fill(lib, pair)[0] == hc.HC_ERR_INVALID_ARG, b
            assert "overlap" in hc.hc_last_error_string()
    # the same input twice (into two outputs), neighbours, in place beside others
    for b in ((0x1000, 0xa000, 16, 0), (0x1040, 0x9040, 16, 0), (0xa000, 0xa000, 16, 0),
              (0x1008, 0x8fc0, 16, 0)):
        assert fill(lib, [a, b])[0] == hc.HC_OK, b
    # in place the same tensor twice would be scaled twice
    assert fill(lib, [a, a], in_place=True)[0] == hc.HC_ERR_INVALID_ARG


def test_calls_refuse(lib):
    _, d = fill(lib, [(0x1000, 0x9000, 16, 0)])
    ref = ctypes.byref(d)
    assert lib.hc_grad_norm(None, P(0x1000), None) == hc.HC_ERR_INVALID_ARG
    assert lib.hc_grad_norm(ref, None, None) == hc.HC_ERR_INVALID_ARG
    assert lib.hc_grad_norm(ref, P(0x1002), None) == hc.HC_ERR_INVALID_ARG
    f = ctypes.c_float
    for args in ((None, P(0x1000), f(1.0)), (ref, None, f(1.0)), (ref, P(0x1001), f(1.0)),
                 (ref, P(0x1000), f(-1.0)), (ref, P(0x1000), f(float("nan")))):
        assert lib.hc_grad_clip(*args, None) == hc.HC_ERR_INVALID_ARG
        assert hc.hc_last_error_string()
    _, empty = fill(lib, [])
    assert lib.hc_grad_clip(ctypes.byref(empty), P(0x1000), f(1.0), None) == hc.HC_OK


def test_binding_refuses(lib):
    z = torch.zeros
    for grads, outs in (([z(3)], None), ([z(3)], [z(3), z(3)]), ([z(3, dtype=torch.float64)], None)):
        with pytest.raises((ValueError, TypeError)):
            hc.hc_tensor_list(grads, outs)
    with pytest.raises(TypeError):
        hc.hc_grad_norm([z(3)], z(1))
