"""Sizes near the largest int that the token operators take or refuse, on the
host: nothing reaches a GPU."""
import ctypes

import pytest

from paper_2608_09388_gb300 import build, hc

torch = pytest.importorskip("torch")

FAKE = ctypes.c_void_p(0x1000)
F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    build.build()
    return hc.load_library()


@pytest.mark.parametrize("C", [2 ** 31 - 1, 2 ** 31 - 1024, 2 ** 31 - 8192])
def test_rows_too_wide_refused(lib, C):
    """Channel counters of 32 bits would run past the end of such rows."""
    calls = (
        lambda: lib.hc_layer_norm_fwd(FAKE, 1, None, 1, C, F(1e-5), None, None, FAKE, None, None, None),
        lambda: lib.hc_layer_norm_bwd(FAKE, FAKE, 1, None, 1, C, None, FAKE, FAKE, FAKE, None, None, None),
        lambda: lib.hc_embedding_fwd(FAKE, 0, 9, C, FAKE, 1, None, 1, F(1.0), FAKE, None),
        lambda: lib.hc_embedding_bwd(FAKE, 0, FAKE, FAKE, 1, 9, C, F(1.0), FAKE, None),
        lambda: lib.hc_quantize_fp8_rows(FAKE, 0, None, 1, C, FAKE, FAKE, None),
        lambda: lib.hc_quantize_fp8_weight(FAKE, 0, C, 8, FAKE, FAKE, None),
        lambda: lib.hc_quantize_fp8_weight(FAKE, 0, 8, C, FAKE, FAKE, None),
        lambda: lib.hc_fp8_linear_fwd(FAKE, FAKE, None, 1, C, 8, FAKE, FAKE, None, 0, 1, FAKE, None),
        lambda: lib.hc_fp8_linear_fwd(FAKE, FAKE, None, 1, 8, C, FAKE, FAKE, None, 0, 1, FAKE, None))
    for k, call in enumerate(calls):
        assert call() == hc.HC_ERR_INVALID_ARG, k
        assert b"too large" in lib.hc_last_error_string(), k


def test_binding_refuses_sizes_past_32_bits(lib):
    """A C int takes the low 32 bits of a size: 2^32 + 5 rows would be five.
    (Expanded and meta tensors: no memory is behind these sizes.)"""
    n = 2 ** 32 + 5
    x1, f1 = torch.zeros(1, 1), torch.zeros(1)
    i1, u1 = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 16, dtype=torch.uint8)
    rows, cols, ids = x1.expand(n, 1), x1.expand(1, n), i1.expand(n)
    far = torch.empty(2, 2 ** 31, dtype=torch.int32, device="meta")[:, 0]
    calls = (
        lambda: hc.hc_layer_norm_fwd(rows, 1e-5, None, None, rows),
        lambda: hc.hc_layer_norm_fwd(cols, 1e-5, None, None, cols),
        lambda: hc.hc_layer_norm_bwd(rows, rows, None, f1.expand(n), f1.expand(n), dx=rows),
        lambda: hc.hc_embedding_fwd(rows, i1, 1.0, x1),
        lambda: hc.hc_embedding_fwd(x1, ids, 1.0, rows),
        lambda: hc.hc_embedding_fwd(x1, far, 1.0, x1.expand(2, 1)),
        lambda: hc.hc_embedding_sort(ids, 3, torch.zeros(4, dtype=torch.int32), ids),
        lambda: hc.hc_embedding_sort(i1, n, i1.expand(n + 1), i1),
        lambda: hc.hc_embedding_bwd(rows, torch.zeros(2, dtype=torch.int32), ids, 1.0, x1),
        lambda: hc.hc_embedding_bwd(x1, i1.expand(n + 1), i1, 1.0, rows),
        lambda: hc.hc_quantize_fp8_rows(rows, u1.expand(n, 16), x1.expand(1, n)),
        lambda: hc.hc_quantize_fp8_weight(cols, u1.expand(n, 16), x1),
        lambda: hc.hc_fp8_linear_fwd(u1.expand(n, 16), x1.expand(1, n), u1, x1, None, 0, rows),
        lambda: hc.hc_fp8_linear_fwd(u1, x1, u1.expand(n, 16), x1, None, 0, cols))
    for k, call in enumerate(calls):
        with pytest.raises(ValueError, match="below 2\\^31"):
            call()
