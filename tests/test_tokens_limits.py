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
