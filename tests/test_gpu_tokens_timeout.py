"""The bounded-wait failure path of the 8-bit linear layer: with the
pipeline-wait limit lowered far below the time its first copies take, the
call gives up instead of finishing and the device status reads
HC_ERR_TIMEOUT; with the limit back at its default the same call is correct
again (the unwind let every copy and MMA it had issued finish and freed the
CTA's tensor memory). No kernel is made to hang: every wait still ends, only
sooner than the work it waits for."""
import pytest

from paper_2608_09388_gb300 import hc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# Far below the microsecond that a first copy from memory takes.
SHORT_LIMIT_NS = 100


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_09388_gb300 import build
    build.build()
    hc.load_library()
    assert hc.hc_get_device_status() == hc.HC_OK


@pytest.fixture
def short_waits():
    yield lambda: hc.hc_test_set_option(hc.HC_TEST_WAIT_LIMIT_NS, SHORT_LIMIT_NS)
    hc.hc_test_set_option(hc.HC_TEST_WAIT_LIMIT_NS, 0)
    hc.hc_get_device_status()


# (rows, K, N): 256 and 128 output channels a tile, tokens on the columns, and
# both with the blocks split over a cluster; one with fewer blocks than stages
@pytest.mark.parametrize("n,K,N", [(5000, 4096, 2048), (3000, 2048, 128), (200, 8192, 256),
                                   (7, 8192, 1000), (40, 4096, 20000), (3000, 256, 128)])
def test_linear_wait_timeout_reported_then_correct(short_waits, n, K, N):
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    x = torch.randn(n, K, generator=g, device="cuda")
    q = torch.empty(n, K, dtype=torch.uint8, device="cuda")
    s = torch.empty(K // 128, n, device="cuda")
    hc.hc_quantize_fp8_rows(x, q, s)
    w = torch.empty(N, K, dtype=torch.uint8, device="cuda")
    ws = torch.empty((N + 127) // 128, K // 128, device="cuda")
    hc.hc_quantize_fp8_weight(torch.randn(K, N, generator=g, device="cuda"), w, ws)
    want, y = (torch.empty(n, N, device="cuda") for _ in range(2))
    hc.hc_fp8_linear_fwd(q, s, w, ws, None, hc.HC_ACT_NONE, want)
    assert hc.hc_get_device_status() == hc.HC_OK
    short_waits()
    seen = set()
    for _ in range(5):
        hc.hc_fp8_linear_fwd(q, s, w, ws, None, hc.HC_ACT_NONE, y)
        seen.add(hc.hc_get_device_status())
    assert seen <= {hc.HC_ERR_TIMEOUT, hc.HC_OK} and hc.HC_ERR_TIMEOUT in seen
    hc.hc_test_set_option(hc.HC_TEST_WAIT_LIMIT_NS, 0)
    for _ in range(3):
        y.fill_(float("nan"))
        hc.hc_fp8_linear_fwd(q, s, w, ws, None, hc.HC_ACT_NONE, y)
        assert hc.hc_get_device_status() == hc.HC_OK
        assert torch.equal(y, want)
