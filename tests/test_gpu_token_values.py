"""The token operators on values at the edge of their arithmetic: what an
activation does with NaN and with values near zero, rows without a spread,
rows with a NaN in a ragged block. Bounds as in test_gpu_tokens.py: U = 2^-24
is the unit roundoff of fp32, a bf16 result is rounded once more by at most
2^-8 of its value."""
import pytest

from paper_2608_09388_gb300 import hc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
BF, F, D64 = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_09388_gb300 import build
    build.build()
    hc.load_library()
    assert hc.hc_get_device_status() == hc.HC_OK


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    assert hc.hc_get_device_status() == hc.HC_OK


def randn(seed, *shape, dtype=F):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def quantise(x):
    n, K = x.shape
    q = torch.full((n, hc.HC_FP8_PITCH(K)), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full(((K + 127) // 128, n), 77.0, device="cuda")
    hc.hc_quantize_fp8_rows(x, q, s)
    return q, s


def quantise_weight(W):
    K, N = W.shape
    q = torch.full((N, hc.HC_FP8_PITCH(K)), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full(((N + 127) // 128, (K + 127) // 128), 77.0, device="cuda")
    hc.hc_quantize_fp8_weight(W, q, s)
    return q, s


# The four ways a tile leaves the 8-bit product: tokens or channels on the
# lanes, the channel blocks by one CTA (K below 512: fewer than four blocks) or
# joined over a cluster; and tokens on the lanes with 256 channels a tile.
EPILOGUES = [(300, 136, 200), (128, 1024, 256), (5, 136, 200), (40, 136, 70), (5, 1024, 200),
             (2400, 392, 2000)]


@pytest.mark.parametrize("out", [BF, F])
@pytest.mark.parametrize("n,K,N", EPILOGUES)
@pytest.mark.parametrize("act", [hc.HC_ACT_NONE, hc.HC_ACT_ELU, hc.HC_ACT_RELU])
def test_linear_keeps_nan(n, K, N, act, out):
    """Every output of a row that holds a NaN or an infinity is NaN, behind an
    activation too, and no other row's is."""
    x = randn(n, n, K)
    x[1, 3], x[2, K - 1], x[n - 2, 0] = float("nan"), float("inf"), float("-inf")
    q, s = quantise(x)
    w, ws = quantise_weight(randn(K, K, N))
    y = torch.empty(n, N, dtype=out, device="cuda")
    hc.hc_fp8_linear_fwd(q, s, w, ws, randn(N, N), act, y)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[[1, 2, n - 2]] = True
    assert y[bad].isnan().all()
    assert y[~bad].isfinite().all()


@pytest.mark.parametrize("out", [BF, F])
@pytest.mark.parametrize("n,K,N", EPILOGUES)
def test_linear_elu_near_zero(n, K, N, out):
    """ELU of small negative sums keeps their leading bits. All products have
    one sign, so the sum's bound (128 products a block and the scaled block
    sums, each addition off by at most 2 U) is relative to the sum; ELU's slope
    is at most 1, and its exponential minus one is off by at most 20 U of the
    result (two units in the last place of a fast exponential below exp(-1/8),
    against 1 - exp(-1/8))."""
    x = randn(n, n, K).abs() * torch.logspace(-9, 1, n, device="cuda")[:, None]
    q, s = quantise(x)
    w, ws = quantise_weight(-randn(K, K, N).abs() * K ** -0.5)
    y = torch.empty(n, N, dtype=out, device="cuda")
    hc.hc_fp8_linear_fwd(q, s, w, ws, None, hc.HC_ACT_ELU, y)
    xv = q.view(torch.float8_e4m3fn).to(D64)[:, :K] * s.to(D64).t().repeat_interleave(128, 1)[:, :K]
    wv = w.view(torch.float8_e4m3fn).to(D64)[:, :K] \
        * ws.to(D64).repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    z = xv @ wv.t()
    ref = torch.expm1(z)
    tol = (2 * 128 + 2 * (K // 128 + 1) + 8) * U * z.abs() + 20 * U * ref.abs() \
        + (2.0 ** -8 if out == BF else U) * ref.abs()
    bad = (y.to(D64) - ref).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off"


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("C", [1, 2, 7, 24, 131, 264, 500, 1000, 2048, 2051, 4104, 8192, 8200, 20001])
def test_layer_norm_constant_rows(C, dtype):
    """A row of one value has that value as its mean and no differences from
    it, whatever the rounding of its sum: beta exactly, with the gradient's
    xh = 0 exactly as well (dgamma = 0)."""
    v = torch.cat([torch.tensor([0.1, 56188.883, -3.3e-3, 1e30, -7.7e-30, 0.0]),
                   1e4 + 9e4 * torch.rand(60, generator=torch.Generator().manual_seed(C))])
    x = v.cuda()[:, None].expand(-1, C).to(dtype).contiguous()
    gamma, beta = 1 + randn(1, C).abs(), randn(2, C)
    y, mean, rstd = torch.empty_like(x), torch.empty(len(v), device="cuda"), torch.empty(len(v), device="cuda")
    hc.hc_layer_norm_fwd(x, 1e-5, gamma, beta, y, mean=mean, rstd=rstd)
    assert torch.equal(mean, x[:, 0].float())
    assert torch.equal(y, beta.to(dtype).expand(len(v), C))
    dg = torch.empty(C, device="cuda")
    hc.hc_layer_norm_bwd(x, torch.ones_like(x), gamma, mean, rstd, dgamma=dg)
    assert (dg == 0).all()


@pytest.mark.parametrize("C", [8, 131, 264, 2048, 2051, 8200])
def test_layer_norm_mean_of_infinities(C):
    """The saved mean of a row with infinities of one sign is that infinity
    (sum x / C); the row's norm is NaN."""
    x = randn(C, 5, C)
    x[1, C - 1], x[2, 0], x[3, 1], x[3, 2] = float("inf"), float("-inf"), float("inf"), float("-inf")
    y, mean, rstd = torch.empty_like(x), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    hc.hc_layer_norm_fwd(x, 1e-5, None, None, y, mean=mean, rstd=rstd)
    assert mean[1] == float("inf") and mean[2] == float("-inf") and mean[3].isnan()
    assert y[1:4].isnan().all() and rstd[1:4].isnan().all()
    assert y[[0, 4]].isfinite().all() and mean[[0, 4]].isfinite().all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("C", [7, 24, 64, 131, 264, 2048, 8200])
def test_layer_norm_rows_apart(C, dtype):
    """A row gives the same bits beside rows far from zero as alone, and such
    rows the same bits as alone."""
    x = randn(C, 40, C, dtype=dtype)
    x[1::3] = (3000 + 4 * randn(C + 1, 13, C)).to(dtype)
    x[2::3] = 1234.5
    y, mean, rstd = torch.empty_like(x), torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
    hc.hc_layer_norm_fwd(x, 1e-5, None, None, y, mean=mean, rstd=rstd)
    one, m, r = torch.empty_like(x[:1]), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    for n in range(40):
        hc.hc_layer_norm_fwd(x[n:n + 1].clone(), 1e-5, None, None, one, mean=m, rstd=r)
        assert torch.equal(one[0], y[n]) and m[0] == mean[n] and r[0] == rstd[n], n


@pytest.mark.parametrize("dtype,C", [(F, 131), (F, 2001), (F, 300), (BF, 131), (BF, 2001),
                                     (BF, 130), (BF, 300), (BF, 2002), (BF, 1), (F, 2)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_quantize_rows_padding_is_zero(dtype, C, value):
    """The bytes of a row beyond C are zero, also where its last block holds a
    NaN or an infinity (the block's channels are then not numbers, or zero)."""
    x = randn(C, 5, C, dtype=dtype)
    x[1, C - 1] = value
    x[3, (C - 1) // 128 * 128] = value
    for t in (x, torch.empty(x.numel() + 1, dtype=dtype, device="cuda")[1:].view(x.shape).copy_(x)):
        q, s = quantise(t)
        assert (q[:, C:] == 0).all()
        assert not s[-1, [1, 3]].isfinite().any() and s[:, [0, 2, 4]].isfinite().all()
        last = q[:, :C].view(torch.float8_e4m3fn).float()
        assert last[1, C - 1].isnan() and last[3, (C - 1) // 128 * 128].isnan()
