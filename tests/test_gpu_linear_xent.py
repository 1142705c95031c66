"""Cross entropy behind a linear layer and its gradients against plain 64-bit
implementations.

Tolerances, derived from the arithmetic. U = 2^-24. The tensor cores add the 16
exact products of a step to an fp32 accumulator; a step is taken to be off by at
most 2^-22 of the sum of all magnitudes S (two truncations), so that a sum of K
terms is off by (K / 16 + 1) 2^-22 S. fp32 operands take six such sums, and what the
split leaves out is below 2^-24 S. A logit l is off by that, T, and the
rounding of its bias. exp is taken of a difference (U |l - lse| and U |lse| of
it), by a base-2 exponential of 2 units in the last place (2^-22) of a rounded product
(2 U |l - lse|); a row's sum of V positive terms is a chain of at most 64
additions behind 1024 joins with two such exponentials each. G is off by what its logit
and lse are, relative to the probability, and, as bf16, by 2^-8 of itself."""
import pytest

from paper_2608_09388_gb300 import hc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from _tokens import BF, D64, F, U, count_of, full, gen, randn, rounding, shifted, within  # noqa: E402


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


def sum_tol(K, dtype, S):
    """Error of a sum of K products of magnitudes that add up to S."""
    steps = (K // 16 + 8) * (6 if dtype == F else 1)
    return (steps * 2.0 ** -22 + (U if dtype == F else 0)) * S


def inputs(seed, cap, V, C, dtype, bias=True, ignored=0.2):
    g = gen(seed)
    W = randn(g, V, C) * C ** -0.5
    t = torch.randint(0, V, (cap,), generator=g, device="cuda")
    lean = 8 * torch.rand(cap, 1, generator=g, device="cuda")
    x = (randn(g, cap, C) + lean * W[t]).to(dtype)
    b = 0.3 * randn(g, V) if bias else None
    gone = torch.rand(cap, generator=g, device="cuda") < ignored
    return x, W.to(dtype), b, torch.where(gone, -1, t).int(), randn(g, cap)


def logits_ref(x, W, b):
    l, S = x.to(D64) @ W.to(D64).t(), x.to(D64).abs() @ W.to(D64).abs().t()
    if b is not None:
        l = l + b.to(D64)
    return l, sum_tol(x.shape[1], x.dtype, S) + U * l.abs()


def fwd_ref(x, W, b, t):
    """loss and lse of the tokens that take part, with their bounds."""
    l, T = logits_ref(x, W, b)
    lse = torch.logsumexp(l, 1)
    p = torch.exp(l - lse[:, None])
    # each term off by its logit, the exponentials and products behind it
    terms = (p * (T + 4 * U * (l - l.amax(1, keepdim=True)).abs())).sum(1)
    tl = terms + 64 * U + 40 * 2.0 ** -22 + 4 * U * lse.abs()
    at = l.gather(1, t[:, None])[:, 0]
    return lse - at, lse, tl + T.gather(1, t[:, None])[:, 0] + U * at.abs(), tl


def bwd_ref(x, W, b, t, lse, dloss):
    l, T = logits_ref(x, W, b)
    d = l - lse.to(D64)[:, None]
    p = torch.exp(d)
    tp = p * (T + 2.0 ** -21 + 4 * U * (d.abs() + lse.to(D64).abs()[:, None]))
    G = p.scatter_add(1, t[:, None], -torch.ones_like(p[:, :1]))
    tg = (tp + U * G.abs()) * dloss.to(D64).abs()[:, None]
    G = G * dloss.to(D64)[:, None]
    xd, Wd = x.to(D64), W.to(D64)
    half = 2.0 ** -8 if x.dtype == BF else 2.0 ** -24
    # the products may take a number below the normal range as zero: all of it is off
    tg16 = tg + half * G.abs() + torch.where(G.abs() < 2.0 ** -126, G.abs(), 0.0)
    dx, dW, db = G @ Wd, G.t() @ xd, G.sum(0)
    Sx, Sw = G.abs() @ Wd.abs(), G.abs().t() @ xd.abs()
    tdx = tg16 @ Wd.abs() + sum_tol(W.shape[0], x.dtype, Sx) + rounding(x.dtype, dx)
    tdw = tg16.t() @ xd.abs() + sum_tol(x.shape[0], x.dtype, Sw) + rounding(x.dtype, dW)
    return dx, dW, db, tdx, tdw, tg.sum(0) + (x.shape[0] + 8) * U * G.abs().sum(0)


def run_all(x, W, b, t, dloss, n, stream=None):
    cap, C = x.shape
    V = W.shape[0]
    o = dict(loss=full((cap,)), lse=full((cap,)), dx=full((cap, C), x.dtype),
             dW=full((V, C), x.dtype), dbias=full((V,)))
    cnt = None if n is None else count_of(n)
    torch.cuda.synchronize()
    hc.hc_linear_cross_entropy_fwd(x, W, b, t, o["loss"], o["lse"], count=cnt, stream=stream)
    hc.hc_linear_cross_entropy_bwd(x, W, b, t, o["lse"], dloss, dx=o["dx"], dW=o["dW"],
                                   dbias=o["dbias"], count=cnt, stream=stream)
    return o


def check(x, W, b, t, dloss, n, o):
    on = torch.nonzero(t[:n] >= 0)[:, 0]
    off = torch.nonzero(t[:n] < 0)[:, 0]
    tt = t[on].long()
    loss, lse, tloss, tlse = fwd_ref(x[on], W, b, tt)
    within(o["lse"][on], lse, tlse, "lse")
    within(o["loss"][on], loss, tloss, "loss")
    dx, dW, db, tdx, tdw, tdb = bwd_ref(x[on], W, b, tt, o["lse"][on], dloss[on])
    within(o["dx"][on], dx, tdx, "dx")
    within(o["dW"], dW, tdw, "dW")
    within(o["dbias"], db, tdb, "dbias")
    for k in ("loss", "lse", "dx"):
        assert (o[k][off] == 0).all(), k
        assert (o[k][n:] == 77).all(), k


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,slack,V,C", [
    (1, 0, 1, 1), (1, 0, 300, 64), (2, 3, 42, 64), (5, 0, 31, 7), (37, 0, 64, 8), (64, 1, 65, 16),
    (63, 0, 128, 63), (65, 5, 129, 65), (128, 0, 256, 128), (129, 0, 257, 129), (255, 9, 1000, 136),
    (256, 0, 2, 256), (257, 300, 511, 264), (300, 0, 5003, 72), (700, 0, 513, 1000),
    (1500, 0, 2049, 200), (4099, 0, 77, 96), (3, 0, 40000, 520), (513, 0, 12, 2056)])
def test_all_outputs(n, slack, V, C, dtype):
    x, W, b, t, dloss = inputs(n + V + C, n + slack, V, C, dtype)
    check(x, W, b, t, dloss, n, run_all(x, W, b, t, dloss, n))


@pytest.mark.parametrize("dtype", [BF, F])
def test_pieces(dtype):
    """A large capacity: G is written and used in pieces of 2048 classes."""
    n, cap, V, C = 300, 150000, 5000, 136
    x, W, b, t, dloss = inputs(1, cap, V, C, dtype)
    check(x, W, b, t, dloss, n, run_all(x, W, b, t, dloss, n))


@pytest.mark.parametrize("dtype", [BF, F])
def test_long_sums(dtype):
    """Many classes for few tokens (the sum of dx in parts), many tokens for few
    classes, each output alone and no bias: the same bits."""
    for n, V, C in ((300, 20000, 264), (9000, 50, 40)):
        x, W, b, t, dloss = inputs(n, n, V, C, dtype, ignored=0.5)
        o = run_all(x, W, b, t, dloss, None)
        check(x, W, b, t, dloss, n, o)
        for k in ("dx", "dW", "dbias"):
            one = torch.full_like(o[k], 77)
            hc.hc_linear_cross_entropy_bwd(x, W, b, t, o["lse"], dloss, **{k: one})
            assert torch.equal(one, o[k]), k
        for k in ("loss", "lse"):
            one = full((n,))
            hc.hc_linear_cross_entropy_fwd(x, W, b, t, **{k: one})
            assert torch.equal(one, o[k]), k
        x2 = x.clone()
        hc.hc_linear_cross_entropy_bwd(x2, W, b, t, o["lse"], dloss, dx=x2)
        assert torch.equal(x2, o["dx"])
        check(x, W, None, t, dloss, n, run_all(x, W, None, t, dloss, n))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [0, 5, 300])
def test_no_token_takes_part(n, dtype):
    x, W, b, t, dloss = inputs(2, 300, 100, 72, dtype)
    t.fill_(-1)
    x.fill_(float("nan"))
    dloss.fill_(float("nan"))
    o = run_all(x, W, b, t, dloss, n)
    assert (o["dW"] == 0).all() and (o["dbias"] == 0).all()
    for k in ("loss", "lse", "dx"):
        assert (o[k][:n] == 0).all() and (o[k][n:] == 77).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_capacity_zero(dtype):
    _, W, b, _, _ = inputs(2, 3, 100, 72, dtype)
    dW, db = full((100, 72), dtype), full((100,))
    e = torch.empty(0, device="cuda")
    hc.hc_linear_cross_entropy_bwd(W[:0], W, b, e.int(), e, e, dW=dW, dbias=db)
    assert (dW == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_what_takes_no_part_has_no_effect(dtype):
    """NaN in tokens that take no part and behind the last one."""
    n, cap, V, C = 200, 300, 150, 72
    x, W, b, t, dloss = inputs(3, cap, V, C, dtype)
    want = run_all(x, W, b, t, dloss, n)
    hole = (t < 0) | (torch.arange(cap, device="cuda") >= n)
    x[hole], dloss[hole] = float("nan"), float("nan")
    got = run_all(x, W, b, t, dloss, n)
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("dtype", [BF, F])
def test_masked_classes(dtype):
    """A bias of -infinity, or of the lowest number, takes a class out; also
    whole tiles of them, and all but one."""
    n, V, C = 70, 700, 40
    for low in (float("-inf"), torch.finfo(F).min):
        x, W, b, t, dloss = inputs(4, n, V, C, dtype, ignored=0.0)
        b[:513], b[600:620] = low, low
        t[:] = torch.where((t < 513) | ((t >= 600) & (t < 620)), 650, t)
        keep = torch.nonzero(b > -1e30)[:, 0]
        inside = torch.searchsorted(keep, t.long())
        o = run_all(x, W, b, t, dloss, n)
        loss, lse, tloss, tlse = fwd_ref(x, W[keep], b[keep], inside)
        within(o["lse"], lse, tlse, "lse")
        within(o["loss"], loss, tloss, "loss")
        dx, dW, db, tdx, tdw, tdb = bwd_ref(x, W[keep], b[keep], inside, o["lse"], dloss)
        within(o["dx"], dx, tdx, "dx")
        within(o["dW"][keep], dW, tdw, "dW")
        within(o["dbias"][keep], db, tdb, "dbias")
        rest = b <= -1e30
        assert (o["dW"][rest] == 0).all() and (o["dbias"][rest] == 0).all()
    b[:] = float("-inf")
    b[699], t[:] = 0.5, 699
    o = run_all(x, W, b, t, dloss, n)
    assert (o["loss"].abs() <= 2.0 ** -20 * o["lse"].abs().clamp_min(1)).all()
    # the lowest number everywhere: as none at all, one step of rounding beside it
    b[:] = torch.finfo(F).min
    hc.hc_linear_cross_entropy_fwd(x, W, b, t, o["loss"], o["lse"])
    assert o["lse"].isfinite().all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_values(dtype):
    """Large logits, a sure token, a NaN in one token."""
    n, V, C = 33, 400, 72
    x, W, b, t, dloss = inputs(5, n, V, C, dtype, ignored=0.0)
    x[:8] *= 100
    x[9] = 0
    check(x, W, b, t, dloss, n, run_all(x, W, b, t, dloss, n))
    want = full((n,))
    hc.hc_linear_cross_entropy_fwd(x, W, b, t, loss=want)
    x[3, 5] = float("nan")
    got, lse = full((n,)), full((n,))
    hc.hc_linear_cross_entropy_fwd(x, W, b, t, loss=got, lse=lse)
    rest = torch.arange(n, device="cuda") != 3
    assert got[3].isnan() and torch.equal(got[rest], want[rest])
    dx, dW = full((n, C), dtype), full((V, C), dtype)
    hc.hc_linear_cross_entropy_bwd(x, W, b, t, lse, dloss, dx=dx, dW=dW)
    assert dx[3].isnan().all() and dx[rest].isfinite().all() and dW.isnan().any()


@pytest.mark.parametrize("dtype", [BF, F])
def test_shifted_rows(dtype):
    """Rows that are not 16-byte aligned, of widths that would allow it."""
    n, V, C = 130, 300, 136
    x, W, b, t, dloss = inputs(6, n, V, C, dtype)
    o = dict(loss=full((n,)), lse=full((n,)), dx=shifted(x), dW=shifted(W), dbias=shifted(b))
    xs, Ws, bs = shifted(x), shifted(W), shifted(b)
    hc.hc_linear_cross_entropy_fwd(xs, Ws, bs, t, o["loss"], o["lse"])
    hc.hc_linear_cross_entropy_bwd(xs, Ws, bs, t, o["lse"], dloss, dx=o["dx"], dW=o["dW"],
                                   dbias=o["dbias"])
    check(x, W, b, t, dloss, n, o)


def test_fp32_range():
    """fp32 operands up to the largest number: what bf16 would round to an
    infinity does not become one; exact products, so exact logits."""
    V, C = 300, 136
    W, x = torch.zeros(V, C, device="cuda"), torch.zeros(6, C, device="cuda")
    top = torch.finfo(F).max
    W[200, 3], x[:, 3] = 2.0 ** -126, torch.tensor([top, -top, 1.0, 2.0 ** 127, 0.0, -1.5], device="cuda")
    t = full((6,), torch.int32, 200)
    loss, lse = full((6,)), full((6,))
    hc.hc_linear_cross_entropy_fwd(x, W, None, t, loss, lse)
    l = x[:, 3].to(D64) * 2.0 ** -126
    want = torch.log(torch.exp(l) + (V - 1))
    within(lse, want, 2.0 ** -20 * want, "lse")
    within(loss, want - l, 2.0 ** -20 * want, "loss")


def test_targets_out_of_range():
    n, V, C = 50, 40, 24
    x, W, b, t, dloss = inputs(7, n, V, C, F)
    clean = t.clone()
    clean[[3, 40]] = -1
    want = run_all(x, W, b, clean, dloss, n)
    t[3], t[40] = V, -2
    got = run_all(x, W, b, t, dloss, n)
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX
    assert all(torch.equal(got[k], want[k]) for k in want)
    hc.hc_linear_cross_entropy_fwd(x, W, b, clean, got["loss"], count=count_of(n + 1))
    assert hc.hc_get_device_status() == hc.HC_ERR_CAPACITY
    assert torch.equal(got["loss"], want["loss"])


def test_equal_weights():
    """A mean over tokens that are far from sure: G's target entries, p - 1 times
    one number, are held to p of it (below 2^-9, p - 1 rounds to -1), the others to
    2^-8 of themselves, whatever that number's mantissa; dx has the target's
    rounding given back."""
    n, V, C = 700, 3000, 264
    x, W, b, t, _ = inputs(12, n, V, C, BF, bias=False, ignored=0.0)
    x = (x.float() * 0.05).to(BF)
    for weight in (1 / 700, -1.9921875 / 512, 3e-30, 1.0):
        dloss = full((n,), value=weight)
        o = run_all(x, W, b, t, dloss, None)
        l, T = logits_ref(x, W, b)
        d = l - o["lse"].to(D64)[:, None]
        p = torch.exp(d)
        assert float(p.max()) < 2.0 ** -9
        w = dloss.to(D64).abs()[:, None]
        tp = p * (T + 2.0 ** -21 + 4 * U * (d.abs() + o["lse"].to(D64).abs()[:, None]))
        at = torch.zeros_like(p).scatter_(1, t.long()[:, None], 1.0)
        G = (p - at) * dloss.to(D64)[:, None]
        tg = (tp + 4 * U * at + 2.0 ** -8 * p) * w
        xd, Wd = x.to(D64), W.to(D64)
        dx, dW = G @ Wd, G.t() @ xd
        within(o["dx"], dx, tg @ Wd.abs() + sum_tol(V, BF, G.abs() @ Wd.abs()) + rounding(BF, dx), "dx")
        within(o["dW"], dW, (tg + p * at * w).t() @ xd.abs() + sum_tol(n, BF, G.abs().t() @ xd.abs())
               + rounding(BF, dW), "dW")
        within(o["dbias"], G.sum(0), ((tp + 4 * U * at) * w).sum(0) + (n + 8) * U * G.abs().sum(0), "dbias")


@pytest.mark.parametrize("dtype", [BF, F])
def test_sums_of_gradients_over_classes(dtype):
    """dbias adds up to the tokens' dloss times what their probabilities miss of
    one: logits and lse are rounded alike, whatever the length of the sums. A
    probability off by the exponential (2^-22), a rounded product (2 U d, d up to 30
    here) and difference (U of lse, up to 16): 100 U in all, and the chains' 512
    channels, which may be cut off differently by their order alone: 16 U of the logit's
    magnitudes (up to 40) over the 4 chains or more that it has."""
    n, V, C = 200, 700, 2056
    x, W, b, t, _ = inputs(14, n, V, C, dtype, ignored=0.0)
    dloss = torch.full((n,), 1.0, device="cuda")
    o = run_all(x, W, b, t, dloss, None)
    assert abs(float(o["dbias"].to(D64).sum())) <= n * (100 + 16 * 40) * U


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,slack,V,C", [
    (1, 0, 5003, 2056), (1, 0, 1000, 11520), (1, 1, 700, 333), (2, 0, 511, 4104), (2, 1, 40000, 264),
    (3, 0, 129, 1000), (3, 1, 2049, 130), (4, 0, 33, 2048), (4, 0, 6000, 65), (0, 4, 300, 520),
    (5, 0, 3001, 1280), (5, 1, 700, 333), (6, 2, 40000, 264), (7, 0, 129, 1028), (8, 0, 2049, 31),
    (8, 0, 33, 1032), (1, 7, 513, 257), (8, 0, 500, 2056)])
def test_few_tokens(n, slack, V, C, dtype):
    """Up to eight tokens, and the same bits of each gradient alone."""
    x, W, b, t, dloss = inputs(n + V + C, n + slack, V, C, dtype, ignored=0.0)
    if n in (4, 7, 8):
        t[1] = -1
        x[1], dloss[1] = float("nan"), float("inf")
    x[n:], dloss[n:] = float("nan"), float("nan")
    o = run_all(x, W, b, t, dloss, n)
    check(x, W, b, t, dloss, n, o)
    for name in ("dx", "dW", "dbias"):
        alone = full(o[name].shape, o[name].dtype)
        hc.hc_linear_cross_entropy_bwd(x, W, b, t, o["lse"], dloss, count=count_of(n), **{name: alone})
        assert torch.equal(alone, o[name]), name


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("cap,C", [(1, 2056), (2, 2056), (3, 2056), (4, 2056), (5, 1280), (8, 1280)])
def test_few_sure_tokens(cap, C, dtype):
    """A logit of about 1000, the others' below 200: their probabilities are zero in fp32
    (exp(-104) is), lse is the logit to the last bit and so every gradient zero."""
    V = 700
    g = gen(cap)
    W = (randn(g, V, C) * C ** -0.5).to(dtype)
    t = torch.randint(0, V, (cap,), generator=g, device="cuda")
    x, b = (1000 * W[t].float()).to(dtype), 0.3 * randn(g, V)
    o = run_all(x, W, b, t.int(), torch.full((cap,), 3.0, device="cuda"), None)
    for name in ("loss", "dx", "dW", "dbias"):
        assert (o[name] == 0).all(), name


@pytest.mark.parametrize("cap,V,C,dtype", [(1, 3000, 520, BF), (4, 900, 264, F), (8, 2000, 1032, BF)])
def test_few_tokens_replayed(cap, V, C, dtype):
    """On two streams at a time, and captured, replayed with other rows and targets."""
    x, W, b, t, dloss = inputs(cap + V, cap, V, C, dtype, ignored=0.0)
    want = run_all(x, W, b, t, dloss, None)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [run_all(x, W, b, t, dloss, None, s) for s in streams]
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(o[k], want[k]) for k in want)
    side, cnt, o = streams[0], count_of(cap), outs[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hc.hc_linear_cross_entropy_fwd(x, W, b, t, o["loss"], o["lse"], count=cnt, stream=side)
        hc.hc_linear_cross_entropy_bwd(x, W, b, t, o["lse"], dloss, dx=o["dx"], dW=o["dW"],
                                       dbias=o["dbias"], count=cnt, stream=side)
    for m in (cap, cap - 1):
        cnt.fill_(m)
        x.copy_(x.flip(1))
        t.copy_((t + 17) % V)
        for v in o.values():
            v.fill_(77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(x, W, b, t, dloss, m, o)


@pytest.mark.parametrize("dtype", [BF, F])
def test_few_tokens_bad_target(dtype):
    """A target outside the classes is reported by either direction, and the token
    takes no part."""
    x, W, b, t, dloss = inputs(5, 3, 900, 264, dtype, ignored=0.0)
    t[1] = -1
    want = run_all(x, W, b, t, dloss, None)
    t[1] = 900
    o = run_all(x, W, b, t, dloss, None)
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX
    assert all(torch.equal(o[k], want[k]) for k in want)
    hc.hc_linear_cross_entropy_bwd(x, W, b, t, o["lse"], dloss, dbias=o["dbias"])
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX


def test_few_tokens_in_place():
    """dx may be x."""
    x, W, b, t, dloss = inputs(3, 4, 900, 520, BF, ignored=0.0)
    o = run_all(x, W, b, t, dloss, None)
    hc.hc_linear_cross_entropy_bwd(x, W, b, t, o["lse"], dloss, dx=x)
    assert torch.equal(x, o["dx"])


def test_first_weight_special():
    """The first token's dloss of zero, infinite, or below the normal numbers:
    the others' gradients are as without it."""
    n, V, C = 300, 500, 136
    x, W, b, t, dloss = inputs(13, n, V, C, BF, ignored=0.0)
    dloss[0] = 0
    want = run_all(x, W, b, t, dloss, None)
    check(x, W, b, t, dloss, n, want)
    for first in (2.0 ** -140, -2.0 ** -149):
        dloss[0] = first
        check(x, W, b, t, dloss, n, run_all(x, W, b, t, dloss, None))
    dloss[0] = float("inf")
    o = run_all(x, W, b, t, dloss, None)
    assert torch.equal(o["dx"][1:], want["dx"][1:]) and not o["dx"][0].isfinite().any()


def test_differences():
    """dx, dW and dbias against central differences of the 64-bit loss, step
    h = 2^-12: the differences' own error is below h^2 times the third
    derivative (a few tens here) plus 2^-50 / h."""
    n, V, C, h = 4, 7, 5, 2.0 ** -12
    x, W, b, t, dloss = inputs(8, n, V, C, F)
    o = run_all(x, W, b, t, dloss, n)

    def loss(x, W, b):
        p = torch.log_softmax(x @ W.t() + b, 1)
        at = p.gather(1, t.long().clamp_min(0)[:, None])[:, 0]
        return float((torch.where(t >= 0, -at, 0.0) * dloss.to(D64)).sum())

    p = [x.to(D64), W.to(D64), b.to(D64)]
    for k, got in ((0, o["dx"]), (1, o["dW"]), (2, o["dbias"])):
        flat = p[k].view(-1)
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + h
            up = loss(*p)
            flat[i] = old - h
            down = loss(*p)
            flat[i] = old
            assert abs((up - down) / (2 * h) - float(got.view(-1)[i])) <= 2e-5, (k, i)


@pytest.mark.parametrize("dtype,V,C", [(BF, 1000, 264), (F, 300, 72), (BF, 77, 33)])
def test_streams_and_graph(dtype, V, C):
    """Two streams at a time, the same bits from run to run, and a captured
    step replayed with other counts and targets."""
    n = 700
    x, W, b, t, dloss = inputs(9, n, V, C, dtype)
    want = run_all(x, W, b, t, dloss, None)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        outs = [run_all(x, W, b, t, dloss, None, s) for s in streams]
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(o[k], want[k]) for k in want)
    side, cnt = streams[0], count_of(n)
    o = outs[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hc.hc_linear_cross_entropy_fwd(x, W, b, t, o["loss"], o["lse"], count=cnt, stream=side)
        hc.hc_linear_cross_entropy_bwd(x, W, b, t, o["lse"], dloss, dx=o["dx"], dW=o["dW"],
                                       dbias=o["dbias"], count=cnt, stream=side)
    for m in (n, 0, 333):
        cnt.fill_(m)
        t[:100] = -1 if m == 333 else t[:100]
        for v in o.values():
            v.fill_(77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if m:
            check(x, W, b, t, dloss, m, o)
        else:
            assert (o["dW"] == 0).all() and (o["loss"] == 77).all() and (o["dx"] == 77).all()


# Far below the microsecond that a first copy from memory takes.
SHORT_LIMIT_NS = 100


@pytest.fixture
def short_waits():
    yield lambda: hc.hc_test_set_option(hc.HC_TEST_WAIT_LIMIT_NS, SHORT_LIMIT_NS)
    hc.hc_test_set_option(hc.HC_TEST_WAIT_LIMIT_NS, 0)
    hc.hc_get_device_status()


@pytest.mark.parametrize("n,V,C,dtype", [(700, 3000, 520, BF), (300, 300, 2056, F)])
def test_wait_timeout_reported_then_correct(short_waits, n, V, C, dtype):
    """With the pipeline-wait limit far below the time its first copies take the
    call gives up and says so; with the limit back it is right again. Every wait
    still ends, only sooner than the work it waits for."""
    x, W, b, t, dloss = inputs(10, n, V, C, dtype)
    want = run_all(x, W, b, t, dloss, None)
    assert hc.hc_get_device_status() == hc.HC_OK
    short_waits()
    seen = set()
    for _ in range(5):
        run_all(x, W, b, t, dloss, None)
        seen.add(hc.hc_get_device_status())
    assert seen <= {hc.HC_ERR_TIMEOUT, hc.HC_OK} and hc.HC_ERR_TIMEOUT in seen
    hc.hc_test_set_option(hc.HC_TEST_WAIT_LIMIT_NS, 0)
    for _ in range(3):
        got = run_all(x, W, b, t, dloss, None)
        assert hc.hc_get_device_status() == hc.HC_OK
        assert all(torch.equal(got[k], want[k]) for k in want)
