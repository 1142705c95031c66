"""The root-mean-square norm with the residual's addition, its 8-bit output and
its gradient, against plain 64-bit implementations.

Tolerances, derived from the arithmetic. U = 2^-24. A row's sum is taken by at
most 512 threads in chains, D(C) = C / 256 + 64 additions deep with the tree
over the threads; its squares are all positive, so the sum is off by D U of
itself, rstd by half of that, 2 units in the last place (4 U) of rsqrtf and
the roundings of the mean and eps (2 U). An output is a product of two more
roundings, then rounded to its type. Stored sums h, and the 8-bit values and
scales of given fp32 rows, are exact."""
import pytest

from paper_2608_09388_gb300 import hc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from _tokens import BF, D64, F, U, count_of, full, gen, randn, rounding, shifted, within  # noqa: E402

Q8 = torch.float8_e4m3fn


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


def depth(C):
    return C / 256 + 64


def inputs(seed, cap, C, dtype):
    g = gen(seed)
    x = (randn(g, cap, C) * (0.5 + torch.rand(cap, 1, generator=g, device="cuda"))).to(dtype)
    res, dy, dres = (randn(g, cap, C, dtype=dtype) for _ in range(3))
    return x, res, dy, dres, 1 + 0.2 * randn(g, C)


def stored(x, res):
    return x if res is None else (x.float() + res.float()).to(x.dtype)


def fwd_ref(h, gamma, eps):
    """v, rstd in 64 bits and their bounds, h as stored."""
    C = h.shape[1]
    h = h.to(D64)
    ga = torch.ones(C, dtype=D64, device="cuda") if gamma is None else gamma.to(D64)
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    v = h * rstd * ga
    rel = (depth(C) / 2 + 6) * U
    return v, rstd[:, 0], (rel + 2 * U) * v.abs(), (rel * rstd)[:, 0]


def quant_ref(v):
    """The 8-bit form of fp32 rows: bytes and scales."""
    n, C = v.shape
    nb, pitch = (C + 127) // 128, hc.HC_FP8_PITCH(C)
    b = torch.nn.functional.pad(v, (0, nb * 128 - C)).view(n, nb, 128)
    top = b.abs().amax(2)
    s = (top / torch.full_like(top, 448.0)).clamp_min(2.0 ** -126)
    q = (b / s[:, :, None]).to(Q8).view(n, -1)
    q = torch.nn.functional.pad(q.view(torch.uint8), (0, max(0, pitch - nb * 128)))[:, :pitch]
    return q, s.t()


def bwd_ref(h, dy, dres, gamma, rstd):
    """dx, dgamma in 64 bits from the fp32 rstd, and their bounds."""
    n, C = h.shape
    h, dy, r = h.to(D64), dy.to(D64), rstd.to(D64)[:, None]
    ga = torch.ones(C, dtype=D64, device="cuda") if gamma is None else gamma.to(D64)
    hh, g = h * r, dy * ga
    c = (g * hh).mean(1, keepdim=True)
    t = r * (g - hh * c)
    D = depth(C) + 8
    tol = r * (4 * U * g.abs() + hh.abs() * (D * U * (g * hh).abs().mean(1, keepdim=True) + 6 * U * c.abs()))
    dx = t if dres is None else t + dres.to(D64)
    return dx, (dy * hh).sum(0), tol + 2 * U * (t.abs() + dx.abs()), (n + 8) * U * (dy * hh).abs().sum(0)


# widths around every change of the kernels' layout: single channels, a vector,
# a warp, several rows per warp or per block, odd and wide rows
WIDTHS = (1, 2, 7, 8, 24, 33, 64, 65, 72, 127, 129, 131, 255, 256, 257, 264, 500, 512, 513, 1000, 1023, 1024,
          1025, 1032, 2047, 2048, 2051, 2056, 4095, 4096, 4100, 4104, 8191, 8192, 8200, 8201, 16384, 20001, 20004)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("C", WIDTHS)
def test_all_outputs(C, dtype):
    n, cap = (203, 211) if C <= 4104 else (19, 23)
    x, res, dy, dres, gamma = inputs(C, cap, C, dtype)
    h, y, dx = (full((cap, C), dtype) for _ in range(3))
    rstd, dg = full((cap,)), full((C,))
    q = full((cap, hc.HC_FP8_PITCH(C)), torch.uint8, 77)
    sc = full(((C + 127) // 128, cap))
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, res=res, h=h, y=y, rstd=rstd, q=q, scales=sc, count=count_of(n))
    want = stored(x, res)
    assert torch.equal(h[:n], want[:n])
    v, rr, tv, tr = fwd_ref(want[:n], gamma, 1e-5)
    within(rstd[:n], rr, tr, "rstd")
    within(y[:n], v, tv + rounding(dtype, v), "y")
    q_ref, s_ref = quant_ref(want[:n].float() * rstd[:n, None] * gamma)
    assert torch.equal(sc[:, :n], s_ref) and torch.equal(q[:n], q_ref)
    assert (h[n:] == 77).all() and (y[n:] == 77).all() and (rstd[n:] == 77).all()
    assert (q[n:] == 77).all() and (sc[:, n:] == 77).all()
    hc.hc_rms_norm_bwd(h, dy, gamma, rstd, dres=dres, dx=dx, dgamma=dg, count=count_of(n))
    rdx, rdg, tdx, tdg = bwd_ref(h[:n], dy[:n], dres[:n], gamma, rstd[:n])
    within(dx[:n], rdx, tdx + rounding(dtype, rdx), "dx")
    within(dg, rdg, tdg, "dgamma")
    assert (dx[n:] == 77).all()


def two_past(t):
    """A copy whose first element lies two past a 16-byte boundary."""
    s = torch.empty(t.numel() + 2, dtype=t.dtype, device="cuda")[2:].view(t.shape)
    return s.copy_(t)


# rows that allow 4-byte loads and no wider ones: by their width, by gamma's place
# alone, by theirs; around the widths where a block's rows of v pass 32 and 48 KiB
@pytest.mark.parametrize("C,moved", [(C, "none") for C in (514, 642, 770, 1022, 2050, 2946, 3078, 4094, 4098, 6018, 6150, 8190)]
                         + [(C, m) for C in (1024, 4096, 8192) for m in ("gamma", "rows")])
def test_8_bits_of_even_rows(C, moved):
    n, cap = 203, 211
    x, res, _, _, gamma = inputs(C + 2, cap, C, BF)
    h, y = full((cap, C), BF), full((cap, C), BF)
    if moved == "gamma":
        gamma = two_past(gamma)
    if moved == "rows":
        x, res, h, y = (two_past(t) for t in (x, res, h, y))
    rstd, q = full((cap,)), full((cap, hc.HC_FP8_PITCH(C)), torch.uint8, 77)
    sc = full(((C + 127) // 128, cap))
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, res=res, h=h, y=y, rstd=rstd, q=q, scales=sc, count=count_of(n))
    want = stored(x, res)
    assert torch.equal(h[:n], want[:n])
    v, rr, tv, tr = fwd_ref(want[:n], gamma, 1e-5)
    within(rstd[:n], rr, tr, "rstd")
    within(y[:n], v, tv + rounding(BF, v), "y")
    q_ref, s_ref = quant_ref(want[:n].float() * rstd[:n, None] * gamma)
    assert torch.equal(sc[:, :n], s_ref) and torch.equal(q[:n], q_ref)
    assert (h[n:] == 77).all() and (y[n:] == 77).all() and (rstd[n:] == 77).all()
    assert (q[n:] == 77).all() and (sc[:, n:] == 77).all()
    # the 8-bit rows alone, of the stored sums
    q1, sc1 = torch.full_like(q, 77), torch.full_like(sc, 77)
    hc.hc_rms_norm_fwd(h, 1e-5, gamma, q=q1, scales=sc1, count=count_of(n))
    assert torch.equal(q1, q) and torch.equal(sc1, sc)


@pytest.mark.parametrize("n", [0, 1, 2, 3, 127, 128, 129, 5000])
@pytest.mark.parametrize("C,dtype", [(64, BF), (131, F), (1024, BF), (4096, F), (8200, BF)])
def test_rows(n, C, dtype):
    cap = n + 3
    x, res, dy, dres, gamma = inputs(n + C, cap, C, dtype)
    h, y, dx = (full((cap, C), dtype) for _ in range(3))
    rstd, dg = full((cap,)), full((C,))
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, res=res, h=h, y=y, rstd=rstd, count=count_of(n))
    hc.hc_rms_norm_bwd(h, dy, gamma, rstd, dres=dres, dx=dx, dgamma=dg, count=count_of(n))
    assert (y[n:] == 77).all() and (dx[n:] == 77).all()
    if n == 0:
        assert (dg == 0).all()
        return
    v, _, tv, _ = fwd_ref(h[:n], gamma, 1e-5)
    within(y[:n], v, tv + rounding(dtype, v), "y")
    rdx, rdg, tdx, tdg = bwd_ref(h[:n], dy[:n], dres[:n], gamma, rstd[:n])
    within(dx[:n], rdx, tdx + rounding(dtype, rdx), "dx")
    within(dg, rdg, tdg, "dgamma")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("C", [40, 131, 1000, 2048, 8191, 12000, 20001])
def test_forms(C, dtype):
    """All rows without a count, no residual, no gamma, each output alone, in
    place, and rows that are not 16-byte aligned."""
    n = 37
    x, res, dy, dres, gamma = inputs(C + 1, n, C, dtype)
    h, y, rstd = full((n, C), dtype), full((n, C), dtype), full((n,))
    q, sc = full((n, hc.HC_FP8_PITCH(C)), torch.uint8, 77), full(((C + 127) // 128, n))
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, res=res, h=h, y=y, rstd=rstd, q=q, scales=sc)
    # each output alone, and in place: the same bits
    y1 = full((n, C), dtype)
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, res=res, y=y1)
    assert torch.equal(y1, y)
    q1, sc1 = torch.empty_like(q).view(Q8), torch.empty_like(sc)
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, res=res, q=q1, scales=sc1)
    assert torch.equal(q1.view(torch.uint8), q) and torch.equal(sc1, sc)
    for hx, yx in ((0, 1), (1, 0)):
        both = [x.clone(), res.clone()]
        hc.hc_rms_norm_fwd(both[0], 1e-5, gamma, res=both[1], h=both[hx], y=both[yx], q=q1, scales=sc1)
        assert torch.equal(both[hx], h) and torch.equal(both[yx], y)
        assert torch.equal(q1.view(torch.uint8), q)
    # without a residual and without gamma
    y1, h1 = x.clone(), full((n, C), dtype)
    hc.hc_rms_norm_fwd(y1, 1e-5, None, h=h1, y=y1, rstd=rstd)
    assert torch.equal(h1, x)
    v, rr, tv, tr = fwd_ref(x, None, 1e-5)
    within(y1, v, tv + rounding(dtype, v), "y of x alone")
    within(rstd, rr, tr, "rstd of x alone")
    dx, dg = full((n, C), dtype), full((C,))
    hc.hc_rms_norm_bwd(x, dy, None, rstd, dx=dx, dgamma=dg)
    rdx, rdg, tdx, tdg = bwd_ref(x, dy, None, None, rstd)
    within(dx, rdx, tdx + rounding(dtype, rdx), "dx without gamma and residual")
    within(dg, rdg, tdg, "dgamma without gamma")
    # each gradient alone, in place of each input
    hc.hc_rms_norm_bwd(h, dy, gamma, rstd, dres=dres, dx=dx, dgamma=dg)
    one = full((C,))
    hc.hc_rms_norm_bwd(h, dy, gamma, rstd, dres=dres, dgamma=one)
    assert torch.equal(one, dg)
    for k in range(3):
        p = [h.clone(), dy.clone(), dres.clone()]
        hc.hc_rms_norm_bwd(p[0], p[1], gamma, rstd, dres=p[2], dx=p[k])
        assert torch.equal(p[k], dx)
    # one element past a 16-byte boundary
    hs, ys, rs = shifted(x), shifted(x), shifted(rstd)
    hc.hc_rms_norm_fwd(shifted(x), 1e-5, shifted(gamma), res=shifted(res), h=hs, y=ys, rstd=rs, q=q1, scales=sc1)
    assert torch.equal(hs, h)
    v, _, tv, _ = fwd_ref(h, gamma, 1e-5)
    within(ys, v, tv + rounding(dtype, v), "y of shifted rows")
    q_ref, s_ref = quant_ref(h.float() * rs[:, None] * gamma)
    assert torch.equal(sc1, s_ref) and torch.equal(q1.view(torch.uint8), q_ref)
    dxs, dgs = shifted(x), shifted(gamma)
    hc.hc_rms_norm_bwd(hs, shifted(dy), shifted(gamma), rs, dres=shifted(dres), dx=dxs, dgamma=dgs)
    rdx, rdg, tdx, tdg = bwd_ref(h, dy, dres, gamma, rs)
    within(dxs, rdx, tdx + rounding(dtype, rdx), "dx of shifted rows")
    within(dgs, rdg, tdg, "dgamma of shifted rows")


@pytest.mark.parametrize("C,dtype", [(24, F), (131, F), (264, BF), (2048, BF), (8200, F), (20001, BF)])
def test_values(C, dtype):
    """Zeros give zeros; squares past the range of fp32, and eps with rows as
    small as it, keep their norm; a NaN fills its row, an infinity makes the
    rest of its row zero; none of them reaches another row."""
    x, _, _, _, gamma = inputs(5, 9, C, dtype)
    x[0] = 0
    x[1] *= 2.0 ** 100
    x[2] *= 2.0 ** 110
    x[3] *= 2.0 ** -60
    x[4] = torch.finfo(dtype).max
    x[5, C - 1], x[6, C // 2] = float("nan"), float("-inf")
    y, rstd = full((9, C), dtype), full((9,))
    q, sc = full((9, hc.HC_FP8_PITCH(C)), torch.uint8, 77).view(Q8), full(((C + 127) // 128, 9))
    for eps in (1e-5, 1e-38):
        hc.hc_rms_norm_fwd(x, eps, gamma, y=y, rstd=rstd, q=q, scales=sc)
        assert (y[0] == 0).all() and (q[0].float() == 0).all()
        keep = [1, 2, 3, 4, 7, 8]
        v, rr, tv, tr = fwd_ref(x[keep], gamma, eps)
        # the largest values' rstd is below the smallest normal number: half
        # of the smallest step besides
        least = torch.where(rr < 2.0 ** -126, 2.0 ** -150, 0.0)
        within(rstd[keep], rr, tr + least, "rstd")
        tv = tv + x[keep].to(D64).abs() * gamma.to(D64).abs() * least[:, None]
        within(y[keep], v, tv + rounding(dtype, v), "y")
        assert y[5].isnan().all()
        assert y[6, C // 2].isnan() and int(y[6].isnan().sum()) == 1 and (y[6].nan_to_num() == 0).all()
        b = (C - 1) // 128
        assert sc[b, 5].isnan() and sc[C // 256, 6].isnan()
    y.fill_(77)
    hc.hc_rms_norm_fwd(x, 0.0, gamma, y=y)
    assert y[0].isnan().all() and (y[1:5].isfinite()).all() and (y[7:].isfinite()).all()


@pytest.mark.parametrize("C,dtype", [(24, F), (24, BF), (131, F), (264, BF), (602, BF), (2048, F), (2051, BF), (8200, F),
                                     (20001, BF)])
def test_smallest_rows(C, dtype):
    """Without eps: rows whose rstd fp32 just holds are normed like any others; below
    that rstd is infinite, and no finite output pretends otherwise. Rows of the
    ordinary size beside them stay what they are."""
    x, _, _, _, gamma = inputs(C, 12, C, F)
    x[::3] *= 2.0 ** -125
    x[1::3] *= 2.0 ** -132
    x = x.to(dtype)
    y, rstd = full((12, C), dtype), full((12,))
    q, sc = full((12, hc.HC_FP8_PITCH(C)), torch.uint8, 77), full(((C + 127) // 128, 12))
    hc.hc_rms_norm_fwd(x, 0.0, gamma, y=y, rstd=rstd, q=q, scales=sc)
    v, rr, tv, tr = fwd_ref(x, gamma, 0.0)
    past = rr >= 2.0 ** 128
    assert past[1::3].all() and not past[::3].any() and not past[2::3].any()
    within(rstd[~past], rr[~past], tr[~past], "rstd")
    within(y[~past], v[~past], (tv + rounding(dtype, v))[~past], "y")
    assert (rstd[past] == float("inf")).all() and not y[past].isfinite().any()
    top = (x[~past].float() * rstd[~past, None] * gamma).abs().amax(1)
    assert torch.equal(sc[:, ~past].amax(0), top / torch.full_like(top, 448.0))


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("C", [64, 131])
def test_stored_sums(C, dtype):
    """The stored sum over all exponents: terms far apart, of opposite signs,
    halfway cases, numbers below the normal range, zeros of both signs."""
    g = gen(C)
    n = 4096
    e = torch.randint(-149, 120, (2, n, C), generator=g, device="cuda")
    e[1, ::2] = e[0, ::2] - torch.randint(0, 12, (n // 2, C), generator=g, device="cuda")
    x, res = ((1 + torch.rand(n, C, generator=g, device="cuda")).double().ldexp(k).float()
              * torch.randint(0, 2, (n, C), generator=g, device="cuda").mul(2).sub(1) for k in e)
    x, res = x.to(dtype), res.to(dtype)
    x[5], res[5] = 0.0, -0.0
    x[6], res[6] = -0.0, -0.0
    h, y = torch.empty_like(x), torch.empty_like(x)
    hc.hc_rms_norm_fwd(x, 1e-5, None, res=res, h=h, y=y)
    want = stored(x, res)
    bits = torch.int16 if dtype == BF else torch.int32
    assert torch.equal(h.view(bits), want.view(bits))


def test_differences():
    """dx (with the residual's share) and dgamma against central differences of
    the 64-bit forward, step h = 2^-12: the differences' own error is below h^2
    times the third derivative (a few hundred here) plus 2^-52 / h."""
    n, C, step = 3, 10, 2.0 ** -12
    x, res, dy, dres, gamma = inputs(11, n, C, F)
    h, y, rstd = full((n, C)), full((n, C)), full((n,))
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, res=res, h=h, y=y, rstd=rstd)
    dx, dg = full((n, C)), full((C,))
    hc.hc_rms_norm_bwd(h, dy, gamma, rstd, dres=dres, dx=dx, dgamma=dg)

    def loss(x, ga):
        s = x + res.to(D64)
        v = s / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-5) * ga
        return float((v * dy.to(D64)).sum() + (s * dres.to(D64)).sum())

    p = [x.to(D64), gamma.to(D64)]
    for k, got in ((0, dx), (1, dg)):
        flat = p[k].view(-1)
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + step
            up = loss(*p)
            flat[i] = old - step
            down = loss(*p)
            flat[i] = old
            assert abs((up - down) / (2 * step) - float(got.view(-1)[i])) <= 1e-4, (k, i)


def test_counts_out_of_range():
    x, _, _, _, gamma = inputs(3, 6, 40, F)
    y = full((6, 40))
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, y=y, count=count_of(9))
    assert hc.hc_get_device_status() == hc.HC_ERR_CAPACITY
    assert (y != 77).any(1).all()
    y.fill_(77)
    hc.hc_rms_norm_fwd(x, 1e-5, gamma, y=y, count=count_of(-1))
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX
    assert (y == 77).all()


@pytest.mark.parametrize("C,dtype", [(131, F), (2048, BF), (9000, BF)])
def test_stream_and_graph(C, dtype):
    """Another stream, and a captured step replayed on new inputs."""
    n = 300
    x, res, dy, dres, gamma = inputs(17, n, C, dtype)
    h, y, dx = (full((n, C), dtype) for _ in range(3))
    rstd, dg, cnt = full((n,)), full((C,)), count_of(n)

    def step(s=None):
        hc.hc_rms_norm_fwd(x, 1e-5, gamma, res=res, h=h, y=y, rstd=rstd, count=cnt, stream=s)
        hc.hc_rms_norm_bwd(h, dy, gamma, rstd, dres=dres, dx=dx, dgamma=dg, count=cnt, stream=s)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (h, y, dx, rstd, dg)]
    side = torch.cuda.Stream()
    for t in (h, y, dx, rstd, dg):
        t.fill_(77)
    torch.cuda.synchronize()
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((h, y, dx, rstd, dg), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for m in (n, 0, 7):
        cnt.fill_(m)
        for t in (h, y, dx, rstd, dg):
            t.fill_(77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y[:m], want[1][:m]) and torch.equal(dx[:m], want[2][:m])
        assert (y[m:] == 77).all() and (dx[m:] == 77).all()
        if m == n:
            assert torch.equal(dg, want[4])
