"""The token operators (row embedding, layer norm, 8-bit quantisation and
linear layer) through the C ABI against plain 64-bit implementations, with
their gradients against the formulas and against central differences.

Tolerances, derived from the arithmetic. u = 2^-24 is the unit roundoff of
fp32, and a sum whose additions form a tree of depth D is off by at most
D * u * (sum of magnitudes). A row's channels are summed by at most 1024
threads in a chain of at most C / 256 + 64 additions each, the tree over the
threads included: D(C) = C / 256 + 64. The channel sums over rows, and a
token's gradient, are bounded by the chain of all n additions. A bf16 result
(8 significant bits) is rounded once more, by at most 2^-8 of its value. Indices, and the 8-bit
values and scales, are exact."""
import numpy as np
import pytest

from paper_2608_09388_gb300 import hc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
BF, F = torch.bfloat16, torch.float32
D64 = torch.float64


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


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def count_of(n):
    return torch.tensor([n], dtype=torch.int32, device="cuda")


def rounding(dtype, v):
    return (2.0 ** -8 if dtype == BF else U) * v.abs()


def within(got, ref, tol, what):
    got = got.to(D64)
    assert got.shape == ref.shape, what
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst "
                           f"{float(((got - ref).abs() - tol).max()):.3e} over its bound")


def depth(C):
    return C / 256 + 64


# ------------------------------------------------------------------ layer norm
def norm_ref(x, gamma, beta, eps):
    """y, mean, rstd in 64 bits and the bound on y's error."""
    C = x.shape[1]
    x = x.to(D64)
    ga = gamma.to(D64) if gamma is not None else torch.ones(C, dtype=D64, device="cuda")
    be = beta.to(D64) if beta is not None else torch.zeros(C, dtype=D64, device="cuda")
    mean = x.mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    xh = (x - mean) * rstd
    y = xh * ga + be
    D = depth(C)
    dm = (D + 2) * U * x.abs().mean(1, keepdim=True)          # the mean's error
    rel = ((D + 6) * U * var + dm ** 2) * rstd ** 2 / 2 + 4 * U  # rstd's relative error
    tol = ga.abs() * (rstd * (dm + 2 * U * (x.abs() + mean.abs())) + xh.abs() * (rel + 4 * U)) \
        + 4 * U * (y.abs() + be.abs())
    return y, mean[:, 0], rstd[:, 0], tol, dm[:, 0], (rel * rstd)[:, 0]


def norm_grad_ref(x, dy, gamma, mean, rstd):
    """dx, dgamma, dbeta in 64 bits from the fp32 mean and rstd, and their bounds."""
    n, C = x.shape
    x, dy, m, r = x.to(D64), dy.to(D64), mean.to(D64)[:, None], rstd.to(D64)[:, None]
    ga = gamma.to(D64) if gamma is not None else torch.ones(C, dtype=D64, device="cuda")
    xh, g = (x - m) * r, dy * ga
    c1, c2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = r * (g - c1 - xh * c2)
    D = depth(C) + 8
    tdx = r.abs() * (4 * U * g.abs() + D * U * g.abs().mean(1, keepdim=True)
                     + D * U * xh.abs() * (g * xh).abs().mean(1, keepdim=True)
                     + 8 * U * (c1.abs() + (xh * c2).abs()))
    return (dx, (dy * xh).sum(0), dy.sum(0), tdx, (n + 8) * U * (dy * xh).abs().sum(0),
            (n + 8) * U * dy.abs().sum(0))


def norm_inputs(seed, cap, C, dtype, level=0.5):
    g = gen(seed)
    x = (randn(g, cap, C) * (0.5 + torch.rand(cap, 1, generator=g, device="cuda"))
         + level * randn(g, cap, 1)).to(dtype)
    return x, randn(g, cap, C, dtype=dtype), 1 + 0.2 * randn(g, C), 0.1 * randn(g, C)


# widths around every change of the kernels' layout: single channels, a vector,
# a warp, several rows per warp or per block, odd and large rows
WIDTHS = (1, 2, 7, 8, 24, 64, 72, 129, 131, 256, 264, 500, 512, 1000, 1023, 1024, 1032, 2048,
          2056, 2051, 4096, 4104, 8192, 8200, 16384, 16392, 20001)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("C", WIDTHS)
def test_layer_norm(C, dtype):
    n, cap = (203, 211) if C <= 4104 else (19, 23)
    x, dy, gamma, beta = norm_inputs(C, cap, C, dtype)
    y = torch.full((cap, C), 77.0, dtype=dtype, device="cuda")
    mean, rstd = (torch.full((cap,), 77.0, device="cuda") for _ in range(2))
    hc.hc_layer_norm_fwd(x, 1e-5, gamma, beta, y, mean=mean, rstd=rstd, count=count_of(n))
    ry, rm, rr, tol, tm, tr = norm_ref(x[:n], gamma, beta, 1e-5)
    within(y[:n], ry, tol + rounding(dtype, ry), "y")
    within(mean[:n], rm, tm + U * rm.abs(), "mean")
    within(rstd[:n], rr, tr, "rstd")
    assert (y[n:] == 77).all() and (mean[n:] == 77).all() and (rstd[n:] == 77).all()
    dx = torch.full((cap, C), 77.0, dtype=dtype, device="cuda")
    dg, db = (torch.full((C,), 77.0, device="cuda") for _ in range(2))
    hc.hc_layer_norm_bwd(x, dy, gamma, mean, rstd, dx=dx, dgamma=dg, dbeta=db, count=count_of(n))
    rdx, rdg, rdb, tdx, tdg, tdb = norm_grad_ref(x[:n], dy[:n], gamma, mean[:n], rstd[:n])
    within(dx[:n], rdx, tdx + rounding(dtype, rdx), "dx")
    within(dg, rdg, tdg, "dgamma")
    within(db, rdb, tdb, "dbeta")
    assert (dx[n:] == 77).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("C", [65, 127, 129, 255, 301, 511, 513, 1025, 2047, 2051, 4095, 4099, 8191])
def test_layer_norm_odd_widths(C, dtype):
    """Rows without 16-byte loads at the widths where their layout changes."""
    test_layer_norm(C, dtype)


@pytest.mark.parametrize("n", [0, 1, 2, 3, 127, 128, 129, 5000])
@pytest.mark.parametrize("C,dtype", [(64, BF), (131, F), (1024, BF), (4096, F)])
def test_layer_norm_rows(n, C, dtype):
    cap = n + 3
    x, dy, gamma, beta = norm_inputs(n + C, cap, C, dtype)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(cap, device="cuda"), torch.empty(cap, device="cuda")
    dg, db = (torch.full((C,), 77.0, device="cuda") for _ in range(2))
    hc.hc_layer_norm_fwd(x, 1e-5, gamma, beta, y, mean=mean, rstd=rstd, count=count_of(n))
    hc.hc_layer_norm_bwd(x, dy, gamma, mean, rstd, dx=dx, dgamma=dg, dbeta=db, count=count_of(n))
    if n == 0:
        assert (dg == 0).all() and (db == 0).all()
        return
    ry, _, _, tol, _, _ = norm_ref(x[:n], gamma, beta, 1e-5)
    within(y[:n], ry, tol + rounding(dtype, ry), "y")
    rdx, rdg, rdb, tdx, tdg, tdb = norm_grad_ref(x[:n], dy[:n], gamma, mean[:n], rstd[:n])
    within(dx[:n], rdx, tdx + rounding(dtype, rdx), "dx")
    within(dg, rdg, tdg, "dgamma")
    within(db, rdb, tdb, "dbeta")


@pytest.mark.parametrize("C,dtype", [(64, BF), (264, F), (1000, BF), (2048, BF), (20001, F)])
def test_layer_norm_forms(C, dtype):
    """All rows without a count, no affine, no saved statistics, each gradient
    alone, in place, and rows that are not 16-byte aligned: the same bits."""
    n = 37
    x, dy, gamma, beta = norm_inputs(C + 1, n, C, dtype)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    hc.hc_layer_norm_fwd(x, 1e-5, gamma, beta, y, mean=mean, rstd=rstd)
    x2 = x.clone()
    hc.hc_layer_norm_fwd(x2, 1e-5, gamma, beta, x2)
    assert torch.equal(x2, y)
    ry, _, _, tol, _, _ = norm_ref(x, None, None, 1e-5)
    y0 = torch.empty_like(x)
    hc.hc_layer_norm_fwd(x, 1e-5, None, None, y0)
    within(y0, ry, tol + rounding(dtype, ry), "y without affine")
    dx, dg, db = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    hc.hc_layer_norm_bwd(x, dy, gamma, mean, rstd, dx=dx, dgamma=dg, dbeta=db)
    one = {k: torch.empty_like(v) for k, v in (("dx", dx), ("dgamma", dg), ("dbeta", db))}
    for k, v in one.items():
        hc.hc_layer_norm_bwd(x, dy, gamma, mean, rstd, **{k: v})
    assert torch.equal(one["dx"], dx) and torch.equal(one["dgamma"], dg)
    assert torch.equal(one["dbeta"], db)
    for which in ("x", "dy"):
        xi, dyi = x.clone(), dy.clone()
        hc.hc_layer_norm_bwd(xi, dyi, gamma, mean, rstd, dx=xi if which == "x" else dyi)
        assert torch.equal(xi if which == "x" else dyi, dx)
    rdx, rdg, rdb, tdx, tdg, tdb = norm_grad_ref(x, dy, None, mean, rstd)
    hc.hc_layer_norm_bwd(x, dy, None, mean, rstd, dx=dx, dgamma=dg, dbeta=db)
    within(dx, rdx, tdx + rounding(dtype, rdx), "dx without gamma")
    # one element past a 16-byte boundary
    def shifted(t):
        s = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape)
        return s.copy_(t)
    ys = shifted(y)
    hc.hc_layer_norm_fwd(shifted(x), 1e-5, shifted(gamma), shifted(beta), ys)
    ry, _, _, tol, _, _ = norm_ref(x, gamma, beta, 1e-5)
    within(ys, ry, tol + rounding(dtype, ry), "y of shifted rows")
    dxs, dgs, dbs = shifted(x), shifted(gamma), shifted(beta)
    hc.hc_layer_norm_bwd(shifted(x), shifted(dy), shifted(gamma), shifted(mean), shifted(rstd),
                         dx=dxs, dgamma=dgs, dbeta=dbs)
    rdx, rdg, rdb, tdx, tdg, tdb = norm_grad_ref(x, dy, gamma, mean, rstd)
    within(dxs, rdx, tdx + rounding(dtype, rdx), "dx of shifted rows")
    within(dgs, rdg, tdg, "dgamma of shifted rows")
    within(dbs, rdb, tdb, "dbeta of shifted rows")


def test_layer_norm_values():
    """Constant rows give beta; a NaN or an infinity stays in its row; a level
    far above the spread does not cost the spread."""
    for C, dtype in ((264, F), (131, F), (2048, BF)):
        x, _, gamma, beta = norm_inputs(5, 6, C, dtype)
        x[0] = 3.0
        x[1, 5], x[2, C - 1] = float("nan"), float("inf")
        x[3] = (1000 + 4 * randn(gen(9), C)).to(dtype)
        y = torch.empty_like(x)
        hc.hc_layer_norm_fwd(x, 1e-5, gamma, beta, y)
        assert torch.equal(y[0], beta.to(dtype))
        assert y[1].isnan().all() and y[2].isnan().all()
        ry, _, _, tol, _, _ = norm_ref(x[3:], gamma, beta, 1e-5)
        within(y[3:], ry, tol + rounding(dtype, ry), "y")


def test_layer_norm_differences():
    """dx, dgamma and dbeta against central differences of the 64-bit forward,
    step h = 2^-12: the differences' own error is below h^2 times the third
    derivative (a few hundred here) plus 2^-52 / h."""
    n, C, h = 3, 10, 2.0 ** -12
    x, dy, gamma, beta = norm_inputs(11, n, C, F)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    hc.hc_layer_norm_fwd(x, 1e-5, gamma, beta, y, mean=mean, rstd=rstd)
    dx, dg, db = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    hc.hc_layer_norm_bwd(x, dy, gamma, mean, rstd, dx=dx, dgamma=dg, dbeta=db)

    def loss(x, ga, be):
        m = x.mean(1, keepdim=True)
        v = ((x - m) ** 2).mean(1, keepdim=True)
        return float((((x - m) / torch.sqrt(v + 1e-5) * ga + be) * dy.to(D64)).sum())

    p = [x.to(D64), gamma.to(D64), beta.to(D64)]
    for k, got in ((0, dx), (1, dg), (2, db)):
        flat = p[k].view(-1)
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + h
            up = loss(*p)
            flat[i] = old - h
            down = loss(*p)
            flat[i] = old
            assert abs((up - down) / (2 * h) - float(got.view(-1)[i])) <= 1e-4, (k, i)


# ------------------------------------------------------------------ embedding
def ids_of(g, cap, V, kind):
    if kind == "one":  # every token the same
        ids = torch.full((cap,), V // 2)
    elif kind == "zipf":
        ids = (torch.exp(torch.rand(cap, generator=g, device="cuda") * np.log(V + 1)) - 1).long() \
            .clamp_(0, V - 1).cpu()
    elif kind == "pad":
        ids = torch.full((cap,), -1)
    else:
        ids = torch.randint(0, V, (cap,), generator=g, device="cuda").cpu()
    ids = ids.int()
    if kind == "uniform":
        ids[::7] = -1
    return ids


def sort_ref(ids, n, V):
    a = ids[:n].cpu().numpy().astype(np.int64)
    key = np.full(ids.shape[0], V, np.int64)
    key[:n] = np.where((a >= 0) & (a < V), a, V)
    order = np.argsort(key, kind="stable")
    return np.searchsorted(key[order], np.arange(V + 1)), order


def embed_all(table, ids, scale, dy, cap, n=None):
    V, C = table.shape
    cnt = None if n is None else count_of(n)
    y = torch.full((cap, C), 77.0, dtype=table.dtype, device="cuda")
    row_ptr = torch.full((V + 1,), 77, dtype=torch.int32, device="cuda")
    order = torch.full((cap,), 77, dtype=torch.int32, device="cuda")
    dt = torch.full((V, C), 77.0, device="cuda")
    hc.hc_embedding_fwd(table, ids, scale, y, count=cnt)
    hc.hc_embedding_sort(ids, V, row_ptr, order, count=cnt)
    hc.hc_embedding_bwd(dy, row_ptr, order, scale, dt)
    return y, row_ptr, order, dt


def check_embed(table, ids, scale, dy, cap, n, out):
    V, C = table.shape
    y, row_ptr, order, dt = out
    i = ids[:n].long()
    ok = ((i >= 0) & (i < V))[:, None]
    want = torch.where(ok, table[i.clamp(0, V - 1)].float() * scale, 0.0).to(table.dtype)
    assert torch.equal(y[:n], want)
    assert (y[n:] == 77).all()
    rp, od = sort_ref(ids, n, V)
    assert np.array_equal(row_ptr.cpu().numpy(), rp)
    assert np.array_equal(order.cpu().numpy(), od)
    d = torch.where(ok, dy[:n].to(D64), 0.0)
    at = i.clamp(0, V - 1)
    ref = torch.zeros(V, C, dtype=D64, device="cuda").index_add_(0, at, d) * scale
    mag = torch.zeros(V, C, dtype=D64, device="cuda").index_add_(0, at, d.abs()) * abs(scale)
    deg = torch.bincount(at[ok[:, 0]], minlength=V).to(D64)[:, None]
    within(dt, ref, (deg + 2) * U * mag, "dtable")


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,slack,V,C,kind", [
    (0, 5, 10, 16, "uniform"), (1, 0, 1, 1, "uniform"), (1, 4, 40000, 64, "zipf"),
    (5, 0, 3, 7, "uniform"), (33, 0, 2048, 8, "zipf"), (31, 3, 2047, 9, "zipf"),
    (64, 0, 64, 131, "one"), (65, 1, 5, 24, "pad"), (700, 77, 655, 45, "uniform"),
    (2048, 0, 2049, 128, "zipf"), (2049, 900, 10475, 128, "zipf"), (4097, 0, 17, 264, "uniform"),
    (5000, 0, 9, 1000, "one"), (20000, 1, 131072, 40, "zipf"), (9000, 0, 300, 2056, "zipf"),
    (150001, 0, 30, 8, "zipf"), (70000, 70000, 4200000, 2, "zipf"), (30, 0, 7, 5000, "uniform")])
def test_embedding(n, slack, V, C, kind, dtype):
    g = gen(n + V)
    cap = n + slack
    ids = ids_of(g, cap, V, kind).cuda()
    table, dy = randn(g, V, C, dtype=dtype), randn(g, cap, C, dtype=dtype)
    out = embed_all(table, ids, 1.7, dy, cap, n)
    check_embed(table, ids, 1.7, dy, cap, n, out)


@pytest.mark.parametrize("cap", [1023, 1024, 1025, 2047, 2048, 2049, 32768, 32769, 65536, 65537,
                                 131073])
def test_embedding_sort_sizes(cap):
    """The sort at the sizes where its tiles change, all rows used and fewer."""
    for n in (cap, cap // 2 + 1):
        for V, kind in ((3, "uniform"), (10475, "zipf")):
            ids = ids_of(gen(cap + V), cap, V, kind).cuda()
            row_ptr = torch.full((V + 1,), 77, dtype=torch.int32, device="cuda")
            order = torch.full((cap,), 77, dtype=torch.int32, device="cuda")
            hc.hc_embedding_sort(ids, V, row_ptr, order, count=count_of(n))
            rp, od = sort_ref(ids, n, V)
            assert np.array_equal(row_ptr.cpu().numpy(), rp)
            assert np.array_equal(order.cpu().numpy(), od)


@pytest.mark.parametrize("n,V,C,dtype", [
    (9000, 500, 45, BF), (20000, 40, 520, F), (20000, 60000, 40, BF), (30000, 50000, 136, F),
    (15000, 200000, 13, BF), (15000, 200000, 24, F), (3000, 40000, 520, BF)])
def test_embedding_frequent_rows_side_by_side(n, V, C, dtype):
    """Low ids far more frequent than the others: most tokens belong to rows
    that are cut into pieces, several of them next to each other."""
    g = gen(n + V)
    ids = (torch.rand(n, generator=g, device="cuda").pow(4) * V).int().clamp_(0, V - 1)
    table, dy = randn(g, V, C, dtype=dtype), randn(g, n, C, dtype=dtype)
    out = embed_all(table, ids, 0.3, dy, n)
    check_embed(table, ids, 0.3, dy, n, n, out)
    assert all(torch.equal(a, b) for a, b in zip(out, embed_all(table, ids, 0.3, dy, n)))


def test_embedding_column_of_coordinates():
    """The vertex column of a coordinate list as ids, as a strided view."""
    g = gen(3)
    V, C, cap, n = 655, 64, 3000, 2711
    coords = torch.randint(0, V, (cap, 2), generator=g, device="cuda", dtype=torch.int32)
    table, dy = randn(g, V, C), randn(g, cap, C)
    out = embed_all(table, coords[:, 1], 0.5, dy, cap, n)
    check_embed(table, coords[:, 1].contiguous(), 0.5, dy, cap, n, out)


def test_embedding_forms():
    """All rows without a count; rows that are not 16-byte aligned; one sort
    for two tables; the same bits from run to run."""
    g = gen(4)
    V, cap = 500, 3001
    ids = ids_of(g, cap, V, "zipf").cuda()
    for C, dtype in ((64, BF), (132, F)):
        table, dy = randn(g, V, C, dtype=dtype), randn(g, cap, C, dtype=dtype)
        out = embed_all(table, ids, 3.0, dy, cap)
        check_embed(table, ids, 3.0, dy, cap, cap, out)
        again = embed_all(table, ids, 3.0, dy, cap)
        assert all(torch.equal(a, b) for a, b in zip(out, again))
        tb = torch.empty(V * C + 1, dtype=dtype, device="cuda")[1:].view(V, C).copy_(table)
        db = torch.empty(cap * C + 1, dtype=dtype, device="cuda")[1:].view(cap, C).copy_(dy)
        check_embed(tb, ids, 3.0, db, cap, cap, embed_all(tb, ids, 3.0, db, cap))


def test_embedding_bad_ids_reported():
    g = gen(5)
    V, C, cap = 20, 16, 50
    ids = torch.randint(0, V, (cap,), generator=g, device="cuda", dtype=torch.int32)
    ids[7], ids[9], ids[11] = V, -2, 2 ** 31 - 1
    table, dy = randn(g, V, C), randn(g, cap, C)
    y = torch.empty(cap, C, device="cuda")
    hc.hc_embedding_fwd(table, ids, 1.0, y)
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX
    assert (y[[7, 9, 11]] == 0).all()
    row_ptr = torch.empty(V + 1, dtype=torch.int32, device="cuda")
    order = torch.empty(cap, dtype=torch.int32, device="cuda")
    hc.hc_embedding_sort(ids, V, row_ptr, order)
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX
    rp, od = sort_ref(ids, cap, V)
    assert np.array_equal(row_ptr.cpu().numpy(), rp) and np.array_equal(order.cpu().numpy(), od)


def test_embedding_bwd_bad_tables_reported():
    """row_ptr and order that hc_embedding_sort did not write: what is out of
    range is reported and skipped, the other rows are right."""
    g = gen(6)
    V, C, cap = 6, 40, 300
    ids = (torch.arange(cap, device="cuda") % V).int()
    dy = randn(g, cap, C)
    _, row_ptr, order, good = embed_all(randn(g, V, C), ids, 1.0, dy, cap)
    dt = torch.empty(V, C, device="cuda")
    bad = row_ptr.clone()
    bad[3] = cap + 5  # rows 2 and 3
    hc.hc_embedding_bwd(dy, bad, order, 1.0, dt)
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX
    assert torch.equal(dt[[0, 1, 4, 5]], good[[0, 1, 4, 5]]) and (dt[2:4] == 0).all()
    bad = order.clone()
    bad[int(row_ptr[1])], bad[int(row_ptr[2])] = -1, cap
    hc.hc_embedding_bwd(dy, row_ptr, bad, 1.0, dt)
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX
    assert torch.equal(dt[[0, 3, 4, 5]], good[[0, 3, 4, 5]])


def test_embedding_differences():
    """The gradient is that of a linear map: <dy, fwd(E)> = <dtable, E> for
    every unit table E, evaluated in 64 bits."""
    g = gen(7)
    V, C, cap = 4, 3, 9
    ids = torch.tensor([0, 2, 2, -1, 1, 2, 0, 1, 2], dtype=torch.int32, device="cuda")
    dy = randn(g, cap, C)
    _, _, _, dt = embed_all(torch.zeros(V, C, device="cuda"), ids, 2.0, dy, cap)
    for v in range(V):
        for c in range(C):
            E = torch.zeros(V, C, device="cuda")
            E[v, c] = 1.0
            y = torch.empty(cap, C, device="cuda")
            hc.hc_embedding_fwd(E, ids, 2.0, y)
            want = (y.to(D64) * dy.to(D64)).sum()
            mag = (y.to(D64) * dy.to(D64)).abs().sum()
            assert abs(float(dt[v, c]) - float(want)) <= 12 * U * float(mag)


# ------------------------------------------------------------------ 8 bits
def q_ref(x):
    """e4m3 bytes, scales and their values by the definition (fp32 quotients)."""
    x = x.float().cpu()
    n, K = x.shape
    nb, P = (K + 127) // 128, hc.HC_FP8_PITCH(K)
    b = torch.nn.functional.pad(x, (0, nb * 128 - K)).view(n, nb, 128)
    top = torch.from_numpy(np.max(np.abs(b.numpy()), axis=2))
    s = torch.from_numpy(np.maximum(top.numpy() / np.float32(448), np.float32(2.0 ** -126)))
    v = torch.from_numpy(b.numpy() / s.numpy()[:, :, None])
    q = v.to(torch.float8_e4m3fn).view(torch.uint8).view(n, nb * 128)[:, :P]
    return q.contiguous(), s.t().contiguous()


def value(q, s, K):
    """[n, K] fp64 values of e4m3 bytes with scales [blocks, n]."""
    v = q.view(torch.float8_e4m3fn).to(D64)[:, :K]
    return v * s.to(D64).t().repeat_interleave(128, 1)[:, :K]


def quantise(x, count=None, cap=None):
    cap, K = x.shape
    q = torch.full((cap, hc.HC_FP8_PITCH(K)), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full(((K + 127) // 128, cap), 77.0, device="cuda")
    hc.hc_quantize_fp8_rows(x, q, s, count=count)
    return q, s


def quantise_weight(W):
    K, N = W.shape
    q = torch.full((N, hc.HC_FP8_PITCH(K)), 0x55, dtype=torch.uint8, device="cuda")
    s = torch.full(((N + 127) // 128, (K + 127) // 128), 77.0, device="cuda")
    hc.hc_quantize_fp8_weight(W, q, s)
    return q, s


def test_embedding_bwd_end_behind_entries():
    """A row_ptr that decreases, a row's end far behind the entries in use: it
    is reported, the chunks' sums stay within their buffer, and the next call
    is right."""
    g = gen(7)
    V, C, cap = 2, 64, 200000
    dy = randn(g, cap, C)
    ids = torch.zeros(cap, dtype=torch.int32, device="cuda")
    _, row_ptr, order, good = embed_all(randn(g, V, C), ids, 1.0, dy, cap)
    bad = torch.tensor([0, cap, 64], dtype=torch.int32, device="cuda")
    dt = torch.empty(V, C, device="cuda")
    hc.hc_embedding_bwd(dy, bad, order, 1.0, dt)
    assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX
    assert (dt[1] == 0).all()
    hc.hc_embedding_bwd(dy, row_ptr, order, 1.0, dt)
    assert torch.equal(dt, good) and hc.hc_get_device_status() == hc.HC_OK


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n,slack,K", [(0, 3, 40), (1, 0, 1), (1, 0, 8192), (7, 2, 15), (33, 7, 16),
                                       (64, 0, 127), (65, 1, 128), (100, 0, 129), (31, 0, 1000),
                                       (513, 5, 264), (40, 0, 2001), (3000, 0, 136)])
def test_quantize_rows(n, slack, K, dtype):
    x = (randn(gen(n + K), n + slack, K) * torch.exp(2 * randn(gen(K), n + slack, 1))).to(dtype)
    q, s = quantise(x, count_of(n))
    rq, rs = q_ref(x[:n])
    assert torch.equal(s[:, :n].cpu(), rs)
    assert torch.equal(q[:n].cpu(), rq)
    assert (q[n:] == 0x55).all() and (s[:, n:] == 77).all()
    xs = torch.empty(x.numel() + 1, dtype=dtype, device="cuda")[1:].view(x.shape).copy_(x)
    q2, s2 = quantise(xs, count_of(n))
    assert torch.equal(q2, q) and torch.equal(s2, s)


def test_quantize_special_values():
    x = torch.zeros(7, 300, device="cuda")
    x[1, 3], x[1, 200] = 1e-44, -2e-40                # below the smallest scale
    x[2, 5] = 3.4e38                                  # the largest magnitudes
    x[3, 7], x[4, 140], x[5, 299] = float("nan"), float("inf"), float("-inf")
    x[3:6] += 1.0
    x[6] = torch.linspace(-448, 448, 300)
    q, s = quantise(x)
    rq, rs = q_ref(x[[0, 1, 2, 6]])
    assert torch.equal(s[:, [0, 1, 2, 6]].cpu(), rs) and torch.equal(q[[0, 1, 2, 6]].cpu(), rq)
    assert s[0, 3].isnan() and s[1, 4].isinf() and s[2, 5].isinf()
    w, ws = quantise_weight(0.1 * randn(gen(1), 300, 70))
    y = torch.empty(7, 70, device="cuda")
    hc.hc_fp8_linear_fwd(q, s, w, ws, None, hc.HC_ACT_NONE, y)
    assert y[3:6].isnan().all() and y[[0, 1, 2, 6]].isfinite().all() and (y[0] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("K,N", [(1, 1), (16, 5), (127, 128), (130, 129), (300, 64), (1152, 260)])
def test_quantize_weight(K, N, dtype):
    W = randn(gen(K + N), K, N, dtype=dtype)
    q, s = quantise_weight(W)
    w = torch.nn.functional.pad(W.float().t(), (0, -K % 128, 0, -N % 128)).cpu().numpy()
    b = w.reshape(w.shape[0] // 128, 128, w.shape[1] // 128, 128)
    rs = np.maximum(np.abs(b).max((1, 3)) / np.float32(448), np.float32(2.0 ** -126))
    v = torch.from_numpy((b / rs[:, None, :, None]).reshape(w.shape)[:N, :hc.HC_FP8_PITCH(K)])
    assert np.array_equal(s.cpu().numpy(), rs)
    assert torch.equal(q.cpu(), v.to(torch.float8_e4m3fn).view(torch.uint8))


def linear_ref(q, s, w, ws, K, bias, act):
    """The layer in 64 bits and the bound on its fp32 sums: 128 products of a
    block and up to K / 128 scaled block sums, each addition off by at most
    2 u (the tensor cores may cut instead of round), the products of the
    scales, and the fast exponential's few 1e-7."""
    N = w.shape[0]
    x = value(q, s, K)
    wv = w.view(torch.float8_e4m3fn).to(D64)[:, :K]
    wv = wv * ws.to(D64).repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    z = x @ wv.t()
    mag = x.abs() @ wv.abs().t()
    if bias is not None:
        z, mag = z + bias.to(D64), mag + bias.to(D64).abs()
    tol = (2 * 128 + 2 * (K // 128 + 1) + 8) * U * mag
    if act == hc.HC_ACT_ELU:
        return torch.where(z > 0, z, torch.expm1(z.clamp_max(0))), tol + 1e-6
    return (z.clamp_min(0) if act == hc.HC_ACT_RELU else z), tol


@pytest.mark.parametrize("out", [BF, F])
@pytest.mark.parametrize("n,slack,K,N,act", [
    (0, 4, 64, 64, 0), (1, 0, 1, 1, 0), (1, 0, 16, 8, 1), (1, 0, 4096, 1000, 0), (2, 5, 128, 128, 2),
    (3, 0, 129, 127, 0), (7, 1, 1000, 136, 1), (8, 0, 8192, 264, 0), (9, 0, 640, 2000, 0),
    (16, 0, 2048, 4096, 0), (17, 3, 250, 129, 2), (33, 0, 2000, 1001, 0), (64, 0, 512, 640, 1),
    (65, 0, 512, 513, 0), (100, 28, 384, 257, 0), (127, 0, 144, 42, 1), (128, 0, 128, 128, 0),
    (129, 0, 256, 256, 0), (255, 2, 1152, 130, 2), (500, 0, 96, 64, 0), (1000, 24, 1152, 128, 1),
    (2050, 0, 272, 640, 0), (4000, 0, 131, 33, 0), (300, 0, 4096, 16, 0), (20000, 3, 64, 24, 0)])
def test_fp8_linear(n, slack, K, N, act, out):
    g = gen(n + K + N)
    cap = n + slack
    x = randn(g, cap, K) * torch.exp(randn(g, cap, 1))
    q, s = quantise(x)
    w, ws = quantise_weight(randn(g, K, N) * torch.exp(randn(g, 1, N)))
    bias = randn(g, N) if (n + N) % 2 else None
    y = torch.full((cap, N), 77.0, dtype=out, device="cuda")
    hc.hc_fp8_linear_fwd(q, s, w, ws, bias, act, y, count=count_of(n))
    ref, tol = linear_ref(q[:n], s[:, :n], w, ws, K, bias, act)
    within(y[:n], ref, tol + rounding(out, ref), "y")
    assert (y[n:] == 77).all()


@pytest.mark.parametrize("n,slack,K,N,act,out", [
    (2400, 30, 392, 2000, 1, BF), (4700, 0, 136, 1001, 2, F), (4700, 150, 520, 2050, 0, BF),
    (9000, 0, 260, 3000, 0, F), (128, 0, 1024, 2048, 0, BF), (90, 3, 4096, 1030, 1, F)])
def test_fp8_linear_tiles(n, slack, K, N, act, out):
    """Tiles of 256 output channels, one and several a block, with whole and
    ragged ends; tiles split over clusters of four and eight."""
    test_fp8_linear(n, slack, K, N, act, out)


def test_fp8_linear_forms():
    """Rows past N' may hold anything, NaN included; no count; an output that
    is not 16-byte aligned; the same bits from run to run."""
    g = gen(8)
    for cap, n, K, N in ((300, 150, 256, 200), (40, 3, 1024, 512), (12, 12, 320, 96)):
        q, s = quantise(randn(g, cap, K))
        w, ws = quantise_weight(randn(g, K, N))
        bias = randn(g, N)
        y = torch.empty(cap, N, dtype=BF, device="cuda")
        hc.hc_fp8_linear_fwd(q, s, w, ws, bias, hc.HC_ACT_NONE, y)
        again = torch.empty_like(y)
        hc.hc_fp8_linear_fwd(q, s, w, ws, bias, hc.HC_ACT_NONE, again)
        assert torch.equal(y, again)
        ref, tol = linear_ref(q, s, w, ws, K, bias, 0)
        within(y, ref, tol + rounding(BF, ref), "y")
        for out in (BF, F):
            odd = torch.empty(cap * N + 1, dtype=out, device="cuda")[1:].view(cap, N)
            hc.hc_fp8_linear_fwd(q, s, w, ws, bias, hc.HC_ACT_NONE, odd)
            within(odd, ref, tol + rounding(out, ref), "y unaligned")
        q[n:], s[:, n:] = 0x7F, float("nan")  # e4m3 NaN
        part = torch.full_like(y, 77.0)
        hc.hc_fp8_linear_fwd(q, s, w, ws, bias, hc.HC_ACT_NONE, part, count=count_of(n))
        within(part[:n], ref[:n], tol[:n] + rounding(BF, ref[:n]), "y of the rows in use")
        assert (part[n:] == 77).all()


def test_fp8_linear_input_gradient():
    """The input gradient is the same product with the transposed weight: the
    8-bit values and scales of W^T are W's, transposed."""
    g = gen(10)
    K, N, n = 256, 384, 70
    W = randn(g, K, N)
    w, ws = quantise_weight(W)
    wt, wts = quantise_weight(W.t().contiguous())
    assert torch.equal(wt, w.t().contiguous()) and torch.equal(wts, ws.t().contiguous())
    dy = randn(g, n, N)
    q, s = quantise(dy)
    dx = torch.empty(n, K, device="cuda")
    hc.hc_fp8_linear_fwd(q, s, wt, wts, None, hc.HC_ACT_NONE, dx)
    ref, tol = linear_ref(q, s, wt, wts, N, None, 0)
    within(dx, ref, tol + rounding(F, ref), "dx")


# ------------------------------------------------------------------ all of them
def test_counts_outside_the_capacity_reported():
    g = gen(12)
    cap, C, V = 12, 32, 9
    x, y = randn(g, cap, C), torch.full((cap, C), 77.0, device="cuda")
    ids = torch.randint(0, V, (cap,), generator=g, device="cuda", dtype=torch.int32)
    table = randn(g, V, C)
    mean, rstd = torch.zeros(cap, device="cuda"), torch.ones(cap, device="cuda")
    row_ptr = torch.empty(V + 1, dtype=torch.int32, device="cuda")
    order = torch.empty(cap, dtype=torch.int32, device="cuda")
    w, ws = quantise_weight(randn(g, C, 24))
    q, s = quantise(x)
    yl = torch.full((cap, 24), 77.0, device="cuda")
    calls = [
        lambda c: hc.hc_layer_norm_fwd(x, 1e-5, None, None, y, count=c),
        lambda c: hc.hc_layer_norm_bwd(x, x, None, mean, rstd, dx=y, count=c),
        lambda c: hc.hc_embedding_fwd(table, ids, 1.0, y, count=c),
        lambda c: hc.hc_embedding_sort(ids, V, row_ptr, order, count=c),
        lambda c: hc.hc_quantize_fp8_rows(x, q, s, count=c),
        lambda c: hc.hc_fp8_linear_fwd(q, s, w, ws, None, 0, yl, count=c)]
    for k, call in enumerate(calls):
        call(count_of(cap + 1))
        assert hc.hc_get_device_status() == hc.HC_ERR_CAPACITY, k
        y.fill_(77.0)
        yl.fill_(77.0)
        call(count_of(-1))
        assert hc.hc_get_device_status() == hc.HC_ERR_INVALID_INDEX, k
        assert (y == 77).all() and (yl == 77).all(), k


def test_other_stream_and_graph():
    """On a stream of their own, and replayed from a CUDA graph with new
    inputs in the same buffers: the results of plain calls."""
    g = gen(13)
    cap, C, V, N = 500, 256, 60, 320
    table = randn(g, V, C)
    gamma, beta = 1 + 0.1 * randn(g, C), 0.1 * randn(g, C)
    w, ws = quantise_weight(randn(g, C, N))
    dyl = randn(g, cap, C)

    def buffers():
        e = dict(device="cuda")
        return dict(x=torch.empty(cap, C, **e), y=torch.empty(cap, C, **e), m=torch.empty(cap, **e),
                    r=torch.empty(cap, **e), q=torch.empty(cap, C, dtype=torch.uint8, **e),
                    s=torch.empty(C // 128, cap, **e), o=torch.empty(cap, N, **e),
                    rp=torch.empty(V + 1, dtype=torch.int32, **e),
                    od=torch.empty(cap, dtype=torch.int32, **e), dx=torch.empty(cap, C, **e),
                    dg=torch.empty(C, **e), db=torch.empty(C, **e), dt=torch.empty(V, C, **e))

    def chain(b, ids, cnt, stream=None):
        hc.hc_embedding_fwd(table, ids, 2.0, b["x"], count=cnt, stream=stream)
        hc.hc_layer_norm_fwd(b["x"], 1e-5, gamma, beta, b["y"], mean=b["m"], rstd=b["r"], count=cnt,
                             stream=stream)
        hc.hc_quantize_fp8_rows(b["y"], b["q"], b["s"], count=cnt, stream=stream)
        hc.hc_fp8_linear_fwd(b["q"], b["s"], w, ws, None, hc.HC_ACT_ELU, b["o"], count=cnt,
                             stream=stream)
        hc.hc_layer_norm_bwd(b["x"], dyl, gamma, b["m"], b["r"], dx=b["dx"], dgamma=b["dg"],
                             dbeta=b["db"], count=cnt, stream=stream)
        hc.hc_embedding_sort(ids, V, b["rp"], b["od"], count=cnt, stream=stream)
        hc.hc_embedding_bwd(b["dx"], b["rp"], b["od"], 2.0, b["dt"], stream=stream)

    ids = torch.randint(0, V, (cap,), generator=g, device="cuda", dtype=torch.int32)
    cnt = count_of(477)
    want, other, replay = buffers(), buffers(), buffers()
    for b in (want, other, replay):
        for t in b.values():
            t.zero_()
    chain(want, ids, cnt)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    chain(other, ids, cnt, stream=side)
    side.synchronize()
    assert all(torch.equal(want[k], other[k]) for k in want)
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            chain(replay, ids, cnt)
    for n in (477, 3, 0, 500):
        ids.copy_(torch.randint(0, V, (cap,), generator=g, device="cuda", dtype=torch.int32))
        cnt.fill_(n)
        for b in (want, replay):
            for t in b.values():
                t.zero_()
        torch.cuda.synchronize()
        chain(want, ids, cnt)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[k], replay[k]) for k in want), n


def test_offsets_past_32_bits():
    """Matrices of more than 2^31 elements: the last rows, against the same
    rows alone."""
    g = gen(14)
    C = 40960
    cap = 2 ** 31 // C + 9
    x = torch.empty(cap, C, dtype=BF, device="cuda")
    x[-9:] = randn(g, 9, C, dtype=BF)
    x[:-9] = 1.0
    tail = x[-9:].clone()
    gamma, beta = randn(g, C), randn(g, C)
    y, m, r = torch.empty_like(x), torch.empty(cap, device="cuda"), torch.empty(cap, device="cuda")
    hc.hc_layer_norm_fwd(x, 1e-5, gamma, beta, y, mean=m, rstd=r)
    yt, mt, rt = torch.empty_like(tail), torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
    hc.hc_layer_norm_fwd(tail, 1e-5, gamma, beta, yt, mean=mt, rstd=rt)
    assert torch.equal(y[-9:], yt) and torch.equal(m[-9:], mt)
    hc.hc_layer_norm_bwd(x, y, gamma, m, r, dx=y)
    hc.hc_layer_norm_bwd(tail, yt, gamma, mt, rt, dx=yt)
    assert torch.equal(y[-9:], yt)
    q, s = quantise(x)
    qt, st = quantise(tail)
    assert torch.equal(q[-9:], qt) and torch.equal(s[:, -9:], st)
    # x as a table, and as the gradient of tokens that read two rows
    ids = torch.tensor([cap - 1, cap - 9, 0, -1], dtype=torch.int32, device="cuda")
    e = torch.empty(4, C, dtype=BF, device="cuda")
    hc.hc_embedding_fwd(x, ids, 1.0, e)
    assert torch.equal(e[0], tail[-1]) and torch.equal(e[1], tail[0]) and (e[2] == 1).all()
    ids = torch.zeros(cap, dtype=torch.int32, device="cuda")
    ids[-1] = 1
    rp = torch.empty(3, dtype=torch.int32, device="cuda")
    od = torch.empty(cap, dtype=torch.int32, device="cuda")
    hc.hc_embedding_sort(ids, 2, rp, od)
    d = torch.empty(2, C, device="cuda")
    hc.hc_embedding_bwd(x, rp, od, 1.0, d)
    assert torch.equal(d[1], tail[-1].float())
    del y, e, d
    # 8-bit rows, and an output, past 2^31 elements
    w, ws = quantise_weight(randn(g, C, 24))
    o = torch.empty(cap, 24, device="cuda")
    hc.hc_fp8_linear_fwd(q, s, w, ws, None, 0, o)
    ot = torch.empty(9, 24, device="cuda")
    hc.hc_fp8_linear_fwd(qt, st.contiguous(), w, ws, None, 0, ot)
    mag = value(qt, st, C).abs() @ value_w(w, ws, C).abs().t()
    within(o[-9:], ot.to(D64), (4 * 128 + 4 * (C // 128) + 16) * U * mag, "the last rows")
    del x, q
    N = 2 ** 31 // 65536 + 24
    q, s = quantise(randn(g, 65536, 16))
    w, ws = quantise_weight(randn(g, 16, N))
    y = torch.empty(65536, N, dtype=BF, device="cuda")
    hc.hc_fp8_linear_fwd(q, s, w, ws, None, 0, y)
    ref, tol = linear_ref(q[-5:], s[:, -5:], w, ws, 16, None, 0)
    within(y[-5:], ref, tol + rounding(BF, ref), "y")


def value_w(w, ws, K):
    v = w.view(torch.float8_e4m3fn).to(D64)[:, :K]
    return v * ws.to(D64).repeat_interleave(128, 0)[:w.shape[0]].repeat_interleave(128, 1)[:, :K]
