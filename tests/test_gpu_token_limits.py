"""Token operators at sizes whose products and sums pass 32 bits. Each case runs in a
process of its own: the workspaces of such sizes are given back with it."""
import os
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_09388_gb300 import hc  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF = torch.bfloat16


def layer_norm_wide():
    """dgamma and dbeta of rows of more than 2^30 channels: 2 C passes 2^31."""
    n, C = 2, 2 ** 30 + 8
    x = torch.ones(n, C, dtype=BF, device="cuda")
    x[1] = -1
    dy = torch.ones(n, C, dtype=BF, device="cuda")
    dy[1, -3:], dy[0, :3] = 2, 4
    mean, rstd = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    dg, db = (torch.full((C,), 77.0, device="cuda") for _ in range(2))
    hc.hc_layer_norm_bwd(x, dy, None, mean, rstd, dgamma=dg, dbeta=db)
    # dy0 - dy1 and dy0 + dy1
    assert (dg[:3] == 3).all() and (db[:3] == 5).all()
    assert (dg[-3:] == -1).all() and (db[-3:] == 3).all()
    assert int((dg[3:-3] == 0).sum()) == C - 6 and int((db[3:-3] == 2).sum()) == C - 6


def linear_rows():
    """An 8-bit product of as many rows as an int counts: the first rows and the last
    ones, which the others, all zero, are not."""
    n, K, N = 2 ** 31 - 1, 16, 8
    q = torch.zeros(n, K, dtype=torch.uint8, device="cuda")
    s = torch.full((1, n), 0.5, device="cuda")
    one, two = 0x38, 0x40  # e4m3
    q[:3], q[-300:] = two, one
    w = torch.full((N, K), one, dtype=torch.uint8, device="cuda")
    ws = torch.full((1, 1), 2.0, device="cuda")
    bias = torch.arange(N, device="cuda").float()
    y = torch.full((n, N), 77.0, dtype=BF, device="cuda")
    hc.hc_fp8_linear_fwd(q, s, w, ws, bias, hc.HC_ACT_NONE, y)
    b = bias.to(BF)
    assert (y[:3] == b + 32).all() and (y[-300:] == b + 16).all()
    for at in range(3, n - 300, 2 ** 28):  # in parts: a comparison of all would take as much memory
        assert (y[at:min(at + 2 ** 28, n - 300)] == b).all(), at


def embedding_tokens():
    """As many tokens as an int counts, nearly all of them one id: the ends of
    the sorted entries, and of the rows' ranges, are the largest int."""
    n, V = 2 ** 31 - 1, 5
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    ids[-61:-41], ids[-41:-21], ids[-21:-1], ids[5] = 1, 3, 4, 4
    rp = torch.empty(V + 1, dtype=torch.int32, device="cuda")
    od = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    hc.hc_embedding_sort(ids, V, rp, od)
    assert rp.tolist() == [0, n - 61, n - 41, n - 41, n - 21, n]
    last = torch.arange(n - 61, n, device="cuda")
    assert torch.equal(od[n - 61:n - 21].long(), last[:40]) and od[n - 21] == 5
    assert torch.equal(od[n - 20:].long(), last[40:60])
    assert torch.equal(od[:5].long(), last[:5] - (n - 61)) and od[5] == 6 and od[n - 62] == n - 1
    del ids
    dy = torch.ones(n, 1, dtype=BF, device="cuda")
    dy[-61:] = 3
    dt = torch.full((V, 1), 77.0, device="cuda")
    hc.hc_embedding_bwd(dy, rp, od, 0.5, dt)
    assert dt[1:, 0].tolist() == [30.0, 0.0, 30.0, 30.5]
    # chunks' sums are exact (below 2^24), their join is not: 1300 additions
    assert abs(float(dt[0, 0]) - 0.5 * (n - 62 + 3)) <= 1300 * 2.0 ** -24 * n
    y = torch.empty(n, 1, dtype=BF, device="cuda")
    ids = torch.ones(n, dtype=torch.int32, device="cuda")
    ids[-3:] = 2
    hc.hc_embedding_fwd(torch.tensor([[5.0], [6.0], [7.0]], dtype=BF, device="cuda"), ids, 1.0, y)
    assert (y[-3:] == 7).all() and y[n - 4] == 6 and int((y[:-3] == 6).sum()) == n - 3


CASES = [layer_norm_wide, linear_rows, embedding_tokens]


@pytest.mark.parametrize("case", [c.__name__ for c in CASES])
def test_sizes_past_32_bits(case):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_09388_gb300 import build
    build.build()
    r = subprocess.run([sys.executable, os.path.abspath(__file__), case], capture_output=True,
                       text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]


if __name__ == "__main__":
    {c.__name__: c for c in CASES}[sys.argv[1]]()
    assert hc.hc_get_device_status() == hc.HC_OK
