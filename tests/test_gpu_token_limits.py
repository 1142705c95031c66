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


CASES = [layer_norm_wide, linear_rows]


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
