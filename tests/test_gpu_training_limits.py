"""The norm, the loss and the clipping at sizes whose products pass 32 bits. Each
case runs in a process of its own: the workspaces of such sizes are given back with
it. What is compared is known without a computation of that size."""
import math
import os
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_09388_gb300 import hc  # noqa: E402

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF = torch.bfloat16


def rms_rows():
    """2^31 and more elements: every row is one of three."""
    n, C = 2 ** 18 + 5, 8192
    base = torch.randn(3, C, device="cuda").to(BF)
    kind = torch.arange(n, device="cuda") % 3
    x, res = base[kind], base.flip(0)[kind]
    y, q = torch.empty_like(x), torch.empty(n, C, dtype=torch.uint8, device="cuda")
    sc, rstd = torch.empty(C // 128, n, device="cuda"), torch.empty(n, device="cuda")
    hc.hc_rms_norm_fwd(x, 1e-5, None, res=res, h=x, y=y, rstd=rstd, q=q, scales=sc)
    for at in range(3, n, 2 ** 16 + 1):  # in parts: a comparison of all would take as much memory
        k = kind[at:at + 2 ** 16 + 1]
        for t in (x, y, q, rstd, sc.t()):
            assert torch.equal(t[at:at + 2 ** 16 + 1], t[:3][k]), at
    dx, dg = res, torch.empty(C, device="cuda")
    hc.hc_rms_norm_bwd(x, y, None, rstd, dres=res, dx=dx, dgamma=dg)
    for at in range(3, n, 2 ** 16 + 1):
        assert torch.equal(dx[at:at + 2 ** 16 + 1], dx[:3][kind[at:at + 2 ** 16 + 1]]), at
    assert dg.isfinite().all()


def loss_rows():
    """Rows whose elements pass 2^32: every token is one of seven, each with its
    own class; its loss and gradient are those of the seven alone, the weight's
    gradient is theirs by how many there are (all sums in fp32 of up to 10^6
    equal terms, then rounded to bf16)."""
    n, C, V = 2 ** 20 + 77, 4096, 300
    base = torch.randn(7, C, device="cuda").to(BF)
    W = (torch.randn(V, C, device="cuda") / 64).to(BF)
    kind = torch.arange(n, device="cuda") % 7
    x, t = base[kind], (kind * 40 + 3).int()
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dloss = torch.full((n,), 2.0 ** -20, device="cuda")
    dW = torch.empty_like(W)
    few = dict(loss=torch.empty(7, device="cuda"), lse=torch.empty(7, device="cuda"))
    hc.hc_linear_cross_entropy_fwd(base, W, None, t[:7], **few)
    hc.hc_linear_cross_entropy_fwd(x, W, None, t, loss=loss, lse=lse)
    assert torch.equal(loss, few["loss"][kind]) and torch.equal(lse, few["lse"][kind])
    l = base.double() @ W.double().t()
    G = torch.exp(l - lse[:7].double()[:, None])
    G[torch.arange(7), t[:7].long()] -= 1
    hc.hc_linear_cross_entropy_bwd(x, W, None, t, lse, dloss, dx=x, dW=dW)
    for at in range(7, n, 2 ** 17):
        assert torch.equal(x[at:at + 2 ** 17], x[:7][kind[at:at + 2 ** 17]]), at
    want = G @ W.double() * 2.0 ** -20
    off = 2.0 ** -7 * (G.abs() @ W.double().abs()) * 2.0 ** -20
    assert ((x[:7].double() - want).abs() <= off).all()
    times = torch.bincount(kind).double()[:, None] * 2.0 ** -20
    want = (G * times).t() @ base.double()
    # 2^-8 of G, 65541 steps of the accumulators at 2^-22 each, the result's 2^-8
    off = (2.0 ** -7 + 65541 * 2.0 ** -22) * ((G.abs() * times).t() @ base.double().abs())
    assert ((dW.double() - want).abs() <= off + 2.0 ** -8 * want.abs()).all()


def loss_classes():
    """A weight of more than 2^31 elements, one token and many: a class far
    behind is found, its gradient written."""
    V, C = 600_001, 4096
    W = torch.zeros(V, C, dtype=BF, device="cuda")
    x = torch.ones(300, C, dtype=BF, device="cuda")
    W[V - 2, :] = 2.0 ** -9   # a logit of 8, all others 0
    t = torch.full((300,), V - 2, dtype=torch.int32, device="cuda")
    want = math.log((V - 1) * math.exp(-8) + 1)
    for n in (1, 300):
        loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        hc.hc_linear_cross_entropy_fwd(x[:n], W, None, t[:n], loss, lse)
        assert ((loss - want).abs() <= 1e-5).all()
        dW = torch.empty_like(W)
        dloss = torch.ones(n, device="cuda")
        hc.hc_linear_cross_entropy_bwd(x[:n], W, None, t[:n], lse, dloss, dW=dW)
        p = math.exp(-8 - want), math.exp(-want) - 1
        assert abs(float(dW[V - 2, 7]) / (n * p[1]) - 1) <= 2.0 ** -6
        assert abs(float(dW[V - 1, C - 1]) / (n * p[0]) - 1) <= 2.0 ** -6
        assert abs(float(dW[0, 0]) / (n * p[0]) - 1) <= 2.0 ** -6
        del dW


def clip_elements():
    """A tensor of more than 2^31 elements beside a small one."""
    big = torch.full((2 ** 31 + 4099,), 2.0, dtype=BF, device="cuda")
    small = torch.full((1000,), 3.0, device="cuda")
    outs = [torch.empty_like(big), torch.empty_like(small)]
    lst, norm = hc.hc_tensor_list([big, small], outs), torch.empty(1, device="cuda")
    hc.hc_grad_norm(lst, norm)
    want = math.sqrt(4.0 * big.numel() + 9.0 * small.numel())
    assert abs(norm.item() / want - 1) <= 10 * 2.0 ** -24
    hc.hc_grad_clip(lst, norm, want / 4)
    for at in range(0, big.numel(), 2 ** 28):
        assert (outs[0][at:at + 2 ** 28] == 0.5).all(), at
    assert ((outs[1] - 0.75).abs() <= 1e-6).all()


CASES = [rms_rows, loss_rows, loss_classes, clip_elements]


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
    torch.manual_seed(0)
    {c.__name__: c for c in CASES}[sys.argv[1]]()
    assert hc.hc_get_device_status() == hc.HC_OK
