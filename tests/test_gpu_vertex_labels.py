"""The network of examples/vertex_labels.py: every operator of a training step
against the formulas in 64 bits on the buffers that the step left, the step
captured and replayed, other types and widths, and single tokens."""
import os
import sys

import pytest

from paper_2608_09388_gb300 import hc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))

D64 = torch.float64


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_09388_gb300 import build
    build.build()
    hc.load_library()
    assert hc.hc_get_device_status() == hc.HC_OK


def values8(q, s, n, C):
    """The numbers that rows or a weight's rows in 8 bits stand for."""
    return q[:n].to(D64)[:, :C] * s.t()[:n].to(D64).repeat_interleave(128, 1)[:, :C]


def weight_values(wq, ws, C_in):
    s = ws.to(D64).repeat_interleave(128, 0)[:wq.shape[0]].repeat_interleave(128, 1)[:, :C_in]
    return wq.to(D64)[:, :C_in] * s


def close(got, ref, what):
    """fp32 sums of up to a thousand terms, gradients of products of a few
    roundings each: 2^-24 * 2000 of the largest of what was summed, which the
    result's own size stands for here."""
    err = (got.to(D64) - ref).abs().max()
    assert err <= 1.2e-4 * ref.abs().max(), (what, float(err), float(ref.abs().max()))


def norm_ref(x, gamma, dy=None, dres=None):
    x = x.to(D64).requires_grad_()
    g = gamma.to(D64).requires_grad_()
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * g
    if dy is None:
        return y.detach()
    y.backward(dy.to(D64))
    return x.grad + (0 if dres is None else dres.to(D64)), g.grad


@pytest.mark.parametrize("C,labels,V", [(256, 42, 655), (136, 300, 500), (260, 7, 101)])
def test_a_step(C, labels, V):
    import vertex_labels as vl
    p = vl.Parameters(V, C, labels, 3)
    ids, want, count = vl.batch(4, V, labels, 0.3, 0.25, 1)
    net = vl.Tokens(p, ids.shape[0])
    n = int(count.item())
    dloss = torch.full((ids.shape[0],), 1 / 300, device="cuda")
    net.sort(ids, count)
    net.forward(ids, want, count)
    net.backward(want, dloss, 0.01, count)
    assert hc.hc_get_device_status() == hc.HC_OK
    x = net.x[:n]
    assert torch.equal(x, p.table[ids[:n].long()] * p.scale)
    n1 = values8(*net.n8, n, C)
    # 8 bits: half a step is at most 2^-4 of a value, or of the smallest normal
    # number of its block
    v = norm_ref(x, p.gamma1)
    blocks = v.abs().split(128, 1)
    floor = torch.cat([b.amax(1, keepdim=True).expand_as(b) / 448 * 2.0 ** -6 for b in blocks], 1)
    assert ((n1 - v).abs() <= (2.0 ** -4 + 1e-5) * torch.maximum(v.abs(), floor)).all()
    close(net.y[:n], n1 @ weight_values(*p.fwd8, C).t(), "y")
    close(net.h[:n], x.to(D64) + net.y[:n].to(D64), "h")
    close(net.z[:n], norm_ref(net.h[:n], p.gamma2), "z")
    on = want[:n] >= 0
    z, W, b = (t.to(D64).requires_grad_() for t in (net.z[:n], p.head, p.bias))
    l = torch.log_softmax(z @ W.t() + b, 1)
    loss = torch.where(on, -l.gather(1, want[:n].long().clamp_min(0)[:, None])[:, 0], 0.0)
    close(net.loss[:n], loss.detach(), "loss")
    (loss.sum() / 300).backward()
    dtable, dgamma1, dgamma2, dhead, dbias = net.grads
    close(net.dz[:n], z.grad, "dz")
    close(dhead, W.grad, "dhead")
    close(dbias, b.grad, "dbias")
    dh, dg2 = norm_ref(net.h[:n], p.gamma2, net.dz[:n])
    close(net.dh[:n], dh, "dh")
    close(dgamma2, dg2, "dgamma2")
    close(net.dn[:n], values8(*net.dh8, n, C) @ weight_values(*p.bwd8, C).t(), "dn")
    dx, dg1 = norm_ref(x, p.gamma1, net.dn[:n], net.dh[:n])
    close(net.dx[:n], dx, "dx")
    close(dgamma1, dg1, "dgamma1")
    ref = torch.zeros(V, C, dtype=D64, device="cuda").index_add_(0, ids[:n].long(), net.dx[:n].to(D64))
    close(dtable, ref * p.scale, "dtable")
    norm = float(torch.stack([g.to(D64).square().sum() for g in net.grads]).sum().sqrt())
    assert norm > 0.01 and abs(float(net.norm) - norm) <= 1e-6 * norm
    for g, c in zip(net.grads, net.clipped):
        close(c, g.to(D64) * (0.01 / norm), "clipped")


def test_example_runs():
    """Training in a replayed graph, then single tokens: alone and in the batch a
    token is rounded to 8 bits alike, only the order of fp32 sums may differ (256
    channels of logits below 2^6, 42 classes)."""
    import vertex_labels as vl
    net, (ids, want, count, dloss), worst = vl.main(say=None)
    assert worst <= 512 * 2.0 ** -24 * 64
    n = int(count.item())
    assert net.loss[:n].isfinite().all() and all(t.isfinite().all() for t in net.p.trained())
    # one more step, eager and replayed, from the same state: the same bits
    start = [t.clone() for t in net.p.trained()]

    def step(stream=None):
        net.forward(ids, want, count)
        net.backward(want, dloss, 1.0, count)
        net.descend(0.5)

    step()
    torch.cuda.synchronize()
    eager = [t.clone() for t in net.p.trained()]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for t, s in zip(net.p.trained(), start):
        t.copy_(s)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(net.p.trained(), eager))
    assert hc.hc_get_device_status() == hc.HC_OK
