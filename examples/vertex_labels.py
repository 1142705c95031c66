"""A semantic label for every active vertex of masked frames: a token network
with a residual stream, its loss and its clipped gradients, trained and served.

Every active (frame, vertex) row of a contact mask is a token whose id is its
vertex. With the number of active rows left on the device:
    x = scale * table[vertex]             hc_embedding_fwd
    y = (rms norm of x) W                 8 bits: hc_rms_norm_fwd, hc_fp8_linear_fwd
    h = x + y, z = rms norm of h          hc_rms_norm_fwd
    loss = cross entropy of z head^T + bias against the vertex's label
                                          hc_linear_cross_entropy_fwd
and backwards
    dz, dhead, dbias                      hc_linear_cross_entropy_bwd
    dh, dgamma2                           hc_rms_norm_bwd
    dn = dh W^T                           8 bits: hc_quantize_fp8_rows, hc_fp8_linear_fwd
    dx, dgamma1                           hc_rms_norm_bwd, with dh on the residual stream
    dtable                                hc_embedding_sort (once per mask), hc_embedding_bwd
    all of them, their norm at most 1     hc_grad_norm, hc_grad_clip
W is given; some vertices have no label. A whole step is captured into a graph
and replayed. Then single tokens are run through the network, and the
probability of each one's label is compared with the batch's.

    python examples/vertex_labels.py
"""
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2608_09388_gb300 import hc  # noqa: E402

EPS = 1e-5


def weight8(W):
    """A weight [C_in, C_out] in 8 bits, laid out once."""
    C_in, C_out = W.shape
    wq = torch.empty(C_out, hc.HC_FP8_PITCH(C_in), dtype=torch.float8_e4m3fn, device="cuda")
    ws = torch.empty((C_out + 127) // 128, (C_in + 127) // 128, device="cuda")
    hc.hc_quantize_fp8_weight(W.contiguous(), wq, ws)
    return wq, ws


def rows8(capacity, C):
    """Buffers for up to `capacity` rows of C channels in 8 bits."""
    return (torch.empty(capacity, hc.HC_FP8_PITCH(C), dtype=torch.float8_e4m3fn, device="cuda"),
            torch.empty((C + 127) // 128, capacity, device="cuda"))


class Parameters:
    def __init__(self, V, C, labels, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        f = dict(generator=g, device="cuda")
        self.scale = math.sqrt(C)
        self.table = torch.randn(V, C, **f) / self.scale
        self.gamma1, self.gamma2 = torch.ones(C, device="cuda"), torch.ones(C, device="cuda")
        self.head = torch.randn(labels, C, **f) / self.scale
        self.bias = torch.zeros(labels, device="cuda")
        W = torch.randn(C, C, **f) / self.scale
        self.fwd8, self.bwd8 = weight8(W), weight8(W.t())

    def trained(self):
        return self.table, self.gamma1, self.gamma2, self.head, self.bias


class Tokens:
    """The buffers of up to `capacity` tokens, and the passes over them."""

    def __init__(self, p, capacity):
        self.p = p
        V, C = p.table.shape
        f = dict(device="cuda")
        self.x, self.y, self.h, self.z = (torch.empty(capacity, C, **f) for _ in range(4))
        self.dz, self.dh, self.dn, self.dx = (torch.empty(capacity, C, **f) for _ in range(4))
        self.rstd1, self.rstd2, self.loss, self.lse = (torch.empty(capacity, **f) for _ in range(4))
        self.n8, self.dh8 = rows8(capacity, C), rows8(capacity, C)
        self.row_ptr = torch.empty(V + 1, dtype=torch.int32, **f)
        self.order = torch.empty(capacity, dtype=torch.int32, **f)
        self.grads = [torch.empty_like(t) for t in p.trained()]
        self.clipped = [torch.empty_like(t) for t in p.trained()]
        self.list = hc.hc_tensor_list(self.grads, self.clipped)
        self.norm = torch.empty(1, **f)

    def forward(self, ids, labels, count=None):
        p = self.p
        hc.hc_embedding_fwd(p.table, ids, p.scale, self.x, count=count)
        hc.hc_rms_norm_fwd(self.x, EPS, p.gamma1, rstd=self.rstd1, q=self.n8[0], scales=self.n8[1],
                           count=count)
        hc.hc_fp8_linear_fwd(*self.n8, *p.fwd8, None, hc.HC_ACT_NONE, self.y, count=count)
        hc.hc_rms_norm_fwd(self.y, EPS, p.gamma2, res=self.x, h=self.h, y=self.z, rstd=self.rstd2,
                           count=count)
        hc.hc_linear_cross_entropy_fwd(self.z, p.head, p.bias, labels, self.loss, self.lse, count=count)

    def sort(self, ids, count):
        hc.hc_embedding_sort(ids, self.p.table.shape[0], self.row_ptr, self.order, count=count)

    def backward(self, labels, dloss, max_norm, count=None):
        p = self.p
        dtable, dgamma1, dgamma2, dhead, dbias = self.grads
        hc.hc_linear_cross_entropy_bwd(self.z, p.head, p.bias, labels, self.lse, dloss, dx=self.dz,
                                       dW=dhead, dbias=dbias, count=count)
        hc.hc_rms_norm_bwd(self.h, self.dz, p.gamma2, self.rstd2, dx=self.dh, dgamma=dgamma2,
                           count=count)
        hc.hc_quantize_fp8_rows(self.dh, *self.dh8, count=count)
        hc.hc_fp8_linear_fwd(*self.dh8, *p.bwd8, None, hc.HC_ACT_NONE, self.dn, count=count)
        hc.hc_rms_norm_bwd(self.x, self.dn, p.gamma1, self.rstd1, dres=self.dh, dx=self.dx,
                           dgamma=dgamma1, count=count)
        hc.hc_embedding_bwd(self.dx, self.row_ptr, self.order, p.scale, dtable)
        hc.hc_grad_norm(self.list, self.norm)
        hc.hc_grad_clip(self.list, self.norm, max_norm)

    def descend(self, rate):
        for t, g in zip(self.p.trained(), self.clipped):
            t.add_(g, alpha=-rate)


def batch(B, V, labels, density, unlabelled, seed):
    """Active rows of masked frames and their labels (-1: none), one for a vertex."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    capacity = B * V
    mask = (torch.rand(B, V, generator=g, device="cuda") < density).to(torch.uint8)
    coords = torch.zeros(capacity, 2, dtype=torch.int32, device="cuda")
    row_of = torch.empty(B, V, dtype=torch.int32, device="cuda")
    offsets = torch.empty(B + 1, dtype=torch.int32, device="cuda")
    count = torch.empty(1, dtype=torch.int32, device="cuda")
    hc.hc_mask_compact(mask, coords, row_of, offsets, count)
    of = torch.randint(0, labels, (V,), generator=g, device="cuda")
    of[torch.rand(V, generator=g, device="cuda") < unlabelled] = -1
    ids = coords[:, 1]
    return ids, of[ids.long()].int(), count


def main(B=8, V=655, C=256, labels=42, density=0.2, steps=60, rate=0.5, say=print):
    """Returns the trained buffers, the batch, and the largest difference between a
    token's loss alone and in the batch."""
    p = Parameters(V, C, labels, 7)
    ids, want, count = batch(B, V, labels, density, 0.2, 0)
    net = Tokens(p, ids.shape[0])
    n = int(count.item())  # for the loss's mean alone: the operators read it on the device
    used = int((want[:n] >= 0).sum())
    dloss = torch.full((ids.shape[0],), 1.0 / used, device="cuda")

    def step():
        net.forward(ids, want, count)
        net.backward(want, dloss, 1.0, count)
        net.descend(rate)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        net.sort(ids, count)
        step()  # workspaces of the stream are there before the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for k in range(1, steps + 1):
        graph.replay()
        if say and (k % 10 == 0 or k == 1):
            say(f"step {k:3d}  {used} labelled of {n} tokens  loss {float(net.loss[:n].sum()) / used:.4f}"
                f"  norm {float(net.norm):.3f}")
    net.forward(ids, want, count)
    torch.cuda.synchronize()

    one, worst = Tokens(p, 1), 0.0
    for t in range(0, n, max(1, n // 16)):
        one.forward(ids[t:t + 1], want[t:t + 1])
        worst = max(worst, float((one.loss[0] - net.loss[t]).abs()))
    status = hc.hc_get_device_status()
    if status != hc.HC_OK:
        raise RuntimeError(f"device status {hc.STATUS_NAMES[status]}")
    if say:
        say(f"largest difference of a token's loss alone: {worst:.2e}")
    return net, (ids, want, count, dloss), worst


if __name__ == "__main__":
    main()
