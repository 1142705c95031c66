"""A token network on the active vertices of masked frames, trained and served
with the token operators.

Every active (frame, vertex) row of a contact mask is a token whose id is its
vertex. The front of the network is
    x = scale * table[vertex]          hc_embedding_fwd on the coordinates' vertex column
    h = layer norm of x                hc_layer_norm_fwd
    y = h W                            8 bits: hc_quantize_fp8_rows, hc_fp8_linear_fwd
with the number of active rows left on the device. The table, gamma and beta
are fitted by gradient descent to the outputs of another table; W is given.
The gradients come from
    dh      the same 8-bit product with the transposed weight
    dx, dgamma, dbeta    hc_layer_norm_bwd
    dtable  hc_embedding_sort (once per mask), hc_embedding_bwd
Then single tokens are run through the trained network, as a decoding loop
would, and compared with the batch.

    python examples/vertex_tokens.py
"""
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2608_09388_gb300 import hc  # noqa: E402

EPS = 1e-5


class Linear8:
    """A weight [C_in, C_out] in 8 bits, laid out once."""

    def __init__(self, W):
        C_in, C_out = W.shape
        self.wq = torch.empty(C_out, hc.HC_FP8_PITCH(C_in), dtype=torch.float8_e4m3fn, device="cuda")
        self.ws = torch.empty((C_out + 127) // 128, (C_in + 127) // 128, device="cuda")
        hc.hc_quantize_fp8_weight(W.contiguous(), self.wq, self.ws)

    def rows(self, capacity):
        """Buffers for up to `capacity` rows in 8 bits."""
        blocks, pitch = self.ws.shape[1], self.wq.shape[1]
        return (torch.empty(capacity, pitch, dtype=torch.float8_e4m3fn, device="cuda"),
                torch.empty(blocks, capacity, device="cuda"))

    def __call__(self, x, rows, y, count=None):
        q, s = rows
        hc.hc_quantize_fp8_rows(x, q, s, count=count)
        hc.hc_fp8_linear_fwd(q, s, self.wq, self.ws, None, hc.HC_ACT_NONE, y, count=count)


class Front:
    """Embedding, layer norm and the 8-bit linear layer, with gradients."""

    def __init__(self, V, C, N, capacity, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.scale = math.sqrt(C)
        self.table = torch.randn(V, C, generator=g, device="cuda") / self.scale
        self.gamma, self.beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
        W = torch.randn(C, N, generator=torch.Generator(device="cuda").manual_seed(1),
                        device="cuda") / math.sqrt(C)
        self.fwd8, self.bwd8 = Linear8(W), Linear8(W.t())
        self.fwd_rows, self.bwd_rows = self.fwd8.rows(capacity), self.bwd8.rows(capacity)
        f = dict(device="cuda")
        self.x, self.h, self.dh = (torch.empty(capacity, C, **f) for _ in range(3))
        self.y = torch.empty(capacity, N, **f)
        self.mean, self.rstd = torch.empty(capacity, **f), torch.empty(capacity, **f)
        self.dtable = torch.empty(V, C, **f)
        self.dgamma, self.dbeta = torch.empty(C, **f), torch.empty(C, **f)
        self.row_ptr = torch.empty(V + 1, dtype=torch.int32, **f)
        self.order = torch.empty(capacity, dtype=torch.int32, **f)

    def forward(self, ids, count):
        hc.hc_embedding_fwd(self.table, ids, self.scale, self.x, count=count)
        hc.hc_layer_norm_fwd(self.x, EPS, self.gamma, self.beta, self.h, mean=self.mean,
                             rstd=self.rstd, count=count)
        self.fwd8(self.h, self.fwd_rows, self.y, count)
        return self.y

    def sort(self, ids, count):
        hc.hc_embedding_sort(ids, self.table.shape[0], self.row_ptr, self.order, count=count)

    def backward(self, dy, count):
        self.bwd8(dy, self.bwd_rows, self.dh, count)
        # dx takes dh's place
        hc.hc_layer_norm_bwd(self.x, self.dh, self.gamma, self.mean, self.rstd, dx=self.dh,
                             dgamma=self.dgamma, dbeta=self.dbeta, count=count)
        hc.hc_embedding_bwd(self.dh, self.row_ptr, self.order, self.scale, self.dtable)

    def step(self, rate, tokens):
        """Gradient descent: a table row moves x by scale^2 times its rate, and
        gamma's and beta's gradients are sums over all tokens."""
        self.table.add_(self.dtable, alpha=-rate / self.scale ** 2)
        self.gamma.add_(self.dgamma, alpha=-rate / tokens)
        self.beta.add_(self.dbeta, alpha=-rate / tokens)


def main(B=8, V=655, C=256, N=192, density=0.2, steps=41, rate=0.1, say=print):
    """Returns the losses of the training steps and the largest difference of a
    token run alone from the same token in the batch."""
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    capacity = B * V
    mask = (torch.rand(B, V, generator=g, device="cuda") < density).to(torch.uint8)
    coords = torch.empty(capacity, 2, dtype=torch.int32, device="cuda")
    row_of = torch.empty(B, V, dtype=torch.int32, device="cuda")
    offsets = torch.empty(B + 1, dtype=torch.int32, device="cuda")
    count = torch.empty(1, dtype=torch.int32, device="cuda")
    hc.hc_mask_compact(mask, coords, row_of, offsets, count)
    ids = coords[:, 1]

    teacher, net = (Front(V, C, N, capacity, seed) for seed in (11, 12))
    n = int(count.item())  # for the loss alone: the operators read it on the device
    want = teacher.forward(ids, count)[:n].clone()
    dy = torch.zeros(capacity, N, device="cuda")
    net.sort(ids, count)
    losses = []
    for k in range(steps):
        out = net.forward(ids, count)[:n]
        losses.append(float((out - want).square().mean()))
        torch.sub(out, want, out=dy[:n])
        net.backward(dy, count)
        net.step(rate, n)
        if say and (k % 10 == 0 or k == steps - 1):
            say(f"step {k:3d}  {n} tokens  loss {losses[-1]:.4f}")

    batch = net.forward(ids, count)[:n].clone()
    worst = 0.0
    one = torch.empty(1, N, device="cuda")
    x, h = torch.empty(1, C, device="cuda"), torch.empty(1, C, device="cuda")
    single = net.fwd8.rows(1)
    for t in range(0, n, max(1, n // 16)):
        hc.hc_embedding_fwd(net.table, ids[t:t + 1], net.scale, x)
        hc.hc_layer_norm_fwd(x, EPS, net.gamma, net.beta, h)
        net.fwd8(h, single, one)
        worst = max(worst, float((one[0] - batch[t]).abs().max()))
    status = hc.hc_get_device_status()
    if status != hc.HC_OK:
        raise RuntimeError(f"device status {hc.STATUS_NAMES[status]}")
    if say:
        say(f"largest difference of a token run alone: {worst:.2e}")
    return losses, worst


if __name__ == "__main__":
    main()
