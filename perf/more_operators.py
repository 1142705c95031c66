"""Measured cases of the operators around a token network's layers: root-mean-square
norm with the residual's addition, the loss, and the clipping of the gradients.

A token is one row of a compact [capacity, C] matrix; rows n < N' are in use,
N' (`count`) is one int32 on the device.

  rms   h = x + residual, held in the rows' type; y = h / rms(h) * gamma, in
        that type, or in 8 bits (e4m3, an fp32 scale per block of 128 channels)
        for the 8-bit linear layer; its gradient, with the gradient of the
        residual stream added
  xent  softmax cross entropy of the logits x W^T + bias against one class per
        token (-1: the token takes no part), and the gradients of x, W and bias
  clip  the norm over all gradients of a network, and the gradients scaled so
        that it is at most max_norm

`run` computes them with elementary torch operations in 32 bits where `own` is
false, and through paper_2608_09388_gb300.hc where it is true.
"""
import math

import torch

own = False

E4M3_MAX = 448.0          # largest finite e4m3 value
TINY = 2.0 ** -126        # smallest scale: the smallest normal binary32
BLOCK = 128               # channels that share a scale
EPS = 1e-5
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token of a decoding step between two layers: residual added, normalised, made the input of an 8-bit product; latency only
        {"name": "rms 1x4096 bf16 8 bits", "op": "rms", "rows": 1, "capacity": 1, "C": 4096, "dtype": "bf16", "out": "q"},
        # active rows of 32 masked 10475-vertex frames (about 5% of the capacity), an odd channel count, one training step
        {"name": "rms 16763x131 f32 train", "op": "rms", "rows": 16763, "capacity": 335200, "C": 131, "dtype": "f32", "out": "train"},
        # a large batch of tokens, one training step
        {"name": "rms 65536x2048 bf16 train", "op": "rms", "rows": 65536, "capacity": 65536, "C": 2048, "dtype": "bf16", "out": "train"},
        # a long prompt in front of an 8-bit product
        {"name": "rms 16384x8192 bf16 8 bits", "op": "rms", "rows": 16384, "capacity": 16384, "C": 8192, "dtype": "bf16", "out": "q"},
        # the probability of one given token, as a scoring loop asks for it: the weight is read once
        {"name": "xent 1 of 32000x4096 bf16 score", "op": "xent", "rows": 1, "capacity": 1, "V": 32000, "C": 4096, "dtype": "bf16", "bias": False, "ignored": 0.0, "train": False},
        # one of 42 semantic labels for every active vertex of 32 masked frames, from 64 channels, some vertices unlabelled; one training step
        {"name": "xent 16763 of 42x64 f32 train", "op": "xent", "rows": 16763, "capacity": 335200, "V": 42, "C": 64, "dtype": "f32", "bias": True, "ignored": 0.25, "train": True},
        # an ordinary training batch
        {"name": "xent 2048 of 32000x1024 bf16 train", "op": "xent", "rows": 2048, "capacity": 2048, "V": 32000, "C": 1024, "dtype": "bf16", "bias": False, "ignored": 0.05, "train": True},
        # a large batch over a large vocabulary
        {"name": "xent 8192 of 131072x2048 bf16 train", "op": "xent", "rows": 8192, "capacity": 8192, "V": 131072, "C": 2048, "dtype": "bf16", "bias": False, "ignored": 0.02, "train": True},
        # the gradients of a small token network (a vertex table, norms, a head), a training step of a few microseconds
        {"name": "clip 5 tensors 0.2M f32", "op": "clip", "tensors": 5, "numel": 200_000, "bf16": 0.0, "max_norm": 1.0, "norm": 7.0},
        # many tensors of all sizes that together fit the L2 cache
        {"name": "clip 60 tensors 20M mixed", "op": "clip", "tensors": 60, "numel": 20_000_000, "bf16": 0.7, "max_norm": 1.0, "norm": 3.0},
        # all gradients of a large network
        {"name": "clip 400 tensors 1.2G mixed", "op": "clip", "tensors": 400, "numel": 1_200_000_000, "bf16": 0.9, "max_norm": 1.0, "norm": 2.5},
    ]


def draw(rng):
    """One case of the same ranges: sizes over their logarithm, half of the
    widths rounded to 8, the others left odd or even."""
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def width(lo, hi):
        c = log(lo, hi)
        return max(lo, c // 8 * 8) if rng.random() < 0.5 else c

    op = rng.choice(("rms", "xent", "clip"))
    dtype = rng.choice(("bf16", "f32"))
    if op == "rms":
        C = width(8, 8192)
        rows = min(log(1, 65536), max(1, (1 << 26) // C))
        slack = rng.choice((0, 0, rng.randrange(0, 3 * rows + 2)))
        return {"op": op, "rows": rows, "capacity": rows + slack, "C": C, "dtype": dtype, "out": rng.choice(("q", "y", "train", "train"))}
    if op == "xent":
        C = width(16, 4096)
        V = width(32, 131072)
        most = (1 << 41 if dtype == "bf16" else 1 << 37) // (V * C)
        rows = min(log(1, 8192), max(1, most))
        slack = rng.choice((0, 0, rng.randrange(0, 3 * rows + 2)))
        return {"op": op, "rows": rows, "capacity": rows + slack, "V": V, "C": C, "dtype": dtype, "bias": rng.random() < 0.5,
                "ignored": rng.choice((0.0, 0.1, 0.5)), "train": rng.random() < 0.75}
    n = log(1, 600)
    norm = math.exp(rng.uniform(math.log(0.3), math.log(30.0)))
    # a norm at the very border would leave the scale to the last bit of the sum
    return {"op": op, "tensors": n, "numel": max(n, log(1000, 1_000_000_000)), "bf16": rng.choice((0.0, 0.5, 1.0)), "max_norm": 1.0,
            "norm": 0.9 if 0.9 < norm < 1.1 else norm}


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _pitch(k):
    return (k + 15) // 16 * 16


def _activations(g, capacity, C, dtype):
    """Rows of a residual stream: a size of its own for each row, and channels
    of unequal size, a few of them outliers."""
    x = torch.randn(capacity, C, generator=g, device="cuda")
    ch = torch.exp(0.5 * torch.randn(C, generator=g, device="cuda"))
    ch = torch.where(torch.rand(C, generator=g, device="cuda") < 0.01, 8 * ch, ch)
    x.mul_(ch).mul_(torch.exp(0.3 * torch.randn(capacity, 1, generator=g, device="cuda")))
    return x.to(dtype)


def _sizes(n, numel, seed):
    """n tensor sizes that add up to numel: a few large matrices, many small
    vectors, as a network's parameters have them."""
    r = torch.Generator().manual_seed(seed)
    w = torch.exp(2.5 * torch.randn(n, generator=r, dtype=torch.float64))
    s = (w / w.sum() * (numel - n)).long() + 1
    s[0] += numel - int(s.sum())
    return s


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"c": c}
    f32 = dict(dtype=torch.float32, device="cuda")
    if c["op"] == "clip":
        # gradients of one type lie one after another in a buffer, each at the
        # next multiple of 8 elements, as a flat allocation holds them
        sizes = _sizes(c["tensors"], c["numel"], 1)
        half = torch.rand(c["tensors"], generator=torch.Generator().manual_seed(2)) < c["bf16"]
        s["grads"], s["outs"], s["flat"], s["flat_out"] = [], [], [], []
        total = float(c["numel"])
        for dt, mine in ((torch.float32, ~half), (torch.bfloat16, half)):
            mine = sizes[mine]
            if mine.numel() == 0:
                continue
            room = (mine + 7) // 8 * 8
            at = torch.cumsum(room, 0) - room
            flat = torch.empty(int(room.sum()), dtype=dt, device="cuda")
            out = torch.zeros_like(flat)
            # a size of its own for each tensor, the whole at about the norm asked for
            size = torch.exp(0.7 * torch.randn(mine.numel(), generator=torch.Generator().manual_seed(seed)))
            for a, m, k in zip(at.tolist(), mine.tolist(), size.tolist()):
                v = torch.randn(m, generator=g, device="cuda")
                flat[a:a + m] = v.mul_(k * c["norm"] / math.sqrt(total) / 1.63)  # 1.63: root mean square of the sizes
                flat[a + m:a + (m + 7) // 8 * 8] = 0
                s["grads"].append(flat[a:a + m])
                s["outs"].append(out[a:a + m])
            s["flat"].append(flat)
            s["flat_out"].append(out)
        s["norm"] = torch.empty(1, **f32)
        # the norm is exactly about what the case says: 2% around it
        have = float(torch.stack([f.double().square().sum() for f in s["flat"]]).sum().sqrt())
        want = c["norm"] * (1 + 0.02 * (seed % 7 - 3) / 3)
        for f in s["flat"]:
            f.mul_(want / have)
        return s
    dt, rows, cap, C = DT[c["dtype"]], c["rows"], c["capacity"], c["C"]
    s["count"] = torch.tensor([rows], dtype=torch.int32, device="cuda")
    if c["op"] == "rms":
        s["x"] = _activations(g, cap, C, dt)
        s["res"] = _activations(g, cap, C, dt)
        s["gamma"] = 1 + 0.2 * torch.randn(C, generator=g, device="cuda")
        s["h"] = torch.empty(cap, C, dtype=dt, device="cuda")
        if c["out"] == "q":
            s["q"] = torch.empty(cap, _pitch(C), dtype=torch.float8_e4m3fn, device="cuda")
            s["scales"] = torch.empty(_blocks(C), cap, **f32)
        else:
            s["y"] = torch.empty(cap, C, dtype=dt, device="cuda")
        if c["out"] == "train":
            s["rstd"] = torch.empty(cap, **f32)
            s["dy"] = torch.randn(cap, C, generator=g, device="cuda").to(dt)
            s["dres"] = torch.randn(cap, C, generator=g, device="cuda").to(dt)
            s["dx"] = torch.empty(cap, C, dtype=dt, device="cuda")
            s["dgamma"] = torch.empty(C, **f32)
        return s
    V = c["V"]
    # classes met with p(rank) ~ 1/rank; the hidden row leans towards its class's
    # row of W by an amount of its own, so that some tokens are sure and others not
    u = torch.rand(cap, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
    t = torch.randperm(V, generator=g, device="cuda")[rank]
    W = torch.randn(V, C, generator=g, device="cuda") * C ** -0.5
    lean = 12 * torch.rand(cap, 1, generator=g, device="cuda")
    s["x"] = (torch.randn(cap, C, generator=g, device="cuda") + lean * W[t]).to(dt)
    s["W"] = W.to(dt)
    s["bias"] = 0.1 * torch.randn(V, generator=g, device="cuda") if c["bias"] else None
    gone = torch.rand(cap, generator=g, device="cuda") < c["ignored"]
    gone[0] = False
    s["targets"] = torch.where(gone, -1, t).int()
    s["loss"], s["lse"] = torch.empty(cap, **f32), torch.empty(cap, **f32)
    if c["train"]:
        # the loss is the mean over the tokens that take part
        s["dloss"] = torch.full((cap,), 1.0 / max(1, int((~gone[:rows]).sum())), **f32)
        s["dx"] = torch.empty(cap, C, dtype=dt, device="cuda")
        s["dW"] = torch.empty(V, C, dtype=dt, device="cuda")
        s["dbias"] = torch.empty(V, **f32) if c["bias"] else None
    return s


def _quantise(x):
    """x [n, C] fp32 -> e4m3 values [n, pitch] (zero beyond C) and scales [blocks, n]."""
    n, C = x.shape
    b = torch.nn.functional.pad(x, (0, _blocks(C) * BLOCK - C)).view(n, _blocks(C), BLOCK)
    top = b.abs().amax(dim=2)
    s = (top / torch.full_like(top, E4M3_MAX)).clamp_min(TINY)
    q = (b / s[:, :, None]).to(torch.float8_e4m3fn).view(n, -1)[:, :_pitch(C)]
    return q.contiguous(), s.t().contiguous()


def _run_plain(s):
    c = s["c"]
    if c["op"] == "clip":
        # squares of up to a billion values: summed in 64 bits
        norm = torch.stack([f.square().sum(dtype=torch.float64) if f.dtype == torch.float32 else f.float().square().sum(dtype=torch.float64)
                            for f in s["flat"]]).sum().sqrt()
        scale = (c["max_norm"] / norm).clamp_max(1.0).float()
        return {"norm": norm.float().view(1), "grads": [(f.float() * scale).to(f.dtype) for f in s["flat"]]}
    dt, n = DT[c["dtype"]], c["rows"]
    if c["op"] == "rms":
        # the residual stream is held in the rows' type: the norm is that of the row as stored
        h = (s["x"][:n].float() + s["res"][:n].float()).to(dt)
        x = h.float()
        rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
        xh = x * rstd[:, None]
        v = xh * s["gamma"]
        out = {"h": h}
        if c["out"] == "q":
            out["q"], out["scales"] = _quantise(v)
            return out
        out["y"] = v.to(dt)
        if c["out"] == "train":
            dy = s["dy"][:n].float()
            t = dy * s["gamma"]
            dx = s["dres"][:n].float() + (t - xh * (t * xh).mean(1, keepdim=True)) * rstd[:, None]
            out.update(rstd=rstd, dx=dx.to(dt), dgamma=(dy * xh).sum(0))
        return out
    x, W = s["x"][:n].float(), s["W"].float()
    logits = x @ W.t()
    if s["bias"] is not None:
        logits = logits + s["bias"]
    t = s["targets"][:n].long()
    there = t >= 0
    at = t.clamp_min(0)[:, None]
    top = logits.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(logits - top).sum(1, keepdim=True))
    out = {"loss": torch.where(there, (lse - logits.gather(1, at))[:, 0], 0.0)}
    if c["train"]:
        G = torch.exp(logits - lse)
        G.scatter_add_(1, at, torch.full_like(lse, -1.0))
        G = G * torch.where(there, s["dloss"][:n], 0.0)[:, None]
        out["dx"], out["dW"] = (G @ W).to(dt), (G.t() @ x).to(dt)
        if s["bias"] is not None:
            out["dbias"] = G.sum(0)
    return out


def _run_own(s):
    from paper_2608_09388_gb300 import hc
    c = s["c"]
    if c["op"] == "clip":
        if "list" not in s:  # a training program makes it once: its gradients stay where they are
            s["list"] = hc.hc_tensor_list(s["grads"], s["outs"])
        hc.hc_grad_norm(s["list"], s["norm"])
        hc.hc_grad_clip(s["list"], s["norm"], c["max_norm"])
        return {"norm": s["norm"], "grads": s["flat_out"]}
    n, count = c["rows"], s["count"]
    if c["op"] == "rms":
        if c["out"] == "q":
            hc.hc_rms_norm_fwd(s["x"], EPS, s["gamma"], res=s["res"], h=s["h"], q=s["q"], scales=s["scales"], count=count)
            return {"h": s["h"][:n], "q": s["q"][:n], "scales": s["scales"][:, :n]}
        hc.hc_rms_norm_fwd(s["x"], EPS, s["gamma"], res=s["res"], h=s["h"], y=s["y"], rstd=s.get("rstd"), count=count)
        out = {"h": s["h"][:n], "y": s["y"][:n]}
        if c["out"] == "train":
            hc.hc_rms_norm_bwd(s["h"], s["dy"], s["gamma"], s["rstd"], dres=s["dres"], dx=s["dx"], dgamma=s["dgamma"], count=count)
            out.update(rstd=s["rstd"][:n], dx=s["dx"][:n], dgamma=s["dgamma"])
        return out
    hc.hc_linear_cross_entropy_fwd(s["x"], s["W"], s["bias"], s["targets"], s["loss"], s["lse"], count=count)
    out = {"loss": s["loss"][:n]}
    if c["train"]:
        hc.hc_linear_cross_entropy_bwd(s["x"], s["W"], s["bias"], s["targets"], s["lse"], s["dloss"], dx=s["dx"], dW=s["dW"], dbias=s["dbias"], count=count)
        out.update(dx=s["dx"][:n], dW=s["dW"])
        if s["bias"] is not None:
            out["dbias"] = s["dbias"]
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


def exact(case, seed):
    """The definitions in 64 bits. An e4m3 value has none: it is rounded by its
    definition, so only the scales are given."""
    s = prepare(case, seed)
    c = s["c"]
    d = torch.float64
    if c["op"] == "clip":
        norm = math.sqrt(sum(float(torch.dot(p, p)) for f in s["flat"] for p in (q.to(d) for q in f.split(1 << 26))))
        scale = min(1.0, c["max_norm"] / norm)
        return {"norm": torch.tensor([norm], dtype=d), "grads": [f.to(d).mul_(scale) for f in s["flat"]]}
    n = c["rows"]
    if c["op"] == "rms":
        total = s["x"][:n].to(d) + s["res"][:n].to(d)
        h = total.to(DT[c["dtype"]]).to(d)
        rstd = torch.rsqrt(torch.einsum("nc,nc->n", h, h) / c["C"] + EPS)
        ga = s["gamma"].to(d)
        v = torch.einsum("nc,n,c->nc", h, rstd, ga)
        out = {"h": total}
        if c["out"] == "q":
            out["q"] = None
            out["scales"] = (torch.stack([p.abs().amax(1) for p in v.split(BLOCK, 1)]) / E4M3_MAX).clamp_min(TINY)
            return out
        out["y"] = v
        if c["out"] == "train":
            dy = s["dy"][:n].to(d)
            dot = torch.einsum("nc,nc,c->n", dy, h, ga)
            # d/dh of h_c (sum h^2 / C + eps)^(-1/2) gamma_c
            dx = torch.einsum("nc,n,c->nc", dy, rstd, ga) - h * (rstd ** 3 * dot / c["C"])[:, None]
            out.update(rstd=rstd, dx=dx + s["dres"][:n].to(d), dgamma=torch.einsum("nc,nc,n->c", dy, h, rstd))
        return out
    V, C = c["V"], c["C"]
    x, W = s["x"][:n].to(d), s["W"].to(d)
    t = s["targets"][:n].long()
    used = torch.nonzero(t >= 0)[:, 0]
    x, t = x[used], t[used]
    b = torch.zeros(V, dtype=d, device="cuda") if s["bias"] is None else s["bias"].to(d)
    loss = torch.zeros(n, dtype=d, device="cuda")
    out = {"loss": loss}
    if c["train"]:
        out["dx"] = torch.zeros(n, C, dtype=d, device="cuda")
        out["dW"] = torch.zeros(V, C, dtype=d, device="cuda")
        if s["bias"] is not None:
            out["dbias"] = torch.zeros(V, dtype=d, device="cuda")
    for at in range(0, used.numel(), 2048):
        i, xi, ti = used[at:at + 2048], x[at:at + 2048], t[at:at + 2048]
        z = torch.addmm(b, xi, W.t())
        p = torch.log_softmax(z, 1)
        loss[i] = -p[torch.arange(ti.numel(), device="cuda"), ti]
        if c["train"]:
            p = p.exp_()
            p[torch.arange(ti.numel(), device="cuda"), ti] -= 1
            p *= s["dloss"][i].to(d)[:, None]
            out["dx"][i] = p @ W
            out["dW"].addmm_(p.t(), xi)
            if s["bias"] is not None:
                out["dbias"] += p.sum(0)
    return out


def work(case):
    c = case
    if c["op"] == "clip":
        e = 4 - 2 * c["bf16"]
        return {"bytes": 2.0 * c["numel"] * e + 4, "flops": 3.0 * c["numel"]}  # gradients in and out
    e, n, C = 2 if c["dtype"] == "bf16" else 4, c["rows"], c["C"]
    if c["op"] == "rms":
        b, f = 3 * n * C * e + 4 * C, 6.0 * n * C                              # x, res, h; gamma
        if c["out"] == "q":
            return {"bytes": b + n * _pitch(C) + 4 * n * _blocks(C), "flops": f + 3.0 * n * C}
        b += n * C * e                                                         # y
        if c["out"] == "train":
            b, f = b + 4 * n * C * e + 8 * n + 8 * C, f + 12.0 * n * C         # h, dy, dres, dx; rstd twice; gamma, dgamma
        return {"bytes": b, "flops": f}
    V, m = c["V"], n * (1 - c["ignored"])
    b, f = m * C * e + V * C * e + 8 * n, 2.0 * m * V * C                      # x, W, targets, loss
    if c["bias"]:
        b += 4 * V
    if c["train"]:
        b, f = b + n * C * e + V * C * e + 4 * n + (4 * V if c["bias"] else 0), f + 4.0 * m * V * C  # dx, dW, dloss, dbias
    return {"bytes": b, "flops": f}
