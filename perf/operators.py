"""Measured cases of the token operators: row embedding, layer norm and the 8-bit linear layer.

A token is one row of a compact [capacity, C] matrix, as the sparse layers hold
them: rows n < N' are in use, N' (`count`) is one int32 on the device. The
operators are the front of a network over such rows, and its training step:

  embed   y[n] = scale * table[ids[n]]; gradient: the rows of dy summed by
          token, in the order of a stable sort of the ids
  norm    layer norm of every row, with the mean and 1/sigma it saves; its
          gradient with the reduction of gamma's and beta's over the rows
  quant   a row cut into blocks of 128 channels, each held in 8 bits (e4m3)
          with one fp32 scale
  linear  the 8-bit product: activations quantised as above, weights in
          128 x 128 blocks with a scale each, bias and activation fused

`run` computes them with elementary torch operations in 32 bits where `own` is
false, and through paper_2608_09388_gb300.hc where it is true.
"""
import math

import torch

own = False

E4M3_MAX = 448.0          # largest finite e4m3 value
TINY = 2.0 ** -126        # smallest scale: the smallest normal binary32
BLOCK = 128               # channels (and output channels) that share a scale
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token of a decoding step through a normalisation: latency only
        {"name": "norm 1x4096 bf16 serve", "op": "norm", "rows": 1, "capacity": 1, "C": 4096, "dtype": "bf16", "train": False},
        # active rows of 32 masked 10475-vertex frames (about 5% of the capacity), an odd channel count, one training step
        {"name": "norm 16763x131 f32 train", "op": "norm", "rows": 16763, "capacity": 335200, "C": 131, "dtype": "f32", "train": True},
        # a large batch of tokens, one training step
        {"name": "norm 65536x2048 bf16 train", "op": "norm", "rows": 65536, "capacity": 65536, "C": 2048, "dtype": "bf16", "train": True},
        # the next token of each of a few sequences looked up in a vocabulary
        {"name": "embed 5 of 32000x4096 bf16 serve", "op": "embed", "rows": 5, "capacity": 5, "V": 32000, "C": 4096, "dtype": "bf16", "stride": 1, "train": False},
        # a learned vector per mesh vertex added to compact rows: the ids are the vertex column of the coordinates (stride 2)
        {"name": "embed 16763 of 10475x128 f32 train", "op": "embed", "rows": 16763, "capacity": 335200, "V": 10475, "C": 128, "dtype": "f32", "stride": 2, "train": True},
        # a training batch over a large vocabulary, frequent tokens first (Zipf), some padding
        {"name": "embed 65536 of 131072x1024 bf16 train", "op": "embed", "rows": 65536, "capacity": 65536, "V": 131072, "C": 1024, "dtype": "bf16", "stride": 1, "train": True},
        # a few odd rows quantised
        {"name": "quant 33x1000 f32", "op": "quant", "rows": 33, "capacity": 40, "K": 1000, "dtype": "f32"},
        # the activations of a large batch quantised
        {"name": "quant 16384x8192 bf16", "op": "quant", "rows": 16384, "capacity": 16384, "K": 8192, "dtype": "bf16"},
        # one token of a decoding step through a linear layer: the weight is read once
        {"name": "linear 1x8192x8192 bf16 serve", "op": "linear", "rows": 1, "capacity": 1, "K": 8192, "N": 8192, "dtype": "bf16", "act": "none"},
        # a small ragged batch
        {"name": "linear 37x2000x1001 f32", "op": "linear", "rows": 37, "capacity": 64, "K": 2000, "N": 1001, "dtype": "f32", "act": "relu"},
        # the compact rows of the 10475-vertex layer (9 taps of 128 channels wide) into 128 channels
        {"name": "linear 16763x1152x128 bf16", "op": "linear", "rows": 16763, "capacity": 335200, "K": 1152, "N": 128, "dtype": "bf16", "act": "elu"},
        # a large batch of tokens
        {"name": "linear 16384x8192x8192 bf16", "op": "linear", "rows": 16384, "capacity": 16384, "K": 8192, "N": 8192, "dtype": "bf16", "act": "none"},
    ]


def draw(rng):
    """One case of the same ranges: rows from one to the largest batch, widths
    over their logarithm (half of them rounded to 8, the others left odd or even)."""
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def width(lo, hi):
        c = log(lo, hi)
        return max(lo, c // 8 * 8) if rng.random() < 0.5 else c

    op = rng.choice(("norm", "embed", "quant", "linear"))
    dtype = rng.choice(("bf16", "f32"))
    rows = log(1, 65536)
    slack = rng.choice((0, 0, rng.randrange(0, 3 * rows + 2)))
    if op == "norm":
        C = width(8, 8192)
        rows = min(rows, max(1, (1 << 26) // C))
        return {"op": op, "rows": rows, "capacity": rows + slack, "C": C, "dtype": dtype, "train": rng.random() < 0.75}
    if op == "embed":
        C = width(8, 4096)
        V = min(log(16, 131072), max(16, (1 << 27) // C))
        rows = min(rows, max(1, (1 << 26) // C))
        return {"op": op, "rows": rows, "capacity": rows + slack, "V": V, "C": C, "dtype": dtype, "stride": rng.choice((1, 2)), "train": rng.random() < 0.75}
    K = width(16, 8192)
    rows = min(rows, 16384)
    slack = min(slack, rows)
    if op == "quant":
        return {"op": op, "rows": rows, "capacity": rows + slack, "K": K, "dtype": dtype}
    return {"op": op, "rows": rows, "capacity": rows + slack, "K": K, "N": width(16, 8192), "dtype": dtype, "act": rng.choice(("none", "elu", "relu"))}


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _pitch(k):
    return (k + 15) // 16 * 16


def _activations(g, capacity, C, dtype):
    """Rows of a residual stream: a level and a size of its own for each row,
    and channels of unequal size, a few of them outliers."""
    x = torch.randn(capacity, C, generator=g, device="cuda")
    ch = torch.exp(0.5 * torch.randn(C, generator=g, device="cuda"))
    ch = torch.where(torch.rand(C, generator=g, device="cuda") < 0.01, 8 * ch, ch)
    row = torch.exp(0.3 * torch.randn(capacity, 1, generator=g, device="cuda"))
    x.mul_(ch).add_(0.25 * torch.randn(capacity, 1, generator=g, device="cuda")).mul_(row)
    return x.to(dtype)


def _ids(g, rows, capacity, V, stride):
    """Token ids drawn with p(rank) ~ 1/rank, ranks in a random order of the
    table's rows, one in fifty a padding entry (-1)."""
    u = torch.rand(capacity, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
    ids = torch.randperm(V, generator=g, device="cuda")[rank].int()
    ids[torch.rand(capacity, generator=g, device="cuda") < 0.02] = -1
    if stride == 1:
        return ids
    pairs = torch.randint(0, 32, (capacity, stride), generator=g, device="cuda", dtype=torch.int32)
    pairs[:, stride - 1] = ids
    return pairs[:, stride - 1]


def _weight(g, K, N):
    """Weights as laid out once: e4m3 [N, pitch], zero beyond K, and a scale for each 128 x 128 block."""
    P, nk, nn = _pitch(K), _blocks(K), _blocks(N)
    w = torch.zeros(nn * BLOCK, nk * BLOCK, device="cuda")
    w[:N, :K] = torch.randn(N, K, generator=g, device="cuda") * (K ** -0.5)
    b = w.view(nn, BLOCK, nk, BLOCK)
    ws = (b.abs().amax(dim=(1, 3)) / E4M3_MAX).clamp_min(TINY)
    q = (b / ws[:, None, :, None]).view(nn * BLOCK, nk * BLOCK)[:N, :P].to(torch.float8_e4m3fn)
    return q.contiguous(), ws.contiguous()


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, rows, cap = DT[c["dtype"]], c["rows"], c["capacity"]
    s = {"c": c, "count": torch.tensor([rows], dtype=torch.int32, device="cuda")}
    f32 = dict(dtype=torch.float32, device="cuda")
    if c["op"] == "norm":
        C = c["C"]
        s["x"] = _activations(g, cap, C, dt)
        s["gamma"] = 1 + 0.2 * torch.randn(C, generator=g, device="cuda")
        s["beta"] = 0.1 * torch.randn(C, generator=g, device="cuda")
        s["y"] = torch.empty(cap, C, dtype=dt, device="cuda")
        s["mean"], s["rstd"] = torch.empty(cap, **f32), torch.empty(cap, **f32)
        if c["train"]:
            s["dy"] = torch.randn(cap, C, generator=g, device="cuda").to(dt)
            s["dx"] = torch.empty(cap, C, dtype=dt, device="cuda")
            s["dgamma"], s["dbeta"] = torch.empty(C, **f32), torch.empty(C, **f32)
    elif c["op"] == "embed":
        V, C = c["V"], c["C"]
        s["scale"] = math.sqrt(C)
        s["table"] = (torch.randn(V, C, generator=g, device="cuda") * 0.02).to(dt)
        s["ids"] = _ids(g, rows, cap, V, c["stride"])
        s["y"] = torch.empty(cap, C, dtype=dt, device="cuda")
        if c["train"]:
            s["dy"] = torch.randn(cap, C, generator=g, device="cuda").to(dt)
            s["row_ptr"] = torch.empty(V + 1, dtype=torch.int32, device="cuda")
            s["order"] = torch.empty(cap, dtype=torch.int32, device="cuda")
            s["dtable"] = torch.empty(V, C, **f32)
    else:
        K = c["K"]
        s["x"] = _activations(g, cap, K, dt)
        s["q"] = torch.empty(cap, _pitch(K), dtype=torch.float8_e4m3fn, device="cuda")
        s["scales"] = torch.empty(_blocks(K), cap, **f32)
        if c["op"] == "linear":
            s["wq"], s["ws"] = _weight(g, K, c["N"])
            s["bias"] = 0.1 * torch.randn(c["N"], generator=g, device="cuda")
            s["y"] = torch.empty(cap, c["N"], dtype=dt, device="cuda")
    return s


def _quantise(x):
    """x [n, K] fp32 -> e4m3 values [n, pitch] (zero beyond K) and scales [blocks, n]."""
    n, K = x.shape
    b = torch.nn.functional.pad(x, (0, _blocks(K) * BLOCK - K)).view(n, _blocks(K), BLOCK)
    top = b.abs().amax(dim=2)
    # a quotient of two tensors: torch multiplies by the reciprocal of a Python
    # scalar, and a scale one bit off moves the values that lie on a tie
    s = (top / torch.full_like(top, E4M3_MAX)).clamp_min(TINY)
    q = (b / s[:, :, None]).to(torch.float8_e4m3fn).view(n, -1)[:, :_pitch(K)]
    return q.contiguous(), s.t().contiguous()


def _act(z, act):
    if act == "elu":
        return torch.where(z > 0, z, torch.expm1(z.clamp_max(0)))
    return z.clamp_min(0) if act == "relu" else z


def _run_plain(s):
    c = s["c"]
    dt, n = DT[c["dtype"]], c["rows"]
    if c["op"] == "norm":
        x = s["x"][:n].float()
        mean = x.mean(1)
        xc = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((xc * xc).mean(1) + 1e-5)
        xh = xc * rstd[:, None]
        out = {"y": (xh * s["gamma"] + s["beta"]).to(dt), "mean": mean, "rstd": rstd}
        if c["train"]:
            dy = s["dy"][:n].float()
            t = dy * s["gamma"]
            dx = (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True)) * rstd[:, None]
            out.update(dx=dx.to(dt), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))
        return out
    if c["op"] == "embed":
        ids = s["ids"][:n].long()
        there = (ids >= 0)[:, None]
        rows = s["table"].index_select(0, ids.clamp_min(0)).float()
        out = {"y": torch.where(there, rows * s["scale"], 0.0).to(dt)}
        if c["train"]:
            dy = torch.where(there, s["dy"][:n].float(), 0.0)
            d = torch.zeros(c["V"], c["C"], device=dy.device).index_add_(0, ids.clamp_min(0), dy)
            out["dtable"] = d * s["scale"]
        return out
    q, sc = _quantise(s["x"][:n].float())
    if c["op"] == "quant":
        return {"q": q, "scales": sc}
    K = q.shape[1]
    xd = q.float() * sc.t().repeat_interleave(BLOCK, 1)[:, :K]
    wd = s["wq"].float() * s["ws"].repeat_interleave(BLOCK, 0)[:c["N"]].repeat_interleave(BLOCK, 1)[:, :K]
    return {"y": _act(xd @ wd.t() + s["bias"], c["act"]).to(dt)}


def _run_own(s):
    from paper_2608_09388_gb300 import hc
    c = s["c"]
    n, count = c["rows"], s["count"]
    if c["op"] == "norm":
        hc.hc_layer_norm_fwd(s["x"], 1e-5, s["gamma"], s["beta"], s["y"], mean=s["mean"], rstd=s["rstd"], count=count)
        out = {"y": s["y"][:n], "mean": s["mean"][:n], "rstd": s["rstd"][:n]}
        if c["train"]:
            hc.hc_layer_norm_bwd(s["x"], s["dy"], s["gamma"], s["mean"], s["rstd"], dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"], count=count)
            out.update(dx=s["dx"][:n], dgamma=s["dgamma"], dbeta=s["dbeta"])
        return out
    if c["op"] == "embed":
        hc.hc_embedding_fwd(s["table"], s["ids"], s["scale"], s["y"], count=count)
        out = {"y": s["y"][:n]}
        if c["train"]:
            hc.hc_embedding_sort(s["ids"], c["V"], s["row_ptr"], s["order"], count=count)
            hc.hc_embedding_bwd(s["dy"], s["row_ptr"], s["order"], s["scale"], s["dtable"])
            out["dtable"] = s["dtable"]
        return out
    hc.hc_quantize_fp8_rows(s["x"], s["q"], s["scales"], count=count)
    if c["op"] == "quant":
        return {"q": s["q"][:n], "scales": s["scales"][:, :n]}
    act = {"none": hc.HC_ACT_NONE, "elu": hc.HC_ACT_ELU, "relu": hc.HC_ACT_RELU}[c["act"]]
    hc.hc_fp8_linear_fwd(s["q"], s["scales"], s["wq"], s["ws"], s["bias"], act, s["y"], count=count)
    return {"y": s["y"][:n]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def exact(case, seed):
    """The definitions in 64 bits. An e4m3 value has none: it is rounded from
    x / scale by its definition, so only the scales are given."""
    s = prepare(case, seed)
    c, n = s["c"], case["rows"]
    d = torch.float64
    if c["op"] == "norm":
        x = s["x"][:n].to(d)
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        rstd = torch.rsqrt(var + 1e-5)
        xh = (x - mean) * rstd
        out = {"y": torch.addcmul(s["beta"].to(d), xh, s["gamma"].to(d)), "mean": mean[:, 0], "rstd": rstd[:, 0]}
        if c["train"]:
            dy = s["dy"][:n].to(d)
            w, C = s["gamma"].to(d), c["C"]
            out["dx"] = rstd / C * (C * dy * w - (dy @ w)[:, None] - xh * torch.einsum("nc,nc,c->n", dy, xh, w)[:, None])
            out["dgamma"], out["dbeta"] = torch.einsum("nc,nc->c", dy, xh), dy.sum(0)
        return out
    if c["op"] == "embed":
        ids = s["ids"][:n].long()
        at = torch.nonzero(ids >= 0)[:, 0]
        y = torch.zeros(n, c["C"], dtype=d, device="cuda")
        y[at] = s["table"].to(d)[ids[at]] * s["scale"]
        out = {"y": y}
        if c["train"]:
            g = torch.zeros(c["V"], c["C"], dtype=d, device="cuda")
            g.index_put_((ids[at],), s["dy"][at].to(d) * s["scale"], accumulate=True)
            out["dtable"] = g
        return out
    x = s["x"][:n].to(d)
    sc = torch.stack([p.abs().amax(1) for p in x.split(BLOCK, 1)]) / E4M3_MAX
    sc = sc.clamp_min(TINY)
    if c["op"] == "quant":
        return {"q": None, "scales": sc}
    # the scale that is kept is the fp32 one, and the e4m3 value is rounded from the fp32 quotient
    s32 = sc.float().to(d)
    y = s["bias"].to(d).expand(n, -1).clone()
    for k, p in enumerate(x.split(BLOCK, 1)):
        q = (p / s32[k][:, None]).float().to(torch.float8_e4m3fn).to(d) * s32[k][:, None]
        w = s["wq"][:, k * BLOCK:k * BLOCK + p.shape[1]].to(d)
        w = w * s["ws"][:, k].to(d).repeat_interleave(BLOCK)[:c["N"], None]
        y.addmm_(q, w.t())
    if c["act"] == "elu":
        y = torch.nn.functional.elu(y)
    elif c["act"] == "relu":
        y = torch.relu(y)
    return {"y": y}


def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    n = c["rows"]
    if c["op"] == "norm":
        C = c["C"]
        b, f = 2 * n * C * e + 8 * n + 8 * C, 8.0 * n * C       # x, y; mean, rstd; gamma, beta
        if c["train"]:
            b, f = b + 3 * n * C * e + 8 * n + 12 * C, f + 14.0 * n * C  # x, dy, dx; mean, rstd; gamma, dgamma, dbeta
        return {"bytes": b, "flops": f}
    if c["op"] == "embed":
        V, C = c["V"], c["C"]
        # distinct rows met by n draws of p(rank) = ln(1 + 1/rank) / ln(V + 1)
        step = max(1, V // 4096)
        met = sum(min(step, V - r) * (1 - (1 - math.log1p(1 / (r + 1 + step // 2)) / math.log(V + 1)) ** n) for r in range(0, V, step))
        b, f = min(n, met) * C * e + n * C * e + 4 * n, 1.0 * n * C    # the rows met, y, ids
        if c["train"]:
            b, f = b + n * C * e + 4 * n + V * C * 4, f + 1.0 * n * C  # dy, ids, dtable
        return {"bytes": b, "flops": f}
    K = c["K"]
    if c["op"] == "quant":
        return {"bytes": n * K * e + n * _pitch(K) + 4 * n * _blocks(K), "flops": 3.0 * n * K}
    N = c["N"]
    return {"bytes": n * K * e + N * _pitch(K) + 4 * _blocks(N) * _blocks(K) + 4 * N + n * N * e, "flops": 2.0 * n * K * N}
