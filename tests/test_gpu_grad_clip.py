"""The norm over a list of tensors and the clipping by it, against 64-bit sums.

Tolerances. U = 2^-24. A thread sums up to 32 squares in two chains of 16 and
adds the two: 17 U of a sum of positive numbers. Their sums are kept in a pair of
fp32 numbers whose lower one takes at most 2^-24 of the upper one a step and
rounds it to 2^-24 of that; for the up to 2^12 steps of a thread here that is
below U. Then 64 bits, a square root and one rounding: the norm is off by at most
(17 + 1) U / 2 + U = 10 U of itself. The scale is a quotient of it (1 U more),
an output one product (1 U) and its rounding."""
import math

import pytest

from paper_2608_09388_gb300 import hc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from _tokens import BF, D64, F, U, full, gen, randn, rounding, shifted, within  # noqa: E402


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


def norm_ref(ts):
    return math.sqrt(sum(float((t.to(D64) ** 2).sum()) for t in ts))


def check(grads, outs, norm, max_norm, before=None):
    ref = norm_ref(before or grads)
    assert abs(float(norm) - ref) <= 10 * U * ref
    scale = 1.0 if float(norm) <= max_norm else max_norm / ref
    for i, (g, o) in enumerate(zip(before or grads, outs)):
        want = g.to(D64) * scale
        within(o, want, 0 if scale == 1 else 13 * U * want.abs() + rounding(g.dtype, want), i)


# one element, pieces that are not full, the border of a unit and of the units
# a block loads together, more units than blocks
SIZES = [[1], [0, 3], [7, 8, 9], [4095, 4096, 4097], [8191, 8192, 8193], [16384, 16385, 1, 65536],
         [1000] * 300, [37, 4100] * 400, [3000000, 5, 0, 70001], [12345678]]


@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES)
def test_norm_and_clip(sizes, kind):
    g = gen(len(sizes) + sizes[0])
    types = {"f32": [F], "bf16": [BF], "mixed": [F, BF]}[kind]
    grads = [randn(g, n, dtype=types[i % len(types)]) for i, n in enumerate(sizes)]
    outs = [full((n,), t.dtype) for n, t in zip(sizes, grads)]
    lst = hc.hc_tensor_list(grads, outs)
    norm = full((1,))
    hc.hc_grad_norm(lst, norm)
    ref = norm_ref(grads)
    for max_norm in (0.7 * ref, 1.3 * ref):
        for o in outs:
            o.fill_(77)
        hc.hc_grad_clip(lst, norm, max_norm)
        check(grads, outs, norm, max_norm)
    again = full((1,))
    hc.hc_grad_norm(lst, again)
    assert torch.equal(again, norm)
    # in place: the same bits, and untouched where the norm is not above
    want = [o.clone() for o in outs]
    here = [t.clone() for t in grads]
    inp = hc.hc_tensor_list(here)
    hc.hc_grad_clip(inp, norm, 1.3 * ref)
    assert all(torch.equal(a, b) for a, b in zip(here, grads))
    hc.hc_grad_clip(lst, norm, 0.3 * ref)
    hc.hc_grad_clip(inp, norm, 0.3 * ref)
    assert all(torch.equal(a, b) for a, b in zip(here, outs)) and len(want) == len(here)


@pytest.mark.parametrize("dtype", [F, BF])
def test_neighbours_and_alignment(dtype):
    """Tensors one after another in one buffer, at every alignment, into outputs
    of other alignments: what lies between and around them stays."""
    g = gen(3)
    sizes = [1, 2, 3, 5, 8, 13, 4095, 4099, 8190, 31, 1, 1]
    total = sum(sizes) + len(sizes) + 9
    src, dst = randn(g, total, dtype=dtype), full((total + 3,), dtype)
    keep = src.clone()
    grads, outs, spans, at = [], [], [], 1
    for n in sizes:
        grads.append(src[at:at + n])
        outs.append(dst[at + 2:at + 2 + n])
        spans.append((at + 2, n))
        at += n + (1 if n % 2 else 0)
    lst = hc.hc_tensor_list(grads, outs)
    norm = full((1,))
    hc.hc_grad_norm(lst, norm)
    hc.hc_grad_clip(lst, norm, 1.0)
    check(grads, outs, norm, 1.0)
    assert torch.equal(src, keep)
    mine = torch.zeros(total + 3, dtype=torch.bool, device="cuda")
    for a, n in spans:
        mine[a:a + n] = True
    assert (dst[~mine] == 77).all()
    before = [t.clone() for t in grads]
    hc.hc_grad_clip(hc.hc_tensor_list(grads), norm, 1.0)
    assert all(torch.equal(a, b) for a, b in zip(grads, outs)) and len(before) == len(outs)
    gap = torch.ones(total, dtype=torch.bool, device="cuda")
    for a, n in spans:
        gap[a - 2:a - 2 + n] = False
    assert torch.equal(src[gap], keep[gap])


def clip_of(ts, max_norm):
    outs = [torch.full_like(t, 77) for t in ts]
    lst, norm = hc.hc_tensor_list(ts, outs), full((1,))
    hc.hc_grad_norm(lst, norm)
    hc.hc_grad_clip(lst, norm, max_norm)
    return norm, outs


def test_values():
    g = gen(5)
    a, b = randn(g, 5000), randn(g, 70000, dtype=BF)
    # squares above the range of fp32
    big = [a * 2.0 ** 100, (b.float() * 2.0 ** 90).to(BF)]
    norm, outs = clip_of(big, 1.0)
    check(big, outs, norm, 1.0)
    # zeros, no elements, no tensors: norm 0, outputs as the inputs
    for ts in ([torch.zeros(5000, device="cuda")], [a[:0]], []):
        norm, outs = clip_of(ts, 0.0)
        assert norm.item() == 0 and all(torch.equal(o, t) for o, t in zip(outs, ts))
    # an infinity, a NaN
    c = a.clone()
    c[4321] = float("-inf")
    norm, outs = clip_of([c, b], 1.0)
    assert norm.item() == math.inf and outs[0][4321].isnan() and int(outs[0].isnan().sum()) == 1
    assert (outs[0].nan_to_num() == 0).all() and (outs[1] == 0).all()
    c[17] = float("nan")
    norm, outs = clip_of([c, b], 1.0)
    assert norm.isnan() and outs[0].isnan().all() and outs[1].isnan().all()
    # exact sums: the norm exactly at the border is not clipped
    d = torch.full((4096, 4), 2.0, device="cuda")
    norm, outs = clip_of([d], 256.0)
    assert norm.item() == 256 and torch.equal(outs[0], d)
    norm, outs = clip_of([d], 64.0)
    assert (outs[0] == 0.5).all()
    norm, outs = clip_of([a], 0.0)
    assert (outs[0] == 0).all()
    norm, outs = clip_of([a], math.inf)
    assert torch.equal(outs[0], a)


@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("size", [2e17, 1e18, 4e18, 5e18, 6.5e18, 1.2e19])
def test_running_sums_past_fp32(size, kind):
    """20 M values whose squares fit fp32, as a thread's sum over a unit does at all
    sizes but the largest (for bf16 the three largest), while its sum over all its
    units does not from 4e18 on."""
    g = gen(11)
    n = {"f32": (20000001, 0), "bf16": (0, 20000001), "mixed": (7000003, 13000001)}[kind]
    ts = [size * (0.9 + 0.1 * torch.rand(k, generator=g, device="cuda")) for k in n]
    ts = [ts[0], ts[1].to(BF)]
    norm, outs = clip_of(ts, 1.0)
    assert norm.isfinite()
    check(ts, outs, norm, 1.0)
    # small ones before and behind the large ones still count
    ones = [torch.full((50000,), size / 1024, device="cuda") for _ in range(2)]
    norm, outs = clip_of([ones[0], *ts, ones[1]], 1.0)
    check([ones[0], *ts, ones[1]], outs, norm, 1.0)


def test_long_sum():
    """2^28 equal values: a plain fp32 chain would stop growing."""
    t = torch.full((2 ** 28,), 0.1, device="cuda")
    norm = full((1,))
    hc.hc_grad_norm(hc.hc_tensor_list([t]), norm)
    ref = math.sqrt(2 ** 28 * float(t[0]) ** 2)
    assert abs(norm.item() - ref) <= 10 * U * ref


def test_stream_graph_and_shapes():
    """Another stream, a captured pass replayed on other gradients, two lists
    at a time on two streams, tensors of several dimensions."""
    g = gen(7)
    sets = [[randn(g, 300, 70), randn(g, 64, 3, 3, 3, dtype=BF), randn(g, 1)] for _ in range(2)]
    outs = [[torch.full_like(t, 77) for t in s] for s in sets]
    lists = [hc.hc_tensor_list(s, o) for s, o in zip(sets, outs)]
    norms = [full((1,)) for _ in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(50):
        for l, n, s in zip(lists, norms, streams):
            hc.hc_grad_norm(l, n, stream=s)
            hc.hc_grad_clip(l, n, 1.0, stream=s)
    torch.cuda.synchronize()
    for s, o, n in zip(sets, outs, norms):
        check(s, o, n, 1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        hc.hc_grad_norm(lists[0], norms[0], stream=streams[0])
        hc.hc_grad_clip(lists[0], norms[0], 1.0, stream=streams[0])
    for by in (3.0, 1e-3):
        for t in sets[0]:
            t.mul_(by)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(sets[0], outs[0], norms[0], 1.0)
    assert shifted(sets[0][0]).shape == sets[0][0].shape


@pytest.mark.parametrize("given", [True, False])
def test_list_dropped_while_another_stream_uses_it(given):
    """A list that goes right behind its calls on another stream than the one it was
    made on: its table's memory goes to nobody before they have run."""
    g = gen(13)
    grads = [randn(g, 300), randn(g, 5000, dtype=BF)]
    outs = [torch.full_like(t, 77) for t in grads]
    norm, side = full((1,)), torch.cuda.Stream()
    # the stream's workspace and the kernels are there: making them would wait
    first = hc.hc_tensor_list(grads, outs)
    hc.hc_grad_norm(first, norm, stream=side)
    hc.hc_grad_clip(first, norm, 1.0, stream=side)
    lst = hc.hc_tensor_list(grads, outs)
    at, size = lst.memory.data_ptr(), lst.memory.numel()
    torch.cuda.synchronize()
    if given:
        with torch.cuda.stream(side):
            torch.cuda._sleep(400_000_000)  # about 0.2 s
        hc.hc_grad_norm(lst, norm, stream=side)
        hc.hc_grad_clip(lst, norm, 1.0, stream=side)
    else:
        with torch.cuda.stream(side):
            torch.cuda._sleep(400_000_000)
            hc.hc_grad_norm(lst, norm)
            hc.hc_grad_clip(lst, norm, 1.0)
    del lst
    new = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(64)]
    assert not side.query()  # still asleep: nothing below is late
    assert all(t.data_ptr() + size <= at or at + size <= t.data_ptr() for t in new)
    torch.cuda.synchronize()
    check(grads, outs, norm, 1.0)


@pytest.mark.parametrize("dtype", [F, BF])
def test_clips_one_after_another(dtype):
    """Each call writes the outputs anew from the gradients, which stay; in place it
    goes on from what it left; rows that start one past 16 bytes in and out."""
    g = gen(17)
    grads = [randn(g, 300, 70, dtype=dtype), randn(g, 4097, dtype=dtype), shifted(randn(g, 211, 3, dtype=dtype))]
    keep = [t.clone() for t in grads]
    outs = [shifted(torch.zeros_like(t)) for t in grads]
    lst, norm = hc.hc_tensor_list(grads, outs), full((1,))
    hc.hc_grad_norm(lst, norm)
    ref = norm_ref(grads)
    done = []
    for part in (0.5, 2.0, 0.25):
        hc.hc_grad_clip(lst, norm, part * ref)
        check(grads, outs, norm, part * ref)
        done.append([o.clone() for o in outs])
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    assert all(torch.equal(a, b) for a, b in zip(done[1], keep))
    assert not any(torch.equal(a, b) for a, b in zip(done[0], done[2]))
    inp = hc.hc_tensor_list(grads)
    hc.hc_grad_clip(inp, norm, 0.5 * ref)
    check(grads, grads, norm, 0.5 * ref, before=keep)
    assert all(torch.equal(a, b) for a, b in zip(grads, done[0]))
    hc.hc_grad_clip(inp, norm, 0.5 * ref)  # the norm given is the same: halved once more
    for t, d in zip(grads, done[0]):
        want = d.to(D64) / 2
        within(t, want, 13 * U * want.abs() + rounding(dtype, want), "halved twice")


def test_other_device_is_refused():
    lst = hc.hc_tensor_list([torch.zeros(3, device="cuda")])
    lst.device += 1
    with pytest.raises(ValueError):
        hc.hc_grad_norm(lst, full((1,)))
