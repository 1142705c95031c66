"""The workspace that the operators of a stream share: a captured graph keeps
the one it was captured with, and threads that share a stream do not share it at one time."""
import threading

import pytest

from paper_2608_09388_gb300 import hc

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_09388_gb300 import build
    build.build()
    hc.load_library()
    assert hc.hc_get_device_status() == hc.HC_OK


class Step:
    """A sort of n ids, the gradient of an embedding with them and of a layer
    norm: three operators that keep sums in the workspace between launches."""

    def __init__(self, n, V, C, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        e = dict(device="cuda")
        self.V = V
        self.ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
        self.x, self.dy = (torch.randn(n, C, generator=g, **e) for _ in range(2))
        self.mean, self.rstd = self.x.mean(1), 1 / self.x.std(1)
        self.rp = torch.empty(V + 1, dtype=torch.int32, **e)
        self.od = torch.empty(n, dtype=torch.int32, **e)
        self.dt, self.dx = torch.empty(V, C, **e), torch.empty(n, C, **e)
        self.dg, self.db = torch.empty(C, **e), torch.empty(C, **e)

    def run(self, stream=None):
        hc.hc_embedding_sort(self.ids, self.V, self.rp, self.od, stream=stream)
        hc.hc_embedding_bwd(self.dy, self.rp, self.od, 0.5, self.dt, stream=stream)
        hc.hc_layer_norm_bwd(self.x, self.dy, None, self.mean, self.rstd, dx=self.dx,
                             dgamma=self.dg, dbeta=self.db, stream=stream)

    def outputs(self):
        return self.rp, self.od, self.dt, self.dx, self.dg, self.db

    def forget(self):
        for t in self.outputs():
            t.zero_()

    def result(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.outputs()]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_graph_after_a_larger_call():
    """A graph captured on a stream gives the same after larger calls on that
    stream have replaced the workspace, twice, and what was allocated since is
    not written by it."""
    small, large, larger = Step(9000, 70, 64, 1), Step(300000, 70, 64, 2), Step(700000, 50, 640, 3)
    side = torch.cuda.Stream()
    want = []
    for s in (small, large, larger):
        s.run()
        want.append(s.result())
        s.forget()
    torch.cuda.synchronize()
    small.run(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        small.run(side)
    for s, w in ((large, want[1]), (larger, want[2])):
        s.run(side)
        assert same(s.result(), w)
        guard = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        for _ in range(2):
            small.forget()
            torch.cuda.synchronize()
            graph.replay()
            assert same(small.result(), want[0])
        assert int(guard.count_nonzero()) == 0
    assert hc.hc_get_device_status() == hc.HC_OK


def test_threads_on_one_stream():
    """Threads that call on one stream at the same time, with sizes that need
    workspaces of different sizes: each gets its own results."""
    steps = [Step(3000, 900, 24, 4), Step(50000, 300, 64, 5), Step(120000, 2000, 40, 6),
             Step(20000, 70, 200, 7)]
    want = []
    for s in steps:
        s.run()
        want.append(s.result())
        s.forget()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    start, failed = threading.Barrier(len(steps)), []

    def work(s):
        try:
            start.wait(60)
            for _ in range(200):
                s.run(side)
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=work, args=(s,)) for s in steps]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not failed and not any(t.is_alive() for t in threads)
    for s, w in zip(steps, want):
        assert same(s.result(), w)
    assert hc.hc_get_device_status() == hc.HC_OK
