"""How the projections are called: on other streams, two at once, in graphs that are replayed, and what the binding refuses."""
import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M
from test_gpu_proj import CODES, FREQ, randn

pytestmark = pytest.mark.gpu


class Calls:
    """All of the calls on one set of tensors, `rows` of 640 columns: fill() puts new inputs in, run() makes the calls, outs() are their results."""

    def __init__(self, rows, dtype=torch.bfloat16, seed=0):
        new = lambda *shape, dtype=dtype: torch.empty(shape, dtype=dtype, device="cuda")
        self.rows, self.seed = rows, seed
        self.x, self.add, self.gu, self.weight = new(rows, 640), new(rows, 640), new(rows, 1280), randn(640, seed=9, dtype=dtype).cuda()
        self.res, self.out, self.y = new(rows, 640), new(rows, 640), new(rows, 900)
        (self.c, self.s), (self.cg, self.sg), (self.cq, self.sq) = (fkv.empty_quant(rows, 640) for _ in range(3))
        self.w, self.ws = fkv.empty_quant(900, 640, tile=128)
        fkv.proj_quant(randn(900, 640, seed=8, dtype=dtype).cuda(), self.w, self.ws, tile=128)
        self.positions, self.freq = new(2, rows, dtype=torch.int32), FREQ.cuda()
        self.q, self.k, self.v = (new(rows, n, 128) for n in (3, 1, 1))
        torch.cuda.synchronize()

    def fill(self, seed):
        for i, t in enumerate((self.x, self.add, self.gu)):
            t.copy_(randn(*t.shape, seed=seed + i, dtype=t.dtype))
        self.positions.copy_(torch.randint(0, 9999, self.positions.shape, generator=torch.Generator().manual_seed(seed), dtype=torch.int32))

    def run(self, stream=None):
        fkv.proj_norm(self.x, self.weight, self.c, self.s, add=self.add, res=self.res, out=self.out, stream=stream)
        fkv.proj_matmul(self.c, self.s, self.w, self.ws, self.y, stream=stream)
        fkv.proj_gate(self.gu, self.cg, self.sg, stream=stream)
        fkv.proj_quant(self.out, self.cq, self.sq, stream=stream)
        fkv.proj_rope(self.res.view(self.rows, 5, 128), self.positions, self.freq, self.q, self.k, self.v, sections=(20, 44), stream=stream)

    def outs(self):
        return [t.float() for t in (self.res, self.out, self.c, self.s, self.y, self.cg, self.sg, self.cq, self.sq, self.q, self.k, self.v)]

    def clear(self):
        for t in (self.res, self.out, self.s, self.y, self.sg, self.sq, self.q, self.k, self.v):
            t.zero_()
        for t in (self.c, self.cg, self.cq):
            t.view(torch.uint8).zero_()


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("rows", [1, 30, 70, 500])
def test_replays_go_by_what_is_there(rows):
    """One graph of all calls, replayed on other inputs, with eager calls of the same and synchronizations between."""
    captured, eager = Calls(rows), Calls(rows)
    captured.fill(0)
    captured.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for seed in range(4):
        captured.fill(10 * seed), eager.fill(10 * seed)
        captured.clear()
        graph.replay()
        if seed % 2:
            torch.cuda.synchronize()
        eager.run()
        torch.cuda.synchronize()
        assert same(captured.outs(), eager.outs()), seed


def test_two_graphs_at_once():
    """The calls keep nothing: two graphs of them run beside each other, on streams of their own, workspaces of products among it."""
    a, b, plain = Calls(120), Calls(300), (Calls(120), Calls(300))
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for calls, seed in ((a, 1), (b, 2)):
        calls.fill(seed)
        calls.run()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls.run()
        graphs.append(g)
    for c, seed in zip(plain, (1, 2)):
        c.fill(seed)
        c.run()
    torch.cuda.synchronize()
    for _ in range(20):
        a.clear(), b.clear()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert same(a.outs(), plain[0].outs()) and same(b.outs(), plain[1].outs())


@pytest.mark.parametrize("named", [False, True])
def test_on_the_stream_that_is_asked_for(named):
    """Inputs arrive late on another stream, and the calls behind them there; the current stream goes on meanwhile."""
    late, plain = Calls(200), Calls(200)
    plain.fill(3)
    plain.run()
    side, ballast = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    x, add, gu, positions = (t.clone() for t in (plain.x, plain.add, plain.gu, plain.positions))
    late.fill(50)
    late.clear()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            ballast @ ballast
        for t, f in ((late.x, x), (late.add, add), (late.gu, gu), (late.positions, positions)):
            t.copy_(f)
        if not named:
            late.run()
    if named:
        late.run(stream=side)
    side.synchronize()
    assert same(late.outs(), plain.outs())


def test_two_streams_at_once():
    calls, plain = [Calls(n) for n in (33, 260, 1000)], [Calls(n) for n in (33, 260, 1000)]
    streams = [torch.cuda.Stream() for _ in calls]
    for i, (c, p) in enumerate(zip(calls, plain)):
        c.fill(i), p.fill(i)
        p.run()
    torch.cuda.synchronize()
    for _ in range(10):
        for c, s in zip(calls, streams):
            c.run(stream=s)
    torch.cuda.synchronize()
    for c, p in zip(calls, plain):
        assert same(c.outs(), p.outs())


def test_a_workspace_of_the_callers():
    """The entry point itself: as many bytes as it asks for, used twice, by another product in between; fewer are refused."""
    import ctypes as C
    L, need = fkv.lib(), C.c_size_t()
    rows, n, cols = 200, 512, 8192
    ops = M.quant(randn(rows, cols, seed=1).double()) + M.quant(randn(n, cols, seed=2).double(), 128)
    x, xs, w, ws = (t.float().to(CODES).cuda() if i % 2 == 0 else t.cuda() for i, t in enumerate(ops))
    assert L.fkv_proj_workspace(rows, n, cols, C.byref(need)) == 0 and need.value > 0
    work = torch.full((need.value + 256,), 77, dtype=torch.uint8, device="cuda")
    out, want = (torch.empty((rows, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fkv.proj_matmul(x, xs, w, ws, want)
    call = lambda size, t=x: L.fkv_proj_matmul(0, 1, t.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), rows, n, cols, out.data_ptr(), work.data_ptr(), size,
                                                 torch.cuda.current_stream().cuda_stream)
    assert call(need.value - 1) == -4
    for _ in range(3):
        assert call(need.value) == 0
        torch.cuda.synchronize()
        assert torch.equal(out, want) and (work[need.value:] == 77).all()
        work[:need.value].random_()


def test_what_the_binding_refuses():
    t = Calls(8)
    big = torch.empty((8, 1300), dtype=torch.bfloat16, device="cuda")
    odd = torch.empty((8 * 640 + 4,), dtype=torch.bfloat16, device="cuda")[4:].view(8, 640)             # (8 bytes behind an aligned place)
    bad = [
        (lambda: fkv.proj_quant(t.x.cpu(), t.c, t.s), "GPU"), (lambda: fkv.proj_quant(t.x, t.c.cpu(), t.s), "codes"), (lambda: fkv.proj_quant(t.x, t.c, t.s.cpu()), "scales"),
        (lambda: fkv.proj_quant(t.x.float(), t.c, t.s), "x:"), (lambda: fkv.proj_quant(big[:, :640], t.c, t.s), "contiguous"), (lambda: fkv.proj_quant(t.x, t.s, t.c), "codes"),
        (lambda: fkv.proj_quant(t.x, t.c, t.s, tile=64), "tile"), (lambda: fkv.proj_quant(t.x, t.c, t.s[:1], tile=1), "scales"), (lambda: fkv.proj_quant(odd, t.c, t.s), "aligned"),
        (lambda: fkv.proj_quant(big[:, :8].contiguous(), *fkv.empty_quant(8, 8)), "cols"),
        (lambda: fkv.proj_norm(t.x, t.weight[:639], t.c, t.s), "weight"), (lambda: fkv.proj_norm(t.x, t.weight.half(), t.c, t.s), "weight"), (lambda: fkv.proj_norm(t.x, t.weight), "wanted"),
        (lambda: fkv.proj_norm(t.x, t.weight, t.c), "wanted"), (lambda: fkv.proj_norm(t.x, t.weight, t.c, t.s, res=t.res), "res"), (lambda: fkv.proj_norm(t.x, t.weight, t.c, t.s, eps=0.0), "eps"),
        (lambda: fkv.proj_norm(t.x, t.weight, t.c, t.s, add=t.add[:7]), "add"), (lambda: fkv.proj_norm(t.x, t.weight, t.c, t.s, add=t.add, res=t.gu), "res"),
        (lambda: fkv.proj_norm(t.x, t.weight, t.c, t.s, out=t.y), "out"),
        (lambda: fkv.proj_gate(t.gu[:, :1279].contiguous(), t.cg, t.sg), "gu"), (lambda: fkv.proj_gate(t.x, t.cg, t.sg), "codes"), (lambda: fkv.proj_gate(t.gu[0], t.cg, t.sg), "gu"),
        (lambda: fkv.proj_matmul(t.c, t.s, t.w, t.ws[:7], t.y), "w_scales"), (lambda: fkv.proj_matmul(t.c, t.s, t.w.T, t.ws, t.y), "w:"), (lambda: fkv.proj_matmul(t.c, t.s, t.w, t.ws, t.y.float()), "out"),
        (lambda: fkv.proj_matmul(t.c, t.s, t.w, t.ws, t.x), "w:"), (lambda: fkv.proj_matmul(t.c.view(torch.uint8), t.s, t.w, t.ws, t.y), "codes"),
    ]
    qkv = t.res.view(8, 5, 128)
    rope = lambda **kw: fkv.proj_rope(**{**dict(qkv=qkv, positions=t.positions, freq=t.freq, q=t.q, k=t.k, v=t.v, sections=(20, 44)), **kw})
    bad += [(lambda: rope(positions=t.positions.long()), "positions"), (lambda: rope(positions=t.positions[:, :7]), "positions"), (lambda: rope(freq=t.freq.double()), "freq"),
            (lambda: rope(sections=(20, 43)), "sections"), (lambda: rope(sections=(20, 20, 24)), "sections"), (lambda: rope(q=t.k), "qkv"), (lambda: rope(v=t.q), "v:"),
            (lambda: rope(positions=torch.zeros((5, 8), dtype=torch.int32, device="cuda"), sections=None), "n_axes")]
    for i, (call, word) in enumerate(bad):
        with pytest.raises(fkv.FreeKVError, match=word):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()
