"""Products that are cut into parts of their long axis, called as programs call them: in graphs, beside each other, on other streams; the forms of the
norm that only the C entry point has; the exactness of products of 33 to 64 rows."""
import ctypes as C

import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M
from test_gpu_proj import CODES, gen, half_step, near, operands, product, randn, same_codes, sum_off

pytestmark = pytest.mark.gpu

PARTS = [(120, 900, 8192), (200, 512, 8192), (203, 1031, 11056), (70, 4096, 14336)]


class Product:
    """A product in parts on tensors of its own: fill() puts other activations in, run() makes the call."""

    def __init__(self, rows, n, cols, seed=0):
        need = C.c_size_t()
        assert fkv.lib().fkv_proj_workspace(rows, n, cols, C.byref(need)) == 0 and need.value > 0
        self.x, self.out = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, n), dtype=torch.bfloat16, device="cuda")
        (self.c, self.s), (self.w, self.ws) = fkv.empty_quant(rows, cols), fkv.empty_quant(n, cols, tile=128)
        fkv.proj_quant(randn(n, cols, seed=100, scale=cols ** -0.5, outliers=False).cuda(), self.w, self.ws, tile=128)
        self.fill(seed)

    def fill(self, seed):
        self.x.copy_(randn(*self.x.shape, seed=seed))

    def run(self, stream=None, out=None):
        fkv.proj_quant(self.x, self.c, self.s, stream=stream)
        fkv.proj_matmul(self.c, self.s, self.w, self.ws, self.out if out is None else out, stream=stream)

    def wanted(self, seed):
        """the call alone"""
        torch.cuda.synchronize()
        self.fill(seed)
        out = torch.empty_like(self.out)
        self.run(out=out)
        torch.cuda.synchronize()
        return out


def captured(run):
    graph = torch.cuda.CUDAGraph()
    run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run()
    return graph


@pytest.mark.parametrize("rows,n,cols", PARTS)
def test_replays_of_a_product_in_parts(rows, n, cols):
    a = Product(rows, n, cols)
    wants = [a.wanted(seed) for seed in range(4)]
    graph = captured(a.run)
    for seed in (2, 0, 3, 1):
        a.fill(seed)
        a.out.zero_()
        graph.replay()
        other = torch.full((1 << 22,), float(seed), device="cuda")         # (eager work, with memory of its own, between the replays)
        if seed % 2:
            torch.cuda.synchronize()
        other.mul_(2)
        torch.cuda.synchronize()
        assert torch.equal(a.out, wants[seed]), seed


def test_two_graphs_of_products_in_parts_at_once():
    """Graphs with pools of their own, and an eager call beside them, each with its own workspace."""
    a, b, c = Product(200, 512, 8192), Product(203, 1031, 11056), Product(120, 900, 8192)
    wants = [t.wanted(i) for i, t in enumerate((a, b, c))]
    graphs, streams = [captured(t.run) for t in (a, b)], [torch.cuda.Stream() for _ in range(3)]
    for _ in range(20):
        for t in (a, b, c):
            t.out.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        c.run(stream=streams[2])
        torch.cuda.synchronize()
        assert all(torch.equal(t.out, w) for t, w in zip((a, b, c), wants))


def test_products_in_parts_on_several_streams():
    calls = [Product(*size) for size in PARTS]
    wants = [t.wanted(10 + i) for i, t in enumerate(calls)]
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(10):
        for t in calls:
            t.out.zero_()
        torch.cuda.synchronize()
        for t, s in zip(calls, streams):
            t.run(stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(t.out, w) for t, w in zip(calls, wants))


@pytest.mark.parametrize("named", [False, True])
def test_a_product_in_parts_behind_late_activations(named):
    """What it reads arrives late on its stream; the current stream takes and gives back memory meanwhile."""
    a = Product(203, 1031, 11056)
    want, late = a.wanted(7), randn(203, 11056, seed=7).cuda()
    a.fill(8)
    a.out.zero_()
    side, ballast = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            ballast @ ballast
        a.x.copy_(late)
        if not named:
            a.run()
    if named:
        a.run(stream=side)
    for i in range(8):
        torch.full((1 << (16 + i),), 9.0, device="cuda")
    side.synchronize()
    assert torch.equal(a.out, want)


@pytest.mark.parametrize("rows,n,cols", PARTS)
def test_a_product_in_parts_gives_the_same_bits(rows, n, cols):
    a = Product(rows, n, cols, seed=3)
    outs = [torch.empty_like(a.out) for _ in range(6)]
    for o in outs:
        a.run(out=o)
    assert all(torch.equal(outs[0], o) for o in outs[1:])
    want, size, cut = M.matmul(a.c.cpu(), a.s.cpu(), a.w.cpu(), a.ws.cpu())
    near(outs[0], want, half_step(torch.bfloat16) * 1.01, sum_off(cols) * size + cut + 2.0 ** -25)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,n,cols", [(33, 300, 512), (47, 1031, 2064), (48, 128, 8192), (49, 17, 144), (64, 2050, 4096), (63, 8192, 128)])
def test_products_of_33_to_64_rows_are_exact_where_it_is_said(rows, n, cols, dtype):
    """n and cols to 8192: no product is cut."""
    x, xs, w, ws = operands(rows, n, cols, seed=rows + n)
    want, size, _ = M.matmul(x, xs, w, ws)
    near(product(x, xs, w, ws, dtype), want, half_step(dtype) * 1.01, sum_off(cols) * size + 2.0 ** -25)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 16), (7, 512), (3, 8192), (5, 8208), (2, 32784)])
def test_norm_of_a_sum_that_is_not_written(rows, cols, dtype):
    """add without res, which the C entry point has: x stays, the norm is that of the sum; and res as all that is written."""
    L, t = fkv.lib(), {torch.float16: 0, torch.bfloat16: 1}[dtype]
    x, add = randn(rows, cols, seed=1, dtype=dtype), randn(rows, cols, seed=2, dtype=dtype, outliers=False)
    w = (1 + 0.2 * torch.randn(cols, generator=gen(3))).to(dtype)
    s, codes_want, scales_want, y = M.norm(x, w, add)
    dx, da, dw = x.cuda(), add.cuda(), w.cuda()
    (codes, scales), out, res = fkv.empty_quant(rows, cols), torch.zeros_like(dx), torch.zeros_like(dx)
    st = torch.cuda.current_stream().cuda_stream
    p = lambda v: None if v is None else v.data_ptr()
    call = lambda res, codes, scales, out: L.fkv_proj_norm(0, t, p(dx), p(da), p(dw), rows, cols, 1e-5, p(res), p(codes), p(scales), p(out), st)
    for want_codes, want_out in ((True, True), (True, False), (False, True)):
        codes.view(torch.uint8).zero_(), scales.zero_(), out.zero_()
        assert call(None, codes if want_codes else None, scales if want_codes else None, out if want_out else None) == 0
        if want_codes:
            same_codes(codes, codes_want)
            near(scales, scales_want, 2.0 ** -24 * 1.001)
        if want_out:
            near(out, y, half_step(dtype) * 1.01 + 2.0 ** -24, 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)
        assert torch.equal(dx.cpu(), x) and torch.equal(da.cpu(), add)
    assert call(res, None, None, None) == 0
    assert torch.equal(res.cpu(), s) and torch.equal(dx.cpu(), x)
