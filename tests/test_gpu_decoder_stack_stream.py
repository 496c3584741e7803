"""DecoderStack over a paged cache on a stream that is not the current one."""
import pytest
import torch

from test_gpu_paged_cache import Pair, ints

pytestmark = pytest.mark.gpu


def test_steps_on_another_stream_are_those_on_the_current_one():
    """Both streams are busy when a step begins.  The step waits for its input, positions are those of the token that is decoded, and what
    the current stream reads next is the result: bit for bit what a sibling gives that is decoded on the current stream."""
    from paper_2505_13109_amd.layer_loop import DecoderStack
    p = Pair(n_layers=2, n_kv=2, G=4, max_seqs=4, max_ctx=256, n_pages=40)
    p.grow([0, 3], [58, 9])
    p.c.fork(ints([0, 3]), ints([1, 2]))
    plain, other = (DecoderStack(p.c, seqs=ints(s), ffn_mult=1.0) for s in ([0, 3], [1, 2]))
    side = torch.cuda.Stream()
    x = torch.randn((2, plain.hidden), generator=p.gen).bfloat16().cuda()
    ballast = torch.randn((4096, 4096), device="cuda")
    a = b = x
    plain.step(x), other.step(x)                         # (the library's products choose their workspaces)
    torch.cuda.synchronize()
    for step in range(12):
        a = plain.step(a)
        torch.cuda.synchronize()
        late = b.clone() if step == 0 else b
        xin = torch.zeros_like(late)
        with torch.cuda.stream(side):
            for _ in range(3):
                ballast @ ballast
        for _ in range(step % 3):
            ballast @ ballast
        xin.copy_(late)                                  # on the current stream, behind its products
        b = other.step(xin, stream=side)
        xin.zero_()                                      # (the step has had its input by the time this runs)
        got = b.clone()
        torch.cuda.synchronize()
        assert torch.equal(a, got), step
        for layer in range(2):
            assert torch.equal(plain.out[layer], other.out[layer]), (step, layer)
    lens = ints([0] * 4)
    p.c.tables(ints([0, 1, 2, 3]), lens)
    assert lens.tolist() == [71, 71, 22, 22]
    p.c.health()


def test_a_step_captured_with_its_own_stream_goes_on():
    """The other stream joins the capture and leaves it again; replays are the eager steps."""
    from paper_2505_13109_amd.layer_loop import DecoderStack
    p = Pair(n_layers=2, n_kv=2, G=4, max_seqs=3, max_ctx=256, n_pages=40)
    p.grow([0], [58])
    p.c.fork(ints([0, 0]), ints([1, 2]))
    eager, captured, warm = (DecoderStack(p.c, seqs=ints([s]), ffn_mult=1.0) for s in (0, 1, 2))
    side, inner = torch.cuda.Stream(), torch.cuda.Stream()
    x = torch.randn((1, eager.hidden), generator=p.gen).bfloat16().cuda()
    for s in (side, inner):                              # (the library's products choose a stream's workspaces before a capture)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            warm.step(x)
    torch.cuda.synchronize()
    xin, graph = x.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        yout = captured.step(xin, stream=inner)
    a = b = x
    for step in range(8):
        a = eager.step(a)
        xin.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        b = yout.clone()
        assert torch.equal(a, b), step
    p.c.health()
