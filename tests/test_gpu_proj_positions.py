"""Rotary positions and frequencies that lie anywhere: a step's of a tensor of all steps'."""
import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M
from test_gpu_proj import FREQ, gen, half_step, near, randn

pytestmark = pytest.mark.gpu


def turned(qkv, positions, freq, stream=None, **kw):
    q, k, v = (torch.zeros((qkv.shape[0], n, 128), dtype=qkv.dtype, device="cuda") for n in (3, 1, 1))
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    fkv.proj_rope(qkv, positions, freq, q, k, v, stream=stream, **kw)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    return q, k, v


@pytest.mark.parametrize("axes,rows", [(1, 1), (3, 1), (2, 5), (4, 33)])
def test_positions_of_one_step_of_many(axes, rows):
    steps = torch.randint(0, 5000, (6, axes, rows), generator=gen(rows), dtype=torch.int32).cuda()
    sections = {1: (64,), 2: (16, 48), 3: (16, 24, 24), 4: (16, 16, 16, 16)}[axes]
    qkv, side = randn(rows, 5, 128, seed=3), torch.cuda.Stream()
    which = [a for a, n in enumerate(sections) for _ in range(n)]
    for t in range(6):
        for stream in (None, side):
            q, k, v = turned(qkv.cuda(), steps[t], FREQ.cuda(), stream, sections=sections)
            wq, wk, wv, oq, ok = M.rope(qkv, steps[t].cpu(), FREQ, 3, 1, which)
            near(q, wq, half_step(qkv.dtype) * 1.01, oq)
            near(k, wk, half_step(qkv.dtype) * 1.01, ok)
            assert torch.equal(v.cpu().double(), wv), t


def test_frequencies_behind_others():
    tables = torch.stack((FREQ, FREQ * 0.5, FREQ * 0.25)).reshape(-1)
    many = torch.cat((torch.zeros(1), tables)).cuda()
    qkv, at = randn(7, 5, 128, seed=4), torch.arange(7, dtype=torch.int32) * 100
    for i in range(3):
        q, k, v = turned(qkv.cuda(), at.cuda(), many[1 + 64 * i:65 + 64 * i])
        wq, wk, wv, oq, ok = M.rope(qkv, at, tables[64 * i:64 * i + 64], 3, 1)
        near(q, wq, half_step(qkv.dtype) * 1.01, oq)
        near(k, wk, half_step(qkv.dtype) * 1.01, ok)


def test_a_replay_goes_by_the_positions_that_are_there():
    steps = torch.randint(0, 5000, (4, 3, 1), generator=gen(2), dtype=torch.int32).cuda()
    qkv, freq = randn(1, 5, 128, seed=5).cuda(), FREQ.cuda()
    here = steps[1]
    turned(qkv, here, freq, sections=(16, 24, 24))
    q, k, v = (torch.zeros((1, n, 128), dtype=qkv.dtype, device="cuda") for n in (3, 1, 1))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fkv.proj_rope(qkv, here, freq, q, k, v, sections=(16, 24, 24))
    for i in range(4):
        new = torch.randint(0, 5000, (3, 1), generator=gen(10 + i), dtype=torch.int32).cuda()
        here.copy_(new)
        graph.replay()
        want = turned(qkv, new, freq, sections=(16, 24, 24))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((q, k, v), want)), i
