"""DecoderStack with weights in 8 bits, beside its arithmetic: layers of different lengths, what it hands out, calls that it refuses."""
import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M
from paper_2505_13109_amd.layer_loop import DecoderStack
from test_gpu_decoder_stack_fp8 import stack_of
from test_gpu_paged_cache import D, Pair, ints

pytestmark = pytest.mark.gpu


def test_layers_of_different_lengths():
    """Each layer's own length is its token's position, as with weights in 16 bits."""
    lens = [520, 713, 520]
    g = fkv.FreeKV(n_layers=3, batch=2, n_q_heads=8, n_kv_heads=2, max_ctx=2048, budget=512, sink=64, window=64, tau=0.8, dtype="bf16", placement=0)
    gen = torch.Generator().manual_seed(1)
    for layer, n in enumerate(lens):
        g.load_prefix(layer, *(torch.randn((2, n, 2, D), generator=gen).bfloat16().cuda() for _ in "kv"))
    x = torch.randn((2, 8 * D), generator=gen).bfloat16().cuda()
    for n_layers in (1, 2, 3):                                # the last of them left its product behind
        stack = DecoderStack(g, weights="fp8", ffn_mult=1.0)
        stack.n_layers = n_layers
        stack.step(x)
        q, k, v = stack.last_qkv[n_layers - 1]
        at = torch.full((2,), lens[n_layers - 1], dtype=torch.int32)
        wq, wk, wv, oq, ok = M.rope(stack.qkv.cpu().view(2, 12, D), at, stack.inv_freq.cpu(), 8, 2)
        for got, want, off in ((q, wq, oq), (k, wk, ok)):
            err = (got.cpu().double() - want).abs() - torch.finfo(torch.bfloat16).eps / 2 * 1.01 * want.abs() - off
            assert (err <= 0).all(), (n_layers, float(err.max()))
        assert torch.equal(v.cpu().double(), wv)
        for layer in range(n_layers):
            lens[layer] += 1
            assert g.context_len(layer) == lens[layer]
    torch.cuda.synchronize()
    g.close()


def test_a_steps_queries_keys_and_values_stay():
    """What a step has handed out is not written again by those behind it."""
    p = Pair(n_layers=2, n_kv=2, G=4, max_seqs=2, max_ctx=256, n_pages=16)
    p.grow([0, 1], [20, 9])
    stack = stack_of(p, [0, 1], ffn_mult=1.0)
    x = torch.randn((2, 8 * D), generator=p.gen).bfloat16().cuda()
    kept = []
    for _ in range(3):
        x = stack.step(x)
        kept.append([(t, t.clone()) for layer in stack.last_qkv for t in layer])
    torch.cuda.synchronize()
    for step in kept:
        assert len(step) == 6 and all(torch.equal(t, then) for t, then in step)


def test_a_refused_step_leaves_the_cache_as_it_was():
    p = Pair(n_layers=1, n_kv=2, G=4, max_seqs=2, max_ctx=256, n_pages=16)
    p.grow([0, 1], [20, 9])
    one, three = stack_of(p, [0, 1], ffn_mult=1.0), stack_of(p, [0, 1], ffn_mult=1.0, rope_sections=(16, 24, 24))
    x = torch.randn((2, 8 * D), generator=p.gen).bfloat16().cuda()
    at = ints([20, 9])
    for bad in (x[:1], x.half(), x.cpu(), x[:, :512], x.T.contiguous().T, None):
        for stack in (one, three):
            with pytest.raises((ValueError, fkv.FreeKVError)):
                stack.step(bad)
    for stack, bad in ((one, at.long()), (one, at[:1]), (one, at.cpu()), (one, at.view(2, 1)), (one, at.repeat(5).view(5, 2)), (one, 20), (three, at),
                       (three, at.repeat(2).view(2, 2)), (three, at.repeat(3).view(2, 3).T)):
        with pytest.raises((ValueError, fkv.FreeKVError)):
            stack.step(x, positions=bad)
    torch.cuda.synchronize()
    p.check_tables()
    p.check_contents()
    given, own = one.step(x, positions=at), one.step(x)                  # (each appends a token)
    assert torch.isfinite(given.float()).all() and torch.isfinite(own.float()).all()
    for sections in ((16, 24), (70, -6), [4] * 64, [-1] + [0] * 63, (16, 16, 16, 8, 8)):
        with pytest.raises((ValueError, fkv.FreeKVError)):
            stack_of(p, [0, 1], ffn_mult=1.0, rope_sections=sections)
