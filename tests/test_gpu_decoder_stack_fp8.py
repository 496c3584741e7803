"""DecoderStack with weights in 8 bits: the run of norm, products, rotary positions, attention and gate, step by step against plain
operations in 64 bits on what each received, and as a whole."""
import pytest
import torch

import proj_model as M
from test_gpu_paged_cache import D, Pair, ints

pytestmark = pytest.mark.gpu


def stack_of(p, seqs, **kw):
    from paper_2505_13109_amd.layer_loop import DecoderStack
    return DecoderStack(p.c, seqs=ints(seqs), weights="fp8", **kw)


def whole_layer(stack, layer, x, attention):
    """(x behind the layer, the product before the rotary positions), by the definitions, in 64 bits between the roundings that a layer has."""
    T = stack.dtype
    weights = lambda w: M.values(w[0].cpu(), w[1].cpu(), 128)
    eight = lambda codes, scales: codes * M.spread(scales, *codes.shape, 1)
    _, codes, scales, _ = M.norm(x)
    qkv = (eight(codes, scales) @ weights(stack.wqkv[layer]).T).to(T)
    y = (eight(*M.quant(attention.double())) @ weights(stack.wo[layer]).T).to(T)
    s, codes, scales, _ = M.norm(x, add=y)
    gu = (eight(codes, scales) @ weights(stack.wgu[layer]).T).to(T)
    down = (eight(*M.quant(M.gate(gu))) @ weights(stack.wd[layer]).T).to(T)
    return (s.float() + down.float()).to(T), qkv


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("batch", [2, 40])
def test_a_layers_run_is_the_definitions(batch, dtype):
    """A layer at a time.  Roundings to 8 bits may fall to either side where sums differ in their last digits, so results are held to the size
    of what one such step moves, and all of them together to what the type's own roundings leave."""
    p = Pair(n_layers=1, n_kv=2, G=4, max_seqs=batch, max_ctx=256, n_pages=8 * batch, dtype=dtype)
    seqs = list(range(batch))
    p.grow(seqs, [5 + 3 * (i % 30) for i in seqs])
    stack = stack_of(p, seqs, ffn_mult=1.375)
    x = torch.randn((batch, 8 * D), generator=p.gen).to(stack.dtype)
    got = stack.step(x.cuda()).cpu()
    want, qkv = whole_layer(stack, 0, x, stack.out[0].reshape(batch, -1).cpu())
    half = torch.finfo(stack.dtype).eps / 2
    err = (got.double() - want.double()).norm() / want.double().norm()
    # every value is rounded to T five times on its way (the product, the sum, the gate's input, the product, the sum), each by less than half a
    # step of what is summed there, and 8-bit codes that fall to the other side (one in 1000, a step of 2^-3) move less than 2^-3 / sqrt(1000) of it
    assert err <= 5 * half + 2.0 ** -3 / 1000 ** 0.5, err
    q, k, v = (t.cpu() for t in stack.last_qkv[0])
    heads = qkv.view(batch, 12, D)
    places = torch.tensor([p.m.len[s] for s in seqs], dtype=torch.int32)
    wq, wk, wv, oq, ok = M.rope(heads, places, stack.inv_freq.cpu(), 8, 2)
    for a, b in ((q, wq), (k, wk), (v, wv)):
        e = (a.double() - b).norm() / b.norm()
        assert e <= 3 * half + 2.0 ** -3 / 1000 ** 0.5, e
    # what went into the cache and came out of it is the cache's own matter
    assert p.m.extend(seqs, [1] * batch)
    p.m.append(0, seqs, [1] * batch, k, v)
    p.check_attention(0, seqs, q=q, got=stack.out[0].cpu())


def test_the_caches_attention_behind_every_layer():
    p = Pair(n_layers=3, n_kv=2, G=4, max_seqs=3, max_ctx=256, n_pages=24)
    p.grow([0, 2], [61, 5])
    stack = stack_of(p, [2, 0], ffn_mult=1.0)
    x = torch.randn((2, 8 * D), generator=p.gen).bfloat16().cuda()
    for step in range(5):
        before = x.clone()
        y = stack.step(x)
        assert torch.equal(x, before) and torch.isfinite(y.float()).all() and p.m.extend([2, 0], [1, 1])
        for layer in range(3):
            q, k, v = stack.last_qkv[layer]
            p.m.append(layer, [2, 0], [1, 1], k.cpu(), v.cpu())
            p.check_attention(layer, [2, 0], q=q.cpu(), got=stack.out[layer].cpu())
        x = y
    p.check_tables()
    p.check_contents()


@pytest.mark.parametrize("batch", [1, 40])
def test_in_a_graph_it_decodes_on(batch):
    """Replays of one captured step, with eager steps of a sibling and other work between them, bit for bit."""
    p = Pair(n_layers=2, n_kv=2, G=4, max_seqs=3 * batch, max_ctx=128, n_pages=20 * batch)
    first, second, third = (list(range(i * batch, (i + 1) * batch)) for i in range(3))
    p.grow(first, [30 + i for i in range(batch)])
    p.c.fork(ints(first * 2), ints(second + third))
    eager, captured = stack_of(p, second, ffn_mult=1.0), stack_of(p, third, ffn_mult=1.0)
    x = torch.randn((batch, 8 * D), generator=p.gen).bfloat16().cuda()
    xin, graph = x.clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        yout = captured.step(xin)
    a, b = x, x
    for step in range(12):
        a = eager.step(a)
        xin.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        b = yout.clone()
        assert torch.equal(a, b), step
    p.c.health()


def test_on_another_stream():
    p = Pair(n_layers=2, n_kv=2, G=4, max_seqs=4, max_ctx=256, n_pages=40)
    p.grow([0, 3], [58, 9])
    p.c.fork(ints([0, 3]), ints([1, 2]))
    plain, other = stack_of(p, [0, 3], ffn_mult=1.0), stack_of(p, [1, 2], ffn_mult=1.0)
    side, ballast = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    x = torch.randn((2, 8 * D), generator=p.gen).bfloat16().cuda()
    a = b = x
    for step in range(6):
        a = plain.step(a)
        torch.cuda.synchronize()
        ballast @ ballast
        b = other.step(b.clone(), stream=side)
        got = b.clone()
        torch.cuda.synchronize()
        assert torch.equal(a, got), step
    p.c.health()


def test_positions_of_several_axes():
    """The same position on all axes is one axis; other positions turn the sections that they are of."""
    p = Pair(n_layers=1, n_kv=2, G=4, max_seqs=4, max_ctx=256, n_pages=40)
    p.grow([0], [40])
    p.c.fork(ints([0, 0, 0]), ints([1, 2, 3]))
    x = torch.randn((1, 8 * D), generator=p.gen).bfloat16().cuda()
    one, three, given, moved = (stack_of(p, [s], ffn_mult=1.0, rope_sections=r) for s, r in ((0, None), (1, (16, 24, 24)), (2, (16, 24, 24)), (3, (16, 24, 24))))
    y = one.step(x)
    assert torch.equal(y, three.step(x)) and torch.equal(y, given.step(x, positions=ints([40] * 3).view(3, 1)))
    moved.step(x, positions=ints([40, 7, 900]).view(3, 1))
    (q0, k0, v0), (q1, k1, v1) = one.last_qkv[0], moved.last_qkv[0]
    same = torch.zeros(D, dtype=torch.bool)
    same[:16] = same[64:80] = True
    assert torch.equal(v0, v1)
    for a, b in ((q0, q1), (k0, k1)):
        differ = (a != b).any(0).any(0).cpu()
        assert not differ[same].any() and differ[~same].float().mean() > 0.75            # (the slowest pairs hardly move)


def test_refusals():
    from paper_2505_13109_amd.layer_loop import DecoderStack
    p = Pair(n_kv=2, G=2)
    for kw in (dict(weights="fp4"), dict(rope_sections=(64,)), dict(weights="fp8", ffn_mult=1.01)):
        with pytest.raises(ValueError):
            DecoderStack(p.c, seqs=ints([0]), **kw)
    with pytest.raises(ValueError):
        DecoderStack(p.c, seqs=ints([0]), ffn_mult=1.0).step(torch.zeros((1, 4 * D), dtype=torch.bfloat16, device="cuda"), positions=ints([0]))


@pytest.mark.parametrize("placement", [0, 1])
def test_over_a_retrieval_context(placement):
    """The layers' own queries, keys and values drive the retrieval loop: every step against the oracle, fed with the same."""
    import numpy as np
    import paper_2505_13109_amd as fkv
    import workloads as W
    from harness import rel_err_per_head, to_dev
    from oracle import freekv_oracle as O
    from paper_2505_13109_amd.layer_loop import DecoderStack
    wl = W.Workload("loop8", 2, 2, 8, 2, "bf16", 2000 - 9, 512, 64, 64, 0.8, 12, 0.9, 0.436, 710, placement=placement)
    g = fkv.FreeKV(n_layers=2, batch=2, n_q_heads=8, n_kv_heads=2, max_ctx=wl.max_ctx, budget=wl.budget, sink=wl.sink, window=wl.window, tau=wl.tau,
                   dtype="bf16", placement=placement)
    oracles = {}
    for layer in range(2):
        loads = []
        for r in range(2):
            (K, Kb), (V, Vb) = W.kv_prefix(wl, layer, r)
            oracles[(layer, r)] = O.FreeKVOracle(8, 2, 128, 32, wl.budget, wl.sink, wl.window, wl.tau, wl.max_ctx)
            oracles[(layer, r)].load_prefix_bulk(K, V)
            loads.append((Kb, Vb))
        g.load_prefix(layer, *(to_dev(np.stack([x[i] for x in loads]), "bf16") for i in (0, 1)))
    stack = DecoderStack(g, weights="fp8", ffn_mult=1.0, copy_stream=torch.cuda.Stream())
    gen = torch.Generator().manual_seed(5)
    state = torch.randn((2, stack.hidden), generator=gen)
    for t in range(wl.steps):
        rho = 0.2 if t % 5 == 4 else 0.97
        state = rho * state + (1 - rho * rho) ** 0.5 * torch.randn((2, stack.hidden), generator=gen)
        y = stack.step(state.bfloat16().cuda())
        torch.cuda.synchronize()
        assert torch.isfinite(y.float()).all()
        for layer in range(2):
            q, k, v = (x.float().cpu().numpy() for x in stack.last_qkv[layer])
            ids, flags = (g.debug_read(layer, what) for what in (fkv.binding.DBG_ACTIVE_IDS, fkv.binding.DBG_FLAGS))
            out = stack.out[layer].cpu().numpy()
            for r in range(2):
                ref = oracles[(layer, r)].step(q[r], k[r], v[r])
                assert np.array_equal(flags[r], ref["flags"]) and np.array_equal(ids[r], ref["new_ids"]), (t, layer, r)
                assert rel_err_per_head(out[r], ref["out"]).max() <= 2e-3, (t, layer, r)
    g.close()
