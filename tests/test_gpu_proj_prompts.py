"""The projections one behind the other on a prompt's rows: what a layer does before and behind the attention."""
import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M
from test_gpu_proj import FREQ, half_step, randn

pytestmark = pytest.mark.gpu

# Values are rounded to T at most three times on their way, each by half a step of what is there; 8-bit codes of the gate's results fall to the other side
# where a product's rounding did (one in 1000 at most, a step of 2^-3): 2^-3 / sqrt(1000) of the whole.
def off(dtype):
    return 3 * half_step(dtype) + 2.0 ** -3 / 1000 ** 0.5


def apart(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


def weights(n, cols, seed, dtype):
    w = fkv.empty_quant(n, cols, tile=128)
    fkv.proj_quant(randn(n, cols, seed=seed, dtype=dtype, scale=cols ** -0.5, outliers=False).cuda(), *w, tile=128)
    return w, M.values(*w, 128)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [65, 300, 1031])
def test_a_prompts_rows_through_a_layer(rows, dtype):
    hidden, ffn, n_q, n_kv, axes = 640, 1424, 5, 1, (16, 24, 24)
    (wqkv, a), (wgu, b), (wd, c) = weights((n_q + 2 * n_kv) * 128, hidden, 1, dtype), weights(2 * ffn, hidden, 2, dtype), weights(hidden, ffn, 3, dtype)
    x, y = randn(rows, hidden, seed=4, dtype=dtype), randn(rows, hidden, seed=5, dtype=dtype, outliers=False)
    gamma = (1 + 0.2 * torch.randn(hidden, generator=torch.Generator().manual_seed(6))).to(dtype)
    positions = torch.randint(0, 5000, (3, rows), generator=torch.Generator().manual_seed(7), dtype=torch.int32)
    new = lambda *shape: torch.empty(shape, dtype=dtype, device="cuda")
    dx, h, f = x.cuda(), fkv.empty_quant(rows, hidden), fkv.empty_quant(rows, ffn)
    qkv, gu, down, (q, k, v) = new(rows, (n_q + 2 * n_kv) * 128), new(rows, 2 * ffn), new(rows, hidden), (new(rows, n, 128) for n in (n_q, n_kv, n_kv))
    fkv.proj_norm(dx, gamma.cuda(), *h, add=y.cuda())
    fkv.proj_matmul(*h, *wqkv, qkv)
    fkv.proj_rope(qkv.view(rows, n_q + 2 * n_kv, 128), positions.cuda(), FREQ.cuda(), q, k, v, sections=axes)
    fkv.proj_matmul(*h, *wgu, gu)
    fkv.proj_gate(gu, *f)
    fkv.proj_matmul(*f, *wd, down)

    s, codes, scales, _ = M.norm(x, gamma, y)
    assert torch.equal(dx.cpu(), s)
    z = codes * M.spread(scales, rows, hidden, 1)
    want = z @ a.T
    assert apart(qkv, want) <= off(dtype)
    which = [i for i, n in enumerate(axes) for _ in range(n)]
    wq, wk, wv, _, _ = M.rope(want.view(rows, n_q + 2 * n_kv, 128), positions, FREQ, n_q, n_kv, which)
    for got, w in ((q, wq), (k, wk), (v, wv)):
        assert apart(got, w) <= off(dtype)
    g = (z @ b.T).to(dtype)
    codes, scales = M.quant(M.gate(g))
    assert apart(down, (codes * M.spread(scales, rows, ffn, 1)) @ c.T) <= off(dtype)
