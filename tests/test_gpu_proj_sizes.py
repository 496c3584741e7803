"""The product in 8 bits where it is cut in other ways: tiles of all sizes, one and several to a block, long axes in parts and runs of scales,
operands past 4 GiB; all of the projections past 4 GiB."""
import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M
from test_gpu_proj import CODES, FREQ, gen, half_step, near, randn, same_codes, same_scales

pytestmark = pytest.mark.gpu


def whole_numbers(rows, n, cols, seed):
    """Codes and scales whose products and sums are whole numbers up to 96, on the GPU: twelve places of a row count, other ones in each."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = dict(generator=g, device="cuda")
    x = torch.zeros((rows, cols), device="cuda")
    k = min(12, cols)
    x.scatter_(1, torch.randint(0, cols, (rows, k), **new), torch.randint(-1, 2, (rows, k), **new).float())
    w = torch.randint(-2, 3, (n, cols), **new).float()
    xs = torch.exp2(torch.randint(0, 2, (rows, -(-cols // 128)), **new).float())
    ws = torch.exp2(torch.randint(0, 2, (-(-n // 128), -(-cols // 128)), **new).float())
    return x.to(CODES), xs, w.to(CODES), ws


def exact(x, xs, w, ws):
    """in 64 bits on the GPU, whatever the order of sums"""
    spread = lambda s, c, tile: (c.float().double() * s.double().repeat_interleave(tile, 0)[:c.shape[0]].repeat_interleave(128, 1)[:, :c.shape[1]])
    return spread(xs, x, 1) @ spread(ws, w, 128).T


FEW = [(1, 33, 33040), (7, 600, 131072), (20, 4099, 20000), (32, 50, 16400), (17, 20000, 272), (9, 9001, 16), (63, 4099, 2064), (49, 1, 8192)]
# rows, n, cols: a tile of 64, 128 (four stages, two) and 256 squared; whole and in parts; one to a block and more; runs of scales of one block to many
MANY = [(33, 1, 16), (130, 16848, 2416), (137, 11029, 400), (198, 10556, 16), (39, 6763, 2080), (414, 18, 464), (232, 116, 128), (36, 16633, 7936), (40, 2958, 10384),
        (254, 1, 2560), (50, 100, 131072), (74, 16811, 2320), (75, 17604, 1216), (66, 5379, 10800), (69, 6135, 3840), (799, 16609, 2064), (1070, 13195, 400),
        (869, 16468, 160), (210, 17959, 2144), (271, 16457, 416), (1361, 4433, 144), (69, 13105, 8640), (65, 5508, 8352), (1560, 10161, 2064), (1169, 14538, 416),
        (2389, 6710, 16), (386, 17590, 2192), (775, 9847, 416), (714, 8648, 16), (140, 16858, 6320), (130, 6298, 5104), (2630, 6370, 3472)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,n,cols", FEW + MANY)
def test_every_place_counts_once(rows, n, cols, dtype):
    ops = whole_numbers(rows, n, cols, rows + n + cols)
    pad = torch.full((rows * n + 512,), 7.0, dtype=dtype, device="cuda")
    out = pad[256:256 + rows * n].view(rows, n)
    for again in range(2):                                       # (the second on used workspaces)
        out.fill_(9.0)
        fkv.proj_matmul(*ops, out)
        want = exact(*ops)
        assert want.abs().max() <= 256 and torch.equal(out.double(), want)
    assert (pad[:256] == 7).all() and (pad[256 + rows * n:] == 7).all()


@pytest.mark.parametrize("rows", [1, 16, 32, 33, 200, 3000])
def test_the_same_call_gives_the_same_bits(rows):
    x, w = randn(rows, 2192, seed=1).cuda(), randn(3001, 2192, seed=2, outliers=False).cuda()
    (c, s), (wc, ws) = fkv.empty_quant(rows, 2192), fkv.empty_quant(3001, 2192, tile=128)
    fkv.proj_quant(x, c, s)
    fkv.proj_quant(w, wc, ws, tile=128)
    outs = [torch.empty((rows, 3001), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    for o in outs:
        fkv.proj_matmul(c, s, wc, ws, o)
    assert all(torch.equal(outs[0], o) for o in outs[1:])


# ---- past 4 GiB ------------------------------------------------------------------------------------------------------

def some_rows(rows):
    return torch.tensor([0, 1, rows // 2, rows - 2, rows - 1])


def big(rows, cols, seed=0):
    """[rows, cols] bf16 on the GPU, rows repeating after 1000"""
    part = randn(1000, cols, seed=seed).cuda()
    return part.repeat(-(-rows // 1000), 1)[:rows].contiguous()


def test_values_past_4_gib():
    rows, cols, at = 600001, 4096, some_rows(600001)
    x = big(rows, cols)
    assert x.numel() * 2 > 2 ** 32
    picked = x[at.cuda()].cpu()
    for tile in (1, 128):
        codes, scales = fkv.empty_quant(rows, cols, tile=tile)
        fkv.proj_quant(x, codes, scales, tile=tile)
        if tile == 1:
            c, s = M.quant(picked.double())
            same_codes(codes[at.cuda()], c)
            same_scales(scales[at.cuda()], s)
        else:
            first = (rows - 1) // 128 * 128
            c, s = M.quant(x[first:].cpu().double(), 128)
            same_codes(codes[first:], c)
            same_scales(scales[-1:], s)
    codes, scales = fkv.empty_quant(rows, cols)
    out = torch.empty_like(x)
    fkv.proj_norm(x, None, codes, scales, out=out)
    _, c, s, y = M.norm(picked)
    same_codes(codes[at.cuda()], c)
    near(scales[at.cuda()], s, 2.0 ** -24 * 1.001)
    near(out[at.cuda()], y, half_step(torch.bfloat16) * 1.01 + 2.0 ** -24)
    fkv.proj_norm(x, None, None, None, add=out, out=out)       # the sum into x, the norm over what was added: a row is read before it is written
    s, _, _, y = M.norm(picked, add=y.bfloat16())
    assert torch.equal(x[at.cuda()].cpu(), s)
    near(out[at.cuda()], y, half_step(torch.bfloat16) * 1.01 + 2.0 ** -24)


def test_gate_and_rope_past_4_gib():
    rows, at = 300001, some_rows(300001).cuda()
    gu = big(rows, 8192, seed=3)
    codes, scales = fkv.empty_quant(rows, 4096)
    fkv.proj_gate(gu, codes, scales)
    y = M.gate(gu[at].cpu())
    near(scales[at], M.block_tops(y, 1) / 448, 9 * 2.0 ** -24)
    q = y / M.spread(scales[at].cpu(), 5, 4096, 1)
    c = codes[at].float().cpu().double()
    assert ((c - M.nearest_e4m3(q * (1 - 9 * 2.0 ** -24))) * (c - M.nearest_e4m3(q * (1 + 9 * 2.0 ** -24))) <= 0).all()
    qkv = gu.view(rows, 64, 128)
    q, k, v = (torch.empty((rows, n, 128), dtype=torch.bfloat16, device="cuda") for n in (48, 8, 8))
    positions = torch.arange(rows, dtype=torch.int32, device="cuda")
    fkv.proj_rope(qkv, positions, FREQ.cuda(), q, k, v)
    wq, wk, wv, oq, ok = M.rope(qkv[at].cpu(), positions[at].cpu(), FREQ, 48, 8)
    near(q[at], wq, half_step(torch.bfloat16) * 1.01, oq)
    near(k[at], wk, half_step(torch.bfloat16) * 1.01, ok)
    assert torch.equal(v[at].cpu().double(), wv)


@pytest.mark.parametrize("rows,n,cols", [(1100000, 70, 4096), (5, 1100000, 4096), (40, 1100000, 4096), (45000, 50000, 16)])
def test_products_past_4_gib(rows, n, cols):
    """Activations, weights and results of more than 4 GiB; a part of them is looked at."""
    x, xs, w, ws = whole_numbers(min(rows, 1000), min(n, 1024), cols, 5)
    if rows > 1000:
        x, xs = (t.repeat(-(-rows // 1000), 1)[:rows].contiguous() for t in (x, xs))
    if n > 1024:
        w, ws = w.repeat(-(-n // 1024), 1)[:n].contiguous(), ws.repeat(-(-n // 1024), 1)[:-(-n // 128)].contiguous()
    assert max(x.numel(), w.numel(), 2 * rows * n) > 2 ** 32 or rows * n > 2 ** 31
    out = torch.full((rows, n), 9.0, dtype=torch.bfloat16, device="cuda")
    fkv.proj_matmul(x, xs, w, ws, out)
    want = exact(x[:1000], xs[:1000], w[:1024], ws[:8])
    for r in range(0, rows, max(1000, rows // 7 // 1000 * 1000)):
        for c in range(0, n, max(1024, n // 7 // 1024 * 1024)):
            part = out[r:r + 1000, c:c + 1024]
            assert torch.equal(part.double(), want[:part.shape[0], :part.shape[1]]), (r, c)
    assert torch.equal(out[-3:, -3:].double(), last(x, xs, w, ws))


def last(x, xs, w, ws):
    """the last three columns of the last three rows"""
    n = w.shape[0]
    first = (n - 3) // 128 * 128
    return exact(x[-3:], xs[-3:], w[first:], ws[first // 128:])[:, -3:]
