"""The projections in 8 bits against their definitions in 64 bits (tests/proj_model.py), on a GPU."""
import math

import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M

pytestmark = pytest.mark.gpu

TYPES = [torch.float16, torch.bfloat16]
CODES = torch.float8_e4m3fn


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(*shape, seed=0, dtype=torch.bfloat16, scale=1.0, outliers=True):
    x = torch.randn(shape, generator=gen(seed)) * scale
    if outliers:
        x[..., ::37] *= 8
    return x.to(dtype)


def fenced(shape, dtype, fill):
    """A tensor between rows that have to stay as they are; (tensor, check)."""
    n = math.prod(shape)
    whole = torch.full((n + 512,), fill, dtype=torch.float32).to(dtype).cuda()
    before = whole.clone()

    def untouched():
        raw = torch.uint8
        assert torch.equal(whole[:256].view(raw), before[:256].view(raw)) and torch.equal(whole[256 + n:].view(raw), before[256 + n:].view(raw))
    return whole[256:256 + n].view(shape), untouched


def fenced_quant(rows, cols, tile=1):
    c, a = fenced((rows, cols), CODES, 3.0)
    s, b = fenced((-(-rows // tile), -(-cols // 128)), torch.float32, -5.0)
    return c, s, lambda: (a(), b())


def same_codes(codes, want):
    assert torch.equal(codes.float().cpu().double(), want.double())


def same_scales(scales, want):
    assert torch.equal(torch.nan_to_num(scales.cpu(), -1.0), torch.nan_to_num(want, -1.0))


def near(got, want, rel, off=0.0):
    """|got - want| <= rel |want| + off, infinities where they are wanted"""
    got = got.cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    err = (got - want).abs() - rel * want.abs() - off
    assert (err[fine] <= 0).all(), (float(err[fine].max()), int(err[fine].argmax()))


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ---- into 8 bits ----------------------------------------------------------------------------------------

SHAPES = [(1, 16), (1, 128), (3, 112), (2, 144), (17, 1040), (130, 256), (128, 128), (257, 4096), (5, 11056)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quant_is_the_definition(rows, cols, tile, dtype):
    x = randn(rows, cols, seed=rows * 7 + cols, dtype=dtype)
    codes, scales, untouched = fenced_quant(rows, cols, tile)
    fkv.proj_quant(x.cuda(), codes, scales, tile=tile)
    want = M.quant(x.double(), tile)
    same_codes(codes, want[0])
    same_scales(scales, want[1])
    untouched()


@pytest.mark.parametrize("dtype", TYPES)
def test_quant_of_every_size_and_of_what_is_next_to_a_border(dtype):
    """Rows from the smallest to the largest numbers of the type; in each all 2^7 mantissas, so that quotients lie on and beside borders."""
    info = torch.finfo(dtype)
    least, most = (-24, 15) if dtype == torch.float16 else (-133, 127)
    base = torch.cat((1 + torch.arange(128) / 128.0, torch.tensor([0.0, 1.0, 2.0 ** -9, 2.0 ** -10, 2.0 ** -10 * 1.0078125, 0.75 * 2.0 ** -9]).repeat(21)[:122], torch.zeros(6)))
    rows = [(base * sign * 2.0 ** e * f).double() for e in range(least, most + 1) for sign, f in ((1, 1.0), (-1, 0.4375))]
    x = torch.stack(rows).clamp(-info.max, info.max).to(dtype)
    codes, scales, untouched = fenced_quant(*x.shape)
    fkv.proj_quant(x.cuda(), codes, scales)
    want = M.quant(x.double())
    same_codes(codes, want[0])
    same_scales(scales, want[1])
    untouched()


def test_quant_of_every_bf16_number_against_some_largest_ones():
    every = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    every = every[torch.isfinite(every)]
    for top in (1.0, 1.9921875, 3.0, 447.0, 2.0 ** -117, 2.0 ** -120, 1e30):
        small = every[every.abs().float() <= top]
        n = -(-small.numel() // 127)
        x = torch.zeros((n, 128), dtype=torch.bfloat16)
        x[:, 1:].reshape(-1)
        flat = torch.zeros(n * 127, dtype=torch.bfloat16)
        flat[:small.numel()] = small
        x[:, 1:] = flat.view(n, 127)
        x[:, 0] = top
        codes, scales, _ = fenced_quant(n, 128)
        fkv.proj_quant(x.cuda(), codes, scales)
        want = M.quant(x.double())
        same_codes(codes, want[0])
        same_scales(scales, want[1])


@pytest.mark.parametrize("tile", [1, 128])
def test_blocks_with_nan_or_infinities_stand_for_nan_alone(tile):
    x = randn(200, 300, seed=4)
    x[3, 5], x[4, 140], x[150, 299], x[6, 256] = math.nan, math.inf, -math.inf, 0.0
    x[8] = 0
    codes, scales, _ = fenced_quant(200, 304, tile)
    y = torch.cat((x, torch.zeros(200, 4, dtype=x.dtype)), 1)
    fkv.proj_quant(y.cuda(), codes, scales, tile=tile)
    want = M.quant(y.double(), tile)
    assert int(torch.isnan(want[1]).sum()) == 3
    same_codes(codes, want[0])
    same_scales(scales, want[1])


# ---- the norm -----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("add,weight,quant,out", [(True, True, True, False), (True, False, True, True), (False, True, True, True), (False, False, False, True), (True, True, False, True)])
@pytest.mark.parametrize("rows,cols", [(1, 16), (33, 1024), (9, 1040), (5, 2048), (3, 2064), (3, 3584), (2, 4112), (65, 8192), (7, 8208), (700, 256), (2, 32784), (3, 131072)])
def test_norm_is_the_definition(rows, cols, add, weight, quant, out, dtype):
    x = randn(rows, cols, seed=1, dtype=dtype)
    a = randn(rows, cols, seed=2, dtype=dtype, outliers=False) if add else None
    w = (1 + 0.2 * torch.randn(cols, generator=gen(3))).to(dtype) if weight else None
    s, codes_want, scales_want, y = M.norm(x, w, a)
    codes, scales, untouched = fenced_quant(rows, cols)
    res, res_same = fenced((rows, cols), dtype, 7.0)
    o, o_same = fenced((rows, cols), dtype, 7.0)
    dev = lambda t: None if t is None else t.cuda()
    fkv.proj_norm(dev(x), dev(w), codes if quant else None, scales if quant else None, add=dev(a), res=res if add else None, out=o if out else None)
    if add:
        assert torch.equal(res.cpu(), s)
    if quant:
        same_codes(codes, codes_want)
        # one rounding, and 2^-40 for what is summed and turned over in fp64
        near(scales, scales_want, 2.0 ** -24 * 1.001)
    if out:
        # rounded to fp32 and then to T
        near(o, y, half_step(dtype) * 1.01 + 2.0 ** -24, 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)
    untouched(), res_same(), o_same()


@pytest.mark.parametrize("cols", [512, 40000])
def test_norm_into_its_input(cols):
    """The stream goes on in place, whether it is named or not; with `out`, too."""
    x, a, w = randn(9, cols, seed=1), randn(9, cols, seed=2), randn(cols, seed=3, outliers=False)
    s, codes_want, scales_want, y = M.norm(x, w, a)
    for named in (False, True):
        for want_out in (False, True):
            at = x.cuda()
            codes, scales = fkv.empty_quant(9, cols)
            out = torch.empty_like(at) if want_out else None
            fkv.proj_norm(at, w.cuda(), codes, scales, add=a.cuda(), res=at if named else None, out=out)
            assert torch.equal(at.cpu(), s)
            same_codes(codes, codes_want)
            near(scales, scales_want, 2.0 ** -24 * 1.001)
            if want_out:
                near(out, y, half_step(torch.bfloat16) * 1.01 + 2.0 ** -24)


def test_norm_of_values_of_all_sizes():
    """bf16 rows from 2^-120 to 2^126, where fp32's squares are nothing or infinite; a row of zeros; eps of all sizes."""
    scales = torch.tensor([2.0 ** e for e in (-120, -100, -70, -60, -10, 0, 20, 62, 64, 100, 120)] + [0.0])
    x = (torch.randn((12, 1024), generator=gen(5)).clamp(-3, 3) * scales[:, None]).bfloat16()
    for eps in (1e-5, 2.0 ** -126, 1e30):
        codes, sc, _ = fenced_quant(12, 1024)
        out = torch.empty((12, 1024), dtype=torch.bfloat16, device="cuda")
        fkv.proj_norm(x.cuda(), None, codes, sc, out=out, eps=eps)
        _, codes_want, scales_want, y = M.norm(x, eps=float(torch.tensor(eps, dtype=torch.float32)))
        same_codes(codes, codes_want)
        near(sc, scales_want, 2.0 ** -24 * 1.001, 2.0 ** -150)
        near(out, y, half_step(torch.bfloat16) * 1.01 + 2.0 ** -24, 2.0 ** -134 + 2.0 ** -150)


def test_norm_of_rows_with_nan_and_infinities():
    x = randn(4, 512, seed=6)
    x[0, 3], x[1, 200] = math.nan, math.inf
    codes, scales = fkv.empty_quant(4, 512)
    out = torch.empty((4, 512), dtype=x.dtype, device="cuda")
    fkv.proj_norm(x.cuda(), None, codes, scales, out=out)
    s, o = scales.cpu(), out.cpu()
    assert torch.isnan(s[0]).all() and torch.isnan(o[0]).all()
    assert torch.isnan(s[1, 1]) and (s[1, [0, 2, 3]] == 0).all() and torch.isnan(o[1, 200]) and not o[1, :200].any()
    _, codes_want, scales_want, _ = M.norm(x[2:])
    same_codes(codes[2:], codes_want)
    near(scales[2:], scales_want, 2.0 ** -24 * 1.001)


# ---- the gate -----------------------------------------------------------------------------------------------

# exp2 within a step of fp32 (2^-23), two roundings around it, the quotient's, the two products': under 8 x 2^-24
GATE = 8 * 2.0 ** -24


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 16), (3, 144), (33, 1040), (200, 12544), (1, 131072)])
def test_gate_is_the_definition(rows, cols, dtype):
    gu = randn(rows, 2 * cols, seed=rows + cols, dtype=dtype, scale=2.0)
    codes, scales, untouched = fenced_quant(rows, cols)
    fkv.proj_gate(gu.cuda(), codes, scales)
    y = M.gate(gu)
    top = M.block_tops(y, 1)
    near(scales, top / 448, GATE + 2.0 ** -24)
    held_to_quotients(codes, scales, y, GATE + 2.0 ** -24)
    untouched()


def held_to_quotients(codes, scales, y, off):
    """Each code is what a value within `off` of y rounds to (y is off by that, the quotient is rounded once)."""
    q = y / M.spread(scales.cpu(), *y.shape, 1)
    lo, hi = M.nearest_e4m3(q * (1 - off)), M.nearest_e4m3(q * (1 + off))
    c = codes.float().cpu().double()
    assert ((c - lo) * (c - hi) <= 0).all()


def test_gate_at_the_ends():
    """Large gates let everything or nothing through; NaN and infinities take their block with them, and no other."""
    g = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 20, -20, 80, -80, 88, -100, 1000, -1000, 60000, -60000, 3, -3]).repeat(8)
    u = torch.tensor([1.0, -2.0, 3.0, 1e4, -1e-4, 0.0, 5.0, 6.0]).repeat_interleave(16)
    gu = torch.cat((g, g, u, u))[None].repeat(3, 1).half()
    gu[1, 130], gu[2, 256] = math.inf, math.nan
    codes, scales = fkv.empty_quant(3, 256)
    fkv.proj_gate(gu.cuda(), codes, scales)
    y = M.gate(gu)
    y[1, 130] = math.nan
    top = M.block_tops(y, 1)
    assert torch.isnan(top).tolist() == [[False, False], [False, True], [True, False]]
    near(scales, top / 448, GATE + 2.0 ** -24)
    fine = ~torch.isnan(M.spread(scales.cpu(), 3, 256, 1))
    assert not codes.float().cpu()[~fine].any()
    q = torch.where(fine, y / M.spread(scales.cpu(), 3, 256, 1), torch.zeros_like(y)).nan_to_num(0.0)
    c = codes.float().cpu().double()
    lo, hi = M.nearest_e4m3(q * (1 - 2 * GATE)), M.nearest_e4m3(q * (1 + 2 * GATE))
    assert ((c - lo) * (c - hi) <= 0).all()


# ---- rotary positions -----------------------------------------------------------------------------------------

FREQ = (500000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).float()


def rope_of(rows, n_q, n_kv, positions, dtype, sections=None, axis_of=None, seed=0, freq=FREQ):
    qkv = randn(rows, n_q + 2 * n_kv, 128, seed=seed, dtype=dtype)
    (q, a), (k, b), (v, c) = (fenced((rows, n, 128), dtype, 9.0) for n in (n_q, n_kv, n_kv))
    fkv.proj_rope(qkv.cuda(), positions.cuda(), freq.cuda(), q, k, v, sections=sections)
    wq, wk, wv, oq, ok = M.rope(qkv, positions, freq, n_q, n_kv, axis_of)
    for got, want, off in ((q, wq, oq), (k, wk, ok)):
        near(got, want, half_step(dtype) * 1.01, off + (2.0 ** -25 if dtype == torch.float16 else 0.0))
    assert torch.equal(v.cpu().double(), wv)
    a(), b(), c()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_q,n_kv", [(1, 1, 1), (6, 4, 1), (1, 32, 8), (5, 28, 4), (67, 7, 1), (1100, 12, 3), (9, 12, 3), (2, 300, 300)])
def test_rope_of_one_axis(rows, n_q, n_kv, dtype):
    positions = torch.randint(0, 40000, (rows,), generator=gen(rows), dtype=torch.int32)
    rope_of(rows, n_q, n_kv, positions, dtype)


@pytest.mark.parametrize("sections", [(16, 24, 24), (0, 64), (64, 0, 0), (10, 20, 30, 4), (1, 63)])
def test_rope_of_several_axes(sections):
    axes = len(sections)
    positions = torch.randint(-50, 5000, (axes, 37), generator=gen(axes), dtype=torch.int32)
    rope_of(37, 6, 2, positions, torch.bfloat16, sections=sections, axis_of=[a for a, n in enumerate(sections) for _ in range(n)])
    turns = [i % axes for i in range(64)]                    # axes in turn
    rope_of(37, 6, 2, positions, torch.float16, sections=turns, axis_of=turns)


def test_rope_without_sections_goes_by_the_first_axis():
    positions = torch.randint(0, 5000, (3, 9), generator=gen(1), dtype=torch.int32)
    rope_of(9, 4, 2, positions, torch.bfloat16)


def test_rope_of_far_positions():
    """Whole turns are taken off exactly: up to the last 32-bit position, either sign, at frequencies near 1 (the angles by rational numbers)."""
    from fractions import Fraction
    ends = [0, 1, -1, 4194303, 4194304, 2 ** 29 - 1, 2 ** 31 - 1, -2 ** 31]
    freq = torch.cat((torch.tensor([1.0, 0.99999994, 0.9]), FREQ[3:]))
    two_pi = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62) * 2
    # positions that stand for the same angle below one turn, in 64 bits
    angle = torch.tensor([[float((p * Fraction(float(f))) % two_pi) for f in freq] for p in ends], dtype=torch.float64)
    qkv = randn(len(ends), 4, 128, seed=8, dtype=torch.float16)
    q, k, v = (torch.empty((len(ends), n, 128), dtype=torch.float16, device="cuda") for n in (2, 1, 1))
    fkv.proj_rope(qkv.cuda(), torch.tensor(ends, dtype=torch.int32).cuda(), freq.cuda(), q, k, v)
    a, b, turn = qkv[:, :3, :64].double(), qkv[:, :3, 64:].double(), angle[:, None]
    want = torch.cat((a * turn.cos() - b * turn.sin(), a * turn.sin() + b * turn.cos()), -1)
    off = 10 * 2.0 ** -24 * (a.abs() + b.abs()).repeat(1, 1, 2) + 2.0 ** -25      # (past 2^29 turns are off by up to 2^-25, 2^-22.3 as an angle)
    off[5:] += 4 * 2.0 ** -24 * (a.abs() + b.abs()).repeat(1, 1, 2)[5:]
    near(torch.cat((q, k), 1), want, half_step(torch.float16) * 1.01, off)


# ---- the product --------------------------------------------------------------------------------------------------

def operands(rows, n, cols, seed=0):
    x, w = randn(rows, cols, seed=seed), randn(n, cols, seed=seed + 1, scale=cols ** -0.5, outliers=False)
    (xc, xs), (wc, ws) = M.quant(x.double()), M.quant(w.double(), 128)
    return xc.float().to(CODES), xs, wc.float().to(CODES), ws


def product(x, xs, w, ws, dtype):
    out, untouched = fenced((x.shape[0], w.shape[0]), dtype, 11.0)
    fkv.proj_matmul(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), out)
    untouched()
    return out


FEW = 32               # rows up to which no product is cut


# 128 products a block and the blocks' sums, each addition off by a step of fp32 of the terms' sizes at most, and the scales' product and its own
def sum_off(cols):
    return (128 + -(-cols // 128) + 3) * 2.0 ** -23


ROWS = [1, 2, 15, 16, 17, 31, 33, 48, 64, 65, 100, 128, 129, 200, 256, 257, 400]
WIDTHS = [(1, 16), (15, 112), (16, 128), (17, 144), (128, 1024), (129, 2064), (300, 512), (1000, 4096), (2050, 400)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,cols", WIDTHS)
@pytest.mark.parametrize("rows", ROWS)
def test_product_is_the_definition(rows, n, cols, dtype):
    x, xs, w, ws = operands(rows, n, cols, seed=rows + n)
    want, size, cut = M.matmul(x, xs, w, ws)
    near(product(x, xs, w, ws, dtype), want, half_step(dtype) * 1.01, sum_off(cols) * size + (rows > FEW) * cut + 2.0 ** -25)


@pytest.mark.parametrize("rows,n,cols", [(1, 300, 4096), (7, 4096, 11056), (40, 1031, 2048), (130, 513, 1040), (300, 700, 8192), (1030, 1100, 1024)])
def test_product_of_small_whole_numbers_is_exact(rows, n, cols):
    """Every place counts once: sums of products of whole numbers with scales that are powers of two are exact in fp32, and here in bf16."""
    g = gen(rows)
    x, w = torch.zeros((rows, cols)), torch.zeros((n, cols))
    at = torch.randint(0, cols, (rows, 12), generator=g)
    x.scatter_(1, at, torch.randint(-1, 2, (rows, 12), generator=g).float())
    w = torch.randint(-2, 3, (n, cols), generator=g).float()
    xs = torch.exp2(torch.randint(0, 2, (rows, -(-cols // 128)), generator=g).float())
    ws = torch.exp2(torch.randint(0, 2, (-(-n // 128), -(-cols // 128)), generator=g).float())
    want, _, _ = M.matmul(x.to(CODES), xs, w.to(CODES), ws)
    assert want.abs().max() <= 256
    got = product(x.to(CODES), xs, w.to(CODES), ws, torch.bfloat16)
    assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_product_keeps_rows_columns_and_blocks_apart(rows):
    """A NaN scale or code reaches what it is a factor of, and nothing else; scales of all sizes."""
    n, cols = 400, 1040
    x, xs, w, ws = operands(rows, n, cols, seed=9)
    xs = xs * torch.exp2(torch.randint(-30, 30, xs.shape, generator=gen(1)).float())
    clean, size, cut = M.matmul(x, xs, w, ws)
    near(product(x, xs, w, ws, torch.bfloat16), clean, half_step(torch.bfloat16) * 1.01, sum_off(cols) * size + (rows > FEW) * cut)
    xs[rows // 2, 3] = math.nan
    ws[1, 8] = math.nan
    wf = w.float()
    wf[399, 1039] = math.nan
    w = wf.to(CODES)
    got = product(x, xs, w, ws, torch.bfloat16).cpu()
    bad = torch.zeros((rows, n), dtype=torch.bool)
    bad[rows // 2] = True
    bad[:, 128:256] = True
    bad[:, 399] = True
    assert torch.equal(torch.isnan(got), bad)
    off = half_step(torch.bfloat16) * 1.01 * clean.abs() + sum_off(cols) * size + (rows > FEW) * cut
    assert ((got.double() - clean).abs()[~bad] <= off[~bad]).all()


def test_product_overflows_to_infinities_in_fp16():
    x, w = torch.full((3, 256), 448.0).to(CODES), torch.full((20, 256), 448.0).to(CODES)
    xs, ws = torch.ones((3, 2)), torch.ones((1, 2))
    assert torch.isinf(product(x, xs, w, ws, torch.float16)).all()
    assert torch.equal(product(x, xs, w, ws * 2.0 ** -12, torch.float16).cpu(), torch.full((3, 20), 448.0 * 448 * 256 / 4096).half())


def test_nothing_to_do():
    x = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    codes, scales = fkv.empty_quant(0, 256)
    w, ws = fkv.empty_quant(256, 256, tile=128)
    fkv.proj_quant(x, codes, scales)
    fkv.proj_norm(x, None, codes, scales)
    fkv.proj_gate(torch.empty((0, 512), dtype=torch.bfloat16, device="cuda"), codes, scales)
    fkv.proj_matmul(codes, scales, w, ws, torch.empty((0, 256), dtype=torch.bfloat16, device="cuda"))
    h = [torch.empty((0, n, 128), dtype=torch.bfloat16, device="cuda") for n in (4, 2, 1, 1)]
    fkv.proj_rope(h[0], torch.empty((0,), dtype=torch.int32, device="cuda"), FREQ.cuda(), *h[1:])
    torch.cuda.synchronize()
