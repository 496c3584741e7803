"""The gated activation where it is hard: gates of all of bf16's sizes, and how far its values are off."""
import math

import pytest
import torch

import paper_2505_13109_amd as fkv
import proj_model as M
from test_gpu_proj import GATE, fenced_quant, gen, held_to_quotients, near, randn

pytestmark = pytest.mark.gpu

ENDS = [-5898240.0, -1e8, -1e20, 1e8, 1e20, 3e38, -3e38, 2.35e38, -2.35e38, 2.4e38, -2.4e38, 80.0, -80.0, 87.0, -87.0, -88.0, 89.0, -89.0, 100.0, -100.0, 1e4, -1e4]


@pytest.mark.parametrize("others", [False, True])
def test_gates_of_all_sizes(others):
    """A row for each end, that is one column of it, with ordinary values beside it or none.  Sigmoids below 2^-126 are nothing."""
    g = torch.zeros((len(ENDS), 128)) if not others else randn(len(ENDS), 128, seed=1, scale=2.0).float()
    u = torch.zeros((len(ENDS), 128)) if not others else randn(len(ENDS), 128, seed=2).float()
    for i, end in enumerate(ENDS):
        g[i, 17] = end
        u[i, 17] = 0.5 if abs(end) < 1e6 else 3.0 / abs(end)           # (products that others can be seen beside)
    g[:, 40], u[:, 40] = -3e38, 0.5                                    # nothing, whatever it meets
    gu = torch.cat((g, u), 1).bfloat16()
    codes, scales, untouched = fenced_quant(len(ENDS), 128)
    fkv.proj_gate(gu.cuda(), codes, scales)
    g, u = gu.double().chunk(2, 1)
    s = torch.sigmoid(g)
    y = g * torch.where(s < 2.0 ** -126, torch.zeros_like(s), s) * u
    assert torch.isfinite(y).all() and (others or (y[:, 40] == 0).all())
    near(scales, torch.maximum(M.block_tops(y, 1) / 448, torch.tensor(2.0 ** -126, dtype=torch.float64)), GATE + 2.0 ** -24)
    held_to_quotients(codes, scales, y, GATE + 2.0 ** -24)
    untouched()


# The result is rounded once, to 2^-24 of it.  The exponential p is off by its instruction's step of fp32 (2 x 2^-24), a rounding, and what its argument
# leaves out (0.72 x 2^-24 at 60, the most here); that counts as p / (1 + p) of the result, and so does a rounding of the quotient's remainder.  What is of the
# second order is below 0.05 x 2^-24 in all.  For gates from 6 on p / (1 + p) is below exp(-6).
@pytest.mark.parametrize("lo,hi,p_counts", [(6.0, 17.0, math.exp(-6)), (-60.0, 60.0, 1.0)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_gate_is_rounded_once(dtype, lo, hi, p_counts):
    """A value to a row: its block's scale is fp32(value / 448), one more rounding."""
    rows = 1 << 17
    gu = torch.zeros((rows, 32))
    gu[:, 5] = lo + (hi - lo) * torch.rand(rows, generator=gen(1))
    gu[:, 16 + 5] = 1e4 * torch.exp2(torch.rand(rows, generator=gen(2)))
    if lo < 0:
        gu[:, 5] = gu[:, 5].clamp(min=-16 if dtype == torch.float16 else lo)
    gu = gu.to(dtype)
    codes, scales = fkv.empty_quant(rows, 16)
    fkv.proj_gate(gu.cuda(), codes, scales)
    y = M.gate(gu)[:, 5].abs()
    off = (scales[:, 0].cpu().double() * 448 / y - 1).abs() * 2.0 ** 24
    fine = y > 0
    print("off by", float(off[fine].max()), "mean", float(off[fine].mean()))
    assert off[fine].max() <= 1 + 1 + p_counts * (2 + 1 + 0.72 + 1) + 0.05
