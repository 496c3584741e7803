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
