"""What the projections say of errors that are not theirs."""
import ctypes as C

import pytest
import torch

import paper_2505_13109_amd as fkv
from test_gpu_proj import FREQ, randn

pytestmark = pytest.mark.gpu


def hip():
    """The runtime that this process has loaded."""
    with open("/proc/self/maps") as maps:
        path = next(line.split()[-1] for line in maps if "libamdhip64" in line)
    return C.CDLL(path)


def test_an_earlier_calls_error_stays_the_programs():
    """A call of the program's has failed and its error has not been fetched: it is not the projections', and they leave it where it is."""
    L, H = fkv.lib(), hip()
    x, gu, add = randn(200, 4096, seed=1).cuda(), randn(200, 8192, seed=2).cuda(), randn(200, 4096, seed=3).cuda()
    (c, s), (w, ws) = fkv.empty_quant(200, 4096), fkv.empty_quant(300, 4096, tile=128)
    w1, ws1 = fkv.empty_quant(200, 4096, tile=128)
    out, out1 = (torch.zeros((n, 300), dtype=torch.bfloat16, device="cuda") for n in (200, 1))
    work = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    positions, freq = torch.zeros(200, dtype=torch.int32, device="cuda"), FREQ.cuda()
    q, k, v = (torch.empty((200, n, 128), dtype=torch.bfloat16, device="cuda") for n in (28, 2, 2))
    st = torch.cuda.current_stream().cuda_stream
    need = C.c_size_t()
    assert L.fkv_proj_workspace(200, 300, 4096, C.byref(need)) == 0 and 0 < need.value <= work.numel()
    p = lambda t: t.data_ptr()
    calls = {
        "quant": lambda: L.fkv_proj_quant(0, 1, p(x), 200, 4096, 1, p(c), p(s), st),
        "weights": lambda: L.fkv_proj_quant(0, 1, p(x), 200, 4096, 128, p(w1), p(ws1), st),
        "norm": lambda: L.fkv_proj_norm(0, 1, p(x), p(add), None, 200, 4096, 1e-5, p(x), p(c), p(s), None, st),
        "gate": lambda: L.fkv_proj_gate(0, 1, p(gu), 200, 4096, p(c), p(s), st),
        "rope": lambda: L.fkv_proj_rope(0, 1, p(x), 200, 28, 2, p(positions), 1, None, p(freq), p(q), p(k), p(v), st),
        "few": lambda: L.fkv_proj_matmul(0, 1, p(c), p(s), p(w), p(ws), 1, 300, 4096, p(out1), None, 0, st),
        "parts": lambda: L.fkv_proj_matmul(0, 1, p(c), p(s), p(w), p(ws), 200, 300, 4096, p(out), p(work), work.numel(), st),
    }
    fkv.proj_quant(randn(300, 4096, seed=4).cuda(), w, ws, tile=128)
    torch.cuda.synchronize()
    assert H.hipGetLastError() == 0
    for name, call in calls.items():
        left = H.hipSetDevice(1000)                      # no such device
        assert left != 0 and H.hipPeekAtLastError() == left
        rc = call()
        still = H.hipGetLastError()
        assert (rc, still) == (0, left), name
    torch.cuda.synchronize()
