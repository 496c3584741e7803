"""Binding of include/freekv_proj.h: a decoder layer's projections in 8 bits.  Argument marshalling and checks; formulas are in the
header.  Functions carry the names of the C entry points they call and write into tensors of the caller's, to be kept until the stream
is done with them; `stream` None is the current stream of the tensors' device.

    codes, scales = empty_quant(rows, cols)            # float8_e4m3fn [rows, cols], fp32 [rows, ceil(cols / 128)]
    proj_norm(x, weight, codes, scales, add=y)         # x += y, the norm of that in 8 bits
    proj_matmul(codes, scales, w, w_scales, out)       # w, w_scales: proj_quant(..., tile=128)
"""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

from .binding import FreeKVError, lib

BLOCK = 128
FEW_ROWS = 32                 # up to here a product needs no workspace
CODES = torch.float8_e4m3fn
_TYPES = {torch.float16: 0, torch.bfloat16: 1}
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else None


def _refuse(t, what, dtype, shape, index):
    where = f"cuda:{index}" if index >= 0 else "a GPU"
    if not isinstance(t, torch.Tensor):
        raise FreeKVError(f"{what}: a tensor is wanted, this is {type(t).__name__}")
    raise FreeKVError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} on {where} is wanted, this is {t.dtype} {tuple(t.shape)} on {t.device}"
                      + ("" if t.is_contiguous() else ", not contiguous"))


# (calls are a few microseconds of GPU time each, so what is right is told with few attribute reads)
def _at(t, what, dtype, shape, index):
    if t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous():
        return t.data_ptr()
    _refuse(t, what, dtype, shape, index)


def _first(x, what, dims):
    """Address, type code, type and device of the tensor that a call's shapes go by."""
    if not isinstance(x, torch.Tensor) or x.dtype not in _TYPES or x.dim() != dims or not x.is_contiguous():
        raise FreeKVError(f"{what}: a contiguous fp16 or bf16 tensor of {dims} dimensions on a GPU is wanted, this is "
                          + (f"{x.dtype} {tuple(x.shape)} on {x.device}" if isinstance(x, torch.Tensor) else type(x).__name__))
    index = x.get_device()
    if index < 0:
        raise FreeKVError(f"{what}: the projections are HIP kernels, this tensor is on {x.device}")
    return x.data_ptr(), _TYPES[x.dtype], x.dtype, index


def _run(fn, what, index, *args, stream):
    rc = fn(index, *args, _raw_stream(index) if stream is None else stream.cuda_stream)
    if rc:
        raise FreeKVError(f"{what}: {rc}: {lib().fkv_proj_last_error().decode()}")


def empty_quant(rows, cols, tile=1, device="cuda"):
    """Codes and scales for [rows, cols] values, not filled; tile: rows that share a scale, 1 or 128."""
    return (torch.empty((rows, cols), dtype=CODES, device=device),
            torch.empty((-(-rows // tile), -(-cols // BLOCK)), dtype=torch.float32, device=device))


def proj_quant(x, codes, scales, tile=1, stream=None):
    """x [rows, cols] into 8 bits; tile 1: activations, 128: weights."""
    at, t, _, dev = _first(x, "x", 2)
    if tile != 1 and tile != BLOCK:
        raise FreeKVError("tile must be 1 or 128 rows")
    rows, cols = x.shape
    _run(lib().fkv_proj_quant, "fkv_proj_quant", dev, t, at, rows, cols, tile, _at(codes, "codes", CODES, (rows, cols), dev),
         _at(scales, "scales", torch.float32, (-(-rows // tile), -(-cols // BLOCK)), dev), stream=stream)


def proj_norm(x, weight, codes=None, scales=None, add=None, res=None, out=None, eps=1e-5, stream=None):
    """The norm of x [rows, cols] (with `add`, of their sum, which is written to `res`, or into x where that is None) in 8 bits and / or, to
    `out`, in 16; weight [cols] or None."""
    at, t, dtype, dev = _first(x, "x", 2)
    rows, cols = x.shape
    if add is None:
        if res is not None:
            raise FreeKVError("res: there is no sum without `add`")
        a = r = None
    else:
        a, r = _at(add, "add", dtype, (rows, cols), dev), at if res is None else _at(res, "res", dtype, (rows, cols), dev)
    if (codes is None) != (scales is None) or (codes is None and out is None):
        raise FreeKVError("codes and scales, or out, or all of them are wanted")
    _run(lib().fkv_proj_norm, "fkv_proj_norm", dev, t, at, a, None if weight is None else _at(weight, "weight", dtype, (cols,), dev), rows, cols, eps, r,
         None if codes is None else _at(codes, "codes", CODES, (rows, cols), dev),
         None if scales is None else _at(scales, "scales", torch.float32, (rows, -(-cols // BLOCK)), dev),
         None if out is None else _at(out, "out", dtype, (rows, cols), dev), stream=stream)


def proj_gate(gu, codes, scales, stream=None):
    """silu(g) u of gu = [g, u], [rows, 2 cols], into 8 bits."""
    at, t, _, dev = _first(gu, "gu", 2)
    rows, cols = gu.shape
    if cols % 2:
        raise FreeKVError("gu: as many columns of the gate as of the other are wanted")
    cols //= 2
    _run(lib().fkv_proj_gate, "fkv_proj_gate", dev, t, at, rows, cols, _at(codes, "codes", CODES, (rows, cols), dev),
         _at(scales, "scales", torch.float32, (rows, -(-cols // BLOCK)), dev), stream=stream)


def proj_rope(qkv, positions, freq, q, k, v, sections=None, stream=None):
    """qkv [rows, n_q + 2 n_kv, 128] apart into q, k, v, q and k turned by positions ([rows] or [axes, rows] int32) times freq ([64] fp32).
    sections: how many pairs of channels each axis has, one axis behind the other (64 in all), or each pair's axis (64 numbers); None: all the
    first axis'."""
    at, t, dtype, dev = _first(qkv, "qkv", 3)
    rows, heads, d = qkv.shape
    n_q, n_kv = (x.shape[1] if isinstance(x, torch.Tensor) and x.dim() == 3 else 0 for x in (q, k))
    if d != 128 or n_q + 2 * n_kv != heads:
        raise FreeKVError(f"qkv: [rows, {n_q} + 2 x {n_kv}, 128] is wanted for this q and k, this is {tuple(qkv.shape)}")
    axes = positions.shape[0] if positions.dim() == 2 else 1
    _run(lib().fkv_proj_rope, "fkv_proj_rope", dev, t, at, rows, n_q, n_kv,
         _at(positions, "positions", torch.int32, (axes, rows) if positions.dim() == 2 else (rows,), dev), axes, _axis_of(sections, axes),
         _at(freq, "freq", torch.float32, (64,), dev), _at(q, "q", dtype, (rows, n_q, 128), dev), _at(k, "k", dtype, (rows, n_kv, 128), dev),
         _at(v, "v", dtype, (rows, n_kv, 128), dev), stream=stream)


_axes_known = {}


def _axis_of(sections, axes):
    """The C array of each pair's axis (arrays of the few sections that a program has are kept)."""
    if sections is None:
        return None
    key = (tuple(sections), axes)
    if key not in _axes_known:
        given = key[0]
        each = given if len(given) == 64 else tuple(a for a, n in enumerate(given) for _ in range(n))
        if len(each) != 64 or any(n < 0 for n in given) or (len(given) != 64 and len(given) > axes) or max(each) >= axes:
            raise FreeKVError(f"sections: parts of 64 pairs for {axes} axes, or 64 axes, are wanted, these are {given}")
        if len(_axes_known) >= 64:
            _axes_known.clear()
        _axes_known[key] = (C.c_int32 * 64)(*each)
    return _axes_known[key]


def proj_matmul(codes, scales, w, w_scales, out, stream=None):
    """out [rows, n] = x [rows, cols] w [n, cols]^T, both in 8 bits: scales [rows, ceil(cols / 128)], w_scales [ceil(n / 128), ceil(cols / 128)]."""
    at, t, _, dev = _first(out, "out", 2)
    rows, n = out.shape
    cols = codes.shape[1] if codes.dim() == 2 else -1
    blocks = -(-cols // BLOCK)
    x, xs = _at(codes, "codes", CODES, (rows, cols), dev), _at(scales, "scales", torch.float32, (rows, blocks), dev)
    ww, ws = _at(w, "w", CODES, (n, cols), dev), _at(w_scales, "w_scales", torch.float32, (-(-n // BLOCK), blocks), dev)
    work, size = None, 0
    if rows > FEW_ROWS:
        need = C.c_size_t()
        if lib().fkv_proj_workspace(rows, n, cols, C.byref(need)) == 0 and need.value:
            size = need.value
            with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):     # (the stream's own memory: it is free again behind this call's work)
                work = torch.empty(size, dtype=torch.uint8, device=out.device)
    _run(lib().fkv_proj_matmul, "fkv_proj_matmul", dev, t, x, xs, ww, ws, rows, n, cols, at, None if work is None else work.data_ptr(), size, stream=stream)
