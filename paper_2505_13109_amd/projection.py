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
MAX_AXES = 4
FEW_ROWS = 32                 # up to here a product needs no workspace
CODES = torch.float8_e4m3fn
F32, I32 = torch.float32, torch.int32
_TYPES = {torch.float16: 0, torch.bfloat16: 1}


# A call's kernel is a few microseconds of GPU time and so is the launch, so what is right is told in one expression, with few attribute
# reads and no call in between (1 us less of 7 for a norm of one row); what is wrong is looked up afterwards.
def _refuse(*wanted):
    """Names the first of (name, tensor, types, shape, device) that is not as wanted."""
    for what, t, types, shape, index in wanted:
        if not isinstance(t, torch.Tensor):
            raise FreeKVError(f"{what}: a tensor is wanted, this is {type(t).__name__}")
        if t.dtype in types and tuple(t.shape) == tuple(shape) and t.is_contiguous() and t.get_device() == index and index >= 0:
            continue
        names = " or ".join(str(x).replace("torch.", "") for x in types)
        where = f"cuda:{index}" if index >= 0 else "a GPU"
        raise FreeKVError(f"{what}: a contiguous {names} tensor of shape {tuple(shape)} on {where} is wanted, this is {t.dtype} {tuple(t.shape)} on {t.device}"
                          + ("" if t.is_contiguous() else ", not contiguous"))
    raise FreeKVError("tensors that do not belong together")


def _shape(t, dims):
    """A tensor's shape, or one that it cannot have."""
    return tuple(t.shape) if isinstance(t, torch.Tensor) and t.dim() == dims else (-1,) * dims


def _device(t):
    return t.get_device() if isinstance(t, torch.Tensor) else -1


def _stream(stream, dev):
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _failed(rc, what):
    raise FreeKVError(f"{what}: {rc}: {lib().fkv_proj_last_error().decode()}")


def empty_quant(rows, cols, tile=1, device="cuda"):
    """Codes and scales for [rows, cols] values, not filled; tile: rows that share a scale, 1 or 128."""
    return (torch.empty((rows, cols), dtype=CODES, device=device),
            torch.empty((-(-rows // tile), -(-cols // BLOCK)), dtype=F32, device=device))


def _eight_bits(what, x, dims, dev, codes, scales, rows, cols, tile=1):
    """What _refuse() looks at for values and what they become."""
    return ((what, x, _TYPES, _shape(x, dims), dev), ("codes", codes, (CODES,), (rows, cols), dev),
            ("scales", scales, (F32,), (-(-rows // tile), -(-cols // BLOCK)), dev))


def proj_quant(x, codes, scales, tile=1, stream=None):
    """x [rows, cols] into 8 bits; tile 1: activations, 128: weights."""
    if tile != 1 and tile != BLOCK:
        raise FreeKVError("tile must be 1 or 128 rows")
    rows, cols = shape = _shape(x, 2)
    dev = _device(x)
    try:
        ok = (dev >= 0 and x.dtype in _TYPES and x.is_contiguous() and codes.dtype is CODES and codes.shape == shape and codes.is_contiguous()
              and codes.get_device() == dev and scales.dtype is F32 and scales.shape == (-(-rows // tile), -(-cols // BLOCK)) and scales.is_contiguous()
              and scales.get_device() == dev)
    except AttributeError:       # (what is no tensor)
        ok = False
    if not ok:
        _refuse(*_eight_bits("x", x, 2, dev, codes, scales, rows, cols, tile))
    rc = lib().fkv_proj_quant(dev, _TYPES[x.dtype], x.data_ptr(), rows, cols, tile, codes.data_ptr(), scales.data_ptr(), _stream(stream, dev))
    if rc:
        _failed(rc, "fkv_proj_quant")


def proj_norm(x, weight, codes=None, scales=None, add=None, res=None, out=None, eps=1e-5, stream=None):
    """The norm of x [rows, cols] (with `add`, of their sum, which is written to `res`, or into x where that is None) in 8 bits and / or, to
    `out`, in 16; weight [cols] or None."""
    rows, cols = shape = _shape(x, 2)
    dev = _device(x)
    if add is None and res is not None:
        raise FreeKVError("res: there is no sum without `add`")
    if (codes is None) != (scales is None) or (codes is None and out is None):
        raise FreeKVError("codes and scales, or out, or all of them are wanted")
    try:
        ok = (dev >= 0 and (dtype := x.dtype) in _TYPES and x.is_contiguous()
              and (weight is None or (weight.dtype is dtype and weight.shape == (cols,) and weight.is_contiguous() and weight.get_device() == dev))
              and (codes is None or (codes.dtype is CODES and codes.shape == shape and codes.is_contiguous() and codes.get_device() == dev
              and scales.dtype is F32 and scales.shape == (rows, -(-cols // BLOCK)) and scales.is_contiguous() and scales.get_device() == dev))
              and (add is None or (add.dtype is dtype and add.shape == shape and add.is_contiguous() and add.get_device() == dev))
              and (res is None or (res.dtype is dtype and res.shape == shape and res.is_contiguous() and res.get_device() == dev))
              and (out is None or (out.dtype is dtype and out.shape == shape and out.is_contiguous() and out.get_device() == dev)))
    except AttributeError:       # (what is no tensor)
        ok = False
    if not ok:
        first, *eight = _eight_bits("x", x, 2, dev, codes, scales, rows, cols)
        types = (x.dtype,) if isinstance(x, torch.Tensor) else ()
        given = [(what, t, types, s, dev) for what, t, s in (("weight", weight, (cols,)), ("add", add, shape), ("res", res, shape), ("out", out, shape)) if t is not None]
        _refuse(first, *(eight if codes is not None else ()), *given)
    at = x.data_ptr()
    rc = lib().fkv_proj_norm(dev, _TYPES[dtype], at, None if add is None else add.data_ptr(), None if weight is None else weight.data_ptr(), rows, cols, eps,
                             None if add is None else at if res is None else res.data_ptr(), None if codes is None else codes.data_ptr(),
                             None if codes is None else scales.data_ptr(), None if out is None else out.data_ptr(), _stream(stream, dev))
    if rc:
        _failed(rc, "fkv_proj_norm")


def proj_gate(gu, codes, scales, stream=None):
    """silu(g) u of gu = [g, u], [rows, 2 cols], into 8 bits."""
    rows, both = _shape(gu, 2)
    cols, dev = both // 2, _device(gu)
    try:
        ok = (dev >= 0 and not both & 1 and gu.dtype in _TYPES and gu.is_contiguous() and codes.dtype is CODES and codes.shape == (rows, cols) and codes.is_contiguous()
              and codes.get_device() == dev and scales.dtype is F32 and scales.shape == (rows, -(-cols // BLOCK)) and scales.is_contiguous() and scales.get_device() == dev)
    except AttributeError:       # (what is no tensor)
        ok = False
    if not ok:
        if both & 1 and both > 0:
            raise FreeKVError("gu: as many columns of the gate as of the other are wanted")
        _refuse(*_eight_bits("gu", gu, 2, dev, codes, scales, rows, cols))
    rc = lib().fkv_proj_gate(dev, _TYPES[gu.dtype], gu.data_ptr(), rows, cols, codes.data_ptr(), scales.data_ptr(), _stream(stream, dev))
    if rc:
        _failed(rc, "fkv_proj_gate")


def proj_rope(qkv, positions, freq, q, k, v, sections=None, stream=None):
    """qkv [rows, n_q + 2 n_kv, 128] apart into q, k, v, q and k turned by positions ([rows] or [axes, rows] int32) times freq ([64] fp32).
    sections: how many pairs of channels each axis has, one axis behind the other (64 in all), or each pair's axis (64 numbers); None: all the
    first axis'.  positions and freq may begin at any of their numbers; the other tensors on 16 bytes, as everywhere here."""
    rows, heads, d = _shape(qkv, 3)
    n_q, n_kv = (q.shape[1], k.shape[1]) if isinstance(q, torch.Tensor) and isinstance(k, torch.Tensor) and q.dim() == k.dim() == 3 else (0, 0)
    dev = _device(qkv)
    axes = positions.shape[0] if isinstance(positions, torch.Tensor) and positions.dim() == 2 else 0
    try:
        ok = (dev >= 0 and d == 128 and n_q + 2 * n_kv == heads and (dtype := qkv.dtype) in _TYPES and qkv.is_contiguous()
              and q.dtype is dtype and q.shape == (rows, n_q, 128) and q.is_contiguous() and q.get_device() == dev
              and k.dtype is dtype and k.shape == (kv := (rows, n_kv, 128)) and k.is_contiguous() and k.get_device() == dev
              and isinstance(v, torch.Tensor) and v.dtype is dtype and v.shape == kv and v.is_contiguous() and v.get_device() == dev
              and isinstance(positions, torch.Tensor) and positions.dtype is I32 and positions.shape == ((axes, rows) if axes else (rows,)) and positions.is_contiguous()
              and positions.get_device() == dev
              and isinstance(freq, torch.Tensor) and freq.dtype is F32 and freq.shape == (64,) and freq.is_contiguous() and freq.get_device() == dev)
    except AttributeError:       # (what is no tensor)
        ok = False
    if not ok:
        types = (qkv.dtype,) if isinstance(qkv, torch.Tensor) else ()
        _refuse(("qkv", qkv, _TYPES, (rows, n_q + 2 * n_kv, 128), dev), ("q", q, types, (rows, n_q, 128), dev), ("k", k, types, (rows, n_kv, 128), dev),
                ("v", v, types, (rows, n_kv, 128), dev), ("positions", positions, (I32,), (axes, rows) if axes else (rows,), dev), ("freq", freq, (F32,), (64,), dev))
    axes = axes or 1
    at, by = positions.data_ptr(), freq.data_ptr()
    if (at | by) & 15:           # (one step's of a tensor of all steps', say: the stream takes a copy to where the entry point wants it)
        with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
            positions, freq = (t.clone() if t.data_ptr() & 15 else t for t in (positions, freq))
        at, by = positions.data_ptr(), freq.data_ptr()
    rc = lib().fkv_proj_rope(dev, _TYPES[dtype], qkv.data_ptr(), rows, n_q, n_kv, at, axes, None if sections is None else _axis_of(sections, axes),
                             by, q.data_ptr(), k.data_ptr(), v.data_ptr(), _stream(stream, dev))
    if rc:
        _failed(rc, "fkv_proj_rope")


_axes_known = {}


def _axis_of(sections, axes):
    """The C array of each pair's axis (arrays of the few sections that a program has are kept)."""
    if sections is None:
        return None
    key = (*sections, axes)
    known = _axes_known.get(key)
    if known is None:
        given = key[:-1]
        each = given if len(given) == 64 else tuple(a for a, n in enumerate(given) for _ in range(n))
        if len(each) != 64 or any(n < 0 for n in given) or (len(given) != 64 and len(given) > axes) or max(each) >= axes:
            raise FreeKVError(f"sections: parts of 64 pairs for {axes} axes, or 64 axes, are wanted, these are {given}")
        if len(_axes_known) >= 64:
            _axes_known.clear()
        known = _axes_known[key] = (C.c_int32 * 64)(*each)
    return known


def axes_of(sections):
    """How many axes' positions `sections` need; refuses what proj_rope would."""
    each = tuple(sections)
    axes = 1 + max(each) if len(each) == 64 else len(each)
    if axes > MAX_AXES:
        raise FreeKVError(f"sections: {axes} axes, {MAX_AXES} are the most")
    _axis_of(each, axes)
    return axes


def proj_matmul(codes, scales, w, w_scales, out, stream=None):
    """out [rows, n] = x [rows, cols] w [n, cols]^T, both in 8 bits: scales [rows, ceil(cols / 128)], w_scales [ceil(n / 128), ceil(cols / 128)]."""
    rows, n = _shape(out, 2)
    cols = _shape(codes, 2)[1]
    dev, blocks = _device(out), -(-cols // BLOCK)
    try:
        ok = (dev >= 0 and out.dtype in _TYPES and out.is_contiguous()
              and codes.dtype is CODES and codes.shape == (rows, cols) and codes.is_contiguous() and codes.get_device() == dev
              and scales.dtype is F32 and scales.shape == (rows, blocks) and scales.is_contiguous() and scales.get_device() == dev
              and w.dtype is CODES and w.shape == (n, cols) and w.is_contiguous() and w.get_device() == dev
              and w_scales.dtype is F32 and w_scales.shape == (-(-n // BLOCK), blocks) and w_scales.is_contiguous() and w_scales.get_device() == dev)
    except AttributeError:       # (what is no tensor)
        ok = False
    if not ok:
        _refuse(("out", out, _TYPES, (rows, n), dev), ("codes", codes, (CODES,), (rows, cols), dev), ("scales", scales, (F32,), (rows, blocks), dev),
                ("w", w, (CODES,), (n, cols), dev), ("w_scales", w_scales, (F32,), (-(-n // BLOCK), blocks), dev))
    L, work, size = lib(), None, 0
    if rows > FEW_ROWS:
        need = C.c_size_t()
        if L.fkv_proj_workspace(rows, n, cols, C.byref(need)) == 0 and need.value:
            size = need.value
            with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):     # (the stream's own memory: it is free again behind this call's work)
                work = torch.empty(size, dtype=torch.uint8, device=out.device)
    rc = L.fkv_proj_matmul(dev, _TYPES[out.dtype], codes.data_ptr(), scales.data_ptr(), w.data_ptr(), w_scales.data_ptr(), rows, n, cols, out.data_ptr(),
                           None if work is None else work.data_ptr(), size, _stream(stream, dev))
    if rc:
        _failed(rc, "fkv_proj_matmul")
