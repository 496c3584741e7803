"""Binding of include/freekv_cache.h: a paged cache in 4 bits for sequences of any lengths, the attention over it, and what
forks, copies, compacts and frees its pages.  Argument marshalling and checks; shapes, rows and token offsets are described in
the header.

    cache = PagedCache(n_layers=32, n_q_heads=32, n_kv_heads=8, max_seqs=64, max_ctx=32768, n_pages=20000)
    cache.extend(seqs, cu)                             # seqs [rows] int32 slots, cu [rows + 1] int32 token offsets (None: one each)
    for layer in range(32):
        cache.append(layer, seqs, k, v, cu)            # [tokens, n_kv, 128]
        cache.attn(layer, seqs, q, out)                # [rows, n_q, 128], one query token a row
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import CacheConfig, FreeKVError, _ptr, lib


class PagedCache:
    """One cache.  Methods carry the names of the C entry points they call; `stream` None is the current stream of the cache's device.
    Tensors are the caller's, to be kept until the stream is done with them."""

    def __init__(self, *, n_layers, n_q_heads, n_kv_heads, max_seqs, max_ctx, n_pages, dtype="bf16", head_dim=128, page_size=32, device="cuda:0"):
        self._h = C.c_void_p()
        self.L = lib()
        self.cfg = CacheConfig(n_layers, n_q_heads, n_kv_heads, head_dim, page_size, max_seqs, max_ctx, n_pages, {"fp16": 0, "bf16": 1}[dtype])
        self.dtype = dtype
        self.torch_dtype = torch.float16 if dtype == "fp16" else torch.bfloat16
        self.device = torch.device(device)
        self.max_pages = max_ctx // page_size
        need = C.c_size_t()
        rc = self.L.fkv_cache_arena_bytes(C.byref(self.cfg), C.byref(need))
        if rc:
            raise FreeKVError(f"fkv_cache_arena_bytes: {rc}: {self.L.fkv_cache_last_error(None).decode()}")
        if self.device.type != "cuda":
            raise FreeKVError(f"device: a cache is on a GPU, not on {self.device}")
        if not torch.cuda.is_available():
            raise FreeKVError("no GPU: the cache's operators are HIP kernels")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self.dev_bytes = need.value
        self.dev_arena = torch.empty(self.dev_bytes, dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self.device):
            rc = self.L.fkv_cache_create(C.byref(self.cfg), _ptr(self.dev_arena), self.dev_bytes, C.byref(self._h))
        if rc:
            raise FreeKVError(f"fkv_cache_create: {rc}: {self.L.fkv_cache_last_error(None).decode()}")

    # -- plumbing ------------------------------------------------------------
    def _check(self, rc, what):
        if rc:
            raise FreeKVError(f"{what}: {rc}: {self.L.fkv_cache_last_error(self._h).decode()}")

    def _stream(self, stream):
        return torch._C._cuda_getCurrentRawStream(self._index) if stream is None else stream.cuda_stream

    # (a decode step's calls are a few microseconds of GPU time each, so what is right is told with few attribute reads)
    def _tensor(self, t, what, dtype, shape):
        if t.dtype is dtype and t.shape == shape and t.get_device() == self._index and t.is_contiguous():
            return t.data_ptr()
        raise FreeKVError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device} is wanted, this is {t.dtype} {tuple(t.shape)} on {t.device}"
                          + ("" if t.is_contiguous() else ", not contiguous"))

    def _rows(self, seqs, cu=None, what="seqs"):
        n = seqs.shape[0] if seqs.dim() == 1 else -1
        at = self._tensor(seqs, what, torch.int32, (n,))
        return at, n, None if cu is None else self._tensor(cu, "cu", torch.int32, (n + 1,))

    def _kv(self, k, v):
        shape = (k.shape[0] if k.dim() else 0, self.cfg.n_kv_heads, self.cfg.head_dim)
        return self._tensor(k, "k", self.torch_dtype, shape), self._tensor(v, "v", self.torch_dtype, shape), shape[0]

    def close(self):
        if self._h:
            self.L.fkv_cache_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- entry points ---------------------------------------------------------
    def extend(self, seqs, cu=None, stream=None):
        at, n, cu = self._rows(seqs, cu)
        self._check(self.L.fkv_cache_extend(self._h, at, n, cu, self._stream(stream)), "fkv_cache_extend")

    def append(self, layer, seqs, k, v, cu=None, stream=None):
        at, n, cu = self._rows(seqs, cu)
        k, v, tokens = self._kv(k, v)
        self._check(self.L.fkv_cache_append(self._h, layer, at, n, cu, k, v, tokens, self._stream(stream)), "fkv_cache_append")

    def attn(self, layer, seqs, q, out, pages=None, sink=0, window=0, stream=None):
        """pages [rows, n_kv, n_list] int32: the full pages to attend per KV head, next to `sink` and `window` tokens' and the open one."""
        at, n, _ = self._rows(seqs)
        shape = (n, self.cfg.n_q_heads, self.cfg.head_dim)
        q, o = self._tensor(q, "q", self.torch_dtype, shape), self._tensor(out, "out", self.torch_dtype, shape)
        n_list = 0
        if pages is not None:
            n_list = pages.shape[-1]
            pages = self._tensor(pages, "pages", torch.int32, (n, self.cfg.n_kv_heads, n_list))
            if n_list == 0:
                pages = at               # (an empty list has no address of its own, and none of its entries is read)
        elif sink or window:
            raise FreeKVError("attn: sink and window need a page list")
        self._check(self.L.fkv_cache_attn(self._h, layer, at, n, q, pages, n_list, sink, window, o, self._stream(stream)), "fkv_cache_attn")

    def read(self, layer, seqs, k, v, cu=None, stream=None):
        at, n, cu = self._rows(seqs, cu)
        k, v, tokens = self._kv(k, v)
        self._check(self.L.fkv_cache_read(self._h, layer, at, n, cu, k, v, tokens, self._stream(stream)), "fkv_cache_read")

    def fork(self, src, dst, stream=None):
        at, n, _ = self._rows(src, what="src")
        to = self._tensor(dst, "dst", torch.int32, (n,))
        self._check(self.L.fkv_cache_fork(self._h, at, to, n, self._stream(stream)), "fkv_cache_fork")

    def copy(self, src, dst, to=None, stream=None):
        """Into `to`, another cache (None: this one)."""
        to = self if to is None else to
        at, n, _ = self._rows(src, what="src")
        into = to._tensor(dst, "dst", torch.int32, (n,))
        to._check(self.L.fkv_cache_copy(self._h, at, to._h, into, n, self._stream(stream)), "fkv_cache_copy")

    def free(self, seqs, stream=None):
        at, n, _ = self._rows(seqs)
        self._check(self.L.fkv_cache_free(self._h, at, n, self._stream(stream)), "fkv_cache_free")

    def compact(self, stream=None):
        self._check(self.L.fkv_cache_compact(self._h, self._stream(stream)), "fkv_cache_compact")

    def tables(self, seqs, lens, pages=None, stream=None):
        """lens [rows], pages [rows, max_ctx // 32] int32 (None: the lengths alone)"""
        at, n, _ = self._rows(seqs)
        lens = self._tensor(lens, "lens", torch.int32, (n,))
        pages = None if pages is None else self._tensor(pages, "pages", torch.int32, (n, self.max_pages))
        self._check(self.L.fkv_cache_tables(self._h, at, n, lens, pages, self._stream(stream)), "fkv_cache_tables")

    def health(self):
        """Raises if the device refused something since the last call (blocking)."""
        self._check(self.L.fkv_cache_health(self._h), "fkv_cache_health")

    def used_pages(self):
        """Pages of the pool that are in use (blocking)."""
        n = self.L.fkv_cache_used_pages(self._h)
        if n < 0:
            self._check(n, "fkv_cache_used_pages")
        return n
