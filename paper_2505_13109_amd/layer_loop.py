"""A decoder layer stack around the retrieval loop (Sec. 3.2 "Speculative retrieval": selection and recall
overlap the rest of the layer -- attention output projection, FFN, the next layer's QKV projection).

The retrieval step itself is `fkv_decode_step` of the HIP library, unchanged.  Around it this module puts
what a Llama-shaped layer does for one token: RMSNorm, the QKV projection, rotary embedding, the output
projection and a SwiGLU FFN, as plain library GEMVs and elementwise PyTorch ops on the compute stream
(they are context for the loop -- something real for the deferred recall to hide behind and a closed loop in
which the layer's own q, k, v drive the selection -- not a tuned layer).  Weights are random (there are no
checkpoints here); the cached context of each layer is synthetic and loaded by the caller.

`step()` feeds one hidden state per request through all layers.  With `external_qkv` the loop's q, k, v are
taken from the caller (seeded synthetic streams with a set adjacent-step similarity) while the projections
still run and are dropped: that keeps a workload's reuse and correction statistics, which random weights
would not produce.

Over a `PagedCache` the stack decodes the sequences `seqs` (int32 slots on the GPU) of any lengths: every layer appends its keys and
values to the 4-bit cache and attends over all of it.  Lengths, and with them the rotary positions, stay on the device, so
`step()` may be captured into a graph and every replay decodes the next token.

With `weights="fp8"` the weights are kept in 8 bits and everything around the loop runs in the library's own kernels (`projection.py`): the
residual's addition with the norm, the products, rotary positions, the gated activation.  Rotary positions may then have several axes.
"""
from __future__ import annotations

import torch

from .binding import FreeKV
from .paged_cache import PagedCache
from .projection import MAX_AXES, axes_of, empty_quant, proj_gate, proj_matmul, proj_norm, proj_quant, proj_rope


class DecoderStack:
    def __init__(self, fkv: FreeKV | PagedCache, *, seqs: torch.Tensor | None = None, ffn_mult: float = 3.5, seed: int = 7, rope_base: float = 500000.0,
                 copy_stream: torch.cuda.Stream | None = None, weights: str | None = None, rope_sections=None):
        """weights: None, the storage type's 16 bits, or "fp8".  rope_sections (fp8 only): `proj_rope`'s, for positions of several axes."""
        c = fkv.cfg
        if weights not in (None, "fp8"):
            raise ValueError(f"weights: None or 'fp8' are known, not {weights!r}")
        if rope_sections is not None and weights is None:
            raise ValueError("positions of several axes go with weights='fp8'")
        self.axes = 1 if rope_sections is None else axes_of(rope_sections)          # (refuses sections that no step could do with)
        self.fkv, self.seqs = fkv, seqs
        self.paged = isinstance(fkv, PagedCache)
        if self.paged != (seqs is not None):
            raise ValueError("a PagedCache, and nothing else, is decoded with the slots of its sequences")
        self.n_layers, self.batch = c.n_layers, seqs.shape[0] if self.paged else c.batch
        self.n_q, self.n_kv, self.d = c.n_q_heads, c.n_kv_heads, c.head_dim
        self.hidden = self.n_q * self.d
        self.ffn = int(ffn_mult * self.hidden)
        self.dtype = fkv.torch_dtype
        dev = fkv.device
        g = torch.Generator(device=dev).manual_seed(seed)

        def mk(*shape, scale):
            return (torch.randn(*shape, generator=g, device=dev, dtype=torch.float32) * scale).to(self.dtype)

        qkv_out = (self.n_q + 2 * self.n_kv) * self.d
        s_in = self.hidden ** -0.5
        keep = (lambda w: w) if weights is None else self._in_8_bits
        if weights is not None and self.ffn % 16:
            raise ValueError(f"weights='fp8' wants a multiple of 16 for the FFN's width, {ffn_mult} x {self.hidden} gives {self.ffn}")
        self.wqkv = [keep(mk(self.hidden, qkv_out, scale=s_in)) for _ in range(self.n_layers)]
        self.wo = [keep(mk(self.hidden, self.hidden, scale=s_in)) for _ in range(self.n_layers)]
        self.wgu = [keep(mk(self.hidden, 2 * self.ffn, scale=s_in)) for _ in range(self.n_layers)]
        self.wd = [keep(mk(self.ffn, self.hidden, scale=self.ffn ** -0.5)) for _ in range(self.n_layers)]
        self.inv_freq = (rope_base ** (-torch.arange(0, self.d, 2, device=dev, dtype=torch.float32) / self.d))
        self.out = torch.empty((self.n_layers, self.batch, self.n_q, self.d), dtype=self.dtype if self.paged else torch.float32, device=dev)
        self.lens = torch.zeros((self.batch,), dtype=torch.int32, device=dev)
        self.copy_stream = copy_stream
        self.last_qkv = [None] * self.n_layers       # what each layer fed to the loop at the last step (for tests)
        self.weight_bytes_per_layer = (self.hidden * qkv_out + self.hidden * self.hidden + 3 * self.hidden * self.ffn) * (2 if weights is None else 1)
        self.weights, self.sections = weights, rope_sections
        if weights is not None:
            def new(*shape, dtype=self.dtype):
                return torch.empty(shape, dtype=dtype, device=dev)

            self.h8, self.f8 = (empty_quant(self.batch, cols, device=dev) for cols in (self.hidden, self.ffn))
            self.qkv, self.gu, self.y = new(self.batch, qkv_out), new(self.batch, 2 * self.ffn), new(self.batch, self.hidden)
            self.x = new(2, self.batch, self.hidden)         # the stream of a layer, before and behind the attention
            self.positions = new(self.batch, dtype=torch.int32)

    @staticmethod
    def _in_8_bits(w):
        """[in, out] of the storage type -> codes [out, in] and a scale for each 128 x 128."""
        codes, scales = empty_quant(w.shape[1], w.shape[0], tile=128, device=w.device)
        proj_quant(w.T.contiguous(), codes, scales, tile=128)
        return codes, scales

    def _rms(self, x):
        return torch.nn.functional.rms_norm(x, (self.hidden,), eps=1e-5)

    def _rope(self, x, cos, sin):
        """x [batch, heads, d]; rotate pairs (i, i + d/2) by pos * inv_freq[i]."""
        a, b = x[..., : self.d // 2], x[..., self.d // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)

    def step(self, x, external_qkv=None, stream=None, positions=None):
        """x [batch, hidden] -> [batch, hidden].  external_qkv: per layer (q [batch,n_q,d], k, v [batch,n_kv,d]).
        positions (fp8 only): rotary positions of the tokens, [batch] or [axes, batch] int32 on the GPU; None: their places in the sequences, on
        every axis (over a FreeKV context, each layer's own).

        Over a PagedCache the whole step runs on `stream`, behind what the current stream has been given and before what it is given next:
        positions come from the device, so the projections have to follow the cache's calls.  Over a FreeKV context, `stream` is the one that
        its calls are launched on; the rest runs on the current stream, which has to be the same."""
        if self.weights is None and positions is not None:
            raise ValueError("positions of the caller's go with weights='fp8'")
        if self.weights is not None:
            self._refuse_step(x, positions)
        run = self._step if self.weights is None else lambda *a: self._step_in_8_bits(*a, positions)
        here = torch.cuda.current_stream(self.fkv.device) if self.paged and stream is not None else None
        if here is None or stream == here:
            return run(x, external_qkv, stream)
        stream.wait_stream(here)
        with torch.cuda.stream(stream):
            y = run(x, external_qkv, stream)
        here.wait_stream(stream)
        y.record_stream(here)
        return y

    def _step(self, x, external_qkv, stream):
        pos_cached, cos, sin = None, None, None
        if self.paged:
            self.fkv.extend(self.seqs, stream=stream)
            self.fkv.tables(self.seqs, self.lens, stream=stream)
            ang = (self.lens - 1).float()[:, None, None] * self.inv_freq
            cos, sin = ang.cos().to(self.dtype), ang.sin().to(self.dtype)
        for layer in range(self.n_layers):
            pos = None if self.paged else self.fkv.context_len(layer)       # position of the token being appended
            if pos != pos_cached:                               # (the layers of one model share it)
                ang = float(pos) * self.inv_freq
                cos, sin, pos_cached = ang.cos().to(self.dtype), ang.sin().to(self.dtype), pos
            qkv = (self._rms(x) @ self.wqkv[layer]).view(self.batch, self.n_q + 2 * self.n_kv, self.d)
            qk = self._rope(qkv[:, : self.n_q + self.n_kv], cos, sin)       # queries and keys in one go
            q, k = qk[:, : self.n_q].contiguous(), qk[:, self.n_q:].contiguous()
            v = qkv[:, self.n_q + self.n_kv:].contiguous()
            if external_qkv is not None:
                q, k, v = external_qkv[layer]
            self.last_qkv[layer] = (q, k, v)
            if self.paged:
                self.fkv.append(layer, self.seqs, k, v, stream=stream)
                self.fkv.attn(layer, self.seqs, q, self.out[layer], stream=stream)
            else:
                self.fkv.decode_step(layer, q, k, v, self.out[layer], stream=stream, copy_stream=self.copy_stream)
            x = x + self.out[layer].to(self.dtype).view(self.batch, self.hidden) @ self.wo[layer]
            gu = self._rms(x) @ self.wgu[layer]
            x = x + (torch.nn.functional.silu(gu[:, : self.ffn]) * gu[:, self.ffn:]) @ self.wd[layer]
        return x

    def _step_in_8_bits(self, x, external_qkv, stream, positions):
        """The same step, the additions of a layer's two halves in the norms behind them."""
        if self.paged:
            self.fkv.extend(self.seqs, stream=stream)
            self.fkv.tables(self.seqs, self.lens, stream=stream)
        given, place_before = positions, None
        if given is None and self.paged:
            positions = self._on_all_axes(self.lens - 1)
        y = None
        for layer in range(self.n_layers):
            if y is None:
                proj_norm(x, None, *self.h8)
            else:
                proj_norm(x, None, *self.h8, add=y, res=self.x[0])
                x = self.x[0]
            proj_matmul(*self.h8, *self.wqkv[layer], self.qkv)
            if given is None and not self.paged:
                place = self.fkv.context_len(layer)                 # (the layers of one model share it)
                if place != place_before:
                    positions, place_before = self._on_all_axes(torch.full_like(self.positions, place)), place
            # (the step's own, as last_qkv hands them out)
            q, k, v = (torch.empty((self.batch, n, self.d), dtype=self.dtype, device=x.device) for n in (self.n_q, self.n_kv, self.n_kv))
            proj_rope(self.qkv.view(self.batch, self.n_q + 2 * self.n_kv, self.d), positions, self.inv_freq, q, k, v, sections=self.sections)
            if external_qkv is not None:
                q, k, v = external_qkv[layer]
            self.last_qkv[layer] = (q, k, v)
            if self.paged:
                self.fkv.append(layer, self.seqs, k, v, stream=stream)
                self.fkv.attn(layer, self.seqs, q, self.out[layer], stream=stream)
            else:
                self.fkv.decode_step(layer, q, k, v, self.out[layer], stream=stream, copy_stream=self.copy_stream)
            proj_quant(self.out[layer].to(self.dtype).view(self.batch, self.hidden), *self.h8)
            proj_matmul(*self.h8, *self.wo[layer], self.y)
            proj_norm(x, None, *self.h8, add=self.y, res=self.x[1])
            x = self.x[1]
            proj_matmul(*self.h8, *self.wgu[layer], self.gu)
            proj_gate(self.gu, *self.f8)
            proj_matmul(*self.f8, *self.wd[layer], self.y)
            y = self.y
        return x + y

    def _refuse_step(self, x, positions):
        """What a kernel of the step would refuse, before the sequences have a token more."""
        dev = self.inv_freq.get_device()
        if not (isinstance(x, torch.Tensor) and x.dtype is self.dtype and x.shape == (self.batch, self.hidden) and x.get_device() == dev and x.is_contiguous()
                and x.data_ptr() % 16 == 0):
            raise ValueError(f"x: a contiguous {self.dtype} tensor of shape {(self.batch, self.hidden)} on cuda:{dev}, 16-byte aligned, is wanted")
        if positions is None:
            return
        shape = tuple(positions.shape) if isinstance(positions, torch.Tensor) else None
        axes = 1 if shape == (self.batch,) else shape[0] if shape and shape[1:] == (self.batch,) else 0
        if not (self.axes <= axes <= MAX_AXES and positions.dtype is torch.int32 and positions.get_device() == dev and positions.is_contiguous()):
            raise ValueError(f"positions: a contiguous int32 tensor on cuda:{dev} is wanted, [axes, {self.batch}] with {self.axes} to {MAX_AXES} axes"
                             + (f", or [{self.batch}]" if self.axes == 1 else ""))

    def _on_all_axes(self, places):
        """[batch] positions as they are, or the same on each of the axes."""
        return places if self.sections is None else places.expand(self.axes, -1).contiguous()
