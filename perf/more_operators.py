"""Performance cases of a decoder layer's projections in 8 bits: what puts activations and weights into e4m3 with scales, the
product of the two, and the rotary positions between the product and the cache.

Values in 8 bits are e4m3 codes (largest 448) with an fp32 scale for each block of 128 columns, of one row (activations) or of
128 rows (weights):

    scale = max(fp32(max |x| / 448), 2^-126)         over the block
    code  = e4m3(fp32(x / scale))                    both rounded to nearest, ties to even

The norm of s with weights w, s_c w_c r with r = 1 / sqrt(mean s^2 + eps), has the codes of the products s_c w_c, which fp32 holds
exactly, and their scales times r: what is next to a border is decided by the inputs alone.

A case is a dict.  kind is
  "quant"    values [rows, cols] into 8 bits; `tile` rows share a scale: 1 for activations, 128 for weights
  "norm"     the residual's addition, the root-mean-square norm of the sum, and that in 8 bits
  "gate"     silu(gate) * up of [rows, 2 cols], in 8 bits
  "rope"     q, k, v [rows, heads, 128] out of the packed product, q and k turned by positions of `axes` axes up to `far`
  "matmul"   x [rows, cols] times w [n, cols], both in 8 bits, into 16
Head dimension is the library's only one, 128.
"""
import math

import torch

own = False

HEAD_DIM, BLOCK, TOP, LEAST = 128, 128, 448.0, 2.0 ** -126
EPS, ROPE_BASE = 1e-5, 500000.0
OUTLIER_SCALE = 8.0                                       # activations have a few large channels
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _case(name, kind, rows, dtype="bf16", **kw):
    return dict(name=name, kind=kind, rows=rows, dtype=dtype, **kw)


def listed():
    return [
        # the outputs of 32 requests' attention, 32 heads, on their way to the output projection
        _case("quant_32_rows", "quant", 32, cols=4096, tile=1),
        # weights as a program starts: gate and up of a 4096-wide layer
        _case("quant_weights", "quant", 28672, cols=4096, tile=128),
        # the smallest call: one fp16 token of a 28-head layer; launch and latency count
        _case("norm_1_row", "norm", 1, "fp16", cols=3584),
        # 4096 tokens of prompts, 64 heads
        _case("norm_4096_rows", "norm", 4096, cols=8192),
        # one step of 33 requests; the width that 3.5 x 28 heads come to
        _case("gate_33_rows", "gate", 33, cols=12544),
        # 4096 tokens of prompts
        _case("gate_4096_rows", "gate", 4096, cols=14336),
        # one token, 32/8 heads, one axis, fp16, far into a long context
        _case("rope_1_row", "rope", 1, "fp16", n_q=32, n_kv=8, axes=1, far=131072),
        # 16381 tokens of prompts with images, 28/4 heads, three axes
        _case("rope_16381_rows_3_axes", "rope", 16381, n_q=28, n_kv=4, axes=3, far=32768),
        # one token through q, k, v of a 28/4-head layer: latency, and the weights' bytes
        _case("matmul_1_row", "matmul", 1, "fp16", cols=3584, n=4608),
        # a decode step of 32 requests, gate and up of a 4096-wide layer: the weights' bytes
        _case("matmul_32_rows", "matmul", 32, cols=4096, n=28672),
        # a batch of 203, down from a width that is no multiple of 128
        _case("matmul_203_rows", "matmul", 203, cols=11056, n=4096),
        # 4096 tokens of prompts, gate and up: the matrix cores
        _case("matmul_4096_rows", "matmul", 4096, cols=4096, n=28672),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quant", "norm", "gate", "rope", "matmul", "matmul", "matmul"])
    dtype = rng.choice(["fp16", "bf16", "bf16"])
    if kind == "rope":
        n_kv = rng.choice([1, 2, 4, 8, 8])
        return dict(kind=kind, rows=_log_int(rng, 1, 16384), dtype=dtype, n_q=n_kv * rng.randint(1, 8), n_kv=n_kv, axes=rng.randint(1, 4),
                    far=_log_int(rng, 100, 4 << 20))
    cols = 16 * _log_int(rng, 4, 1792)
    if kind == "matmul":
        n = _log_int(rng, 16, 28672)
        rows = _log_int(rng, 1, max(1, min(4096, (4096 * 28672 * 4096) // (cols * n))))
        return dict(kind=kind, rows=rows, dtype=dtype, cols=cols, n=n)
    case = dict(kind=kind, rows=_log_int(rng, 1, max(1, min(16384, (50 << 20) // cols))), dtype=dtype, cols=cols)
    if kind == "quant":
        case["tile"] = rng.choice([1, 128])
    return case


# ---- what the cases are made of -----------------------------------------------------------------

def _generator(seed, what):
    return torch.Generator(device="cuda").manual_seed(((seed & 0xffffffff) * 1000003 + what + 1) & 0x7fffffffffff)


def _activations(rows, cols, seed, what):
    """fp32, normal, about one channel in 64 eight times larger."""
    g = _generator(seed, what)
    scale = torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 64, OUTLIER_SCALE, 1.0)
    return torch.randn((rows, cols), generator=g, device="cuda") * scale


def _weights(rows, cols, seed, what):
    """fp32, normal, rows of somewhat different sizes."""
    g = _generator(seed, what)
    size = torch.exp(0.3 * torch.randn((rows, 1), generator=g, device="cuda")) * cols ** -0.5
    return torch.randn((rows, cols), generator=g, device="cuda") * size


def _sections(axes):
    """Pairs of channels for each axis, 64 in all: a quarter for time, the rest in equal parts, as heights and widths have."""
    if axes == 1:
        return [HEAD_DIM // 2]
    rest = (HEAD_DIM // 2 - 16) // (axes - 1)
    return [HEAD_DIM // 2 - rest * (axes - 1)] + [rest] * (axes - 1)


def prepare(case, seed):
    kind, rows, dt = case["kind"], case["rows"], TYPES[case["dtype"]]
    st = dict(case=case)
    if kind == "rope":
        n_q, n_kv, axes = case["n_q"], case["n_kv"], case["axes"]
        g = _generator(seed, 1)
        st["qkv"] = torch.randn((rows, n_q + 2 * n_kv, HEAD_DIM), generator=g, device="cuda").to(dt)
        # tokens one behind the other; the axes behind the first walk over pictures of 24 x 32 patches
        at = case["far"] - rows + torch.arange(rows, device="cuda") if case["far"] >= rows else torch.arange(rows, device="cuda")
        begin = torch.randint(0, 768, (), generator=g, device="cuda")
        patch = (torch.arange(rows, device="cuda") + begin) % 768
        walks = [at, at - patch + patch // 32, at - patch + patch % 32, at // 2]
        st["positions"] = torch.stack([w.clamp(min=0) for w in walks[:axes]]).to(torch.int32)
        half = torch.arange(0, HEAD_DIM, 2, dtype=torch.float64, device="cuda") / HEAD_DIM
        st["freq"] = (ROPE_BASE ** -half).float()
        st["sections"] = _sections(axes)
        st["q"], st["k"], st["v"] = (torch.empty((rows, n, HEAD_DIM), dtype=dt, device="cuda") for n in (n_q, n_kv, n_kv))
        return st
    cols = case["cols"]
    blocks = -(-cols // BLOCK)
    if kind == "matmul":
        n = case["n"]
        st["codes"], st["scales"] = _in_8_bits(_activations(rows, cols, seed, 1).to(dt).float(), 1)
        st["w"], st["w_scales"] = _in_8_bits(_weights(n, cols, seed, 2).to(dt).float(), BLOCK)
        st["out"] = torch.empty((rows, n), dtype=dt, device="cuda")
        return st
    tile = case.get("tile", 1)
    st["codes"] = torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device="cuda")
    st["scales"] = torch.empty((-(-rows // tile), blocks), dtype=torch.float32, device="cuda")
    if kind == "quant":
        st["x"] = (_weights if tile > 1 else _activations)(rows, cols, seed, 1).to(dt)
    elif kind == "norm":
        st["x"], st["add"] = (_activations(rows, cols, seed, k).to(dt) for k in (1, 2))
        st["weight"] = (1.0 + 0.2 * torch.randn(cols, generator=_generator(seed, 3), device="cuda")).to(dt)
        st["res"] = torch.empty((rows, cols), dtype=dt, device="cuda")
    else:
        st["gu"] = torch.cat([_activations(rows, cols, seed, k) for k in (1, 2)], 1).to(dt)
    return st


# ---- the plain form: elementary operations in 32 bits -----------------------------------------------

def _blocks(y, tile):
    """y [rows, cols] as [row blocks, tile, column blocks, 128], zeros behind the ends."""
    rows, cols = y.shape
    y = torch.nn.functional.pad(y, (0, -cols % BLOCK, 0, -rows % tile))
    return y.view(-1, tile, y.shape[1] // BLOCK, BLOCK)


def _in_8_bits(y, tile):
    rows, cols = y.shape
    y = _blocks(y, tile)
    scales = (y.abs().amax((1, 3), keepdim=True).double() / TOP).float().clamp(min=LEAST)
    codes = (y / scales).to(torch.float8_e4m3fn)
    return codes.view(codes.shape[0] * tile, -1)[:rows, :cols].contiguous(), scales[:, 0, :, 0].contiguous()


def _values(codes, scales, tile):
    """fp32 values that codes stand for."""
    rows, cols = codes.shape
    y = _blocks(codes.float(), tile) * scales[:, None, :, None]
    return y.view(y.shape[0] * tile, -1)[:rows, :cols]


def _run_plain(st):
    case, kind = st["case"], st["case"]["kind"]
    if kind == "quant":
        return dict(zip(("codes", "scales"), _in_8_bits(st["x"].float(), case["tile"])))
    if kind == "norm":
        res = (st["x"].float() + st["add"].float()).to(st["x"].dtype)
        s = res.float()
        codes, scales = _in_8_bits(s * st["weight"].float(), 1)
        return {"codes": codes, "scales": scales * torch.rsqrt((s * s).mean(1, keepdim=True) + EPS), "res": res}
    if kind == "gate":
        g, u = st["gu"].float().chunk(2, 1)
        return dict(zip(("codes", "scales"), _in_8_bits(g / (1.0 + torch.exp(-g)) * u, 1)))
    if kind == "rope":
        n_q, n_kv, half = case["n_q"], case["n_kv"], HEAD_DIM // 2
        axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"), torch.tensor(st["sections"], device="cuda"), output_size=half)
        angle = st["positions"].double().T[:, axis] * st["freq"].double()          # far positions: in 64 bits
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        x = st["qkv"][:, :n_q + n_kv].float()
        a, b = x[..., :half], x[..., half:]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1).to(st["qkv"].dtype)
        return {"q": y[:, :n_q].contiguous(), "k": y[:, n_q:].contiguous(), "v": st["qkv"][:, n_q + n_kv:].contiguous()}
    x, w = _values(st["codes"], st["scales"], 1), _values(st["w"], st["w_scales"], BLOCK)
    return {"out": torch.matmul(x, w.T).to(st["out"].dtype)}


# ---- a pass ---------------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    import paper_2505_13109_amd as fkv
    kind = st["case"]["kind"]
    if kind == "quant":
        fkv.proj_quant(st["x"], st["codes"], st["scales"], tile=st["case"]["tile"])
    elif kind == "norm":
        fkv.proj_norm(st["x"], st["weight"], st["codes"], st["scales"], add=st["add"], res=st["res"], eps=EPS)
        return {"codes": st["codes"], "scales": st["scales"], "res": st["res"]}
    elif kind == "gate":
        fkv.proj_gate(st["gu"], st["codes"], st["scales"])
    elif kind == "rope":
        fkv.proj_rope(st["qkv"], st["positions"], st["freq"], st["q"], st["k"], st["v"], sections=st["sections"])
        return {"q": st["q"], "k": st["k"], "v": st["v"]}
    else:
        fkv.proj_matmul(st["codes"], st["scales"], st["w"], st["w_scales"], st["out"])
        return {"out": st["out"]}
    return {"codes": st["codes"], "scales": st["scales"]}


def work(case):
    rows, kind = case["rows"], case["kind"]
    if kind == "rope":
        heads = case["n_q"] + 2 * case["n_kv"]
        return {"bytes": rows * (2 * heads * HEAD_DIM * 2 + 4 * case["axes"]) + 256, "flops": rows * (case["n_q"] + case["n_kv"]) * HEAD_DIM * 3}
    cols = case["cols"]
    blocks = -(-cols // BLOCK)
    if kind == "matmul":
        n = case["n"]
        moved = (rows + n) * cols + 4 * blocks * (rows + -(-n // BLOCK)) + 2 * rows * n
        return {"bytes": moved, "flops": 2 * rows * n * cols}
    out = rows * cols + 4 * blocks * -(-rows // case.get("tile", 1))
    if kind == "quant":
        return {"bytes": 2 * rows * cols + out, "flops": 3 * rows * cols}
    if kind == "norm":
        return {"bytes": 6 * rows * cols + 2 * cols + out, "flops": 8 * rows * cols}
    return {"bytes": 4 * rows * cols + out, "flops": 8 * rows * cols}


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def _spread(scales, rows, cols, tile):
    """A block's scale at each of its values."""
    return scales.double().repeat_interleave(tile, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def _exact_8_bits(y, tile):
    rows, cols = y.shape
    size = y.abs()
    if rows % tile:
        size = torch.cat((size, size.new_zeros(tile - rows % tile, cols)))
    if cols % BLOCK:
        size = torch.cat((size, size.new_zeros(size.shape[0], BLOCK - cols % BLOCK)), 1)
    largest = size.unflatten(1, (-1, BLOCK)).amax(2).unflatten(0, (-1, tile)).amax(1)
    scales = torch.maximum((largest / 448).float(), torch.full_like(largest, 2.0 ** -126, dtype=torch.float32))
    q = (y / _spread(scales, rows, cols, tile)).float().double()
    # e4m3: three bits behind the leading one, none smaller than 2^-9
    step = torch.exp2((torch.frexp(q)[1] - 4).clamp(min=-9).double())
    return {"codes": torch.round(q / step) * step, "scales": scales}


def exact(case, seed):
    st, kind = prepare(case, seed), case["kind"]
    if kind == "quant":
        return _exact_8_bits(st["x"].double(), case["tile"])
    if kind == "norm":
        res = (st["x"].double() + st["add"].double()).to(st["x"].dtype).double()
        out = _exact_8_bits(res * st["weight"].double(), 1)
        r = 1 / torch.sqrt(res.square().sum(1, keepdim=True) / case["cols"] + EPS)
        return {"codes": out["codes"], "scales": out["scales"].double() * r, "res": res}
    if kind == "gate":
        g, u = st["gu"][:, :case["cols"]].double(), st["gu"][:, case["cols"]:].double()
        return _exact_8_bits(g * u / (1 + torch.exp(-g)), 1)
    if kind == "rope":
        x, n_q, n_kv = st["qkv"].double(), case["n_q"], case["n_kv"]
        which = [a for a, n in enumerate(st["sections"]) for _ in range(n)]
        angle = torch.stack([st["positions"][a].double() * st["freq"][i].double() for i, a in enumerate(which)], 1)
        turn = torch.complex(torch.cos(angle), torch.sin(angle))[:, None]
        z = torch.complex(x[..., :HEAD_DIM // 2], x[..., HEAD_DIM // 2:])[:, :n_q + n_kv] * turn
        y = torch.cat((z.real, z.imag), 2)
        return {"q": y[:, :n_q], "k": y[:, n_q:], "v": x[:, n_q + n_kv:]}
    rows, cols, n = case["rows"], case["cols"], case["n"]
    x = st["codes"].float().double() * _spread(st["scales"], rows, cols, 1)
    w = st["w"].float().double() * _spread(st["w_scales"], n, cols, BLOCK)
    return {"out": x @ w.T}
