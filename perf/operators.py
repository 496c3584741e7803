"""Performance cases of the paged cache in 4 bits: keys and values of many sequences in one pool of 4-bit pages, what
fills it, the attention that reads it, and what forks, copies, compacts and frees its pages.

A sequence's full pages (32 tokens of all layers and KV heads) lie in the pool in 4 bits, relative to each channel's
smallest value in the page; the tokens of its open page stay in 16 bits.  Full pages never change, so sequences share them.
Of a page, a KV head's keys (and likewise its values) are, for every channel c over the page's 32 tokens t:

    lo_c   = min_t x_tc                                  in the storage type
    w_c    = (max_t x_tc - lo_c) / 15                    in fp32
    E      = floor(log2(max_c w_c))                      one exponent for the 128 channels
    step_c = fp16(w_c 2^-E) 2^E
    code   = round((x_tc - lo_c) / step_c), 0 to 15      ties to even, 0 where step_c is 0
    value  = lo_c + step_c code

A case is a dict.  kind is
  "attn"     one token's attention of `rows` sequences over what the cache holds of them; with `n_list`, over listed pages
             per KV head between `sink` and `window` tokens (what a page selection gives)
  "fill"     tokens of `rows` sequences put into the cache and read back; with `base`, behind a shared prompt of that length
  "step"     a decode step of `rows` branches of `bases` sequences: fork, room for a token, append and attention in every
             layer, and the branches given up again
  "compact"  half of `rows` sequences written into pages of their own, their old pages given back, the pool compacted, and
             the moved sequences read
Head dimension and page size are the library's only ones, 128 and 32.
"""
import math

import torch

own = False

HEAD_DIM, PAGE = 128, 32
UNIT = 2 * (PAGE * HEAD_DIM // 2 + 4 * HEAD_DIM)          # bytes of one page of one KV head: codes, steps and minima of keys and values
OUTLIER_CHANNELS, OUTLIER_SCALE = (7, 43, 71, 101), 8.0   # keys and values have a few large channels
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}

_BASE = dict(kind="attn", layers=1, rows=1, bases=0, n_q=32, n_kv=8, dtype="bf16", ctx=4096, spread=1, base=0, n_list=0, sink=0, window=0)


def _case(name, **kw):
    return dict(_BASE, name=name, **kw)


def listed():
    return [
        # the smallest call: the second page of one fp16 sequence has just begun; launch and latency count
        _case("attn_45_tokens", dtype="fp16", ctx=45),
        # the ordinary one: a request at 32K tokens, 32/8 heads
        _case("attn_32k", ctx=32768),
        # a batch of 32 requests of all lengths between 500 and 16K tokens, 28/4 heads
        _case("attn_ragged_batch32_g7", rows=32, n_q=28, n_kv=4, ctx=16384, spread=32),
        # a few very long requests: four of 128K tokens
        _case("attn_batch4_128k", rows=4, ctx=131072),
        # the attention behind a page selection: 64/8 heads, 64K tokens, a budget of 4096 of them
        _case("attn_list_64k_g8", rows=8, n_q=64, ctx=65536, n_list=96, sink=512, window=512),
        # seven answers to one prompt of 1000 tokens handed over, of different lengths, fp16; every page boundary is inside
        _case("fill_behind_prompt", kind="fill", layers=4, rows=7, n_q=40, dtype="fp16", base=1000, ctx=1500, spread=8),
        # a prompt of 32K tokens handed over in four layers
        _case("fill_32k", kind="fill", layers=4, ctx=32768),
        # eight samples of one request's next token, a short context, all layers of a small model
        _case("step_8_samples_2k", kind="step", layers=28, rows=8, bases=1, n_q=28, n_kv=4, ctx=2047),
        # a beam step: 32 branches of 16 requests of up to 8K tokens, 8 layers
        _case("step_32_branches_8k", kind="step", layers=8, rows=32, bases=16, ctx=8191, spread=4),
        # upkeep of a small pool: six short fp16 sequences in two layers, 2 KV heads
        _case("compact_small", kind="compact", layers=2, rows=6, n_q=2, n_kv=2, dtype="fp16", ctx=601, spread=2),
        # upkeep of a large one: 16 sequences of 4K tokens in 8 layers, 0.67 GB of pages
        _case("compact_16x4k", kind="compact", layers=8, rows=16, ctx=4103),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "fill", "step", "compact"])
    n_kv = rng.choice([1, 2, 4, 8, 8])
    case = dict(_BASE, kind=kind, n_kv=n_kv, n_q=n_kv * rng.randint(1, 8), dtype=rng.choice(["fp16", "bf16", "bf16"]), spread=rng.choice([1, 3, 10, 40]))
    if kind == "attn":
        case["ctx"] = _log_int(rng, 1, 262144)
        case["rows"] = _log_int(rng, 1, max(1, min(64, (4 << 20) // (case["ctx"] * n_kv))))
        if rng.random() < 0.4:
            case["n_list"], case["sink"], case["window"] = rng.randint(1, 200), PAGE * rng.randint(0, 16), PAGE * rng.randint(0, 16)
    elif kind == "fill":
        case["ctx"] = _log_int(rng, 1, 32768)
        case["rows"] = _log_int(rng, 1, max(1, min(32, 32768 // case["ctx"])))
        case["base"] = rng.choice([0, 0, rng.randint(1, 2000)])
        case["layers"] = max(1, min(8, (1 << 20) // ((case["ctx"] + case["base"]) * case["rows"] * n_kv)))
    elif kind == "step":
        case["ctx"] = _log_int(rng, 1, 32768)
        case["bases"] = _log_int(rng, 1, max(1, min(16, 131072 // case["ctx"])))
        case["rows"] = case["bases"] * rng.randint(1, max(1, min(4, 262144 // (case["ctx"] * case["bases"]))))
        case["layers"] = _log_int(rng, 1, max(1, min(16, (4 << 20) // (case["ctx"] * case["rows"] * n_kv))))
    else:
        case["ctx"] = _log_int(rng, 20, 8192)
        case["rows"] = _log_int(rng, 2, max(2, min(24, 65536 // case["ctx"])))
        case["layers"] = _log_int(rng, 1, max(1, min(8, (4 << 20) // (case["ctx"] * case["rows"] * n_kv))))
    return case


# ---- what the cases are made of -----------------------------------------------------------------

def _lengths(case, n):
    """n lengths, the longest case["ctx"], spread evenly in the logarithm down to ctx / spread, not in order."""
    spread = min(case["spread"], case["ctx"])
    at = [i / max(1, n - 1) for i in range(n)]
    lens = [max(1, round(case["ctx"] * spread ** -a)) for a in at]
    return [lens[(i * 5 + 3) % n] for i in range(n)] if n % 5 else lens


def _generator(seed, *what):
    mixed = seed & 0xffffffff
    for w in what:
        mixed = (mixed * 1000003 + w + 1) & 0x7fffffffffff
    return torch.Generator(device="cuda").manual_seed(mixed)


def _tokens(case, n, seed, *what):
    """Keys and values of n tokens, [n, n_kv, d] each: normal, a few channels eight times larger."""
    g = _generator(seed, *what)
    scale = torch.ones(HEAD_DIM, device="cuda")
    scale[list(OUTLIER_CHANNELS)] = OUTLIER_SCALE
    return tuple((torch.randn((n, case["n_kv"], HEAD_DIM), generator=g, device="cuda") * scale).to(TYPES[case["dtype"]]) for _ in "kv")


def _queries(case, n, seed, *what):
    return torch.randn((n, case["n_q"], HEAD_DIM), generator=_generator(seed, 77, *what), device="cuda").to(TYPES[case["dtype"]])


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cu(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _shape(case):
    """Sequence slots, pages and the longest sequence that a program would give the cache for this case, and its prompts' lengths."""
    kind, rows = case["kind"], case["rows"]
    if kind == "attn":
        first = _lengths(case, rows)
        return rows, sum(-(-n // PAGE) for n in first) + 1, max(first), first
    if kind == "fill":
        more = _lengths(case, rows)
        return rows + 1, case["base"] // PAGE + sum((n + PAGE) // PAGE for n in more) + 1, case["base"] + max(more), [case["base"]]
    if kind == "step":
        first = _lengths(case, case["bases"])
        return case["bases"] + rows, sum(n // PAGE for n in first) + rows + 1, max(first) + 1, first
    first = _lengths(case, rows)
    pages = [n // PAGE for n in first]
    return rows + rows // 2, sum(pages) + sum(pages[1::2]) + 1, max(first), first


def _page_lists(case, lens, seed):
    """Ascending page positions [rows, n_kv, n_list] between sink and window, -1 behind the last; some lists are short."""
    g = _generator(seed, 5)
    lists = torch.full((len(lens), case["n_kv"], case["n_list"]), -1, dtype=torch.int32, device="cuda")
    sink, window = case["sink"] // PAGE, case["window"] // PAGE
    for r, n in enumerate(lens):
        free = n // PAGE - sink - window
        if free <= 0:
            continue
        for h in range(case["n_kv"]):
            k = min(free, case["n_list"] if (r + h) % 3 else (case["n_list"] + 1) // 2)
            lists[r, h, :k] = (torch.randperm(free, generator=g, device="cuda")[:k].sort().values + sink).to(torch.int32)
    return lists


# ---- the plain form: the same cache as tensors, elementary operations -----------------------------

class _Plain:
    """Page pool, tables and open pages as tensors; lengths are known to the host, as they are to a program."""

    def __init__(self, case, slots, n_pages, max_ctx):
        dt, kv, layers = TYPES[case["dtype"]], case["n_kv"], case["layers"]
        new = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device="cuda")
        self.case = case
        self.codes = new(layers, n_pages, 2, PAGE, kv, HEAD_DIM // 2, dtype=torch.uint8)
        self.lo = new(layers, n_pages, 2, 1, kv, HEAD_DIM, dtype=dt)
        self.step = new(layers, n_pages, 2, 1, kv, HEAD_DIM, dtype=torch.float32)
        self.open = new(layers, slots, 2, PAGE, kv, HEAD_DIM, dtype=dt)
        self.table = torch.full((slots, max_ctx // PAGE + 1), -1, dtype=torch.int64, device="cuda")
        self.ref = new(n_pages, dtype=torch.int32)
        self.lens = [0] * slots
        self.added = [0] * slots

    def _take(self, n):
        ids = torch.argsort((self.ref > 0).to(torch.uint8), stable=True)[:n]      # the lowest free pages
        self.ref[ids] = 1
        return ids

    def extend(self, seqs, new):
        counts = [(self.lens[s] + n) // PAGE - self.lens[s] // PAGE for s, n in zip(seqs, new)]
        ids, at = self._take(sum(counts)), 0
        for s, n, c in zip(seqs, new, counts):
            first = self.lens[s] // PAGE
            self.table[s, first:first + c] = ids[at:at + c]
            self.lens[s], self.added[s], at = self.lens[s] + n, n, at + c

    def append(self, layer, seqs, k, v):
        x, at = torch.stack((k, v), 1), 0                                        # [tokens, 2, kv, d]
        for s in seqs:
            n, end = self.added[s], self.lens[s]
            held = (end - n) % PAGE
            both = torch.cat((self.open[layer, s, :, :held].transpose(0, 1), x[at:at + n]))
            at += n
            full = (held + n) // PAGE
            if full:
                pages = both[:full * PAGE].view(full, PAGE, 2, -1, HEAD_DIM).transpose(1, 2)     # [full, 2, 32, kv, d]
                ids = self.table[s, end // PAGE - full:end // PAGE]
                self.codes[layer, ids], self.lo[layer, ids], self.step[layer, ids] = _pack(pages)
            rest = both[full * PAGE:]
            self.open[layer, s, :, :rest.shape[0]] = rest.transpose(0, 1)

    def values(self, layer, s, pages=None):
        """fp32 keys and values [2, tokens, kv, d] of a sequence (of these pages of it) and its open page."""
        n = self.lens[s]
        ids = self.table[s, :n // PAGE] if pages is None else self.table[s, pages]
        codes = self.codes[layer, ids]
        codes = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
        x = self.lo[layer, ids].float() + self.step[layer, ids] * codes
        return torch.cat((x.transpose(0, 1).flatten(1, 2), self.open[layer, s, :, :n % PAGE].float()), 1)

    def read(self, layer, seqs):
        x = torch.cat([self.values(layer, s) for s in seqs], 1).to(TYPES[self.case["dtype"]])
        return x[0], x[1]

    def attn(self, layer, seqs, q, lists=None):
        case, out = self.case, torch.empty_like(q)
        kv, g = case["n_kv"], case["n_q"] // case["n_kv"]
        for r, s in enumerate(seqs):
            query = q[r].float().view(kv, g, HEAD_DIM)
            if lists is None:
                x = self.values(layer, s).transpose(1, 2)                         # [2, kv, tokens, d]
                out[r] = _softmax_product(query, x[0], x[1]).view(-1, HEAD_DIM)
                continue
            full, sink, window = self.lens[s] // PAGE, case["sink"] // PAGE, case["window"] // PAGE
            sink = min(sink, full)
            window = min(window, full - sink)
            ends = torch.cat((torch.arange(sink, device="cuda"), torch.arange(full - window, full, device="cuda")))
            for h in range(kv):
                listed_ = lists[r, h].long()
                # a place that lists nothing brings tokens that weigh nothing
                x = self.values(layer, s, torch.cat((listed_.clamp(min=0), ends)))[:, :, h]
                weighs = torch.ones(x.shape[1], dtype=torch.bool, device="cuda")
                weighs[:listed_.numel() * PAGE] = (listed_ >= 0).repeat_interleave(PAGE)
                out[r, h * g:(h + 1) * g] = _softmax_product(query[h], x[0], x[1], weighs)
        return out

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.ref.index_add_(0, self.table[a, :self.lens[a] // PAGE], torch.ones(self.lens[a] // PAGE, dtype=torch.int32, device="cuda"))
            self.table[b] = self.table[a]
            self.open[:, b] = self.open[:, a]
            self.lens[b], self.added[b] = self.lens[a], 0

    def copy(self, src, dst):
        for a, b in zip(src, dst):
            full = self.lens[a] // PAGE
            ids, old = self._take(full), self.table[a, :full]
            self.codes[:, ids], self.lo[:, ids], self.step[:, ids] = self.codes[:, old], self.lo[:, old], self.step[:, old]
            self.table[b, :full] = ids
            self.open[:, b] = self.open[:, a]
            self.lens[b], self.added[b] = self.lens[a], 0

    def free(self, seqs):
        for s in seqs:
            full = self.lens[s] // PAGE
            self.ref.index_add_(0, self.table[s, :full], torch.full((full,), -1, dtype=torch.int32, device="cuda"))
            self.lens[s] = 0

    def compact(self, live, moved):
        """live pages are held, the `moved` last of them lie behind the others: they go to the lowest free places."""
        used = self.ref > 0
        holes = torch.argsort(used.to(torch.uint8), stable=True)[:moved]
        tail = torch.argsort((~used).to(torch.uint8), stable=True)[live - moved:live]
        to = torch.arange(self.ref.numel(), device="cuda")
        to[tail] = holes
        self.codes[:, holes], self.lo[:, holes], self.step[:, holes] = self.codes[:, tail], self.lo[:, tail], self.step[:, tail]
        self.ref[holes] = self.ref[tail]
        self.ref[tail] = 0
        self.table = torch.where(self.table >= 0, to[self.table.clamp(min=0)], self.table)

    def tables(self, seqs):
        lens = _int32([self.lens[s] for s in seqs])
        held = torch.arange(self.table.shape[1], device="cuda") < (lens // PAGE)[:, None]
        return lens, torch.where(held, self.table[seqs], -1).to(torch.int32)


def _pack(x):
    """[n, 2, 32, kv, d] of the storage type -> codes, two channels a byte, minima and steps.  In 64 bits where a code may lie at a border."""
    lo, hi = x.amin(2, keepdim=True), x.amax(2, keepdim=True)
    fifteen = torch.full((), 15.0, dtype=torch.float64, device=x.device)
    w = ((hi.double() - lo.double()) / fifteen).float()
    e = torch.frexp(w.amax(-1, keepdim=True))[1] - 1
    step = torch.ldexp(torch.ldexp(w, -e).half().float(), e)
    codes = ((x.double() - lo.double()) / step.double()).round().clamp(0, 15).nan_to_num(0.0).to(torch.uint8)
    return codes[..., 0::2] | codes[..., 1::2] << 4, lo, step


def _softmax_product(q, k, v, weighs=None):
    """fp32 softmax(q k^T / sqrt(d)) v, [..., g, d]; zeros where nothing weighs."""
    s = torch.matmul(q, k.transpose(-1, -2)) * HEAD_DIM ** -0.5
    if weighs is not None:
        s = s.masked_fill(~weighs, -math.inf)
    if not s.shape[-1]:
        return torch.zeros_like(q)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top.clamp(min=torch.finfo(s.dtype).min))
    z = p.sum(-1, keepdim=True)
    return torch.matmul(p / torch.where(z > 0, z, torch.ones_like(z)), v)


# ---- a case's state and its pass -------------------------------------------------------------------

def prepare(case, seed):
    slots, n_pages, max_ctx, first = _shape(case)
    kind, rows = case["kind"], case["rows"]
    st = dict(case=case, own=own, first=first)
    if own:
        from paper_2505_13109_amd import PagedCache
        cache = PagedCache(n_layers=case["layers"], n_q_heads=case["n_q"], n_kv_heads=case["n_kv"], max_seqs=slots,
                           max_ctx=-(-max_ctx // PAGE) * PAGE, n_pages=n_pages, dtype=case["dtype"])
    else:
        cache = _Plain(case, slots, n_pages, -(-max_ctx // PAGE) * PAGE)
    st["cache"] = cache
    # the sequences that are there before the pass; in a pool that lives for long their pages lie among each other's
    ids = list(range(len(first)))
    chunk = 512 if kind == "compact" else max(first, default=0) + 1
    for at in range(0, max(first), chunk):
        here = [s for s in ids if first[s] > at]
        new = [min(chunk, first[s] - at) for s in here]
        if own:
            cu, seqs = _int32(_cu(new)), _int32(here)
            cache.extend(seqs, cu)
        else:
            cache.extend(here, new)
        for layer in range(case["layers"]):
            parts = [_tokens(case, n, seed, layer, s, at) for s, n in zip(here, new)]
            k, v = (torch.cat([p[i] for p in parts]) for i in (0, 1))
            del parts
            cache.append(layer, seqs, k, v, cu) if own else cache.append(layer, here, k, v)
    if kind == "attn":
        st["seqs"] = _int32(ids) if own else ids
        st["q"] = _queries(case, rows, seed)
        st["lists"] = _page_lists(case, first, seed) if case["n_list"] else None
        st["out"] = torch.empty_like(st["q"])
    elif kind == "fill":
        new = _lengths(case, rows)
        st["new"], st["work"] = new, list(range(1, rows + 1))
        st["kv"] = [_tokens(case, sum(new), seed, layer, 1000) for layer in range(case["layers"])]
        total = sum(new) + rows * case["base"]
        shape = (case["layers"], total, case["n_kv"], HEAD_DIM)
        st["k"], st["v"] = (torch.empty(shape, dtype=TYPES[case["dtype"]], device="cuda") for _ in "kv")
        if own:
            st["cu"], st["cu_read"] = _int32(_cu(new)), _int32(_cu([n + case["base"] for n in new]))
            st["seqs"], st["src"] = _int32(st["work"]), _int32([0] * rows)
    elif kind == "step":
        st["from"], st["work"] = [i % case["bases"] for i in range(rows)], [case["bases"] + i for i in range(rows)]
        st["kv"] = [_tokens(case, rows, seed, layer, 1000) for layer in range(case["layers"])]
        st["q"] = [_queries(case, rows, seed, layer) for layer in range(case["layers"])]
        st["out"] = torch.empty((case["layers"], rows, case["n_q"], HEAD_DIM), dtype=TYPES[case["dtype"]], device="cuda")
        if own:
            st["seqs"], st["src"] = _int32(st["work"]), _int32(st["from"])
    else:
        half = rows // 2
        st["stay"], st["held"], st["spare"] = ids[0::2], ids[1::2], list(range(rows, rows + half))
        total = sum(first[1::2])
        shape = (case["layers"], total, case["n_kv"], HEAD_DIM)
        st["k"], st["v"] = (torch.empty(shape, dtype=TYPES[case["dtype"]], device="cuda") for _ in "kv")
        if own:
            st["cu"] = _int32(_cu(first[1::2]))
            for name in ("stay", "held", "spare"):
                st[name] = _int32(st[name])
    if own and kind != "attn":
        n = rows
        st["lens"] = torch.empty((n,), dtype=torch.int32, device="cuda")
        st["pages"] = torch.empty((n, -(-max_ctx // PAGE)), dtype=torch.int32, device="cuda")
    return st


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(st):
    case, cache, kind = st["case"], st["cache"], st["case"]["kind"]
    layers = range(case["layers"])
    if kind == "attn":
        cache.attn(0, st["seqs"], st["q"], st["out"], pages=st["lists"], sink=case["sink"], window=case["window"])
        return st["out"]
    if kind == "fill":
        if case["base"]:
            cache.fork(st["src"], st["seqs"])
        cache.extend(st["seqs"], st["cu"])
        for layer in layers:
            cache.append(layer, st["seqs"], *st["kv"][layer], st["cu"])
        for layer in layers:
            cache.read(layer, st["seqs"], st["k"][layer], st["v"][layer], st["cu_read"])
        cache.tables(st["seqs"], st["lens"], st["pages"])
        cache.free(st["seqs"])
        return st["k"], st["v"], st["lens"], st["pages"]
    if kind == "step":
        cache.fork(st["src"], st["seqs"])
        cache.extend(st["seqs"])
        for layer in layers:
            cache.append(layer, st["seqs"], *st["kv"][layer])
            cache.attn(layer, st["seqs"], st["q"][layer], st["out"][layer])
        cache.tables(st["seqs"], st["lens"], st["pages"])
        cache.free(st["seqs"])
        return st["out"], st["lens"], st["pages"]
    cache.copy(st["held"], st["spare"])
    cache.free(st["held"])
    cache.compact()
    st["held"], st["spare"] = st["spare"], st["held"]
    for layer in layers:
        cache.read(layer, st["held"], st["k"][layer], st["v"][layer], st["cu"])
    n = len(st["first"][0::2])
    cache.tables(st["stay"], st["lens"][:n], st["pages"][:n])
    cache.tables(st["held"], st["lens"][n:], st["pages"][n:])
    return st["k"], st["v"], st["lens"], st["pages"]


def _run_plain(st):
    case, cache, kind = st["case"], st["cache"], st["case"]["kind"]
    layers = range(case["layers"])
    if kind == "attn":
        return cache.attn(0, st["seqs"], st["q"], st["lists"])
    if kind == "fill":
        if case["base"]:
            cache.fork([0] * case["rows"], st["work"])
        cache.extend(st["work"], st["new"])
        for layer in layers:
            cache.append(layer, st["work"], *st["kv"][layer])
        for layer in layers:
            st["k"][layer], st["v"][layer] = cache.read(layer, st["work"])
        lens, pages = cache.tables(st["work"])
        cache.free(st["work"])
        return st["k"], st["v"], lens, pages[:, :_max_pages(case)]
    if kind == "step":
        cache.fork(st["from"], st["work"])
        cache.extend(st["work"], [1] * case["rows"])
        for layer in layers:
            cache.append(layer, st["work"], *st["kv"][layer])
            st["out"][layer] = cache.attn(layer, st["work"], st["q"][layer])
        lens, pages = cache.tables(st["work"])
        cache.free(st["work"])
        return st["out"], lens, pages[:, :_max_pages(case)]
    first = st["first"]
    live, moved = sum(n // PAGE for n in first), sum(n // PAGE for n in first[1::2])
    cache.copy(st["held"], st["spare"])
    cache.free(st["held"])
    cache.compact(live, moved)
    st["held"], st["spare"] = st["spare"], st["held"]
    for layer in layers:
        st["k"][layer], st["v"][layer] = cache.read(layer, st["held"])
    lens, pages = cache.tables(st["stay"] + st["held"])
    return st["k"], st["v"], lens, pages[:, :_max_pages(case)]


def _max_pages(case):
    return -(-_shape(case)[2] // PAGE)


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _kept(x):
    """What the cache stands for of a sequence's tokens [n, kv, d], in 64 bits."""
    n = x.shape[0] // PAGE * PAGE
    y = x.double()
    p = y[:n].reshape(-1, PAGE, *x.shape[1:])
    if not n:
        return y
    least = p.min(dim=1, keepdim=True).values
    width = ((p.max(dim=1, keepdim=True).values - least) / 15.0).to(torch.float32)
    widest = width.max(dim=-1, keepdim=True).values
    scale = torch.exp2(torch.floor(torch.log2(widest.double())))
    scale = torch.where(widest > 0, scale, torch.ones_like(scale))
    step = (width.double() / scale).to(torch.float32).to(torch.float16).double() * scale
    code = torch.where(step > 0, torch.round((p - least) / torch.where(step > 0, step, torch.ones_like(step))), torch.zeros_like(p))
    y[:n] = (least + step * code.clamp(0, 15)).reshape(n, *x.shape[1:])
    return y


def _dense(q, k, v):
    """q [n_q, d], k and v [tokens, kv, d] in 64 bits -> [n_q, d]"""
    kv = k.shape[1]
    g = q.shape[0] // kv
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    if k.shape[0]:
        for h in range(kv):
            s = (q[h * g:(h + 1) * g].double() @ k[:, h].t().contiguous()) / math.sqrt(HEAD_DIM)
            out[h * g:(h + 1) * g] = torch.softmax(s, -1) @ v[:, h].contiguous()
    return out


def exact(case, seed):
    _, _, _, first = _shape(case)
    kind, rows = case["kind"], case["rows"]

    def prompt(layer, s):
        chunk = 512 if kind == "compact" else max(first) + 1
        parts = [_tokens(case, min(chunk, first[s] - at), seed, layer, s, at) for at in range(0, first[s], chunk)]
        if not parts:
            return _tokens(case, 0, seed, layer, s, 0)
        return tuple(torch.cat([p[i] for p in parts]) for i in (0, 1))

    if kind == "attn":
        q = _queries(case, rows, seed)
        lists = _page_lists(case, first, seed).tolist() if case["n_list"] else None
        out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
        g = case["n_q"] // case["n_kv"]
        for r in range(rows):
            k, v = (_kept(x) for x in prompt(0, r))
            if lists is None:
                out[r] = _dense(q[r], k, v)
                continue
            full = first[r] // PAGE
            sink = min(case["sink"] // PAGE, full)
            window = min(case["window"] // PAGE, full - sink)
            for h in range(case["n_kv"]):
                pages = [j for j in range(full) if j < sink or j >= full - window] + [j for j in lists[r][h] if j >= 0]
                at = [t for j in pages for t in range(j * PAGE, j * PAGE + PAGE)] + list(range(full * PAGE, first[r]))
                at = torch.tensor(at, dtype=torch.int64, device="cuda")
                out[r, h * g:(h + 1) * g] = _dense(q[r, h * g:(h + 1) * g], k[at, h:h + 1], v[at, h:h + 1])
        return out
    if kind == "fill":
        new, ks, vs = _lengths(case, rows), [], []
        at = _cu(new)
        for layer in range(case["layers"]):
            more, base = _tokens(case, sum(new), seed, layer, 1000), prompt(layer, 0)
            for i, into in ((0, ks), (1, vs)):
                into.append(torch.cat([_kept(torch.cat((base[i], more[i][at[r]:at[r + 1]]))) for r in range(rows)]))
        return torch.stack(ks), torch.stack(vs), None, None
    if kind == "step":
        out = []
        for layer in range(case["layers"]):
            more, q = _tokens(case, rows, seed, layer, 1000), _queries(case, rows, seed, layer)
            prompts = [prompt(layer, s) for s in range(case["bases"])]
            for r in range(rows):
                k, v = (_kept(torch.cat((prompts[r % case["bases"]][i], more[i][r:r + 1]))) for i in (0, 1))
                out.append(_dense(q[r], k, v))
        return torch.stack(out).view(case["layers"], rows, case["n_q"], HEAD_DIM), None, None
    ks, vs = [], []
    for layer in range(case["layers"]):
        kept = [[_kept(x) for x in prompt(layer, s)] for s in range(1, rows, 2)]
        ks.append(torch.cat([x[0] for x in kept]))
        vs.append(torch.cat([x[1] for x in kept]))
    return torch.stack(ks), torch.stack(vs), None, None


def work(case):
    """Bytes and operations that a pass cannot do without: pages read in 4 bits, open tokens and what comes and goes in 16."""
    slots, n_pages, max_ctx, first = _shape(case)
    kind, rows, kv, n_q, layers = case["kind"], case["rows"], case["n_kv"], case["n_q"], case["layers"]
    token = 4 * HEAD_DIM * kv                                             # bytes of a token's keys and values in one layer
    page = UNIT * kv

    def attention(n, branches=1):
        full = n // PAGE
        if case["n_list"] and kind == "attn":
            ends = min(full, (case["sink"] + case["window"]) // PAGE)
            full = ends + min(full - ends, case["n_list"])
        return full * page + (n % PAGE) * token, 4 * n_q * HEAD_DIM * (full * PAGE + n % PAGE) * branches

    if kind == "attn":
        each = [attention(n) for n in first]
        return {"bytes": sum(b for b, _ in each) + 4 * rows * n_q * HEAD_DIM, "flops": sum(f for _, f in each)}
    if kind == "fill":
        new, nbytes = _lengths(case, rows), 0
        for n in new:
            held, end = case["base"] % PAGE, case["base"] + n
            written = end // PAGE - case["base"] // PAGE
            nbytes += 2 * held * token                                    # the shared open page, copied
            nbytes += n * token + written * page + (end % PAGE) * token   # tokens in, pages and open tokens out
            nbytes += end // PAGE * page + (end % PAGE) * token + end * token   # read back
        return {"bytes": nbytes * layers, "flops": 8 * (sum(new) * 2 + rows * case["base"]) * 2 * HEAD_DIM * kv * layers}
    if kind == "step":
        nbytes = flops = 0
        for s, n in enumerate(first):
            branches = len(range(s, rows, case["bases"]))
            b, f = attention(n, branches)                                 # branches share the pages of their prompt
            nbytes += b + branches * (2 * (n % PAGE) * token + 2 * token + 4 * n_q * HEAD_DIM)
            flops += f
        return {"bytes": nbytes * layers, "flops": flops * layers}
    moved = first[1::2]
    pages = sum(n // PAGE for n in moved) * page
    tail = sum(n % PAGE for n in moved) * token
    return {"bytes": layers * (2 * pages + 2 * tail + 2 * pages + pages + tail + sum(moved) * token), "flops": layers * 2 * sum(moved) * 2 * HEAD_DIM * kv}
