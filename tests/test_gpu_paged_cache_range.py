"""The paged cache's attention at the ends of what the types hold, against the same model in 64 bits."""
import math

import pytest
import torch

from paged_model import D
from test_gpu_paged_cache import TYPES, Pair, ints

pytestmark = pytest.mark.gpu


def dead(channel, at=0.0):
    """keys that hold the same number at every token of one channel"""
    def make(x, gen):
        x[0, ..., channel] = at
        return x
    return make


@pytest.mark.parametrize("dtype,powers", [("bf16", (8, 12, 13, 16, 24, 27, 30, 40, 70, 120)), ("fp16", (8, 11, 13, 15))])
@pytest.mark.parametrize("at", [0.0, 2.0 ** -13])
def test_a_querys_largest_channel_may_meet_keys_that_do_not_change(dtype, powers, at):
    """Its product counts for nothing, or the same at every token: what decides is 2^r below.  With heads beside it that have no such
    channel, in a page alone, in many, and in the open one."""
    p = Pair(n_kv=2, G=4, max_seqs=3, max_ctx=512, n_pages=40, dtype=dtype)
    p.grow([0, 1, 2], [32, 460, 37], dead(0, at))
    for r in powers:
        q = p.queries(3)
        q[:, 1::2, 0] = 2.0 ** r
        q[:, 5, 0] = -2.0 ** r
        if at:                                           # a logit that all share may be as large as fp32 still tells the others' differences
            q[:, :, 0] = q[:, :, 0].clamp(-2.0 ** 15, 2.0 ** 15)
        p.check_attention(0, [0, 1, 2], q=q)


@pytest.mark.parametrize("dtype,span", [("bf16", 20), ("bf16", 40), ("fp16", 10)])
def test_queries_and_keys_whose_channels_span_much(dtype, span):
    """Channels of queries 2^-span to 2^span, of keys the other way round, and a page of keys that are all of one size behind them."""
    p = Pair(n_kv=1, G=5, max_seqs=2, max_ctx=512, n_pages=40, dtype=dtype)
    e = torch.linspace(-span, span, D).round()
    low = -14 if dtype == "fp16" else -200
    for shuffled in range(2):
        s = shuffled
        p.grow([s], [200], lambda x, gen: torch.stack((x[0] * torch.exp2((-e).clamp(min=low)), x[1])))
        q = (torch.randn((1, 5, D), generator=p.gen) * torch.exp2(e)).to(TYPES[dtype])
        p.check_attention(0, [s], q=q)
        p.grow([s], [100], lambda x, gen: x * 2.0 ** -span)
        p.check_attention(0, [s], q=q)
        e = e[torch.randperm(D, generator=p.gen)]


def test_branches_with_wide_queries():
    """The same where branches are read together: one row's large channel changes nothing for the others."""
    p = Pair(n_kv=32, G=2, max_seqs=6, max_ctx=1536, n_pages=100)
    p.grow([0], [1300], dead(5))
    p.c.fork(ints([0] * 4), ints([1, 2, 3, 4]))
    p.m.fork([0] * 4, [1, 2, 3, 4])
    p.grow([0, 1, 3, 4], [70, 1, 40, 99], dead(5))
    q = p.queries(5)
    q[2, ::3, 5] = 2.0 ** 45
    q[4, :, 5] = -2.0 ** 33
    p.check_attention(0, [0, 1, 2, 3, 4], q=q)


@pytest.mark.parametrize("keys,queries", [(100, 20), (100, -100), (-100, 100), (-60, -60), (60, 50)])
def test_logits_of_all_sizes(keys, queries):
    """Products from far below 1 to near fp32's largest."""
    p = Pair(n_kv=1, G=3, max_seqs=1, max_ctx=512, n_pages=40)
    p.grow([0], [300], lambda x, gen: torch.stack((x[0] * 2.0 ** keys, x[1])))
    p.check_attention(0, [0], scale=2.0 ** queries)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("power", [22, 24, 26, 27, 28, 30])
def test_tokens_whose_logits_are_the_same_weigh_the_same(power, dtype):
    """Logits of about 2^power in powers of two, the same at two tokens of three and 0 at the third: the mean of the two's values, whatever
    the maximum is rounded to when it is set, in full pages, in the open one, and where they are joined.  (Keys are 0 and 15 steps.)"""
    p = Pair(n_kv=1, G=2, max_seqs=2, max_ctx=4096, n_pages=130, dtype=dtype)
    key = 15.0 * 2.0 ** 8

    def same(x, gen):
        x[0] = 0
        x[0, ..., 0] = key
        x[0, ::3, :, 0] = 0
        x[1] = torch.randn(x[1].shape, generator=gen)
        return x

    p.grow([0, 1], [71, 3011], same)
    q = torch.zeros((2, 2, D), dtype=TYPES[dtype])
    size = 2.0 ** power / key * math.sqrt(D) / math.log2(math.e)
    if dtype == "fp16":
        size = min(size, 60000.0)
    q[:, 0, 0], q[:, 1, 0] = size, size * 0.93
    out = torch.empty_like(q, device="cuda")
    p.c.attn(0, ints([0, 1]), q.cuda(), out)
    half = torch.finfo(TYPES[dtype]).eps / 2
    for s in (0, 1):
        value, lo, step = p.m.values(0, s)
        far = p.m.tokens[0][s][:, 0, 0, 0] == 0
        # the mean's own rounding, that of weights (half a step of 2^-11, which all share), and sums of values of up to 5
        want = value[~far][:, 1, 0].mean(0)
        off = (out[s].cpu().double() - want).abs() - half * 1.01 * want.abs() - 2.0 ** -24 * 512 * 5
        assert float(off.max()) <= 0, s


@pytest.mark.parametrize("lens", [[5], [64], [100], [3000, 20, 257]])
@pytest.mark.parametrize("scale", [0.0, 1.0])
def test_values_near_the_largest_number(lens, scale):
    """bf16 values of up to 3e38, in full pages and the open one, alone and joined, among branches; weights all the same or not.  Their mean
    is a number, and the sums on the way to it have to be."""
    p = Pair(n_kv=32, G=2, max_seqs=5, max_ctx=4096, n_pages=130)
    seqs = list(range(len(lens)))

    def large(x, gen):
        x[1] = torch.sign(x[1]) * 3.0e38 * torch.rand(x[1].shape, generator=gen)
        x[1, ..., 64:] = x[1, ..., 64:].abs()            # (means near the largest, too)
        x[1, ..., 100] = 3.3e38                          # (a step of 0)
        return x

    p.grow(seqs, lens, large)
    p.check_attention(0, seqs, scale=scale)
    p.c.fork(ints([0]), ints([4]))
    p.m.fork([0], [4])
    p.grow([0, 4], [40, 3], large)
    p.check_attention(0, seqs + [4], scale=scale)


@pytest.mark.parametrize("power", [-100, -60, 60, 110])
def test_values_of_all_sizes(power):
    """Outputs as near to the definition as those of values of 1 are, relative to their size."""
    p = Pair(n_kv=2, G=4, max_seqs=2, max_ctx=512, n_pages=40)
    p.grow([0, 1], [300, 45], lambda x, gen: torch.stack((x[0], x[1] * 2.0 ** power)))
    q = p.queries(2)
    out = torch.empty_like(q, device="cuda")
    p.c.attn(0, ints([0, 1]), q.cuda(), out)
    for s in (0, 1):
        for layer in p.m.tokens:                         # the same of a model whose values are 2^power smaller, where the bound's absolute part counts
            layer[s] = torch.stack((layer[s][:, 0].double(), layer[s][:, 1].double() * 2.0 ** -power), 1).bfloat16()
    scaled = (out.double() * 2.0 ** -power).cpu()
    p.check_attention(0, [0, 1], q=q, got=scaled)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("branches", [0, 4])
def test_an_infinite_value_in_the_open_page_gives_an_infinity(branches, dtype):
    """Open tokens are kept as they are: a channel with one infinity is infinite, with two of one sign as well, NaN with two signs or a NaN; all
    others are as if there were none.  Weights that are all of a size."""
    p = Pair(n_kv=32, G=2, max_seqs=6, max_ctx=1536, n_pages=100, dtype=dtype)

    def bad(x, gen):
        x[1, 0, 0, 3] = math.inf
        x[1, 8, 1, 4] = -math.inf
        x[1, 2, 2, 5], x[1, 9, 2, 5] = math.inf, math.inf
        x[1, 1, 3, 6], x[1, 3, 3, 6] = math.inf, -math.inf
        x[1, 5, 4, 7] = math.nan
        return x

    p.grow([0], [1280])
    rows = list(range(1 + branches))
    if branches:
        p.c.fork(ints([0] * branches), ints(rows[1:]))
        p.m.fork([0] * branches, rows[1:])
    s = rows[-1]
    p.grow([s], [10], bad)
    for r in rows[:-1]:
        p.grow([r], [7])
    q = p.queries(len(rows), 0.1)
    out = torch.empty_like(q, device="cuda")
    p.c.attn(0, ints(rows), q.cuda(), out)
    got = out.cpu()
    mine = got[-1].view(32, 2, D)
    assert (mine[0, :, 3] == math.inf).all() and (mine[1, :, 4] == -math.inf).all() and (mine[2, :, 5] == math.inf).all()
    assert mine[3, :, 6].isnan().all() and mine[4, :, 7].isnan().all()
    assert int((~torch.isfinite(got)).sum()) == 10
    for h, channel in ((0, 3), (1, 4), (2, 5), (3, 6), (4, 7)):
        mine[h, :, channel] = 0
        p.m.tokens[0][s] = p.m.tokens[0][s].clone()
        p.m.tokens[0][s][:, 1, h, channel] = 0
    p.check_attention(0, rows, q=q, got=got)
