"""How near the paged cache's attention comes to the definition in 64 bits, beyond bounds that add all roundings up, and whether every
page counts once."""
import math
import random

import pytest
import torch

from paged_model import D, PG
from test_gpu_paged_cache import TYPES, Pair, ints

pytestmark = pytest.mark.gpu


def not_nearest(p, seqs, q, got, layer=0):
    """Of the outputs that are not small against their row: the share that is not the definition's value rounded to the type."""
    other = total = 0
    for r, s in enumerate(seqs):
        value = p.m.values(layer, s)[0]
        for h in range(p.kv):
            x = q[r, h * p.G:(h + 1) * p.G].double() @ value[:, 0, h].T / math.sqrt(D)
            want = torch.softmax(x, -1) @ value[:, 1, h]
            large = want.abs() >= want.pow(2).mean(-1, keepdim=True).sqrt() / 4
            differs = got[r, h * p.G:(h + 1) * p.G] != want.to(q.dtype)
            other += int((differs & large).sum())
            total += int(large.sum())
    return other / total


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kv,G,rows,branches", [(2, 4, 1, 0), (1, 16, 1, 0), (32, 4, 1, 3), (32, 2, 1, 5)])
def test_outputs_are_the_nearest_numbers_but_for_few(kv, G, rows, branches, dtype):
    """An output that is off by e before it is rounded comes out as another number in e of its distance to the next one.  Logits are off by
    1e-5 (products cut some 24 bits below the largest), weights by 2^-21, and so an output of 2000 tokens by less than 2^-15 of its size.
    The distance is eps / 2 to eps of an output, and over normally distributed ones of which the smallest are left out 1 / |output| is
    1.8 of 1 / rms on average: at most 2 x 1.8 x 2^-15 / eps, 1.4 % for bf16 and 11 % for fp16.  (Weights of 11 bits come to 3.4 and 27 %.)"""
    p = Pair(n_kv=kv, G=G, max_seqs=1 + branches, max_ctx=2560, n_pages=110, dtype=dtype)
    p.grow([0], [2010])
    if branches:
        p.c.fork(ints([0] * branches), ints(list(range(1, 1 + branches))))
        p.m.fork([0] * branches, list(range(1, 1 + branches)))
    seqs = list(range(1 + branches))
    q = p.queries(len(seqs))
    out = torch.empty_like(q, device="cuda")
    p.c.attn(0, ints(seqs), q.cuda(), out)
    share = not_nearest(p, seqs, q, out.cpu())
    assert share <= 2 * 1.8 * 2.0 ** -15 / torch.finfo(q.dtype).eps, share


GROUP = 6 * D                                            # pages that one query head tells apart: six binary digits in each channel


def told_apart(p, s, n):
    """n tokens of slot s.  Page i is one of group i / GROUP, which its keys name, and its values are one binary digit in one channel, the
    same in all of the page's tokens: exact in 4 bits.  Head g attends to group g alone, all of its pages with the same weight, so a channel
    of its output is the sum of six digits over the number of the group's pages.  A page that is missed or counts twice changes one by 1 / 63
    at least, less what one page more or less changes of the number: more than the two roundings to bf16, 2^-7."""
    pages = -(-n // PG)
    k, v = (torch.zeros((pages, p.kv, D)) for _ in "kv")
    for i in range(pages):
        for h in range(p.kv):
            j = (i + 131 * h) % pages                    # another page's for every KV head
            k[i, h, j // GROUP] = 64.0
            v[i, h, j % GROUP % D] = 2.0 ** (j % GROUP // D)
    k, v = (x.repeat_interleave(PG, 0)[:n].to(TYPES[p.dtype]) for x in (k, v))
    cu = ints([0, n])
    p.c.extend(ints([s]), cu)
    p.c.append(0, ints([s]), k.cuda(), v.cuda(), cu)
    return k, v


def group_queries(p):
    q = torch.zeros((1, p.kv * p.G, D))
    for h in range(p.kv * p.G):
        q[0, h, h % p.G] = 64.0                          # logits of 64 x 64 / sqrt(128) = 362 and 0
    return q.to(TYPES[p.dtype])


def check_told_apart(p, got, k, v, q, attended=None):
    """attended[h]: token numbers.  The mean's own rounding; weights are all the same, sums of whole numbers below 2^24 exact."""
    half = torch.finfo(q.dtype).eps / 2
    for h in range(p.kv):
        at = torch.arange(k.shape[0]) if attended is None else attended[h]
        x = q[0, h * p.G:(h + 1) * p.G].double() @ k[at][:, h].double().T / math.sqrt(D)
        want = torch.softmax(x, -1) @ v[at][:, h].double()
        off = (got[h * p.G:(h + 1) * p.G].double() - want).abs()
        assert float((off - half * 1.001 * want - 2.0 ** -22).max()) <= 0, h


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kv,G,n", [(1, 6, 130000), (1, 3, 70001), (2, 2, 40010), (1, 1, 20001), (8, 2, 32769), (1, 16, 9000), (4, 3, 2111)])
def test_every_page_counts_once(kv, G, n, dtype):
    """Up to as many splits as a row may have (256: one KV head and more than 65536 tokens), in one and two levels."""
    p = Pair(n_kv=kv, G=G, max_seqs=1, max_ctx=-(-n // PG) * PG, n_pages=n // PG + 1, dtype=dtype)
    k, v = told_apart(p, 0, n)
    q = group_queries(p)
    out = torch.empty_like(q, device="cuda")
    p.c.attn(0, ints([0]), q.cuda(), out)
    check_told_apart(p, out[0].cpu(), k, v, q)
    p.c.health()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kv,G,n_list,sink,window", [(1, 2, 700, 64, 96), (2, 4, 150, 0, 320), (8, 2, 101, 512, 0), (4, 7, 33, 32, 32), (1, 16, 1, 0, 0)])
def test_every_listed_page_counts_once(kv, G, n_list, sink, window, dtype):
    """Lists of more positions than one level of joining takes (12 splits of 8), and of few, between sink and window; some entries are none."""
    n, full = 40010, 1250
    p = Pair(n_kv=kv, G=G, max_seqs=2, max_ctx=40960, n_pages=1252, dtype=dtype)
    k, v = told_apart(p, 1, n)
    rng = random.Random(n_list)
    first, last = sink // PG, full - window // PG
    lists = [rng.sample(range(first, last), n_list) for _ in range(kv)]
    for l in lists:
        for i in range(3, n_list, 7):
            l[i] = rng.choice([-1, full, full + 5, 0 if first else -9, last if last < full else -1])
    attended = []
    for l in lists:
        pages = list(range(first)) + list(range(last, full)) + [i for i in l if first <= i < last]
        attended.append(torch.tensor([t for i in pages for t in range(i * PG, i * PG + PG)] + list(range(full * PG, n))))
    q = group_queries(p)
    out = torch.empty_like(q, device="cuda")
    p.c.attn(0, ints([1]), q.cuda(), out, pages=ints(lists).view(1, kv, n_list), sink=sink, window=window)
    check_told_apart(p, out[0].cpu(), k, v, q, attended)
    p.c.health()


@pytest.mark.parametrize("kv,G,rows", [(32, 4, 4), (32, 8, 2), (32, 1, 16), (16, 2, 9), (32, 7, 3)])
def test_every_shared_page_counts_once(kv, G, rows):
    """Branches that are read together, and each one's own pages behind: every head of every row has all of them."""
    p = Pair(n_kv=kv, G=G, max_seqs=rows, max_ctx=8192, n_pages=180 + 40 * rows)
    k, v = told_apart(p, 0, 5600)
    seqs = list(range(rows))
    p.c.fork(ints([0] * (rows - 1)), ints(seqs[1:]))
    tails = [(s * 37 + 11) % 300 for s in seqs]
    cu = [0]
    for t in tails:
        cu.append(cu[-1] + t)
    own_k, own_v = torch.zeros((2, cu[-1], kv, D))
    own_k[..., 0] = 64.0
    for s in seqs:
        own_v[cu[s]:cu[s + 1], :, s] = 3.0
    own_k, own_v = own_k.bfloat16(), own_v.bfloat16()
    p.c.extend(ints(seqs), ints(cu))
    p.c.append(0, ints(seqs), own_k.cuda(), own_v.cuda(), ints(cu))
    q = group_queries(p)
    out = torch.empty((rows, kv * G, D), dtype=q.dtype, device="cuda")
    p.c.attn(0, ints(seqs), q.repeat(rows, 1, 1).cuda(), out)
    for s in seqs:
        a, b = (torch.cat((x, y[cu[s]:cu[s + 1]])) for x, y in ((k, own_k), (v, own_v)))
        check_told_apart(p, out[s].cpu(), a, b, q)
    p.c.health()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_listed_pages_come_out_as_near(dtype):
    """Random keys and values, lists of several requests: within the bound, and the nearest numbers but for few."""
    p = Pair(n_kv=2, G=4, max_seqs=3, max_ctx=4096, n_pages=300, dtype=dtype)
    p.grow([0, 1, 2], [4000, 1999, 700])
    rng = random.Random(5)
    lists = [[sorted(rng.sample(range(2, 120), 60)) for _ in range(2)] for _ in range(3)]
    got = p.check_attention(0, [0, 1, 2], lists, sink=64, window=96)
    assert torch.isfinite(got.float()).all()
