"""A plain model of the paged cache in 4 bits: the definition of include/freekv_cache.h in 64 bits, one sequence, page and head
after the other.  Shares no code with the kernels."""
import math

import torch

D, PG = 128, 32


def kept(x):
    """What a full page [32, kv, d] of the storage type stands for, in 64 bits: (value, lo, step) with lo, step [kv, d]."""
    y = x.double()
    lo = y.min(0).values
    bad = ~torch.isfinite(y).all(0)
    w = ((y.max(0).values - lo) / 15.0).float()
    w = torch.where(bad, torch.zeros_like(w), w)
    value, step = torch.empty_like(y), torch.zeros_like(lo)
    for m in range(x.shape[1]):
        top = float(w[m].max())
        e = max(math.frexp(top)[1] - 1, -126) if top > 0 else 0
        step[m] = (w[m].double() * 2.0 ** -e).float().half().double() * 2.0 ** e
    code = torch.where(step > 0, torch.round((y - lo) / torch.where(step > 0, step, torch.ones_like(step))), torch.zeros_like(y)).clamp(0, 15)
    value = lo + step * code
    value[:, bad] = math.nan
    lo[bad] = math.nan
    return value, lo, step


class Model:
    def __init__(self, *, n_layers, n_kv, max_seqs, max_ctx, n_pages, dtype):
        self.n_layers, self.n_kv, self.max_ctx, self.dtype = n_layers, n_kv, max_ctx, dtype
        self.ref = [0] * n_pages
        self.pages = [[] for _ in range(max_seqs)]
        empty = torch.empty((0, 2, n_kv, D), dtype=dtype)
        self.tokens = [[empty] * max_seqs for _ in range(n_layers)]       # raw tokens, [n, 2, kv, d]
        self.len = [0] * max_seqs
        self.packed = {}                                                 # the values of pages already worked out

    def take(self, n):
        ids = [p for p, r in enumerate(self.ref) if r == 0][:n]
        for p in ids:
            self.ref[p] = 1
        return ids

    def extend(self, seqs, new):
        need = [(self.len[s] + n) // PG - self.len[s] // PG for s, n in zip(seqs, new)]
        if sum(need) > self.ref.count(0):
            return False
        for s, n, k in zip(seqs, new, need):
            self.pages[s] = self.pages[s] + self.take(k)
            self.len[s] += n
        return True

    def append(self, layer, seqs, new, k, v):
        at = 0
        for s, n in zip(seqs, new):
            x = torch.stack((k[at:at + n], v[at:at + n]), 1).cpu()
            self.tokens[layer][s] = torch.cat((self.tokens[layer][s], x))
            at += n

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.pages[b] = list(self.pages[a])
            for p in self.pages[a]:
                self.ref[p] += 1
            self.len[b] = self.len[a]
            for layer in range(self.n_layers):
                self.tokens[layer][b] = self.tokens[layer][a]

    def copy(self, src, dst, to=None):
        to = self if to is None else to
        if sum(len(self.pages[a]) for a in src) > to.ref.count(0):
            return False
        for a, b in zip(src, dst):
            to.pages[b] = to.take(len(self.pages[a]))
            to.len[b] = self.len[a]
            for layer in range(self.n_layers):
                to.tokens[layer][b] = self.tokens[layer][a]
        return True

    def free(self, seqs):
        for s in seqs:
            for p in self.pages[s]:
                self.ref[p] -= 1
            self.pages[s], self.len[s] = [], 0
            for layer in range(self.n_layers):
                self.tokens[layer][s] = self.tokens[layer][s][:0]

    def used(self):
        return sum(r > 0 for r in self.ref)

    def compact(self):
        live = self.used()
        holes = [p for p in range(live) if self.ref[p] == 0]
        tail = [p for p in range(live, len(self.ref)) if self.ref[p] > 0]
        new = dict(zip(tail, holes))
        for f, t in new.items():
            self.ref[t], self.ref[f] = self.ref[f], 0
        self.pages = [[new.get(p, p) for p in ids] for ids in self.pages]

    def values(self, layer, s):
        """(value, lo, step) of a sequence's tokens [n, 2, kv, d] in 64 bits; lo the value and step 0 in the open page."""
        x = self.tokens[layer][s]
        out = []
        for p in range(0, x.shape[0], PG):
            page = x[p:p + PG]
            if page.shape[0] < PG:
                y = page.double()
                out.append((y, y, torch.zeros_like(y)))
                continue
            key = (page.data_ptr(), p, tuple(page.shape))
            a = [kept(page[:, i]) for i in (0, 1)]
            out.append(tuple(torch.stack([z.expand(PG, *z.shape[-2:]) if z.dim() == 2 else z for z in (a[0][j], a[1][j])], 1) for j in range(3)))
        if not out:
            e = torch.empty((0, 2, self.n_kv, D), dtype=torch.float64)
            return e, e, e
        return tuple(torch.cat([o[j] for o in out]) for j in range(3))

    def attended(self, s, h, pages=None, sink=0, window=0):
        """token numbers, in any order"""
        n = self.len[s]
        full = n // PG
        if pages is None:
            return list(range(n))
        a = min(sink // PG, full)
        b = full - min(window // PG, full - a)
        at = list(range(a)) + list(range(b, full)) + [j for j in pages if a <= j < b]
        return [t for j in at for t in range(j * PG, j * PG + PG)] + list(range(full * PG, n))


def attention(q, value, lo, step, eps_half):
    """One KV head: q [g, d] of T, value / lo / step [n, 2, d] in 64 bits -> (out [g, d], how far off the kernel may be).

    The bound: the output's own rounding; weights are fp16 (half a step, 2^-11 of each, or 2^-28 where they are below fp16's normal
    range) and normalised by the sum of what they were rounded to, so they tell on the spread of the values around the
    output alone; logits are sums of 128 products and the 8 of lo in fp32, each operation 2^-24 of the terms' sizes; the weighted
    sums likewise, over fewer than 512 additions."""
    g, n = q.shape[0], value.shape[0]
    if n == 0:
        return torch.zeros((g, D), dtype=torch.float64), torch.zeros((g, D), dtype=torch.float64)
    q = q.double()
    k, v = value[:, 0], value[:, 1]
    x = (q @ k.T) / math.sqrt(D)
    w = torch.softmax(x, -1)
    out = w @ v
    size_k = lo[:, 0].abs() + 15 * step[:, 0]
    size_v = lo[:, 1].abs() + 15 * step[:, 1]
    dx = 2.0 ** -24 * 300 * (q.abs() @ size_k.T) / math.sqrt(D)
    tol = torch.empty_like(out)
    for i in range(g):
        dev = (v - out[i]).abs()
        tol[i] = ((w[i] * (2.0 ** -11 * 1.02 + 2 * dx[i])) @ dev) + n * 2.0 ** -28 * dev.max(0).values / 1.0
        tol[i] += 2.0 ** -24 * 512 * (w[i] @ size_v)
    return out, tol + eps_half * 1.01 * out.abs() + 2.0 ** -24 * eps_half
