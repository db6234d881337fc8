"""Paged caches for the tests of drafted tokens, and plain implementations in 64 bits."""
import math

import torch


def half_step(dtype):
    """What a rounding to this type is off by at most, relative to the value."""
    return torch.finfo(dtype).eps / 2


class Cache:
    """Keys and values of n sequences in pages of any order.  Everything that is no sequence's place holds `filler`."""

    def __init__(self, lens, m, kv_heads, d, page, dtype, seed=0, filler=math.nan, spare=2, layers=None):
        gen = torch.Generator().manual_seed(seed)
        self.lens_list, self.m, self.kv_heads, self.d, self.page, self.dtype = list(lens), m, kv_heads, d, page, dtype
        each = [-(-(max(at, 0) + m) // page) for at in lens]
        total = sum(each) + spare
        order = torch.randperm(total, generator=gen).tolist()
        most = max(each)
        table, at = [], 0
        for count in each:
            table.append(order[at:at + count] + [-1] * (most - count))
            at += count
        self.table = table
        more = () if layers is None else (layers,)
        self.k = torch.full((*more, total, kv_heads, page, d), filler, dtype=dtype)
        self.v = torch.full((*more, total, kv_heads, page // 8, d, 8), filler, dtype=dtype)
        for s, length in enumerate(lens):
            for p in range(max(length, 0)):
                if layers is None:
                    self.put(s, p, torch.randn(kv_heads, d, generator=gen), torch.randn(kv_heads, d, generator=gen))

    def put(self, s, place, k, v):
        page, off = self.table[s][place // self.page], place % self.page
        self.k[page, :, off] = k.to(self.dtype)
        self.v[page, :, off // 8, :, off % 8] = v.to(self.dtype)

    def get(self, s, place):
        page, off = self.table[s][place // self.page], place % self.page
        return self.k[page, :, off], self.v[page, :, off // 8, :, off % 8]

    def pages(self):
        return torch.tensor(self.table, dtype=torch.int32)

    def lens(self):
        return torch.tensor(self.lens_list, dtype=torch.int32)

    def gpu(self):
        return self.k.cuda(), self.v.cuda(), self.pages().cuda(), self.lens().cuda()


def branch(parents, i):
    """Row i and its ancestors; parents None: a chain."""
    if parents is None:
        return set(range(i + 1))
    out = set()
    while True:
        out.add(i)
        up = int(parents[i])
        if not 0 <= up < i:
            return out
        i = up


def plain_attention(q, k_cache, v_cache, pages, lens, parents=None, counts=None, scale=None):
    """-> (out, lse, the sum of weights times |v|, the sum of |q||k| of the largest score) in 64 bits; all tensors on the CPU."""
    n, m, heads, d = q.shape
    n_pages, kv_heads, page, _ = k_cache.shape
    share, scale = heads // kv_heads, d ** -0.5 if scale is None else scale
    out = torch.zeros((n, m, heads, d), dtype=torch.float64)
    lse = torch.full((n, m, heads), -math.inf, dtype=torch.float64)
    size = torch.zeros((n, m, heads, d), dtype=torch.float64)
    reach = torch.zeros((n, m, heads, 1), dtype=torch.float64)
    table = pages.tolist()
    for s in range(n):
        length = max(int(lens[s]), 0)
        count = m if counts is None else min(max(int(counts[s]), 0), m)
        here = [p for p in range(length + count) if p // page < len(table[s]) and 0 <= table[s][p // page] < n_pages]
        if not count or not here:
            continue
        at = torch.tensor([table[s][p // page] for p in here]), torch.tensor([p % page for p in here])
        k = k_cache[at[0], :, at[1]].double()                                        # [places][kv_heads][d]
        v = v_cache[at[0], :, at[1] // 8, :, at[1] % 8].double()
        place_of = {p: i for i, p in enumerate(here)}
        for i in range(count):
            rows = branch(None if parents is None else parents[s], i)
            seen = [place_of[p] for p in here if p < length or p - length in rows]
            if not seen:
                continue
            ks, vs = k[seen].repeat_interleave(share, dim=1), v[seen].repeat_interleave(share, dim=1)
            x = q[s, i].double()
            score = (ks * x).sum(dim=2) * scale                                      # [seen][heads]
            w = torch.softmax(score, dim=0)[:, :, None]
            out[s, i] = (w * vs).sum(dim=0)
            lse[s, i] = torch.logsumexp(score, dim=0)
            size[s, i] = (w * vs.abs()).sum(dim=0)
            reach[s, i] = (ks.abs() * x.abs()).sum(dim=2).amax(dim=0)[:, None] * abs(scale)
    return out, lse, size, reach


def tree(n, m, seed, chain_bias=0.5):
    """Random parents [n][m]."""
    gen = torch.Generator().manual_seed(seed)
    parents = torch.full((n, m), -1, dtype=torch.int32)
    for s in range(n):
        for i in range(1, m):
            near = torch.rand((), generator=gen) < chain_bias
            parents[s, i] = i - 1 if near else int(torch.randint(-1, i, (), generator=gen))
    return parents


def rotate(x, positions, inv_freq, interleaved, amplitude):
    """Rows [rows][heads][d] turned by their positions, in 64 bits."""
    y = x.double().clone()
    half = inv_freq.numel()
    if half:
        angle = positions.double()[:, None] * inv_freq.double()
        cos, sin = (angle.cos() * amplitude)[:, None, :], (angle.sin() * amplitude)[:, None, :]
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        p, r = y[..., a].clone(), y[..., b].clone()
        y[..., a], y[..., b] = p * cos - r * sin, r * cos + p * sin
    return y
