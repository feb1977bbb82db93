"""Caches in pages for the tests: made of lists, read back as lists."""
import random

import torch

from paper_2604_15356_amd.paged import PagedKVCache

DEV = "cuda"


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def offsets(counts):
    return ints([sum(counts[:i]) for i in range(len(counts) + 1)])


def make_cache(dtype, d, H, B, lens, seed, L=1, spare=3, layout="plain", fill=float("nan"), width=None):
    """A cache of these lengths on pages in random order, and its rows [rows, L, H, d], sessions one behind the other; rows
    that no session has hold `fill`."""
    rng = random.Random(seed)
    gen = torch.Generator(DEV).manual_seed(seed)
    counts = [-(-n // B) for n in lens]
    P, M = sum(counts) + spare, max(counts) + 1 if width is None else width
    if layout == "plain":
        k, v = (torch.full((P, L, H, B, d), fill, dtype=dtype, device=DEV) for _ in range(2))
    else:  # rows of all heads next to each other, components with a gap behind
        k, v = (torch.full((P, L, B, H, d + 8), fill, dtype=dtype, device=DEV)[..., :d].permute(0, 1, 3, 2, 4) for _ in range(2))
    free = rng.sample(range(P), P)
    table = [[free.pop() for _ in range(c)] for c in counts]
    refs = [0] * P
    for row in table:
        for page in row:
            refs[page] = 1
    cache = PagedKVCache(k, v, ints([row + [-1] * (M - len(row)) for row in table]), ints(lens), ints(refs))
    rows = [torch.randn((sum(lens), L, H, d), device=DEV, generator=gen).to(dtype) for _ in range(2)]
    if sum(lens):
        cache.store(*rows, offsets(lens))
    cache.check_status()
    return cache, rows


def rows_of(cache, s):
    """K and V of a session [n, L, H, d], read through its table."""
    n, B = int(cache.lens[s]), cache.B
    pages = cache.table[s].long()[: -(-n // B)]
    return [x[pages].permute(0, 3, 1, 2, 4).reshape(-1, cache.L, cache.H, cache.d)[:n].clone() for x in (cache.k, cache.v)]


def same_bits(a, b):
    return a.dtype == b.dtype and torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))
