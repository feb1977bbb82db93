"""plc_pages_evict against a model in plain Python: positions, rows, weights, tables, lengths and counts, all of them equal."""
import math
import random

import pytest
import torch

from paged_util import DEV, ints, make_cache, offsets, rows_of, same_bits
from paper_2604_15356_amd import plc

pytestmark = pytest.mark.gpu


def chosen(w, keep, first, last):
    """Positions that stay of those with weights w (a list)."""
    n = len(w)
    mid = sorted(range(first, n - last), key=lambda i: (not math.isnan(w[i]), -w[i] if not math.isnan(w[i]) else 0.0, i))
    return sorted(list(range(first)) + mid[:keep - first - last] + list(range(n - last, n)))


def check(cache, weights, keep, first=0, last=0, refused=(), max_len=None, W=None):
    lens = cache.lens.tolist()
    rows = [rows_of(cache, s) if s not in refused else None for s in range(cache.S)]
    table, refs, w0 = cache.table.tolist(), cache.refs.tolist(), weights.clone()
    pool = cache.k.clone(), cache.v.clone()
    W = max(min(k, n) for k, n in zip(keep, lens)) if W is None else W
    kept = torch.full((cache.S, cache.L, cache.H, W), -7, dtype=torch.int32, device=DEV)
    assert cache.evict(ints(keep), weights, kept, first=first, last=last, max_len=max_len) is kept
    if refused:
        with pytest.raises(plc.PlcError):
            cache.check_status()
    else:
        cache.check_status()
    w_list = w0.tolist()
    for s in range(cache.S):
        n, now = lens[s], min(lens[s], keep[s])
        if s in refused:
            assert int(cache.lens[s]) == n and cache.table[s].tolist() == table[s] and bool((kept[s] == -7).all())
            assert torch.equal(weights[s].view(torch.int32), w0[s].view(torch.int32))
            for page in table[s]:
                if 0 <= page < cache.P:
                    assert same_bits(cache.k[page], pool[0][page]) and same_bits(cache.v[page], pool[1][page])
            continue
        for j in range(-(-now // cache.B), -(-n // cache.B)):
            refs[table[s][j]] -= 1
            table[s][j] = -1
        assert int(cache.lens[s]) == now and cache.table[s].tolist() == table[s]
        got_k, got_v = rows_of(cache, s)
        for layer in range(cache.L):
            for h in range(cache.H):
                stay = list(range(n)) if now == n else chosen(w_list[s][layer][h][:n], now, first, last)
                assert kept[s, layer, h].tolist() == stay + [-7] * (W - now), (s, layer, h)
                idx = torch.tensor(stay, dtype=torch.long, device=DEV)
                assert same_bits(got_k[:, layer, h], rows[s][0][idx, layer, h]) and same_bits(got_v[:, layer, h], rows[s][1][idx, layer, h])
                bits = lambda x: x.view(torch.int32)  # noqa: E731
                assert torch.equal(bits(weights[s, layer, h, :now].contiguous()), bits(w0[s, layer, h][idx]))
                assert torch.equal(bits(weights[s, layer, h, now:].contiguous()), bits(w0[s, layer, h, now:].contiguous()))
    assert cache.refs.tolist() == refs
    return kept


def random_weights(cache, seed, kind="spread"):
    gen = torch.Generator(DEV).manual_seed(seed)
    shape = (cache.S, cache.L, cache.H, cache.M * cache.B)
    w = (torch.randn(shape, device=DEV, generator=gen) * 3).exp()
    if kind == "ties":
        w = torch.randint(0, 4, shape, device=DEV, generator=gen).float()
    elif kind == "zeros":
        w[torch.rand(shape, device=DEV, generator=gen) < 0.9] = 0.0
        w[torch.rand(shape, device=DEV, generator=gen) < 0.1] = -0.0
    elif kind == "odd":
        for value in (float("nan"), float("inf"), float("-inf"), -1.0, 1e-42, 0.0):
            w[torch.rand(shape, device=DEV, generator=gen) < 0.1] = value
    elif kind == "same":
        w.fill_(1.0)
    elif kind == "rising":
        w = torch.arange(shape[3], device=DEV).float().expand(shape).clone()
    return w


@pytest.mark.parametrize("kind", ["spread", "ties", "zeros", "odd", "same", "rising"])
@pytest.mark.parametrize("B,d,dtype", [(16, 64, torch.float16), (64, 80, torch.bfloat16)])
def test_weights_of_every_kind(kind, B, d, dtype):
    lens = [100, 37, 300, 20, 0, 1]
    cache, _ = make_cache(dtype, d, 2, B, lens, seed=d, L=2)
    check(cache, random_weights(cache, 1, kind), [50, 20, 128, 20, 5, 1], first=3, last=8 if kind != "same" else 0)
    check(cache, random_weights(cache, 2, kind), [17, 19, 100, 30, 0, 0] if kind == "zeros" else [20, 11, 99, 11, 0, 1], first=2, last=9,
          refused=(5,) if kind == "zeros" else ())  # (of one position none may stay, but the first and the last would)


@pytest.mark.parametrize("d", [8, 40, 128, 136, 256])
@pytest.mark.parametrize("layout", ["plain", "gaps"])
def test_components_and_layouts(d, layout):
    cache, _ = make_cache(torch.float16, d, 3, 16, [90, 33], seed=d, L=2, layout=layout)
    wide = torch.zeros((2, 3, 2, 256), device=DEV)
    weights = wide.permute(0, 2, 1, 3)[..., 32:32 + cache.M * 16]  # heads before layers, more positions than there are
    weights.copy_(random_weights(cache, d))
    check(cache, weights, [40, 10], first=1, last=4)
    assert bool((wide[..., :32] == 0).all()) and bool((wide[..., 32 + cache.M * 16:] == 0).all())


@pytest.mark.parametrize("n,keep,max_len", [(4096, 2048, 4096), (4097, 4000, 4097), (20000, 7777, None), (9001, 1, None),
                                            (5000, 4999, 1 << 30), (2049, 2048, 4096), (1024, 1023, 1024)])
def test_long_sessions(n, keep, max_len):
    cache, _ = make_cache(torch.float16, 16, 1, 64, [n, 77], seed=n, L=2)
    check(cache, random_weights(cache, n, "ties" if n % 2 else "spread"), [keep, 60], max_len=max_len, first=min(1, keep - 1))
    check(cache, random_weights(cache, n + 1), [max(1, keep // 2), 60], max_len=max_len, last=min(1, keep // 2))


@pytest.mark.parametrize("L,H,n,max_len", [(8, 8, 900, 900), (8, 40, 400, 5000), (2, 3, 6000, 6000)])
def test_rows_past_the_caches(L, H, n, max_len):
    """More than 96 MB in and out, moved by the workgroups that choose and by others: sampled heads, and all rows against what `kept` says."""
    cache, rows = make_cache(torch.float16, 256, H, 64, [n, n], seed=n, L=L)
    weights = random_weights(cache, n)
    w0, k0, v0 = weights.clone(), *(x.view(2, n, L, H, 256).clone() for x in rows)
    kept = cache.evict(ints([n // 2, n - 1]), weights, first=2, last=5, max_len=max_len)
    cache.check_status()
    for s, now in enumerate((n // 2, n - 1)):
        got_k, got_v = rows_of(cache, s)
        assert got_k.shape[0] == now
        idx = kept[s, :, :, :now].long()
        for layer in range(L):
            at = idx[layer].t()[..., None].expand(now, H, 256)
            assert same_bits(got_k[:, layer], torch.gather(k0[s, :, layer], 0, at)) and same_bits(got_v[:, layer], torch.gather(v0[s, :, layer], 0, at))
        for layer, h in ((0, 0), (L - 1, H - 1), (L // 2, 1)):
            assert kept[s, layer, h, :now].tolist() == chosen(w0[s, layer, h, :n].tolist(), now, 2, 5)
        assert torch.equal(weights[s, :, :, :now], torch.gather(w0[s], 2, idx))


def test_borders_of_what_may_stay():
    lens = [64, 64, 64, 64, 64]
    cache, _ = make_cache(torch.float16, 32, 2, 16, lens, seed=1)
    check(cache, random_weights(cache, 1), [10, 11, 63, 64, 1 << 30], first=4, last=6, W=64)  # nobody but the first and last; one more; all but one
    check(cache, random_weights(cache, 2), [0, 0, 1, 0, 16], first=0, last=0)
    assert cache.lens.tolist() == [0, 0, 1, 0, 16] and int(cache.refs.sum()) == 2


def test_sessions_that_cannot_be_shortened_stay_as_they_were():
    lens = [100, 100, 100, 100, 60, 30]
    cache, _ = make_cache(torch.float16, 64, 2, 16, lens, seed=3)
    cache.refs[cache.table[1, 2].long()] += 1  # shared, and would be written
    cache.table[2, 6] = 12345                  # none, behind the new end
    kept = check(cache, random_weights(cache, 1), [50, 50, 50, 9, 50, -1], first=5, last=5, refused=(1, 2, 3, 5))
    assert bool((kept[0] >= 0).all())
    check(cache, random_weights(cache, 2), [41, 100, 100, 100, 100, 100], refused=(1, 2, 3), W=50)  # more of them than W stay
    cache.lens[3] = 5000
    check(cache, random_weights(cache, 2), [30, 20, 20, 20, 20, 20], refused=(2, 3))  # session 1's shared page is not written now
    check(cache, random_weights(cache, 3), [20, 100, 100, 20, 45, 100], refused=(2, 3), max_len=40, W=100)
    narrow = random_weights(cache, 4)[..., :40].contiguous()
    check(cache, narrow, [10, 10, 10, 10, 10, 10], refused=(2, 3))


def test_a_shared_prefix_stays():
    """Sessions that share their first pages are shortened behind them."""
    cache, _ = make_cache(torch.float16, 64, 2, 16, [48, 0], seed=5, spare=20, width=10)
    cache.fork(ints([0, 0]))
    cache.extend(ints([40, 61]))
    k, v = (torch.randn((101, 2, 64), device=DEV).to(torch.float16) for _ in range(2))
    cache.store(k, v, offsets([40, 61]))
    cache.check_status()
    check(cache, random_weights(cache, 1), [60, 75], first=48, last=3)
    check(cache, random_weights(cache, 2), [55, 70], first=47, last=3, refused=(0, 1))  # one less, and their common page would be written
    cache.fork(ints([0, -1]))
    check(cache, random_weights(cache, 3), [20, 5], first=2)


def test_many_sessions():
    rng = random.Random(1)
    lens = [rng.randrange(0, 40) for _ in range(1024)]
    cache, _ = make_cache(torch.float16, 8, 1, 16, lens, seed=1)
    check(cache, random_weights(cache, 1), [max(2, n // 2) for n in lens], first=1, last=1)


def test_pages_given_back_are_taken_again():
    cache, _ = make_cache(torch.float16, 32, 2, 16, [64, 64], seed=1, spare=0, width=8)
    check(cache, random_weights(cache, 1), [20, 30])
    cache.extend(ints([44, 34]))
    cache.check_status()
    assert cache.lens.tolist() == [64, 64] and int(cache.refs.sum()) == 8 and int(cache.refs.max()) == 1


def test_a_pool_beyond_31_bits():
    d, H, B = 128, 8, 16
    from paper_2604_15356_amd.paged import PagedKVCache
    P = 2 ** 31 // (H * B * d) + 8
    k, v = (torch.empty((P, 1, H, B, d), dtype=torch.float16, device=DEV) for _ in range(2))
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    refs[[P - 1, 3, P - 3]] = 1
    cache = PagedKVCache(k, v, ints([[P - 1, 3, P - 3]]), ints([48]), refs)
    cache.store(*(torch.randn((48, H, d), device=DEV).to(torch.float16) for _ in range(2)), offsets([48]))
    weights = random_weights(cache, 1)
    rows = rows_of(cache, 0)
    kept = cache.evict(ints([20]), weights)
    cache.check_status()
    got = rows_of(cache, 0)
    for h in range(H):
        idx = kept[0, 0, h, :20].long()
        assert same_bits(got[0][:, 0, h], rows[0][idx, 0, h]) and same_bits(got[1][:, 0, h], rows[1][idx, 0, h])


def test_another_stream_and_a_graph():
    cache, _ = make_cache(torch.float16, 64, 2, 16, [90, 40], seed=1)
    weights = random_weights(cache, 1)
    state = [x.clone() for x in (cache.k, cache.v, cache.table, cache.lens, cache.refs, weights)]
    live = (cache.k, cache.v, cache.table, cache.lens, cache.refs, weights)

    def put_back():
        for x, y in zip(live, state):
            x.copy_(y)

    keep, kept = ints([40, 30]), torch.zeros((2, 1, 2, 40), dtype=torch.int32, device=DEV)
    cache.evict(keep, weights, kept, first=1)
    want = [x.clone() for x in live] + [kept.clone()]
    put_back()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        cache.evict(keep, weights, kept, first=1)
    stream.synchronize()
    bits = lambda x: x.view(torch.int16 if x.element_size() == 2 else torch.int32)  # noqa: E731
    same = lambda: all(torch.equal(bits(x), bits(y)) for x, y in zip(live + (kept,), want))  # noqa: E731
    assert same()
    put_back()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.evict(keep, weights, kept, first=1)
    for _ in range(3):
        put_back(), kept.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same()
    cache.check_status()
