"""plc_attend against the formula in 64 bits, over the shapes, trees and values where it can go wrong."""
import math
import random

import pytest
import torch

from paper_2604_15356_amd import plc
from paper_2604_15356_amd.paged import PagedKVCache

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def offsets(counts):
    return ints([sum(counts[:i]) for i in range(len(counts) + 1)])


def random_tree(rng, t):
    return [rng.randrange(max(-1, i - 9), i) for i in range(t)]


def make(dtype, d, H, B, lens, seed, L=1, layout="plain", fill=float("nan")):
    """A cache with these lengths, on pages in random order; rows that no session has hold `fill`."""
    rng = random.Random(seed)
    torch.manual_seed(seed)
    counts = [-(-n // B) for n in lens]
    P, M = sum(counts) + 3, max(counts) + 1
    if layout == "plain":
        k, v = (torch.full((P, L, H, B, d), fill, dtype=dtype, device=DEV) for _ in range(2))
    else:  # rows of all heads next to each other, components with a gap behind
        k, v = (torch.full((P, L, B, H, d + 8), fill, dtype=dtype, device=DEV)[..., :d].permute(0, 1, 3, 2, 4) for _ in range(2))
    free = rng.sample(range(P), P)
    table = [[free.pop() for _ in range(c)] for c in counts]
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    refs[ints([p for row in table for p in row]).long()] = 1
    cache = PagedKVCache(k, v, ints([row + [-1] * (M - len(row)) for row in table]), ints(lens), refs)
    rows = [torch.randn((sum(lens), L, H, d), device=DEV).to(dtype) for _ in range(2)]
    if sum(lens):
        cache.store(*rows, offsets(lens))
    cache.check_status()
    return cache, rows


def definition(q, k, v, lens, counts, parents, G, scale):
    """(out, lse, sum of weights times |v|, largest sum |q k|) in 64 bits; k, v [rows, H, d] packed over the sessions.
    Positions that a node does not see take no part, whatever they hold."""
    N, heads, d = q.shape
    H = heads // G
    out, absolute = (torch.zeros((N, heads, d), dtype=torch.float64) for _ in range(2))
    lse = torch.full((N, heads), -math.inf, dtype=torch.float64)
    size = torch.zeros((N, heads), dtype=torch.float64)
    q, k, v = (x.double().cpu() for x in (q, k, v))
    row0 = x = 0
    for n, t in zip(lens, counts):
        for i in range(t):
            seen, a = list(range(n - t)), i
            while a >= 0:
                seen.append(n - t + a)
                a = parents[x - i + a] if parents is not None else a - 1
            seen = torch.tensor(seen) + row0
            for h in range(H):
                qs, ks, vs = q[x, h * G:(h + 1) * G], k[seen, h], v[seen, h]
                s = scale * (qs @ ks.T)
                lse[x, h * G:(h + 1) * G] = torch.logsumexp(s, 1)
                w = torch.softmax(s, 1)
                out[x, h * G:(h + 1) * G] = w @ vs
                absolute[x, h * G:(h + 1) * G] = w @ vs.abs()
                size[x, h * G:(h + 1) * G] = (scale * (qs.abs() @ ks.abs().T)).amax(1)
            x += 1
        row0 += n
    return out, lse, absolute, size


def bounds(dtype, d, n, out, lse, absolute, size, vmax):
    """How far a right result can be off, from the roundings: a score's products are exact in 32 bits and their sum of d has
    d additions; multiplying by the scale, the subtraction of the maximum and exp2 add a few; a weight is then off by the
    score's error, relatively, and by half a step of its type; the sums of n weights and of n products add up to n + 2 more
    roundings in 32 bits each (joins of chunks included); the result is rounded once.  Weights far below 1 are held in steps
    of 2^-24 in fp16 (its smallest), of nothing that matters in bf16."""
    half = torch.finfo(dtype).eps / 2
    u = 2.0 ** -24
    score = size * (d + 4) * u + (lse.abs() + size) * 4 * u + 8 * u
    weight = 2 * score + 2 * (n + 4) * u
    tol = (half * 1.01 + weight)[..., None] * absolute + half * 1.01 * out.abs()
    if dtype == torch.float16:
        tol = tol + n * 2.0 ** -25 * vmax + 2.0 ** -25
    else:
        tol = tol + 1e-30
    return tol, score + (n + 4) * u


def check(dtype, d, G, H, B, lens, counts, tree, seed, layout="plain", scale=None, L=1, layer=0, hints=True, sharp=1.0):
    rng = random.Random(seed)
    cache, (k, v) = make(dtype, d, H, B, lens, seed, L=L, layout=layout)
    N = sum(counts)
    q = (sharp * torch.randn((N, H * G, d + (8 if layout != "plain" else 0)), device=DEV)).to(dtype)[..., :d]
    parents = [p for t in counts for p in random_tree(rng, t)] if tree else None
    kw = dict(max_nodes=max(counts + [1]), max_len=max(lens + [1])) if hints else {}
    got, lse = cache.attend(q, offsets(counts), parents=None if parents is None else ints(parents), layer=layer, scale=scale, **kw)
    cache.check_status()
    scale = d ** -0.5 if scale is None else scale
    want, want_lse, absolute, size = definition(q, k[:, layer], v[:, layer], lens, counts, parents, G, scale)
    tol, tol_lse = bounds(dtype, d, max(lens), want, want_lse, absolute, size, float(v.abs().max()) if v.numel() else 0)
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    off = (lse.double().cpu() - want_lse).abs()
    assert bool((off <= tol_lse).all()), float((off / tol_lse).max())
    return cache, q, parents, got, lse


BOTH = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])


@BOTH
@pytest.mark.parametrize("d", [8, 40, 64, 80, 128, 136, 256])
@pytest.mark.parametrize("G,t", [(1, 1), (3, 7), (4, 12), (5, 33)])
def test_components_and_rows(dtype, d, G, t):
    """Every width of the kernels, whole and not, with rows for each of their arrangements."""
    check(dtype, d, G, 2, 16, [t + 100, t], [t, t], True, seed=d + t)


@BOTH
@pytest.mark.parametrize("lens,counts", [([1], [1]), ([2, 1, 3], [1, 1, 1]), ([16, 17, 15, 31, 32, 33], [1] * 6),
                                         ([127, 128, 129, 300], [1] * 4), ([5, 0, 40, 9], [5, 0, 0, 2]), ([1000, 257], [1, 3])])
@pytest.mark.parametrize("B", [16, 64])
def test_lengths(dtype, lens, counts, B):
    check(dtype, 64, 2, 2, B, lens, counts, False, seed=len(lens) + B)


@BOTH
@pytest.mark.parametrize("t", [2, 63, 64, 65, 130, 256])
def test_trees_across_the_words_of_their_masks(dtype, t):
    check(dtype, 64, 1, 2, 32, [t + 45, t], [t, t], True, seed=t)


@pytest.mark.parametrize("t,n", [(17, 17), (100, 333), (300, 300), (513, 700)])
def test_chains_of_a_prompts_pieces(t, n):
    check(torch.bfloat16, 128, 2, 1, 16, [n, 40], [t, 40], False, seed=t)


@BOTH
@pytest.mark.parametrize("n", [5000, 20011])
@pytest.mark.parametrize("t,G", [(1, 4), (9, 4), (40, 4)])
def test_long_contexts_are_joined_from_chunks(dtype, n, t, G):
    check(dtype, 128, G, 1, 16, [n, 700, t], [t, t, t], True, seed=n + t)


@pytest.mark.parametrize("d", [64, 96, 256])
@pytest.mark.parametrize("G,t", [(2, 3), (20, 2), (40, 2)])
def test_many_tiles_and_heads(d, G, t):
    """Several tiles and heads for each compute unit: the smaller workgroups, each of their arrangements."""
    lens = [t + 5 * i for i in range(16)]
    check(torch.bfloat16, d, G, 64, 16, lens, [t] * 16, True, seed=d + G)


@pytest.mark.parametrize("lens", [[17 * i + 1 for i in range(100)], [9] * 70 + [5000], [1601 - 8 * i for i in range(200)],
                                  [20000] + [3] * 59])
def test_chunks_follow_the_sessions_lengths(lens):
    """Contexts of which the host knows the longest only: many sessions, one long one among short ones."""
    check(torch.float16, 64, 2, 1, 16, lens, [1 + (i % 2) * (n > 1) for i, n in enumerate(lens)], True, seed=len(lens))


@pytest.mark.parametrize("d", [64, 128, 200, 256])
@pytest.mark.parametrize("G,t", [(2, 1), (5, 9), (6, 30)])
def test_contexts_cut_in_some_parts(d, G, t):
    """A dozen tiles and heads: parts enough for several groups of lanes to join, in every arrangement of rows."""
    check(torch.bfloat16, d, G, 1, 32, [1500 + 97 * i for i in range(12)], [t - i % 2 * (t > 1) for i in range(12)], True, seed=d + t)


def test_strides_layers_and_scales():
    for layer in range(3):
        check(torch.float16, 80, 2, 3, 16, [50, 7], [5, 7], True, seed=layer, layout="gaps", L=3, layer=layer, scale=0.3)
    check(torch.bfloat16, 128, 4, 2, 1024, [1500, 3], [2, 1], False, seed=9, hints=False)


def test_sharp_scores():
    """Scores of a hundred and more: the maximum moves by leaps, most weights vanish."""
    for dtype in (torch.float16, torch.bfloat16):
        check(dtype, 64, 2, 2, 16, [900, 70], [4, 4], True, seed=3, sharp=30.0)


@BOTH
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_a_node_does_not_see_has_no_effect(dtype, bad):
    """Infinities and NaN in the rows of other branches, and behind the end: the results are those without, bit for bit."""
    t, n, d, H, G, B = 30, 75, 64, 2, 2, 16
    for rows_per in (1, 8):
        cache, (k, v) = make(dtype, d, H, B, [n], seed=4, fill=bad)
        G = rows_per
        q = torch.randn((t, H * G, d), device=DEV).to(dtype)
        parents = [-1 if i % 2 == 0 and i < 4 else i - 2 if i >= 2 else -1 for i in range(t)]  # even and odd branches
        clean, clean_lse = cache.attend(q, offsets([t]), parents=ints(parents))
        odd = torch.zeros(n, dtype=torch.bool, device=DEV)
        odd[n - t + 1:: 2] = True
        k2, v2 = k.clone(), v.clone()
        k2[odd], v2[odd, :, :, ::3] = bad, bad
        cache.store(k2, v2, offsets([n]))
        got, lse = cache.attend(q, offsets([t]), parents=ints(parents))
        cache.check_status()
        assert torch.isfinite(clean).all() and torch.equal(got[::2], clean[::2]) and torch.equal(lse[::2], clean_lse[::2])
        if bad != bad:
            assert torch.isnan(got[1::2][..., ::3]).all() and torch.isnan(lse[1::2]).all()


@BOTH
def test_infinite_values_that_are_seen(dtype):
    """Of V, in the context and in the tree: the components they are in come out infinite, the others as ever."""
    t, n, d = 6, 70, 64
    cache, (k, v) = make(dtype, d, 1, 16, [n], seed=6)
    q = torch.randn((t, 1, d), device=DEV).to(dtype)
    parents = [-1, 0, 1, -1, 3, 4]
    clean, _ = cache.attend(q, offsets([t]), parents=ints(parents))
    v2 = v.clone()
    v2[3, 0, 0, 5] = math.inf      # everybody sees it
    v2[n - t + 1, 0, 0, 9] = -math.inf  # nodes 1 and 2 see it
    cache.store(k, v2, offsets([n]))
    got, _ = cache.attend(q, offsets([t]), parents=ints(parents))
    cache.check_status()
    assert (got[:, 0, 5] == math.inf).all() and (got[1:3, 0, 9] == -math.inf).all()
    rest = torch.ones((t, d), dtype=torch.bool, device=DEV)
    rest[:, 5] = False
    rest[1:3, 9] = False
    assert torch.equal(got[:, 0][rest], clean[:, 0][rest])


def test_scores_of_the_lowest_value():
    """Rows of which nothing is left but the lowest scores: zeros, and a sum of minus infinity."""
    cache, (k, v) = make(torch.bfloat16, 64, 1, 16, [40], seed=8)
    q = torch.zeros((2, 1, 64), device=DEV, dtype=torch.bfloat16)
    q[0] = 1.0
    k2 = torch.full_like(k, -math.inf)
    cache.store(k2, v, offsets([40]))
    got, lse = cache.attend(q[:1], offsets([1]))
    assert (got == 0).all() and (lse == -math.inf).all()
    k2.fill_(torch.finfo(torch.bfloat16).min)  # as far down as fp32 goes: equal weights, or none
    cache.store(k2, v, offsets([40]))
    got, lse = cache.attend(q[:1] * 0 + 2.0 ** -120, offsets([1]))
    cache.check_status()
    want = v[:, 0, 0].double().mean(0)
    assert torch.allclose(got[0, 0].double(), want, atol=2.0 ** -8 * float(v.abs().max()))
    cache.check_status()


def test_broken_descriptions_raise_status():
    def refused(call):
        cache, _ = make(torch.float16, 64, 1, 16, [40, 30], seed=2)
        q = torch.randn((6, 2, 64), device=DEV, dtype=torch.float16)
        out = torch.full_like(q, 5.0)
        call(cache, q, out)
        with pytest.raises(plc.PlcError) as e:
            cache.check_status()
        assert e.value.code == plc.PLC_ERR_INVALID
        return out

    three = offsets([3, 3])
    refused(lambda c, q, o: c.attend(q, three, parents=ints([-1, 1, 0, -1, 0, 1]), out=o))  # a node that is its own parent
    refused(lambda c, q, o: c.attend(q, three, parents=ints([-1, 0, 2, -1, 0, 1]), out=o))
    refused(lambda c, q, o: c.attend(q, three, parents=ints([-2, 0, 1, -1, 0, 1]), out=o))
    out = refused(lambda c, q, o: c.attend(q, three, max_nodes=2, out=o))
    assert (out == 5).all()
    out = refused(lambda c, q, o: c.attend(q, three, max_len=39, out=o))
    assert (out[:3] == 5).all() and not (out[3:] == 5).any()
    for off in ([0, 3, 7], [-1, 3, 6], [0, 3, 2]):
        refused(lambda c, q, o: c.attend(q, ints(off), out=o))
    for page in (-1, 100, 2**31 - 1, -2**31):
        def broken(c, q, o):
            c.table[0, 1] = page
            c.attend(q, three, out=o)
        refused(broken)
    for length in (-1, 2, 65, 2**31 - 1):
        def broken(c, q, o):
            c.lens[0] = length
            c.attend(q, three, out=o)
        refused(broken)


def test_another_stream_and_a_graph():
    """A step on a stream of its own, eagerly and captured, gives the same as on the default one, at every replay."""
    torch.manual_seed(1)
    S, L, H, G, d, B, t = 3, 2, 2, 4, 64, 16, 5
    start = [40, 16, 3]
    counts, path, path_off = [t] * S, ints([0, 2, 1, 3, 4, 0]), offsets([2, 3, 1])
    parents = ints([-1, 0, 0, 2, -1] * S)
    k, v = (torch.randn((S * t, L, H, d), device=DEV, dtype=torch.float16) for _ in range(2))
    q = torch.randn((S * t, H * G, d), device=DEV, dtype=torch.float16)
    off, grow, src = offsets(counts), ints(counts), ints([0, 1, 1])
    cache, _ = make(torch.float16, d, H, B, start, seed=1, L=L, fill=0.0)
    state = (cache.k, cache.v, cache.table, cache.lens, cache.refs)
    before = [x.clone() for x in state]
    cache.reserve(G, S * t, t, 4 * B)
    outs = [torch.zeros_like(q) for _ in range(L)]

    def step():
        cache.fork(src)
        cache.extend(grow)
        cache.store(k, v, off)
        for layer in range(L):
            cache.attend(q, off, parents=parents, layer=layer, max_nodes=t, max_len=4 * B, out=outs[layer])
        cache.accept(off, path, path_off)
        cache.compact()

    def rewind():
        for x, b in zip(state, before):
            x.copy_(b)

    step()
    cache.check_status()
    want = [x.clone() for x in outs + list(state)]
    side = torch.cuda.Stream()
    rewind()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in outs:
            x.zero_()
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(outs + list(state), want))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        rewind()
        for x in outs:
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outs + list(state), want))
        cache.check_status()
    many, off = torch.zeros((400, H * G, d), dtype=torch.float16, device=DEV), ints([0, 400, 400, 400])
    with pytest.raises(RuntimeError, match="reserve"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            cache.attend(many, off, max_len=1 << 20)


def test_no_nodes():
    cache, _ = make(torch.float16, 64, 1, 16, [40], seed=2)
    out, lse = cache.attend(torch.zeros((0, 2, 64), dtype=torch.float16, device=DEV), offsets([0]))
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
    cache.check_status()


def test_a_cache_beyond_32_bits():
    """Rows on pages whose elements lie beyond 2^31, and a page that every session shares."""
    H, B, d, G = 2, 1024, 128, 2
    P = (1 << 31) // (H * B * d) + 4
    k, v = (torch.empty((P, 1, H, B, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pages = [P - 1, 0, P - 2]
    torch.manual_seed(3)
    for p in pages:
        k[p], v[p] = (torch.randn((1, H, B, d), device=DEV).to(torch.bfloat16) for _ in range(2))
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    cache = PagedKVCache(k, v, ints([pages, pages]), ints([3 * B - 5, B + 1]), refs)
    q = torch.randn((4, H * G, d), device=DEV).to(torch.bfloat16)
    got, lse = cache.attend(q, offsets([3, 1]), parents=ints([-1, -1, 0, -1]))
    cache.check_status()
    rows = [torch.cat([x[p, 0].transpose(0, 1) for p in pages]) for x in (k, v)]
    lens = [3 * B - 5, B + 1]
    packed = [torch.cat([x[:n] for n in lens]) for x in rows]
    want, want_lse, absolute, size = definition(q, *packed, lens, [3, 1], [-1, -1, 0, -1], G, d ** -0.5)
    tol, tol_lse = bounds(torch.bfloat16, d, 3 * B, want, want_lse, absolute, size, 0)
    assert bool(((got.double().cpu() - want).abs() <= tol).all()) and bool(((lse.double().cpu() - want_lse).abs() <= tol_lse).all())


@BOTH
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("G,H,d", [(1, 1, 64), (8, 1, 64), (16, 1, 64), (2, 1, 256), (8, 1, 256), (16, 1, 256), (16, 1024, 8)])
def test_infinite_values_where_context_and_tree_meet(dtype, bad, G, H, d):
    """A context that ends inside a block of 32 positions, an infinity or a NaN in V of its last rows, others in the tree and
    behind the end: what everybody sees reaches everybody, what a node does not see has no effect on it."""
    t, n = 6, 76
    parents = [-1, 0, 1, -1, 3, 4]
    cache, (k, v) = make(dtype, d, H, 16, [n], seed=G + d, fill=bad)
    q = torch.randn((t, H * G, d), device=DEV).to(dtype)
    clean, clean_lse = cache.attend(q, offsets([t]), parents=ints(parents), max_nodes=t)
    assert torch.isfinite(clean).all()
    v2 = v.clone()
    v2[n - t - 4, 0, :, 5] = bad   # in the context
    v2[n - t + 1, 0, :, 3] = bad   # nodes 1 and 2 see it
    cache.store(k, v2, offsets([n]))
    got, lse = cache.attend(q, offsets([t]), parents=ints(parents), max_nodes=t)
    cache.check_status()
    touched = torch.zeros((t, H * G, d), dtype=torch.bool, device=DEV)
    touched[..., 5] = True
    touched[1:3, :, 3] = True
    is_bad = torch.isnan(got) if bad != bad else got == bad
    assert is_bad[touched].all() and torch.equal(got[~touched], clean[~touched]) and torch.equal(lse, clean_lse)


def definition_by_heads(q, k, v, lens, counts, parents, G, scale):
    """What `definition` gives, a session at a time with all of its heads, on the device."""
    N, heads, d = q.shape
    H = heads // G
    out, absolute = (torch.zeros((N, heads, d), dtype=torch.float64, device=DEV) for _ in range(2))
    lse, size = (torch.zeros((N, heads), dtype=torch.float64, device=DEV) for _ in range(2))
    row0 = x = 0
    for n, t in zip(lens, counts):
        if t:
            sees = torch.zeros((t, n), dtype=torch.bool)
            sees[:, : n - t] = True
            for i in range(t):
                a = i
                while a >= 0:
                    sees[i, n - t + a] = True
                    a = parents[x + a] if parents is not None else a - 1
            hidden = ~sees.to(DEV).repeat_interleave(G, 0)  # [t G, n]
            qs = q[x: x + t].double().view(t, H, G, d).transpose(0, 1).reshape(H, t * G, d)
            ks, vs = (r[row0: row0 + n].double().transpose(0, 1).contiguous() for r in (k, v))
            turned = ks.transpose(1, 2).contiguous()
            s = (scale * (qs @ turned)).masked_fill(hidden, -math.inf)
            w = torch.softmax(s, 2)
            back = lambda y: y.view(H, t, G, -1).transpose(0, 1).reshape(t, heads, -1)  # noqa: E731
            out[x: x + t], absolute[x: x + t] = back(w @ vs), back(w @ vs.abs())
            lse[x: x + t] = back(torch.logsumexp(s, 2, keepdim=True))[..., 0]
            size[x: x + t] = back((scale * (qs.abs() @ turned.abs())).masked_fill(hidden, 0).amax(2, keepdim=True))[..., 0]
        x += t
        row0 += n
    return out.cpu(), lse.cpu(), absolute.cpu(), size.cpu()


def check_by_heads(dtype, d, G, H, B, lens, counts, tree, seed, **kw):
    """`check` for many heads and long contexts."""
    rng = random.Random(seed)
    cache, (k, v) = make(dtype, d, H, B, lens, seed)
    q = torch.randn((sum(counts), H * G, d), device=DEV).to(dtype)
    parents = [p for t in counts for p in random_tree(rng, t)] if tree else None
    got, lse = cache.attend(q, offsets(counts), parents=None if parents is None else ints(parents), max_nodes=max(counts),
                            max_len=max(lens), **kw)
    cache.check_status()
    want, want_lse, absolute, size = definition_by_heads(q, k[:, 0], v[:, 0], lens, counts, parents, G, d ** -0.5)
    tol, tol_lse = bounds(dtype, d, max(lens), want, want_lse, absolute, size, float(v.abs().max()))
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    off = (lse.double().cpu() - want_lse).abs()
    assert bool((off <= tol_lse).all()), float((off / tol_lse).max())


@BOTH
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("d", [64, 96, 128, 200])
@pytest.mark.parametrize("G,t", [(2, 3), (20, 2), (9, 9), (7, 23)])
def test_workgroups_that_take_several_chunks(dtype, tree, d, G, t):
    """2560 tiles and heads and more, of which 2048 workgroups take one or several: what one chunk has left in the shared
    memory is not what the next one reads."""
    lens = [t + (13 * i) % 90 for i in range(40)]
    check_by_heads(dtype, d, G, 64, 16, lens, [t - (i % 3) * (t > 3) for i in range(40)], tree, seed=d + G)


@BOTH
@pytest.mark.parametrize("d", [64, 128, 200])
@pytest.mark.parametrize("S,H,longest", [(8, 32, 9000), (8, 64, 9000), (4, 64, 25000), (20, 64, 9000)])
@pytest.mark.parametrize("G,t", [(2, 1), (20, 2), (4, 23)])
def test_many_tiles_and_heads_of_long_contexts(dtype, d, S, H, longest, G, t):
    """As many tiles and heads as there are compute units, or more, and a context that is cut all the same: partial results
    of every arrangement of rows, of short sessions beside them, and of workgroups that take several chunks."""
    lens = [t + (37 * i) % 200 for i in range(S)]
    lens[S // 2] = longest
    check_by_heads(dtype, d, G, H, 16, lens, [t] * S, True, seed=d + S)


@BOTH
@pytest.mark.parametrize("d,B", [(64, 64), (96, 16), (256, 32)])
@pytest.mark.parametrize("t,n", [(130, 130), (257, 700), (600, 2500)])
def test_chains_of_many_nodes(dtype, d, B, t, n):
    """A prompt's pieces in other types, widths and pages than `test_chains_of_a_prompts_pieces`."""
    check_by_heads(dtype, d, 3, 2, B, [n, 77], [t, 40], False, seed=t)


def test_the_same_call_gives_the_same():
    """Parts are joined in a fixed order: a call repeats itself bit for bit."""
    for lens, t, G in (([5000, 20011, 700], 9, 4), ([3000], 1, 4), ([4000, 90, 1200, 40], 40, 3)):
        cache, _ = make(torch.bfloat16, 128, 2, 16, lens, seed=t)
        q = torch.randn((t * len(lens), 2 * G, 128), device=DEV).to(torch.bfloat16)
        first = cache.attend(q, offsets([t] * len(lens)), max_nodes=t)
        for _ in range(5):
            again = cache.attend(q, offsets([t] * len(lens)), max_nodes=t)
            assert all(torch.equal(a, b) for a, b in zip(first, again))
        cache.check_status()


@BOTH
@pytest.mark.parametrize("d,G,t,n", [(64, 4, 5, 600), (128, 8, 5, 3000), (128, 8, 30, 900), (256, 8, 4, 500)])
def test_a_rows_result_is_its_own(dtype, d, G, t, n):
    """Other rows of a tile with larger scores, whose maxima move in other places, do not show in a row's result."""
    cache, _ = make(dtype, d, 1, 16, [n], seed=t)
    q = torch.randn((t, G, d), device=DEV).to(dtype)
    parents = ints(random_tree(random.Random(t), t))
    first, first_lse = cache.attend(q, offsets([t]), parents=parents, max_nodes=t)
    for factor in (4.0, 30.0):
        other = q.clone()
        other[:, 1:] *= factor
        got, lse = cache.attend(other, offsets([t]), parents=parents, max_nodes=t)
        assert torch.equal(got[:, 0], first[:, 0]) and torch.equal(lse[:, 0], first_lse[:, 0])
    cache.check_status()


@pytest.mark.parametrize("exponent", [11, 20, 40, 50, 58])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("d,G,n", [(64, 1, 40), (64, 40, 700), (128, 2, 9000), (256, 3, 300)])
def test_scores_of_any_size(d, G, n, sign, exponent):
    """Scores all over the range of fp32, to both sides: equal ones share their weight, those of twice the size have none or
    all of it.  (Powers of two: every product and sum is exact, so that equal scores are equal.)"""
    cache, (k, v) = make(torch.bfloat16, d, 1, 16, [n], seed=8)
    big = torch.arange(n) % 7 < 3
    size = torch.where(big, 2.0, 1.0) * 2.0 ** exponent
    cache.store(size.to(DEV).to(torch.bfloat16)[:, None, None, None].expand_as(k).contiguous(), v, offsets([n]))
    q = torch.full((1, G, d), sign * 2.0 ** exponent, dtype=torch.bfloat16, device=DEV)
    got, lse = cache.attend(q, offsets([1]))
    cache.check_status()
    kept = big if sign > 0 else ~big
    score = sign * (2.0 if sign > 0 else 1.0) * 4.0 ** exponent * d ** 0.5
    count = int(kept.sum())
    want, absolute = v[:, 0, 0].double().cpu()[kept].mean(0), v[:, 0, 0].double().cpu()[kept].abs().mean(0)
    # the weights' rounding and the result's, each half a step of bf16, and sums in 32 bits
    tol = (2.0 ** -8 * 1.01 + 4 * (n + 4) * 2.0 ** -24) * absolute + 2.0 ** -8 * 1.01 * want.abs()
    assert bool(((got[0].double().cpu() - want).abs() <= tol).all())
    assert bool(((lse.double().cpu() - (score + math.log(count))).abs() <= abs(score) * 4 * 2.0 ** -24 + (n + 4) * 2.0 ** -24).all())


@pytest.mark.parametrize("G,t,n", [(4, 5, 600), (8, 30, 900), (4, 2, 9000)])
def test_far_scores_of_other_rows_do_not_show(G, t, n):
    cache, _ = make(torch.bfloat16, 128, 2, 16, [n], seed=t)
    q = torch.randn((t, 2 * G, 128), device=DEV).to(torch.bfloat16)
    first, first_lse = cache.attend(q, offsets([t]), max_nodes=t)
    other = q.clone()
    other[:, 1::2] *= 2.0 ** 30
    got, lse = cache.attend(other, offsets([t]), max_nodes=t)
    cache.check_status()
    assert torch.equal(got[:, ::2], first[:, ::2]) and torch.equal(lse[:, ::2], first_lse[:, ::2])


@BOTH
@pytest.mark.parametrize("gap", [20.0, 40.0, 300.0])
@pytest.mark.parametrize("d,G,n,t", [(64, 1, 70, 1), (64, 8, 300, 6), (64, 20, 300, 6), (128, 2, 900, 5), (128, 8, 9000, 12), (256, 2, 500, 6),
                                     (256, 20, 9000, 6)])
def test_infinite_values_of_little_weight(dtype, gap, d, G, n, t):
    """An infinity reaches whoever sees it, however small its weight: the formula's are above zero.  Its position's scores lie
    e^-20 to e^-300 below the others, at the beginning (the maximum leaps later), in the middle and in the tree."""
    cache, (k, v) = make(dtype, d, 1, 16, [n], seed=n)
    q = torch.zeros((t, G, d), dtype=dtype, device=DEV)
    q[..., 0] = 8.0
    k2 = k.clone()
    k2[..., 0] = gap * d ** 0.5 / 8
    places = {3: range(t), n - t - 1: range(t), n - t: range(t), n // 2: range(t)}  # position: who sees it, in a chain
    if t > 2:
        places[n - t + 2] = range(2, t)
    for p in places:
        k2[p, 0, 0, 0] = 0.0
    k2[:3, 0, 0, 0] = 0.0
    cache.store(k2, v, offsets([n]))
    clean, clean_lse = cache.attend(q, offsets([t]), max_nodes=t)
    assert torch.isfinite(clean).all()
    for i, (p, seeing) in enumerate(places.items()):
        v2 = v.clone()
        v2[p, 0, 0, 5] = math.inf
        v2[p, 0, 0, 9] = -math.inf
        cache.store(k2, v2, offsets([n]))
        got, lse = cache.attend(q, offsets([t]), max_nodes=t)
        rest = torch.ones((t, G, d), dtype=torch.bool, device=DEV)
        rest[list(seeing)] &= (torch.arange(d, device=DEV) != 5) & (torch.arange(d, device=DEV) != 9)
        assert (got[list(seeing)][..., 5] == math.inf).all() and (got[list(seeing)][..., 9] == -math.inf).all(), p
        assert torch.equal(got[rest], clean[rest]) and torch.equal(lse, clean_lse), p
    cache.check_status()


@BOTH
def test_many_small_weights_beside_a_large_one(dtype):
    """A first position that most of the weight goes to, and 130,000 others in one piece with the same small weight each
    (2^-20 of the first, between two of fp16's smallest numbers): together an eighth of the sum."""
    n, t, H, d, gap = 131072, 2048, 64, 8, 13.8125 if dtype == torch.bfloat16 else 13.8359375
    cache, (k, v) = make(dtype, d, H, 1024, [n + t], seed=1)
    k.zero_()
    k[0, ..., 0] = gap
    v.fill_(1.0)
    v[0] = 0.0
    cache.store(k, v, offsets([n + t]))
    q = torch.zeros((t, H, d), dtype=dtype, device=DEV)
    q[..., 0] = 1.0
    got, lse = cache.attend(q, offsets([t]), scale=1.0, max_nodes=t, max_len=n + t)
    cache.check_status()
    small = torch.arange(n, n + t, dtype=torch.float64) * math.exp(-gap)  # those that a node sees, less the first
    want = (small / (1 + small))[:, None, None]
    # half a step of the type, of a weight and of the result; fp16's smallest steps next to a largest weight of 2^7; sums in 32
    # bits, to which 16 products at a time and 32 weights are added
    half, u = torch.finfo(dtype).eps / 2, 2.0 ** -24
    tol = (2.02 * half + 2 * (n + t) / 16 * u + (n + t) / 32 * u) * want + (n + t) * 2.0 ** -32
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    assert bool(((lse.double().cpu() - (gap + (1 + small).log())[:, None]).abs() <= ((n + t) / 32 + 64) * u).all())


@pytest.mark.parametrize("d,G,t,n", [(64, 1, 6, 40), (128, 8, 6, 300), (64, 20, 6, 500), (256, 20, 6, 300), (128, 1, 6, 5000),
                                     (128, 8, 6, 9000), (128, 20, 6, 20011), (256, 9, 6, 9000), (200, 20, 6, 9000)])
def test_rows_of_broken_sessions_are_left_alone(d, G, t, n):
    """A page that is none, wherever in the context, or a parent that is none: the session's rows stay as they were, those of
    the others are what they are without it, and so is the next call's result."""
    H, B = 2, 16
    cache, _ = make(torch.float16, d, H, B, [n, n // 2 + t, n], seed=d + G)
    q = torch.randn((3 * t, H * G, d), device=DEV).to(torch.float16)
    off, tree = offsets([t] * 3), random_tree(random.Random(n), t) * 3

    def call(parents):
        out, lse = torch.full_like(q, 5.0), torch.full((3 * t, H * G), 5.0, device=DEV)
        cache.attend(q, off, parents=ints(parents), max_nodes=t, max_len=n, out=out, lse=lse)
        return out, lse

    clean = call(tree)
    cache.check_status()

    def check_broken(got, s):
        with pytest.raises(plc.PlcError) as e:
            cache.check_status()
        assert e.value.code == plc.PLC_ERR_INVALID
        here = slice(s * t, (s + 1) * t)
        for x, y in zip(got, clean):
            assert (x[here] == 5).all()
            assert torch.equal(x[: here.start], y[: here.start]) and torch.equal(x[here.stop:], y[here.stop:])
        assert all(torch.equal(x, y) for x, y in zip(call(tree), clean))
        cache.check_status()

    for s, slot in ((0, 0), (1, (n // 2 + t - 1) // B), (2, n // B // 2), (2, (n - 1) // B)):
        for page in (-1, cache.P, 2**31 - 1):
            was = int(cache.table[s, slot])
            cache.table[s, slot] = page
            got = call(tree)
            cache.table[s, slot] = was
            check_broken(got, s)
    for s, node, parent in ((0, 0, 0), (1, 3, 4), (2, t - 1, -2)):
        parents = list(tree)
        parents[s * t + node] = parent
        check_broken(call(parents), s)
