"""plc_attend_weights against the formula in 64 bits."""
import math

import pytest
import torch

from paged_util import DEV, ints, make_cache, offsets
from paper_2604_15356_amd import plc

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BOTH = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])


def definition(q, k, lse, lens, counts, G, scale, before, decay):
    """(weights, how far a right result may be off) [S, H, width] in 64 bits; k [rows, H, d] packed.  A score's products are exact in
    32 bits, their sum of d has d additions, the scale, the product of the log-sum-exp and their difference a few more roundings; a
    weight is off by that, relatively, and by exp2's step; their sum adds a rounding each, the sum with what was before two."""
    H, d = k.shape[1], k.shape[2]
    want, tol = before.double().cpu().clone(), torch.zeros(before.shape, dtype=torch.float64)
    q, k, lse = q.double().cpu(), k.double().cpu(), lse.double().cpu()
    row0 = x0 = 0
    for s, (n, t) in enumerate(zip(lens, counts)):
        for h in range(H if t else 0):
            qs = q[x0:x0 + t, h * G:(h + 1) * G].reshape(t * G, d)
            ls = lse[x0:x0 + t, h * G:(h + 1) * G].reshape(t * G, 1)
            ks = k[row0:row0 + n, h]
            sees = (torch.arange(n)[None] <= (n - t + torch.arange(t).repeat_interleave(G))[:, None])
            seen = torch.where(sees.any(0)[:, None], ks, torch.zeros_like(ks))
            w = torch.where(sees, (scale * (qs @ seen.T) - ls).exp(), torch.zeros((), dtype=torch.float64))
            size = scale * (qs.abs() @ seen.abs().T)
            sums = w.sum(0)
            err = torch.where(sees, w * (size * (d + 4) * U + (ls.abs() + size) * 4 * U + 8 * U), torch.zeros((), dtype=torch.float64)).sum(0)
            err = err + sums * (t * G + 4) * U
            old = want[s, h, :n - t] * decay if decay else 0.0
            want[s, h, :n] = sums
            want[s, h, :n - t] += old
            tol[s, h, :n] = err + want[s, h, :n].abs() * 3 * U + 1e-36
        row0 += n
        x0 += t
    return want, tol


def run(dtype, d, G, H, B, lens, counts, seed, decay=1.0, layout="plain", L=1, layer=0, scale=None, hints=True, sharp=1.0, pad=0):
    cache, (k, _) = make_cache(dtype, d, H, B, lens, seed, L=L, layout=layout)
    torch.manual_seed(seed)
    N = sum(counts)
    q = (sharp * torch.randn((N + pad, H * G, d + (8 if layout != "plain" else 0)), device=DEV)).to(dtype)[..., :d]
    kw = dict(max_nodes=max(counts + [1]), max_len=max(lens + [1])) if hints else {}
    off = offsets(counts)
    _, lse = cache.attend(q, off, layer=layer, scale=scale, **kw)
    weights = torch.rand((cache.S, L, H, cache.M * B), device=DEV) * 3
    before = weights.clone()
    if decay == 0.0:
        weights.fill_(float("nan"))
    cache.add_weights(q, off, lse, weights, decay=decay, layer=layer, scale=scale, **kw)
    cache.check_status()
    want, tol = definition(q, k[:, layer], lse, lens, counts, G, d ** -0.5 if scale is None else scale, before[:, layer], decay)
    for s, (n, t) in enumerate(zip(lens, counts)):
        got = weights[s, layer].double().cpu()
        if t:
            off_by = (got[:, :n] - want[s, :, :n]).abs()
            assert bool((off_by <= tol[s, :, :n]).all()), (s, float((off_by / tol[s, :, :n]).max()))
        rest = weights[s, :, :, n if t else 0:]  # behind the end, or of a session without nodes: as it was
        assert bool((torch.isnan(rest) if decay == 0.0 else rest == before[s, :, :, n if t else 0:])[layer].all())
    others = [x for x in range(L) if x != layer]
    assert decay == 0.0 or torch.equal(weights[:, others], before[:, others])
    return cache, q, lse, weights


@BOTH
@pytest.mark.parametrize("d", [8, 40, 64, 80, 128, 136, 256])
@pytest.mark.parametrize("G,t", [(1, 1), (3, 7), (4, 12), (5, 33)])
def test_components_and_rows(dtype, d, G, t):
    run(dtype, d, G, 2, 16, [t + 100, t], [t, t], seed=d + t)


@BOTH
@pytest.mark.parametrize("lens,counts", [([1], [1]), ([2, 1, 3], [1, 1, 1]), ([16, 17, 15, 31, 32, 33], [1] * 6),
                                         ([127, 128, 129, 300], [1] * 4), ([5, 0, 40, 9], [5, 0, 0, 2]), ([1000, 257], [1, 3]),
                                         ([600, 90], [200, 90])])
@pytest.mark.parametrize("B", [16, 64])
@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
def test_lengths(dtype, lens, counts, B, decay):
    run(dtype, 64, 2, 2, B, lens, counts, seed=len(lens) + B, decay=decay)


@pytest.mark.parametrize("lens,counts,G,H", [([3000], [513], 4, 2), ([700, 1500, 33], [257, 64, 33], 7, 1), ([9000], [100], 8, 1),
                                             ([400] * 20, [3] * 20, 4, 16), ([2050], [2050], 1, 1)])
def test_many_rows(lens, counts, G, H):
    run(torch.bfloat16, 128, G, H, 16, lens, counts, seed=sum(counts))
    run(torch.float16, 96, G, H, 32, lens, counts, seed=sum(counts), decay=0.25)


@BOTH
@pytest.mark.parametrize("d", [64, 128, 256])
def test_more_tiles_than_a_wavefront_takes(dtype, d):
    """So many sessions and heads that a wavefront takes several tiles: lengths that end in each of them."""
    lens = [500, 1, 33, 64, 65, 127, 128, 129, 200, 257, 300, 512] * 8
    run(dtype, d, 1, 64 if d < 256 else 32, 16, lens, [1] * len(lens), seed=d)


def test_a_layer_of_several_and_rows_with_gaps():
    run(torch.float16, 64, 2, 3, 16, [77, 20], [5, 2], seed=8, L=3, layer=1, layout="gaps")
    run(torch.bfloat16, 72, 4, 2, 64, [500, 20], [64, 2], seed=9, L=2, layer=1, layout="gaps", decay=0.0)


def test_bounds_from_the_host_and_other_scales():
    run(torch.float16, 64, 2, 2, 16, [90, 200], [3, 1], seed=1, hints=False)
    run(torch.float16, 64, 2, 2, 16, [90, 200], [3, 1], seed=1, scale=0.5, sharp=3.0)
    run(torch.bfloat16, 64, 2, 2, 16, [90, 200], [40, 1], seed=1, scale=1.0, sharp=30.0)  # one position takes all
    run(torch.bfloat16, 64, 2, 2, 16, [90, 200], [3, 1], seed=1, pad=5)  # rows behind the last session's


@BOTH
@pytest.mark.parametrize("t", [3, 90])
def test_what_a_row_does_not_see_has_no_effect(dtype, t):
    """Infinities and NaN in keys behind a node, and in a session's unused rows (make_cache fills them with NaN)."""
    lens, H = [100, 95], 2
    cache, _ = make_cache(dtype, 64, H, 16, lens, seed=t)
    q = torch.randn((2 * t, H, 64), device=DEV).to(dtype)
    off = offsets([t, t])
    _, lse = cache.attend(q, off)
    clean = cache.make_weights()
    cache.add_weights(q, off, lse, clean)
    for value in (float("nan"), float("inf")):
        k = cache.k.clone()
        pos = 99  # seen by session 0's last node alone
        cache.k[cache.table[0, pos // 16].long(), 0, :, pos % 16] = value
        weights = cache.make_weights()
        cache.add_weights(q, off, lse, weights)
        assert torch.equal(weights[0, :, :, :99], clean[0, :, :, :99]) and torch.equal(weights[1], clean[1])
        assert bool(torch.isnan(weights[0, 0, :, 99]).all()) or value == float("inf")
        cache.k.copy_(k)
    # minus infinity as a score: no weight, not NaN, also where a tile has rows that are none
    cache.k[cache.table[0, 0].long(), 0, :, 5] = 0
    cache.k[cache.table[0, 0].long(), 0, :, 5, 0] = float("-inf")
    q[:, :, 0] = 1.0
    _, lse = cache.attend(q, off)
    weights = cache.make_weights()
    cache.add_weights(q, off, lse, weights)
    assert bool((weights[0, 0, :, 5] == 0).all()) and bool(torch.isfinite(weights).all())


def test_the_weights_of_a_chain_sum_to_its_rows():
    """Each row gives one in all.  The scores behind lse and these are sums of 128 products of a size of 8 in all, off by 132 steps of
    2^-24 each at most: 1.3e-4 of a weight, twice; all else is far below."""
    cache, q, lse, weights = run(torch.float16, 128, 4, 2, 16, [1000], [16], seed=3, decay=0.0)
    total = weights[0, 0, :, :1000].double().sum(1)
    assert bool(((total - 64).abs() < 64 * 3e-4).all())


def test_the_same_bits_every_time_and_whatever_else_is_in_the_call():
    lens, counts = [700, 64, 300], [70, 3, 1]
    cache, _ = make_cache(torch.bfloat16, 128, 2, 16, lens, seed=6)
    q = torch.randn((74, 8, 128), device=DEV).to(torch.bfloat16)
    _, lse = cache.attend(q, offsets(counts))
    weights = [cache.make_weights() for _ in range(4)]
    for w in weights[:3]:
        cache.add_weights(q, offsets(counts), lse, w, max_nodes=70, max_len=700)
    assert torch.equal(weights[0], weights[1]) and torch.equal(weights[0], weights[2])
    cache.add_weights(q[:70], offsets([70, 0, 0]), lse[:70].contiguous(), weights[3])
    assert torch.equal(weights[0][0], weights[3][0])


@BOTH
@pytest.mark.parametrize("d", [40, 64, 80, 128, 256])
@pytest.mark.parametrize("G,t", [(1, 1), (1, 9), (4, 1), (4, 8), (3, 10), (5, 6), (32, 1), (1, 32)])
def test_a_session_s_bits_whatever_bounds_the_call_has(dtype, d, G, t):
    """Up to 32 rows of a session are added in the same order in a call for few rows and in one for many: what decides between them (max_nodes,
    by default the rows of all sessions) does not show."""
    lens, counts = [300, 129, t], [t, max(1, t - 1), t]
    cache, _ = make_cache(dtype, d, 2, 16, lens, seed=t)
    q = (2 * torch.randn((sum(counts), 2 * G, d), device=DEV)).to(dtype)
    off = offsets(counts)
    _, lse = cache.attend(q, off)
    start = torch.rand(cache.make_weights().shape, device=DEV)
    results = []
    for most in (t, 32 // G + 1, 1000):
        weights = start.clone()
        cache.add_weights(q, off, lse, weights, decay=0.75, max_nodes=most, max_len=300)
        results.append(weights)
    cache.check_status()
    assert t * G <= 32 < (32 // G + 1) * G
    assert torch.equal(results[0], results[1]) and torch.equal(results[0], results[2])


@pytest.mark.parametrize("d,counts", [(64, {0: 1, 5: 3}), (72, {0: 2, 5: 1}), (200, {0: 1, 5: 2}),
                                      (64, {0: 100, 5: 130}), (40, {0: 70, 5: 64}), (128, {0: 33, 5: 129}), (200, {0: 64, 5: 40})])
def test_more_positions_than_the_workgroups_take_at_once(d, counts):
    """4096 sessions and heads: a workgroup takes 16 times its 128, or few rows 512 (d > 128: 256), positions and more of the long sessions, one lot after the
    other; of few rows and of many, of which the lots have one stage, or two, or three."""
    S, H = 64, 64
    lens = [9500 if s == 0 else 5000 if s == 5 else 40 + s for s in range(S)]
    counts = [counts.get(s, 1) for s in range(S)]
    cache, (k, _) = make_cache(torch.float16, d, H, 16, lens, seed=d)
    q = torch.randn((sum(counts), H, d), device=DEV).to(torch.float16)
    off, bounds = offsets(counts), dict(max_nodes=max(counts), max_len=9500)
    _, lse = cache.attend(q, off, **bounds)
    weights = torch.rand((S, 1, H, cache.M * 16), device=DEV)
    before = weights.clone()
    cache.add_weights(q, off, lse, weights, decay=0.5, **bounds)
    cache.check_status()
    heads = [0, 31, 63]
    want, tol = definition(q[:, heads], k[:, 0, heads], lse[:, heads], lens, counts, 1, d ** -0.5, before[:, 0, heads], 0.5)
    for s, n in enumerate(lens):
        got = weights[s, 0, heads].double().cpu()
        assert bool(((got[:, :n] - want[s, :, :n]).abs() <= tol[s, :, :n]).all()), s
        assert torch.equal(weights[s, 0, :, n:], before[s, 0, :, n:])


def test_sessions_that_are_not_as_described():
    """Status, and their weights as they were; the others' as ever."""
    lens, counts = [50, 60, 40], [2, 3, 2]
    cache, _ = make_cache(torch.float16, 64, 2, 16, lens, seed=2)
    q = torch.randn((7, 2, 64), device=DEV).to(torch.float16)
    off = offsets(counts)
    _, lse = cache.attend(q, off)
    want = torch.ones_like(cache.make_weights())
    cache.add_weights(q, off, lse, want)
    cache.check_status()
    for bad in (dict(max_nodes=2), dict(max_len=55)):
        weights = torch.ones_like(want)
        cache.add_weights(q, off, lse, weights, **bad)
        with pytest.raises(plc.PlcError):
            cache.check_status()
        assert bool((weights[1] == 1).all()) and torch.equal(weights[[0, 2]], want[[0, 2]])
    narrow = torch.ones((3, 1, 2, 52), device=DEV)
    cache.add_weights(q, off, lse, narrow)
    with pytest.raises(plc.PlcError):
        cache.check_status()
    assert bool((narrow[1] == 1).all()) and torch.equal(narrow[0], want[0, :, :, :52])
    cache.table[1, 1] = 77777  # no page: positions 16..31
    weights = torch.ones_like(want)
    cache.add_weights(q, off, lse, weights)
    with pytest.raises(plc.PlcError):
        cache.check_status()
    assert bool((weights[1, :, :, 16:32] == 1).all())
    keep = [x for x in range(60) if not 16 <= x < 32]
    assert torch.equal(weights[1][:, :, keep], want[1][:, :, keep]) and torch.equal(weights[[0, 2]], want[[0, 2]])


def test_another_stream_and_a_graph():
    cache, q, lse, want = run(torch.float16, 64, 2, 2, 16, [90, 200], [3, 1], seed=1, decay=0.0)
    off, weights = offsets([3, 1]), cache.make_weights()
    want = torch.nan_to_num(want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        cache.add_weights(q, off, lse, weights)
    stream.synchronize()
    assert torch.equal(weights, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.add_weights(q, off, lse, weights)
    for _ in range(3):
        weights.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(weights, want)
    cache.check_status()
