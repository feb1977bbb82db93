"""plc_score_tokens against the definition in 64 bits, over types, sizes, ties and rows where it can go wrong."""
import math

import pytest
import torch

from paper_2604_15356_amd import plc
from paper_2604_15356_amd.scores import TokenScorer

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TYPES = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])


def check(logits, k, tokens=None, temperature=1.0, scorer=None):
    """All results of valid rows.  How far they may be off: c = scale * log2(e) is rounded twice, which scales all of a row's logits
    alike: 2 U times what a logit differs from the mean; c x - c m and exp2 are rounded, U |a| and 2 U; sums of V weights take V / (256 pieces) + 24
    additions at most, one after the other; logarithms and what follows a few more roundings."""
    N, V = logits.shape
    scorer = scorer or TokenScorer(V, k)
    got = scorer.score(logits, tokens, temperature=temperature)
    scorer.check_status()
    scale = float(torch.tensor(1.0 / temperature, dtype=torch.float32))
    x = logits.double().cpu() * scale
    lse = torch.logsumexp(x, 1)
    logs = x - lse[:, None]
    p = logs.exp()
    fin = torch.where(p > 0, logs, torch.zeros_like(logs))
    entropy = -(p * fin).sum(1)
    top = x.amax(1)
    away = torch.where(p > 0, top[:, None] - x, torch.zeros_like(x))
    A, A2 = (p * away).sum(1), (p * away * away).sum(1)
    steps = V / (256 * (4 if logits.dtype == torch.float32 else 8)) + 40
    err = U * (4 * A + steps)
    tol_lse = err + U * 6 * (lse.abs() + top.abs())
    off = lambda a, b: (a.double().cpu() - b).abs()  # noqa: E731
    assert bool((off(got.lse, lse) <= tol_lse).all()), float((off(got.lse, lse) / tol_lse).max())
    tol = U * (4 * A2 + (A + entropy + 1) * (steps + 8))
    assert bool((off(got.entropy, entropy) <= tol).all()), float((off(got.entropy, entropy) / tol).max())

    def near(value, want, where):
        tol = err[where] + U * (6 * want.abs() + 8)
        same = (value.double().cpu() == want) | ((value.double().cpu() - want).abs() <= tol)  # (minus infinities)
        assert bool(same.all())

    if tokens is not None:
        t = tokens.cpu().long()
        rows = t >= 0
        near(got.logprob[rows.to(DEV)], logs[rows, t[rows]], rows)
        assert bool((got.logprob.cpu()[~rows] == 0).all())
    if k:
        # by value, equal ones by number: a stable sort
        ids = torch.sort(logits.float().cpu() + 0.0, dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(got.ids.cpu().long(), ids)
        want = torch.gather(logs, 1, ids)
        each = torch.arange(N)[:, None].expand(N, k)
        near(got.logprobs.flatten(), want.flatten(), each.flatten())
        tol = want.exp() * (err[:, None] + U * (12 * torch.where(want > -1e30, want.abs(), torch.zeros_like(want)) + 16)) + 1e-37
        assert bool((off(got.probs, want.exp()) <= tol).all())
        if tokens is not None:
            hit = ids == t[:, None]
            assert torch.equal(got.chosen.cpu().long(), torch.where(hit.any(1), hit.int().argmax(1), torch.tensor(-1)))
    return got


def draw(N, V, dtype, seed=0, spread=3.0):
    gen = torch.Generator(DEV).manual_seed(seed + N + V)
    x = (torch.randn((N, V), device=DEV, generator=gen) * spread).to(dtype)
    tokens = torch.randint(0, V, (N,), device=DEV, generator=gen, dtype=torch.int32)
    tokens[N // 2:] = x[N // 2:].float().argmax(1).to(torch.int32)
    tokens[4::5] = -1
    return x, tokens


@TYPES
@pytest.mark.parametrize("V,k", [(1, 1), (2, 2), (7, 3), (8, 8), (9, 0), (32, 32), (33, 32), (255, 4), (2047, 20), (2048, 1), (2049, 32),
                                 (8191, 8), (8192, 20), (8193, 31), (50016, 8), (50257, 32), (131071, 20)])
@pytest.mark.parametrize("N", [1, 3, 40])
def test_vocabularies(dtype, V, k, N):
    x, tokens = draw(N, V, dtype)
    check(x, k, tokens)


@TYPES
def test_many_rows(dtype):
    for N, V, k in ((511, 2500, 8), (512, 20011, 20), (513, 9000, 32), (4099, 1000, 4)):
        x, tokens = draw(N, V, dtype)
        check(x, k, tokens)


@TYPES
@pytest.mark.parametrize("shift", range(8))
def test_rows_that_begin_anywhere(dtype, shift):
    """Rows at every distance from a 16-byte boundary; what lies in front of and behind them has no effect."""
    N, V = 9, 1003
    wide = torch.full((N, V + 14), float("nan"), device=DEV, dtype=dtype)
    x, tokens = draw(N, V, dtype, seed=shift)
    wide[:, shift:shift + V] = x
    got = check(wide[:, shift:shift + V], 20, tokens)
    for a, b in zip(got, check(x, 20, tokens)):
        assert bool((a - b).abs().max() <= 1e-5)
    odd = wide.flatten()[shift:shift + (N - 1) * (V + 3) + V + 3]  # rows an odd number of elements apart
    odd = torch.as_strided(odd, (N, V), (V + 3, 1))
    odd.copy_(x)
    check(odd, 20, tokens)


@TYPES
@pytest.mark.parametrize("temperature", [0.25, 0.7, 1.0, 3.0, 100.0])
def test_temperatures(dtype, temperature):
    x, tokens = draw(5, 3001, dtype)
    check(x, 8, tokens, temperature=temperature)


@TYPES
@pytest.mark.parametrize("N", [2, 600])
def test_ties_and_orders(dtype, N):
    """Equal logits go by their numbers; rising, falling and clustered rows, where all that is large is seen last, first or by one thread."""
    V = 20000
    base = torch.arange(V, device=DEV) / 1000.0
    rows = [torch.zeros(V, device=DEV), base, -base, (base * 50).floor() / 50, torch.where(torch.arange(V, device=DEV) % 2048 < 8, 5.0, -5.0),
            torch.where(torch.arange(V, device=DEV) % 2048 < 8, 5.0 + base, -5.0), torch.where(torch.arange(V, device=DEV) % 8192 < 32, 9.0, 8.5),
            torch.where(torch.arange(V, device=DEV) >= V - 40, 3.0, -3.0), torch.randint(0, 3, (V,), device=DEV).float()]
    x = torch.stack([rows[i % len(rows)] for i in range(N)]).to(dtype) if N > 2 else None
    for i in range(0, len(rows), 2):
        pair = torch.stack([rows[i], rows[(i + 1) % len(rows)]]).to(dtype)
        tokens = torch.tensor([3, V - 1], dtype=torch.int32, device=DEV)
        for k in (1, 4, 32):
            check(pair, k, tokens)
    if x is not None:
        check(x, 20, torch.arange(N, device=DEV, dtype=torch.int32))


@TYPES
@pytest.mark.parametrize("N", [2, 520])
@pytest.mark.parametrize("V", [20000, 8192, 140000])
def test_many_large_logits_with_few_threads(dtype, N, V):
    """Thousands of candidates: 31 fours of threads see nothing but large logits, one more a few that are smaller, the others none."""
    at = torch.arange(V, device=DEV) // (4 if dtype == torch.float32 else 8) % 256 // 4  # the four that reads a logit
    noise = torch.rand((2, V), device=DEV)
    x = torch.where(at < 31, 5 + 2 * noise, torch.where(at == 31, noise, torch.full_like(noise, -1.0)))
    x = x.to(dtype)[torch.arange(N, device=DEV) % 2].contiguous()
    tokens = x.float().argmax(1).to(torch.int32)
    for k in (32, 20):
        check(x, k, tokens)


@TYPES
@pytest.mark.parametrize("N", [3, 520])
def test_masked_tokens(dtype, N):
    x, tokens = draw(N, 9999, dtype)
    x[:, ::3] = -math.inf
    check(x, 20, tokens)
    x[0] = -math.inf
    x[0, 7777] = -3.0  # one token left, fewer than k
    x[1, 100:] = -math.inf
    tokens[0], tokens[1] = 7777, 5000
    got = check(x, 32, tokens)
    assert float(got.entropy[0]) < 1e-6 and abs(float(got.logprob[0])) < 1e-6 and got.ids[0].tolist() == [7777] + list(range(31))
    assert float(got.logprob[1]) == -math.inf
    lowest = torch.finfo(dtype).min
    x, tokens = draw(N, 9999, dtype)
    x[:, ::2] = lowest
    check(x, 20, tokens)


@TYPES
@pytest.mark.parametrize("N,V", [(2, 8200), (600, 8200), (2, 140000)])
def test_logits_of_any_size(dtype, N, V):
    """Nothing but the type's lowest value; the largest ones; differences that overflow where they are scaled.  Whole rows, and
    rows in parts, of which one has a larger logit than the others, and one none."""
    most = torch.finfo(dtype).max
    for value in (-most, most, most / 2):
        x = torch.full((N, V), value, device=DEV, dtype=dtype)
        x[1, 77] = -most
        got = TokenScorer(V, 4).score(x, torch.full((N,), 77, dtype=torch.int32, device=DEV))
        even = math.log(V)
        assert abs(float(got.entropy[0]) - even) < 1e-5 and abs(float(got.logprob[0]) + even) < 1e-5
        # V equal logits: lse = x + log V, which is 11.85 for 140000 of them, and its sum one fp32 rounding, 2^-24 of it
        assert abs(float(got.lse[0].double()) - (float(x[0, 0].double()) + even)) <= 1e-5 + 2.0 ** -23 * float(x[0, 0].abs().double())
        assert got.ids[0].tolist() == [0, 1, 2, 3] and got.chosen[0] == -1
        if value > 0:
            assert got.logprob[1] < -1e3 and abs(float(got.entropy[1]) - math.log(V - 1)) < 1e-5
    x, tokens = draw(N, V, dtype, spread=1e4)
    check(x, 8, tokens)
    x = torch.full((N, V), -most, device=DEV, dtype=dtype)
    x[:, V // 2:V // 2 + 100] = draw(N, 100, dtype)[0]
    x[:, : V // 3] = -math.inf
    check(x, 32, torch.full((N,), V // 2 + 50, dtype=torch.int32, device=DEV))


def check_far(logits, k, tokens, temperature=1.0):
    """Valid rows of logits of any size: as check, with a definition that takes all differences from the row's largest logit, as 64 bits have
    no fractions either at 1e16.  The tolerances are check's."""
    N, V = logits.shape
    scorer = TokenScorer(V, k)
    got = scorer.score(logits, tokens, temperature=temperature)
    scorer.check_status()
    scale = float(torch.tensor(1.0 / temperature, dtype=torch.float32))
    steps = V / (256 * (4 if logits.dtype == torch.float32 else 8)) + 40
    logits, t = logits.double().cpu(), tokens.cpu().long()
    top = logits.amax(1)
    below = (logits - top[:, None]) * scale
    norm = torch.logsumexp(below, 1)
    logs, lse = below - norm[:, None], top * scale + norm
    p = logs.exp()
    away = torch.where(p > 0, -below, torch.zeros_like(below))
    A, A2 = (p * away).sum(1), (p * away * away).sum(1)
    entropy = norm + A
    err = U * (4 * A + steps)
    within = lambda a, b, tol: bool(((a.double().cpu() == b) | ((a.double().cpu() - b).abs() <= tol)).all())  # noqa: E731
    assert within(got.lse, lse, err + U * 6 * (lse.abs() + top.abs() * scale))
    assert within(got.entropy, entropy, U * (4 * A2 + (A + entropy + 1) * (steps + 8)))
    want = torch.where(t >= 0, logs.gather(1, t.clamp(min=0)[:, None])[:, 0], torch.zeros_like(top))
    assert within(got.logprob, want, err + U * (6 * want.abs() + 8)) and bool((got.logprob.cpu()[t < 0] == 0).all())
    if k:
        ids = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(got.ids.cpu().long(), ids)
        want = torch.gather(logs, 1, ids)
        assert within(got.logprobs, want, err[:, None] + U * (6 * want.abs() + 8))
        assert within(got.probs, want.exp(), want.exp() * (err[:, None] + U * (12 * want.abs() + 16)) + 1e-37)
        hit = ids == t[:, None]
        assert torch.equal(got.chosen.cpu().long(), torch.where(hit.any(1), hit.int().argmax(1), torch.tensor(-1)))


def rows_with_masks(V, dtype, value, seed):
    """Rows in which tokens are masked by a finite value: all but a few, whole runs in front, behind or up to the last token; and rows of nothing but
    such values, of one size and of several, of both signs."""
    gen = torch.Generator(DEV).manual_seed(seed)
    x = torch.randn((9, V), device=DEV, generator=gen) * 3
    few = torch.randint(0, V, (7,), device=DEV, generator=gen)
    x[0] = torch.full_like(x[0], value).scatter(0, few, x[0][few])
    x[1, :2 * V // 3] = value
    x[2, V // 3:] = value
    x[3, :V - 1] = value
    x[4], x[5] = value, -value
    x[6:8] = torch.rand((2, V), device=DEV, generator=gen) + 0.5
    x[6] *= value
    x[7] *= -value
    x[8] = torch.where(torch.arange(V, device=DEV) < V // 2, value, 2 * value)
    return x.to(dtype)


MASKS = {torch.float16: ((-3e4, -2e4, -1e3), (1e-3, 1e-4, 1e-6)),
         torch.bfloat16: ((-1e7, -1e8, -1e9, -1e10, -1e15, -1e20, -1e29), (1.0, 0.7, 0.1)),
         torch.float32: ((-1e7, -1e8, -1e9, -1e10, -1e15, -1e20, -1e29), (1.0, 0.7, 0.1))}


@TYPES
@pytest.mark.parametrize("which", range(3))
@pytest.mark.parametrize("N,V", [(2, 100), (2, 3000), (2, 9001), (2, 140000), (600, 9001)])
def test_finite_values_that_mask(dtype, which, N, V):
    """Where fp32 does not hold the fractions of what a row is scaled to; such rows are valid (check_far looks at the status)."""
    values, temperatures = MASKS[dtype]
    x = torch.cat([rows_with_masks(V, dtype, value, i) for i, value in enumerate(values)])
    tokens = x.float().argmax(1).to(torch.int32)
    tokens[1::3] = V // 2
    tokens[2::5] = -1
    if N > len(x):
        at = torch.arange(N, device=DEV) % len(x)
        for k in (0, 32):
            check_far(x[at].contiguous(), k, tokens[at], temperature=temperatures[which])
        return
    for i in range(0, len(x) - 1, 2):
        check_far(x[i:i + 2], (32, 0, 8)[i // 2 % 3], tokens[i:i + 2], temperature=temperatures[which])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V", [(2, 3000), (2, 140000), (600, 9001)])
def test_logits_about_the_size_that_a_row_is_gone_through_again_from(dtype, N, V):
    """2^24 over log2(e), 11,629,000: a little below and above, all of a row and a run of it (of which parts have one, or two), of both signs."""
    for i, size in enumerate((1.1e7, 1.16e7, 1.1629e7, 1.163e7, 1.2e7, 1.3e7)):
        x, tokens = draw(N, V, torch.float32, seed=i)
        x[0::4] += size
        x[1::4] -= size
        x[2::4, V // 2:] += size
        x[3::4, :V // 2] -= size
        if N == 2:
            x = torch.cat([x, draw(N, V, torch.float32, seed=i + 10)[0]])
            x[2, V // 2:] += size
            x[3, :V // 2] -= size
        x = x.to(dtype)
        for a in range(0, len(x), N):
            check_far(x[a:a + N], (0, 20, 32)[i % 3], tokens)


@TYPES
def test_rows_and_tokens_that_are_none(dtype):
    for N in (4, 700):
        x, tokens = draw(N, 6000, dtype)
        tokens[:] = 17
        clean = check(x, 8, tokens)
        bad = x.clone()
        bad[0, 5999] = float("nan")
        bad[1, 3] = math.inf
        bad[2] = -math.inf
        tokens[3] = 6000
        scorer = TokenScorer(6000, 8)
        got = scorer.score(bad, tokens)
        with pytest.raises(plc.PlcError):
            scorer.check_status()
        scorer.check_status()  # told once
        for name, a, b in zip(got._fields, got, clean):
            if name in ("ids", "chosen"):
                assert bool((a[:3] == -1).all())
            else:
                assert bool(torch.isnan(a[:3]).all())
            assert torch.equal(a[4:], b[4:])
        assert bool(torch.isnan(got.logprob[3])) and int(got.chosen[3]) == -1 and torch.equal(got.probs[3], clean.probs[3])
        tokens[3] = -2
        scorer.score(x, tokens)
        with pytest.raises(plc.PlcError):
            scorer.check_status()


def test_zeros_of_both_signs_are_equal():
    x = torch.zeros((1, 100), device=DEV)
    x[0, ::2] = -0.0
    assert check(x, 5).ids[0].tolist() == [0, 1, 2, 3, 4]


def test_shapes_and_no_rows():
    x = torch.randn((2, 3, 500), device=DEV).to(torch.float16)
    tokens = torch.randint(0, 500, (2, 3), device=DEV, dtype=torch.int32)
    scorer = TokenScorer(500, 4)
    got, flat = scorer.score(x, tokens), scorer.score(x.view(6, 500), tokens.view(6))
    for a, b in zip(got, flat):
        assert a.shape[:2] == (2, 3) and torch.equal(a.reshape(b.shape), b)
    one = scorer.score(x[0, 0], tokens[0, 0])
    assert one.logprob.shape == () and one.probs.shape == (4,) and torch.equal(one.ids, flat.ids[0])
    none = scorer.score(x[:0].reshape(0, 500))
    assert none.logprob is None and none.chosen is None and none.probs.shape == (0, 4)
    rest = TokenScorer(500).score(x, tokens)
    assert rest.ids is None and rest.probs is None and torch.equal(rest.logprob, got.logprob)
    scorer.check_status()


def test_a_row_by_itself_and_among_others():
    """The alternatives are the same, and the sums to their roundings, however many rows there are (rows are cut into parts
    where they are few)."""
    x, tokens = draw(600, 50016, torch.bfloat16)
    many = check(x[:, :], 20, tokens)
    for i in (0, 1, 599):
        one = check(x[i:i + 1], 20, tokens[i:i + 1])
        assert torch.equal(one.ids[0], many.ids[i]) and torch.equal(one.chosen[0], many.chosen[i])
    assert all(torch.equal(a, b) for a, b in zip(many, TokenScorer(50016, 20).score(x, tokens)))  # and the same bits again


def test_logits_beyond_31_bits():
    N, V = 43000, 50016  # 4.3 GB
    x = torch.zeros((N, V), device=DEV, dtype=torch.float16)
    last, tokens = draw(40, V, torch.float16)
    x[-40:] = last
    got = TokenScorer(V, 4).score(x, torch.cat([torch.zeros(N - 40, dtype=torch.int32, device=DEV), tokens]))
    want = check(last, 4, tokens)
    assert torch.equal(got.ids[-40:], want.ids) and bool(((got.lse[-40:] - want.lse).abs() < 1e-5).all())
    assert got.ids[0].tolist() == [0, 1, 2, 3] and int(got.chosen[0]) == 0


def test_another_stream_and_a_graph():
    for N in (2, 700):
        x, tokens = draw(N, 9000, torch.bfloat16)
        scorer = TokenScorer(9000, 8)
        want = scorer.score(x, tokens)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            got = scorer.score(x, tokens)
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = scorer.score(x, tokens)
        for _ in range(3):
            for t in got:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            scorer.score(x * 0.5, tokens)  # the program's own, with the same workspace
        scorer.check_status()


def test_probs_and_chosen_are_what_the_codec_takes():
    """Logits of a model, its candidates and the tokens that came: coded and decoded as any probabilities are."""
    from paper_2604_15356_amd.codec import KVDeltaCodec
    S, L, H, n, k, d = 1, 2, 2, 64, 4, 32
    x, tokens = draw(n, 1000, torch.float32)
    tokens[tokens < 0] = 11
    s = TokenScorer(1000, k).score(x.view(S, n, 1000), tokens.view(S, n))
    cand_k, cand_v = (torch.randn((S, L, H, n, k, d), device=DEV).to(torch.float16) for _ in range(2))
    at = s.chosen.long().clamp(min=0)[:, None, None, :, None, None].expand(S, L, H, n, 1, d)
    act_k, act_v = (torch.gather(c, 4, at)[:, :, :, :, 0].contiguous() for c in (cand_k, cand_v))
    codec = KVDeltaCodec(S, L, H, n, k, d, 0.02)
    codec.encode_cond(cand_k, cand_v, s.probs, act_k, act_v, chosen=s.chosen)
    out_k, out_v = torch.empty_like(act_k), torch.empty_like(act_v)
    codec.decode_cond(cand_k, cand_v, s.probs, out_k, out_v)
    codec.check_status()
    # (fp16 beside the half step: values below 8 are rounded by 2^-9 at most)
    assert float((out_k.float() - act_k.float()).abs().max()) <= 0.0101 + 2.0 ** -9
