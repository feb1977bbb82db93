"""The calls of a step together, as a serving loop makes them: sessions whose caches may not grow beyond a budget, against the same
loop in plain Python and 64 bits."""
import math

import pytest
import torch

from paged_util import DEV, ints, offsets
from paper_2604_15356_amd.paged import PagedKVCache
from paper_2604_15356_amd.rotary import Rotary
from paper_2604_15356_amd.scores import TokenScorer

pytestmark = pytest.mark.gpu
S, L, H, G, d, B, V, K = 3, 2, 2, 3, 32, 16, 300, 8
BUDGET, KEEP, FIRST, LAST = 40, 29, 2, 10
HALF = 2.0 ** -11  # of fp16: half a step


def rotated(x, pos, theta):
    """x [heads, d] in 64 bits."""
    a = pos * torch.tensor(theta, dtype=torch.float64)
    p, q = x[..., : d // 2], x[..., d // 2:]
    return torch.cat([p * a.cos() - q * a.sin(), q * a.cos() + p * a.sin()], -1)


class Session:
    """Per layer and head: keys, values and weights of the positions that are there."""

    def __init__(self):
        self.seen, self.k, self.v, self.w = 0, *([[[] for _ in range(H)] for _ in range(L)] for _ in range(3))

    def step(self, layer, q, k, v, pos, theta):
        """One token; returns (out [H*G, d], how far it may be off)."""
        k, q = rotated(k, pos, theta), rotated(q, pos, theta)
        out, tol = torch.zeros(H * G, d, dtype=torch.float64), torch.zeros(H * G, d, dtype=torch.float64)
        for h in range(H):
            self.k[layer][h].append(k[h]), self.v[layer][h].append(v[h]), self.w[layer][h].append(0.0)
            ks, vs, qs = torch.stack(self.k[layer][h]), torch.stack(self.v[layer][h]), q[h * G:(h + 1) * G]
            score = qs @ ks.T * d ** -0.5
            w = torch.softmax(score, 1)
            # rotated keys and queries are rounded to fp16 there, half a step each: a score moves by 2 HALF of its size, a weight by
            # twice that with its sum, and by half a step of its own
            err = 4.2 * HALF * (qs.abs() @ ks.abs().T * d ** -0.5).amax() + 1.1 * HALF
            out[h * G:(h + 1) * G] = w @ vs
            tol[h * G:(h + 1) * G] = err * (w @ vs.abs()) + 1.1 * HALF * (w @ vs).abs() + 1e-6
            self.w[layer][h] = [a + float(b) for a, b in zip(self.w[layer][h], w.sum(0))]
            self.err = max(getattr(self, "err", 0.0), float(err))
        return out, tol

    def shorten(self, kept):
        """To the positions that the device kept, which have to be such as may be kept."""
        for layer in range(L):
            for h in range(H):
                w, stay = self.w[layer][h], kept[layer][h]
                n = len(w)
                assert len(stay) == KEEP and stay == sorted(set(stay)) and stay[:FIRST] == list(range(FIRST)) and stay[-LAST:] == list(range(n - LAST, n))
                mid = [w[i] for i in stay[FIRST:-LAST]]
                gone = [w[i] for i in range(n) if i not in stay]
                assert min(mid) >= max(gone) * (1 - 2.2 * self.err)
                for x in (self.k, self.v, self.w):
                    x[layer][h] = [x[layer][h][i] for i in stay]


def test_sessions_within_a_budget():
    torch.manual_seed(7)
    cache = PagedKVCache.create(16, L, H, d, S, 64, B=B)
    rotary, scorer, weights = Rotary(d, base=1000.0), TokenScorer(V, K), cache.make_weights()
    head = torch.randn((H * G * d, V), device=DEV) / 8
    sessions = [Session() for _ in range(S)]
    seen = torch.zeros(S, dtype=torch.int32, device=DEV)
    evicted = 0
    for step in range(70):
        # a prompt first, of another length each, then a token each, but for a session that rests now and then
        counts = [17, 3, 30] if step == 0 else [1, 1 if step % 7 else 0, 1]
        N, off = sum(counts), offsets(counts)
        cache.extend(ints(counts))
        x = None
        for layer in range(L):
            q, k, v = (torch.randn((N, n, d), device=DEV).to(torch.float16) for n in (H * G, H, H))
            q *= 2
            q_rot = cache.store_rotated(k, v, off, rotary, q=q, base=seen, layer=layer)
            out, lse = cache.attend(q_rot, off, layer=layer)
            cache.add_weights(q_rot, off, lse, weights, layer=layer)
            i = 0
            for s, t in enumerate(counts):
                for j in range(t):
                    want, tol = sessions[s].step(layer, q[i].double().cpu(), k[i].double().cpu(), v[i].double().cpu(), sessions[s].seen + j, rotary.theta)
                    off_by = (out[i].double().cpu() - want).abs()
                    assert bool((off_by <= tol).all()), (step, layer, s, float((off_by / tol).max()))
                    i += 1
            x = out
        for s, t in enumerate(counts):
            sessions[s].seen += t
        seen += ints(counts)
        logits = x.reshape(N, -1).float() @ head
        scores = scorer.score(logits, logits.argmax(1).to(torch.int32))
        logs = torch.log_softmax(logits.double(), 1)
        assert bool((scores.chosen == 0).all()) and torch.equal(scores.ids.long(), torch.topk(logits, K, 1).indices)
        assert bool(((scores.logprobs.double() - torch.topk(logs, K, 1).values).abs() < 1e-5).all())
        assert bool(((scores.entropy.double() + (logs.exp() * logs).sum(1)).abs() < 1e-5).all())
        if max(len(s.w[0][0]) for s in sessions) > BUDGET:
            lens = [len(s.w[0][0]) for s in sessions]
            kept = cache.evict(ints([KEEP] * S), weights, first=FIRST, last=LAST).tolist()
            cache.check_status()
            for s in range(S):
                if lens[s] > KEEP:
                    sessions[s].shorten([[kept[s][layer][h][:KEEP] for h in range(H)] for layer in range(L)])
                    evicted += 1
        assert cache.lens.tolist() == [len(s.w[0][0]) for s in sessions]
        for s in range(S):
            for layer in range(L):
                for h in range(H):
                    want = torch.tensor(sessions[s].w[layer][h], dtype=torch.float64)
                    got = weights[s, layer, h, : len(want)].double().cpu()
                    assert bool(((got - want).abs() <= 1.1 * sessions[s].err * want + 1e-6).all())
    cache.check_status()
    assert evicted >= 6 and int(cache.refs.sum()) == sum(-(-n // B) for n in cache.lens.tolist())


def test_a_drafted_tree_s_accepted_nodes():
    """What accepted nodes give positions is what a chain of them gives."""
    torch.manual_seed(3)
    rotary = Rotary(d, interleaved=True)
    parents, path = [-1, 0, 0, 1, 2, 4], [0, 2, 4]
    depths = [0, 1, 1, 2, 2, 3]
    k, v = (torch.randn((26, L, H, d), device=DEV).to(torch.float16) for _ in range(2))
    q = torch.randn((6, H * G, d), device=DEV).to(torch.float16)
    results = []
    for tree in (True, False):
        cache = PagedKVCache.create(8, L, H, d, 1, 64, B=B)
        weights = cache.make_weights()
        cache.extend(ints([20]))
        cache.store_rotated(k[:20].contiguous(), v[:20].contiguous(), ints([0, 20]), rotary)
        if tree:
            cache.extend(ints([6]))
            q_rot = cache.store_rotated(k[20:], v[20:], ints([0, 6]), rotary, q=q, rel=ints(depths))
            out, lse = cache.attend(q_rot, ints([0, 6]), parents=ints(parents), layer=1)
            cache.accept(ints([0, 6]), ints(path), ints([0, 3]))
            out, q_rot, lse = out[path], q_rot[path], lse[path].contiguous()
        else:
            rows = [20 + i for i in path]
            cache.extend(ints([3]))
            q_rot = cache.store_rotated(k[rows], v[rows], ints([0, 3]), rotary, q=q[path])
            out, lse = cache.attend(q_rot, ints([0, 3]), layer=1)
        cache.add_weights(q_rot, ints([0, 3]), lse, weights, layer=1)
        cache.check_status()
        results.append((out, lse, weights))
    (out, lse, w), (out2, lse2, w2) = results
    # (the same scores, summed in another order)
    assert bool(((out - out2).abs() <= 2 * HALF * 1.1 * out2.abs() + 4 * HALF).all())
    assert bool(((lse - lse2).abs() < 1e-5).all()) and bool(((w - w2).abs() <= 4e-5 * w2 + 1e-6).all())


def test_a_session_s_place_given_to_another():
    """The weights of those before count for rows that come without add_weights, also behind what was evicted or trimmed; with zeros put there
    first all is as in a cache of its own."""
    torch.manual_seed(5)
    prompt = [torch.randn((50, L, H, d), device=DEV).to(torch.float16) for _ in range(2)]
    new = [torch.randn((2, L, H, d), device=DEV).to(torch.float16) for _ in range(2)]
    q = torch.randn((2, H * G, d), device=DEV).to(torch.float16)

    def conversation(cache, weights):
        cache.extend(ints([50]))
        cache.store(*prompt, ints([0, 50]))
        cache.extend(ints([2]))
        cache.store(*new, ints([0, 2]))
        for layer in range(L):
            _, lse = cache.attend(q, ints([0, 2]), layer=layer)
            cache.add_weights(q, ints([0, 2]), lse, weights, layer=layer)
        return weights.clone(), cache.evict(ints([20]), weights, first=1, last=3)[..., :20].clone()

    caches = [PagedKVCache.create(8, L, H, d, 1, 64, B=B) for _ in range(3)]
    weights = [cache.make_weights() for cache in caches]
    for cache, w in zip(caches[1:], weights[1:]):  # another conversation had this place, and was shortened in both ways
        cache.extend(ints([60]))
        cache.store(*(torch.randn((60, L, H, d), device=DEV).to(torch.float16) for _ in range(2)), ints([0, 60]))
        w.copy_(torch.rand(w.shape, device=DEV) * 5)
        cache.evict(ints([30]), w, first=1, last=3)
        cache.trim(ints([0]))
    before = weights[2].clone()
    weights[1][0, :, :, 0:] = 0
    (own, kept), (reused, kept2), (stale, _) = (conversation(*x) for x in zip(caches, weights))
    for cache in caches:
        cache.check_status()
    assert torch.equal(own[..., :52], reused[..., :52]) and torch.equal(kept, kept2)
    want = own.double()[..., :50] + before.double()[..., :50]
    assert bool(((stale.double()[..., :50] - want).abs() <= 2.0 ** -23 * want).all()) and torch.equal(stale[..., 50:52], own[..., 50:52])


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_thinned_cache_back_to_the_coder_and_into_pages_again(interleaved):
    """After an eviction a row is another position in each layer and head: rotate takes them one by one."""
    torch.manual_seed(11)
    rotary, n, now = Rotary(d, base=1000.0, interleaved=interleaved), 60, 23
    cache = PagedKVCache.create(8, L, H, d, 1, 64, B=B)
    weights = cache.make_weights()
    k, v = (torch.randn((n, L, H, d), device=DEV).to(torch.float16) for _ in range(2))
    cache.extend(ints([n]))
    cache.store_rotated(k, v, ints([0, n]), rotary)
    weights.copy_(torch.rand(weights.shape, device=DEV))
    kept = cache.evict(ints([now]), weights, first=1, last=3)[0, :, :, :now].permute(2, 0, 1).contiguous()  # [now, L, H]
    rows = [torch.empty((now, L, H, d), dtype=torch.float16, device=DEV) for _ in range(2)]
    cache.load(*rows, ints([0, now]))
    cache.check_status()
    each = lambda x: x.reshape(-1, 1, d)  # noqa: E731
    positions = kept.flatten()
    at = kept.long()[..., None].expand(now, L, H, d)
    before, values = torch.gather(k, 0, at), torch.gather(v, 0, at)
    assert torch.equal(rows[1], values) and torch.equal(rotary.rotate(each(before), positions), each(rows[0]))
    back = rotary.rotate(each(rows[0]), positions, inverse=True).view(now, L, H, d)
    # stored rows are off by half a step each, of which the inverse turns two together; then half a step of its own; sines and products far below
    x = before.double()
    size = torch.cat([x[..., : d // 2].abs() + x[..., d // 2:].abs()] * 2, -1) if not interleaved else \
        (x[..., ::2].abs() + x[..., 1::2].abs()).repeat_interleave(2, -1)
    assert bool(((back.double() - x).abs() <= 2.001 * HALF * size + 1.001 * HALF * x.abs() + 2.0 ** -24).all())
    other = PagedKVCache.create(8, L, H, d, 1, 64, B=B)
    other.extend(ints([now]))
    other.store(rotary.rotate(each(before), positions).view(now, L, H, d), values, ints([0, now]))
    q = torch.randn((1, H * G, d), device=DEV).to(torch.float16)
    outs = []
    for c in (cache, other):  # the next token of either: after what the session has seen
        c.extend(ints([1]))
        turned = c.store_rotated(k[:1], v[:1], ints([0, 1]), rotary, q=q, base=ints([n]))
        outs.append(c.attend(turned, ints([0, 1]), layer=1)[0])
        c.check_status()
    assert torch.equal(*outs)
