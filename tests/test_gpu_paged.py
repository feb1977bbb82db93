"""The paged cache's bookkeeping and moves against a model of them in plain Python: tables, lengths, reference counts and
every element of the pool, bit for bit, after each call of a sequence; and what the calls do with data they cannot use."""
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


class Model:
    """The definition, one session after the other, on the host."""

    def __init__(self, cache):
        self.B, self.M, self.S, self.P = cache.B, cache.M, cache.S, cache.P
        self.k, self.v = cache.k.cpu().clone(), cache.v.cpu().clone()
        self.pages = [[] for _ in range(self.S)]
        self.lens = [0] * self.S

    def refs(self):
        r = [0] * self.P
        for row in self.pages:
            for p in row:
                r[p] += 1
        return r

    def fork(self, src):
        self.pages = [list(self.pages[f]) if f >= 0 else [] for f in src]
        self.lens = [self.lens[f] if f >= 0 else 0 for f in src]

    def extend(self, grow):
        # all pages are chosen among those free at the start of the call
        free = [p for p, r in enumerate(self.refs()) if r == 0]
        refs = self.refs()
        for s, g in enumerate(grow):
            n, B = self.lens[s], self.B
            if g and n % B and refs[self.pages[s][-1]] > 1:
                old, new = self.pages[s][-1], free.pop(0)
                refs[old] -= 1
                self.pages[s][-1] = new
                for x in (self.k, self.v):
                    x[new, :, :, : n % B] = x[old, :, :, : n % B]
            while len(self.pages[s]) < -(-(n + g) // B):
                self.pages[s].append(free.pop(0))
            self.lens[s] = n + g

    def trim(self, new):
        for s, n in enumerate(new):
            self.lens[s] = n
            self.pages[s] = self.pages[s][: -(-n // self.B)]

    def row(self, x, s, pos):
        return x[self.pages[s][pos // self.B], :, :, pos % self.B]

    def store(self, k, v, counts, layers):
        at = 0
        for s, t in enumerate(counts):
            for i in range(t):
                pos = self.lens[s] - t + i
                self.row(self.k, s, pos)[layers] = k[at]
                self.row(self.v, s, pos)[layers] = v[at]
                at += 1

    def load(self, counts, layers):
        out = [[self.row(x, s, self.lens[s] - t + i)[layers] for s, t in enumerate(counts) for i in range(t)]
               for x in (self.k, self.v)]
        return [torch.stack(o) for o in out]

    def accept(self, counts, paths):
        for s, (t, path) in enumerate(zip(counts, paths)):
            c = self.lens[s] - t
            for x in (self.k, self.v):
                rows = [self.row(x, s, c + node).clone() for node in path]
                for r, row in enumerate(rows):
                    self.row(x, s, c + r).copy_(row)
        self.trim([self.lens[s] - t + len(p) for s, (t, p) in enumerate(zip(counts, paths))])

    def compact(self):
        refs = self.refs()
        used = sum(r > 0 for r in refs)
        movers = [p for p in range(used, self.P) if refs[p]]
        holes = [p for p in range(used) if not refs[p]]
        home = dict(zip(movers, holes))
        for f, t in home.items():
            self.k[t], self.v[t] = self.k[f], self.v[f]
        self.pages = [[home.get(p, p) for p in row] for row in self.pages]
        return used

    def check(self, cache):
        cache.check_status()
        assert cache.lens.tolist() == self.lens
        assert cache.table.tolist() == [row + [-1] * (self.M - len(row)) for row in self.pages]
        assert cache.refs.tolist() == self.refs()
        assert torch.equal(cache.k.cpu().view(torch.int16), self.k.view(torch.int16))
        assert torch.equal(cache.v.cpu().view(torch.int16), self.v.view(torch.int16))


def make(P, L, H, B, d, S, M, dtype=torch.float16, heads_first=False):
    shape = (P, L, H, B, d)
    if heads_first:  # rows of all heads next to each other, a gap behind each page
        k, v = (torch.randn((P, L * B * H + 1, d), device=DEV).to(dtype) for _ in range(2))
        k, v = (x[:, : L * B * H].view(P, L, B, H, d).permute(0, 1, 3, 2, 4) for x in (k, v))
        assert k.shape == shape and not k.is_contiguous()
    else:
        k, v = (torch.randn(shape, device=DEV).to(dtype) for _ in range(2))
    zeros = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    return PagedKVCache(k, v, torch.full((S, M), -1, dtype=torch.int32, device=DEV), zeros(S), zeros(P))


def rows_like(cache, n, layers):
    return [torch.randn((n, layers, cache.H, cache.d), device=DEV).to(cache.dtype) for _ in range(2)]


@pytest.mark.parametrize("L,H,B,d,S,M,dtype,heads_first", [
    (2, 3, 16, 8, 5, 9, torch.float16, False),
    (1, 1, 32, 80, 1, 6, torch.bfloat16, False),
    (3, 2, 16, 128, 7, 17, torch.bfloat16, True),
    (5, 7, 64, 40, 3, 4, torch.float16, True),
    (2, 4, 16, 64, 33, 5, torch.float16, False)])
def test_a_life_of_a_cache(L, H, B, d, S, M, dtype, heads_first):
    rng = random.Random(L * 1000 + d + S)
    torch.manual_seed(d)
    P = S * M + 3
    cache = make(P, L, H, B, d, S, M, dtype, heads_first)
    model = Model(cache)
    room = M * B
    for step in range(12):
        # room for a few rows, up to the table's end for some, and the rows
        grow = [rng.choice([0, 1, 2, B - 1, B, B + 1, 2 * B]) for _ in range(S)]
        grow = [min(g, room - n) for g, n in zip(grow, model.lens)]
        cache.extend(ints(grow))
        model.extend(grow)
        model.check(cache)
        counts = [rng.randint(0, g) for g in grow]
        first = rng.randrange(L)
        layers = slice(first, rng.randint(first + 1, L))
        k, v = rows_like(cache, sum(counts), layers.stop - first)
        cache.store(k, v, offsets(counts), layer=first)
        model.store(k.cpu(), v.cpu(), counts, layers)
        model.check(cache)
        # what is there, packed
        counts = [rng.randint(0, n) for n in model.lens]
        if sum(counts):
            out = [torch.zeros_like(x) for x in rows_like(cache, sum(counts), L)]
            cache.load(*out, offsets(counts))
            for got, want in zip(out, model.load(counts, slice(0, L))):
                assert torch.equal(got.cpu().view(torch.int16), want.view(torch.int16))
        # some of the last rows are drafted, and some of those accepted: pages that are the session's own by extend
        tree = [min(g, rng.randint(0, 70)) for g in grow]
        paths = [sorted(rng.sample(range(t), rng.randint(0, t))) for t in tree]
        cache.accept(offsets(tree), ints([x for p in paths for x in p]), offsets([len(p) for p in paths]))
        model.accept(tree, paths)
        model.check(cache)
        src = [rng.choice([s, s, rng.randrange(S), -1 if step % 3 == 2 else s]) for s in range(S)]
        cache.fork(ints(src))
        model.fork(src)
        model.check(cache)
        if step % 4 == 3:
            new = [rng.randint(0, n) for n in model.lens]
            cache.trim(ints(new))
            model.trim(new)
            model.check(cache)
            used = cache.compact()
            assert int(used.item()) == model.compact()
            model.check(cache)


def test_a_shared_tail_is_copied_for_all_but_the_last_holder():
    cache = make(12, 2, 2, 16, 16, 4, 3)
    model = Model(cache)
    for grow, src in (([21, 0, 0, 0], [0, 0, 0, 0]), ([1, 2, 0, 3], [3, 2, 1, 0]), ([1, 1, 1, 1], [1, 1, 1, 1]),
                      ([4, 4, 4, 4], [0, 1, 2, 3])):
        cache.extend(ints(grow))
        model.extend(grow)
        model.check(cache)
        cache.fork(ints(src))
        model.fork(src)
        model.check(cache)


def test_many_sessions_and_pages():
    """1024 sessions, more pages than a round of the scan takes, and tables wider than a strip."""
    S, M, B = 1024, 40, 16
    P = 20000
    cache = make(P, 1, 1, B, 8, S, M)
    model = Model(cache)
    rng = random.Random(5)
    for src in ([rng.randrange(S) for _ in range(S)], [rng.choice([s, -1]) for s in range(S)]):
        grow = [rng.randint(0, 17 * B) for _ in range(S)]
        cache.extend(ints(grow))
        model.extend(grow)
        model.check(cache)
        cache.fork(ints(src))
        model.fork(src)
        model.check(cache)
    used = cache.compact()
    assert int(used.item()) == model.compact()
    model.check(cache)


@pytest.mark.parametrize("n,d,B", [(1, 128, 16), (37, 80, 32), (130, 256, 64)])
def test_the_codecs_layout_goes_in_and_out(n, d, B):
    S, L, H = 3, 4, 2
    torch.manual_seed(n)
    cache = PagedKVCache.create(S * (-(-n // B)) + 1, L, H, d, S, n, B=B, device=DEV)
    full = torch.randn((S, L, n, H, d), device=DEV, dtype=torch.float16).permute(0, 1, 3, 2, 4)  # heads inner
    full2 = torch.randn((S, L, n, H, d), device=DEV, dtype=torch.float16).permute(0, 1, 3, 2, 4)
    counts = [n, n // 2, n]
    cache.extend(ints(counts))
    cache.store(full, full2, offsets(counts))
    out, out2 = torch.full_like(full, 7), torch.full_like(full2, 7)
    cache.load(out, out2, offsets(counts))
    cache.check_status()
    for got, want in ((out, full), (out2, full2)):
        for s, t in enumerate(counts):
            assert torch.equal(got[s, :, :, :t], want[s, :, :, :t])
            assert (got[s, :, :, t:] == 7).all()
    # one layer, the rows of a step
    k, v = (torch.randn((3, H, d), device=DEV, dtype=torch.float16) for _ in range(2))
    cache.trim(ints([max(0, t - 1) for t in counts]))
    cache.extend(ints([1] * S))
    cache.store(k, v, offsets([1] * S), layer=2)
    got, got2 = torch.zeros_like(k), torch.zeros_like(v)
    cache.load(got, got2, offsets([1] * S), layer=2)
    cache.check_status()
    assert torch.equal(got, k) and torch.equal(got2, v)


def test_a_full_pool_or_table_changes_nothing():
    cache = make(6, 1, 2, 16, 8, 3, 3)
    model = Model(cache)
    cache.extend(ints([40, 17, 0]))  # five pages
    model.extend([40, 17, 0])
    model.check(cache)
    for grow in ([0, 0, 17], [9, 0, 0], [1, 1, 49]):
        cache.extend(ints(grow))
        with pytest.raises(plc.PlcError) as e:
            cache.check_status()
        assert e.value.code == plc.PLC_ERR_CAPACITY
        model.check(cache)
    cache.extend(ints([8, 15, 16]))
    model.extend([8, 15, 16])
    model.check(cache)


def test_data_that_cannot_be_used_is_refused():
    """Numbers out of range, shared pages written to, offsets that are none: status tells, the rows stay, nothing else is
    touched."""
    def fresh():
        c = make(8, 2, 2, 16, 16, 3, 3)
        c.extend(ints([20, 33, 0]))
        c.check_status()
        return c, c.k.clone()

    def refused(cache, code=plc.PLC_ERR_INVALID):
        with pytest.raises(plc.PlcError) as e:
            cache.check_status()
        assert e.value.code == code

    for call in (lambda c: c.fork(ints([0, 3, 0])), lambda c: c.fork(ints([-2, 1, 2])), lambda c: c.extend(ints([-1, 0, 0])),
                 lambda c: c.trim(ints([21, 0, 0])), lambda c: c.trim(ints([20, -1, 0])),
                 lambda c: c.accept(offsets([5, 0, 0]), ints([0, 0]), offsets([2, 0, 0])),
                 lambda c: c.accept(offsets([5, 0, 0]), ints([5]), offsets([1, 0, 0])),
                 lambda c: c.accept(offsets([5, 0, 0]), ints([-1]), offsets([1, 0, 0])),
                 lambda c: c.accept(offsets([21, 0, 0]), ints([1]), offsets([1, 0, 0])),
                 lambda c: c.accept(offsets([2, 0, 0]), ints([0, 1, 2]), offsets([3, 0, 0])),
                 lambda c: c.accept(offsets([2, 2, 0]), ints([0, 1]), ints([0, 1, 9, 9]))):
        cache, before = fresh()
        call(cache)
        refused(cache)
        assert torch.equal(cache.k, before)
    # rows
    for off in ([0, 21, 21, 21], [1, 2, 2, 2], [0, 5, 3, 3], [0, 0, 0, 9], [0, -4, 0, 0]):
        for call in ("store", "load"):
            cache, before = fresh()
            k, v = rows_like(cache, 8, 2)
            getattr(cache, call)(k, v, ints(off))
            refused(cache)
    # pages that others hold
    cache, before = fresh()
    cache.fork(ints([0, 1, 0]))
    k, v = rows_like(cache, 2, 2)
    cache.store(k, v, offsets([2, 0, 0]))
    refused(cache)
    cache.accept(offsets([3, 0, 0]), ints([1]), offsets([1, 0, 0]))
    refused(cache)
    assert torch.equal(cache.k, before)
    # a table that names pages there are none of
    for bad in (8, -1, -7, 2**31 - 1):
        cache, before = fresh()
        cache.table[0, 1] = bad
        k, v = rows_like(cache, 3, 2)
        for call in (lambda: cache.store(k, v, offsets([3, 0, 0])), lambda: cache.load(k, v, offsets([3, 0, 0])),
                     lambda: cache.extend(ints([1, 0, 0])), lambda: cache.accept(offsets([3, 0, 0]), ints([2]), offsets([1, 0, 0]))):
            call()
            refused(cache)
        assert torch.equal(cache.k, before)
        cache, before = fresh()
        cache.table[0, 1] = bad
        cache.trim(ints([0, 33, 0]))
        refused(cache)
        cache, before = fresh()
        cache.table[0, 1] = bad
        cache.compact()
        if bad == -1:
            cache.check_status()  # an entry behind a session's pages is none
        else:
            refused(cache)
    for length in (-1, 49, 2**31 - 1):  # beyond the table
        cache, before = fresh()
        cache.lens[1] = length
        k, v = rows_like(cache, 3, 2)
        for call in (lambda: cache.store(k, v, offsets([0, 3, 0])), lambda: cache.load(k, v, offsets([0, 3, 0])),
                     lambda: cache.extend(ints([0, 1, 0])), lambda: cache.trim(ints([20, 0, 0])),
                     lambda: cache.accept(offsets([0, 3, 0]), ints([2]), offsets([0, 1, 0]))):
            call()
            refused(cache)
        assert torch.equal(cache.k, before)


@pytest.mark.parametrize("n", [3001, 4097])
def test_rows_on_both_sides_of_what_the_caches_hold(n):
    """As many rows as are stored through the caches, and more: every element, and nothing else, is where it belongs."""
    L, H, B, d = 4, 8, 16, 128
    assert (n * L * H * d * 8 > 96 << 20) == (n > 4000)
    torch.manual_seed(n)
    cache = make(-(-n // B) + 2, L, H, B, d, 1, -(-n // B))
    before = cache.k.clone()
    cache.extend(ints([n]))
    k, v = (torch.randn((1, L, H, n, d), device=DEV, dtype=torch.float16) for _ in range(2))
    cache.store(k, v, offsets([n]))
    cache.check_status()
    for pool, rows in ((cache.k, k), (cache.v, v)):
        used = pool[cache.table[0].long()].permute(1, 2, 0, 3, 4).flatten(2, 3)  # [L, H, rows, d]
        assert torch.equal(used[:, :, :n], rows[0])
    rest = torch.ones(cache.P, dtype=torch.bool, device=DEV)
    rest[cache.table[0].long()] = False
    assert torch.equal(cache.k[rest], before[rest])
    last = int(cache.table[0, -1])
    assert n % B == 0 or torch.equal(cache.k[last, :, :, n % B:], before[last, :, :, n % B:])
    out, out2 = torch.zeros_like(k), torch.zeros_like(v)
    cache.load(out, out2, offsets([n]))
    assert torch.equal(out, k) and torch.equal(out2, v)


def test_pages_beyond_32_bits():
    """A pool whose halves have more than 2^31 elements: the last page is as good as the first."""
    L, H, B, d = 4, 8, 64, 128
    P = (1 << 31) // (L * H * B * d) + 3
    k, v = (torch.empty((P, L, H, B, d), dtype=torch.float16, device=DEV) for _ in range(2))
    k[-2:] = 0
    v[-2:] = 0
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    cache = PagedKVCache(k, v, ints([[P - 1, -1], [-1, -1]]), ints([10, 0]), refs)
    refs[P - 1] = 1
    rows, rows2 = rows_like(cache, 10, L)
    cache.store(rows, rows2, offsets([10, 0]))
    cache.accept(offsets([4, 0]), ints([1, 3]), offsets([2, 0]))
    out, out2 = torch.zeros_like(rows[:8]), torch.zeros_like(rows[:8])
    cache.load(out, out2, offsets([8, 0]))
    keep = [0, 1, 2, 3, 4, 5, 7, 9]
    assert torch.equal(out, rows[keep]) and torch.equal(out2, rows2[keep])
    cache.fork(ints([0, 0]))
    refs[:P - 2] += 1  # taken by others
    cache.extend(ints([1, 0]))
    cache.load(out, out2, offsets([0, 8]))
    assert torch.equal(out, rows[keep])
    cache.trim(ints([8, 8]))
    cache.load(out, out2, offsets([8, 0]))
    assert torch.equal(out, rows[keep]) and cache.table[0, 0] == P - 2
    refs[:P - 2] = 0
    cache.compact()
    cache.check_status()
    cache.load(out, out2, offsets([0, 8]))
    assert torch.equal(out2, rows2[keep]) and cache.table[:, 0].tolist() == [0, 1]


@pytest.mark.parametrize("S", [64, 65])
def test_more_room_than_32_bits_count(S):
    """Tables so wide that the pages asked for in one call are 2^32 and more: refused like any other, and nothing changes."""
    M, B = 1 << 26, 16
    cache = make(6, 1, 1, B, 8, 1, 1)
    table = torch.empty((S, M), dtype=torch.int32, device=DEV)  # (entries behind a session's pages are not looked at)
    table[:2, :2] = ints([[3, -1], [3, -1]])
    lens, refs = ints([5, 5] + [0] * (S - 2)), ints([0, 0, 0, 2, 0, 0])
    cache = PagedKVCache(cache.k, cache.v, table, lens, refs)
    before = [x.clone() for x in (cache.k, cache.v, table[:, :2].contiguous(), lens, refs)]
    for grow in ([M * B - 5] * 2 + [M * B] * (S - 2), [M * B - 5] + [0] * (S - 1), [M * B - 5] * 2 + [1 << 29] * (S - 2)):
        cache.extend(ints(grow))
        with pytest.raises(plc.PlcError) as e:
            cache.check_status()
        assert e.value.code == plc.PLC_ERR_CAPACITY
        for x, b in zip((cache.k, cache.v, table[:, :2], lens, refs), before):
            assert torch.equal(x.contiguous().view(torch.int16), b.view(torch.int16))
    cache.extend(ints([1, 1] + [0] * (S - 2)))  # what there is room for is still given
    cache.check_status()
    assert lens.tolist() == [6, 6] + [0] * (S - 2) and refs.tolist() == [1, 0, 0, 1, 0, 0] and table[:2, 0].tolist() == [0, 3]


@pytest.mark.parametrize("L,H,d,sessions", [(2, 2, 16, 1), (9, 8, 128, 1), (2, 2, 16, 4), (9, 8, 128, 4)])
@pytest.mark.parametrize("path", [[0, 0], [5, 3], [2, 40], [-1], [0, 2, 30, 31, 33, 34, 35, 36, 37, 36], list(range(1, 38))])
def test_a_refused_path_changes_nothing(L, H, d, sessions, path):
    """Every form of the call: a path that cannot be followed, wherever it breaks off, leaves its session's rows, length, pages
    and counts; the other sessions' are accepted."""
    t, B = 37, 16
    cache = make(12 * sessions, L, H, B, d, sessions, 6)
    model = Model(cache)
    lens = [60 + i for i in range(sessions)]
    cache.extend(ints(lens))
    model.extend(lens)
    good = [1, 2, 20, 36]
    for s in range(sessions):
        cache.accept(offsets([t] * sessions), ints(good * s + path + good * (sessions - 1 - s)),
                     offsets([len(good)] * s + [len(path)] + [len(good)] * (sessions - 1 - s)))
        with pytest.raises(plc.PlcError) as e:
            cache.check_status()
        assert e.value.code == plc.PLC_ERR_INVALID
        kept = [list(range(t)) if i == s else good for i in range(sessions)]
        model.accept([t] * sessions, kept)
        model.check(cache)
        grow = [lens[i] - n for i, n in enumerate(model.lens)]
        cache.extend(ints(grow))
        model.extend(grow)


def test_a_page_given_back_in_the_call_was_not_the_sessions_own():
    """Two sessions on the same pages: one gives up all of its tree, which would leave the pages to the other alone; but it is
    not to write on them in this call, in whatever order the sessions come."""
    for turned in (False, True):
        cache = make(12, 2, 2, 16, 16, 2, 4)
        model = Model(cache)
        cache.extend(ints([40, 0]))
        model.extend([40, 0])
        cache.fork(ints([0, 0]))
        model.fork([0, 0])
        paths = [[], [1, 3]][:: -1 if turned else 1]
        cache.accept(offsets([24, 24]), ints([1, 3]), offsets([len(p) for p in paths]))
        with pytest.raises(plc.PlcError):
            cache.check_status()
        model.accept([24, 24], [[] if not p else list(range(24)) for p in paths])
        model.check(cache)


def test_more_heads_than_a_grid_is_wide():
    L, H, B, d = 300, 1024, 16, 8
    torch.manual_seed(2)
    cache = make(3, L, H, B, d, 2, 2)
    cache.extend(ints([20, 3]))
    before = cache.k.clone()
    k, v = rows_like(cache, 7, L)
    cache.store(k, v, offsets([5, 2]))
    out, out2 = torch.zeros_like(k), torch.zeros_like(v)
    cache.load(out, out2, offsets([5, 2]))
    cache.check_status()
    assert torch.equal(out, k) and torch.equal(out2, v)
    t = cache.table.tolist()
    for i, (page, row) in enumerate([(t[0][0], 15), (t[0][1], 0), (t[0][1], 1), (t[0][1], 2), (t[0][1], 3), (t[1][0], 1), (t[1][0], 2)]):
        assert torch.equal(cache.k[page, :, :, row], k[i])
        before[page, :, :, row] = k[i]
    assert torch.equal(cache.k, before)
