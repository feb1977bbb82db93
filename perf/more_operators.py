"""Workloads for what a model's step needs around the paged cache and the codec: rotary positions, the attention that
positions have received, eviction by it, and what logits say of tokens.

A case names the operator and its shape.
  "rotate"  rotary positions.  `form` "step": the new tokens' queries rotated, their keys rotated into the pages, their values
            stored; "restore": a cache whose keys were coded unrotated, in the codec's [S, L, H, n, d], into pages; "back": rows
            of a cache, rotated back for the encoder.  r of the d components are rotated, in halves or interleaved; `scaling`
            stretches the angles.  `past`: positions that lie before those in the cache (a cache that was thinned out).
  "weigh"   the attention weights that the last T positions of each session give to all that they see, in one layer, summed over
            them and the G query heads of a KV head, added to `decay` times what has been added up before.
  "evict"   of each session the `keep` part of the positions stays: the first, the last quarter, and of the others those of the
            largest weights, for each layer and head by itself.
  "score"   log-probabilities of N given tokens under logits over V, the entropy, and the k largest.
S sessions, L layers, H KV heads, pages of B rows, contexts of up to n rows; with `ragged` the sessions' lengths lie evenly
between one row and n.

The plain forms are the definitions in elementary torch operations.  What a pass changes of a cache (tables, lengths, counts,
the weights) is put back at its start, so that a pass can follow another.
"""
import math
import random

import torch

own = False

_BASE = dict(S=1, L=1, H=8, G=1, d=128, B=16, n=1024, T=1, dtype="fp16", ragged=False,
             form="step", r=128, interleaved=False, scaling="none", base=10000.0, past=0,
             decay=1.0, keep=0.5, N=1, V=50016, k=8, temperature=1.0)
_DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _case(**kw):
    return {**_BASE, **kw}


def listed():
    return [
        # one token of one short session of a small model: latency
        _case(name="rotate_tiny", op="rotate", H=4, d=64, r=64, n=512),
        # drafted tokens of sessions of all lengths, a quarter of the head rotated, interleaved, far positions
        _case(name="rotate_part", op="rotate", S=21, H=5, G=3, d=80, r=20, interleaved=True, scaling="parts", base=500000.0,
              past=150000, n=777, T=9, dtype="bf16", ragged=True),
        # a whole cache that was coded unrotated, into its pages
        _case(name="rotate_restore", op="rotate", form="restore", L=32, n=4096),
        # one token of one short session
        _case(name="weigh_tiny", op="weigh", H=4, d=64, n=512),
        # a serving batch, one token a session, contexts of all lengths
        _case(name="weigh_batched", op="weigh", S=64, G=4, n=4096, decay=0.95, ragged=True),
        # the next piece of a prompt
        _case(name="weigh_prompt", op="weigh", G=4, n=8192, T=512, decay=0.0, dtype="bf16"),
        # a small model's session
        _case(name="evict_tiny", op="evict", L=2, H=4, d=64, n=512),
        # sessions of odd lengths, some of them below what may stay
        _case(name="evict_ragged", op="evict", S=5, L=7, H=5, d=80, n=1777, B=64, keep=0.45, ragged=True, dtype="bf16"),
        # long sessions with every layer
        _case(name="evict_layers", op="evict", S=4, L=32, n=2048),
        # the next token of one session
        _case(name="score_token", op="score", V=50016, k=4, dtype="bf16"),
        # drafted tokens of a batch, odd vocabulary, 32-bit logits
        _case(name="score_drafts", op="score", N=37, V=32003, k=20, dtype="fp32", temperature=0.7),
        # a prompt
        _case(name="score_prompt", op="score", N=4096, V=50016, k=8, dtype="bf16"),
    ]


_MOST_BYTES = 1.07e9   # of one pass: that of "rotate_restore"
_MOST_FLOPS = 3.5e10   # of one pass: that of "weigh_prompt"
_MOST_STATE = 3.0e9    # bytes of the pool's two halves


def draw(rng):
    log_uniform = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        op = rng.choice(["rotate", "rotate", "weigh", "weigh", "evict", "score"])
        c = _case(op=op, H=rng.choice([1, 2, 4, 5, 8, 16, 64]), d=rng.choice([64, 80, 96, 128, 128, 256]),
                  B=rng.choice([16, 16, 32, 64, 128]), S=log_uniform(1, 64), dtype=rng.choice(["fp16", "bf16"]),
                  ragged=rng.random() < 0.5)
        if op == "rotate":
            c.update(form=rng.choice(["step", "step", "restore", "back"]), G=rng.choice([1, 2, 3, 4, 7, 8]),
                     r=2 * rng.choice([c["d"] // 2, c["d"] // 4, c["d"] // 8, rng.randint(1, c["d"] // 2)]),
                     interleaved=rng.random() < 0.5, scaling=rng.choice(["none", "linear", "stretched", "parts", "ramp"]),
                     base=rng.choice([10000.0, 500000.0]), past=rng.choice([0, 0, log_uniform(1, 1000000)]),
                     n=log_uniform(1, 4096))
            if c["form"] == "step":
                c.update(T=rng.choice([1, 1, log_uniform(2, 512)]))
            else:
                c.update(L=log_uniform(1, 32))
        elif op == "weigh":
            c.update(G=rng.choice([1, 2, 3, 4, 7, 8]), n=log_uniform(65, 32768), T=rng.choice([1, 1, log_uniform(2, 512)]),
                     decay=rng.choice([0.0, 0.9, 1.0]))
        elif op == "evict":
            c.update(L=log_uniform(1, 32), n=log_uniform(17, 8192), keep=rng.uniform(0.2, 0.95))
        else:
            c.update(N=log_uniform(1, 4096), V=log_uniform(2000, 131072), k=rng.choice([0, 1, 4, 8, 20, 32]),
                     dtype=rng.choice(["fp16", "bf16", "fp32"]), temperature=rng.choice([1.0, 0.7, 1.3]))
        w = work(c)
        pool = 4.0 * _pages(c) * c["B"] * c["L"] * c["H"] * c["d"] if op != "score" else 0.0
        padded = 4.0 * c["S"] * c["H"] * c["G"] * c["T"] * (c["n"] + c["T"]) if op == "weigh" else 0.0
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS and pool <= _MOST_STATE and padded <= 2 * _MOST_STATE:
            return c


# ---- shapes of a case ---------------------------------------------------------------------------------------------

def _contexts(c):
    """Rows of each session before a call: by the case alone, so that every seed does the same work."""
    return [max(1, c["n"] * (i + 1) // c["S"]) if c["ragged"] else c["n"] for i in range(c["S"])]


def _tokens(c):
    """New rows of each session."""
    if c["op"] == "rotate" and c["form"] != "step":
        return _contexts(c)
    half = c["T"] // 2 + 1
    return [c["T"] - (7 * i) % half if c["ragged"] else c["T"] for i in range(c["S"])]


def _lengths(c):
    """Rows of each session that the call finds."""
    if c["op"] == "evict" or (c["op"] == "rotate" and c["form"] != "step"):
        return _contexts(c)
    return [r + t for r, t in zip(_contexts(c), _tokens(c))]


def _kept(c):
    """(rows that stay, of them the first ones and the last ones), of a session that has more."""
    keep = max(1, int(c["n"] * c["keep"]))
    return keep, min(4, keep // 4), keep // 4


def _pages_of(rows, B):
    return -(-rows // B)


def _slots(c):
    """Width of the table."""
    return _pages_of(max(_lengths(c)), c["B"]) + 1


def _pages(c):
    """Pages of the pool."""
    return sum(_pages_of(r, c["B"]) for r in _lengths(c)) + 3


def work(case):
    c = {**_BASE, **case}
    if c["op"] == "score":
        size = 4 if c["dtype"] == "fp32" else 2
        return {"bytes": float(c["N"] * (size * c["V"] + 20 + 12 * c["k"])), "flops": 0.0}
    new, lens = _tokens(c), _lengths(c)
    row = 2.0 * c["L"] * c["H"] * c["d"]  # bytes of a row's keys in all layers
    if c["op"] == "rotate":
        rows = sum(new)
        if c["form"] == "back":
            return {"bytes": 2 * row * rows, "flops": 0.0}
        queries = 2.0 * c["H"] * c["G"] * c["d"] if c["form"] == "step" else 0.0
        return {"bytes": 2 * rows * (2 * row + queries), "flops": 0.0}
    if c["op"] == "weigh":
        seen = sum(t * (n - t) + t * (t + 1) // 2 for t, n in zip(new, lens))
        olds = 4.0 if c["decay"] else 0.0
        return {"bytes": sum(lens) * (row + c["H"] * (4 + olds)) + sum(new) * c["H"] * c["G"] * (2 * c["d"] + 4),
                "flops": 2.0 * c["d"] * c["H"] * c["G"] * seen}
    keep, first, _ = _kept(c)
    heads = c["L"] * c["H"]
    total = 0.0
    for n in lens:
        if n > keep:  # weights looked at, those and the rows that stay behind the first ones moved, their old places told
            total += heads * (4.0 * n + 8.0 * keep) + (keep - first) * 4 * row
        else:
            total += heads * 4.0 * n
    return {"bytes": total, "flops": 0.0}


# ---- inputs -------------------------------------------------------------------------------------------------------

_FACTOR, _TRAINED = 8.0, 4096  # stretched to so many times the positions that a model was trained on


def _scaling(c):
    """What a user says of the angles: see _angles for what it means."""
    return {"none": {}, "linear": dict(scaling="linear", factor=_FACTOR), "stretched": dict(scaling="stretched", factor=_FACTOR),
            "parts": dict(scaling="parts", factor=_FACTOR, low=1.0, high=4.0, trained=_TRAINED),
            "ramp": dict(scaling="ramp", factor=_FACTOR, low=1.0, high=32.0, trained=_TRAINED,
                         magnitude=0.1 * math.log(_FACTOR) + 1.0)}[c["scaling"]]


def _angles(c):
    """Radians a position, of each pair, and the factor of the results."""
    r, base = c["r"], c["base"]
    kind = c["scaling"]
    if kind == "stretched" and r > 2:
        base = base * _FACTOR ** (r / (r - 2))
    theta = [base ** (-2.0 * i / r) for i in range(r // 2)]
    if kind == "linear":
        theta = [t / _FACTOR for t in theta]
    elif kind == "parts":  # whole where there are 4 turns or more within the trained positions, divided at one or fewer
        for i, t in enumerate(theta):
            g = min(1.0, max(0.0, (_TRAINED * t / (2 * math.pi) - 1.0) / (4.0 - 1.0)))
            theta[i] = (1 - g) * t / _FACTOR + g * t
    elif kind == "ramp":  # the same along the pairs' numbers, between the pairs of 32 turns and of one
        pair = lambda turns: r * math.log(_TRAINED / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), r - 1)
        for i, t in enumerate(theta):
            g = 1.0 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            theta[i] = (1 - g) * t / _FACTOR + g * t
    return theta, _scaling(c).get("magnitude", 1.0)


def _logits(c, gen):
    """A model's: most tokens far below a few, some of the vocabulary masked."""
    x = torch.randn((c["N"], c["V"]), generator=gen, device="cuda", dtype=_DTYPES[c["dtype"]]) * 2.5
    peaks = torch.randint(0, c["V"], (c["N"], 12), generator=gen, device="cuda")
    x.scatter_add_(1, peaks, torch.rand((c["N"], 12), generator=gen, device="cuda").to(x.dtype) * 12)
    x[:, torch.randint(0, c["V"], (c["V"] // 100,), generator=gen, device="cuda")] = -math.inf
    tokens = torch.where(torch.rand(c["N"], generator=gen, device="cuda") < 0.7, peaks[:, 0],
                         torch.randint(0, c["V"], (c["N"],), generator=gen, device="cuda")).to(torch.int32)
    tokens[torch.rand(c["N"], generator=gen, device="cuda") < 0.05] = -1  # padding
    return x, tokens


def prepare(case, seed):
    c = {**_BASE, **case}
    rng = random.Random(seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    st = {"case": c}
    if c["op"] == "score":
        st["logits"], st["tokens"] = _logits(c, gen)
        return st
    S, L, H, G, d, B, op = (c[x] for x in ("S", "L", "H", "G", "d", "B", "op"))
    dt, P, M = _DTYPES[c["dtype"]], _pages(c), _slots(c)
    order = rng.sample(range(S), S) if op == "evict" or c["form"] == "step" else list(range(S))
    new, lens = ([v[i] for i in order] for v in (_tokens(c), _lengths(c)))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda", dtype=dt)  # noqa: E731

    free = rng.sample(range(P), P)
    table, refs = [], [0] * P
    for n in lens:
        table.append([free.pop() for _ in range(_pages_of(n, B))])
    for row in table:
        for page in row:
            refs[page] += 1
    flat = [p for row in table for p in row + [-1] * (M - len(row))]
    meta = ints(lens + flat + refs)  # lengths, table and reference counts in one piece: put back by one copy
    st["start"], st["meta"] = meta, meta.clone()
    st["lens"] = st["meta"][:S]
    st["table"] = st["meta"][S:S + S * M].view(S, M)
    st["refs"] = st["meta"][S + S * M:]
    if op != "evict":
        st["off"] = ints([sum(new[:i]) for i in range(S + 1)])

    def rows(*shape):  # keys have a few strong channels, as those of a model have
        k = normal(*shape)
        k[..., : d // 16] *= 3
        return k

    if op == "rotate":
        N = sum(new)
        if c["form"] == "back":
            st["x"] = rows(N, L, H, d)
            st["positions"] = torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in lens]) + c["past"]
            return st
        st["k"], st["v"] = (torch.zeros((P, L, H, B, d), device="cuda", dtype=dt) for _ in range(2))
        # the positions in front of the new rows: those in the cache, and those that are there no more
        st["base"] = ints([n - t + c["past"] for n, t in zip(lens, new)]) if c["past"] else None
        if c["form"] == "step":
            st["new_k"], st["new_v"], st["q"] = rows(N, L, H, d), normal(N, L, H, d), normal(N, H * G, d)
            # drafted tokens: each follows one of those before it, a few steps deep
            depth = [min(i, rng.randrange(0, 6)) for t in new for i in range(t)]
            st["rel"] = ints(depth) if c["T"] > 1 and c["ragged"] else None
        else:
            st["new_k"], st["new_v"] = rows(S, L, H, c["n"], d), normal(S, L, H, c["n"], d)
        return st
    if op == "weigh":
        st["k"] = rows(P, L, H, B, d)
        st["v"] = torch.zeros_like(st["k"])  # of no account here
        st["q"] = normal(sum(new), H * G, d) * 1.5
        score, back = _scores(st)
        st["lse"] = back(torch.logsumexp(score, 3))
        st["weights_start"] = torch.rand((S, L, H, M * B), generator=gen, device="cuda") * 4
    else:
        st["k"], st["v"] = rows(P, L, H, B, d), normal(P, L, H, B, d)
        # a few positions hold most of it; some have received nothing at all
        w = (torch.randn((S, L, H, M * B), generator=gen, device="cuda") * 2).exp_()
        w[torch.rand(w.shape, generator=gen, device="cuda") < 0.1] = 0.0
        st["weights_start"] = w
        st["keep"] = ints([min(_kept(c)[0], n) for n in lens])
        st["kept"] = torch.full((S, L, H, _kept(c)[0]), -1, dtype=torch.int32, device="cuda")
    st["weights"] = st["weights_start"].clone()
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state)


def _run_own(st):
    c = st["case"]
    op = c["op"]
    if op == "score":
        scorer = st.get("scorer")
        if scorer is None:  # the handle that a user's program makes once
            from paper_2604_15356_amd.scores import TokenScorer
            scorer = st["scorer"] = TokenScorer(c["V"], c["k"])
        s = scorer.score(st["logits"], st["tokens"], temperature=c["temperature"])
        return (s.logprob, s.entropy, s.lse) + ((s.ids, s.logprobs, s.probs, s.chosen) if c["k"] else ())
    rotary = st.get("rotary")
    if op == "rotate" and rotary is None:
        from paper_2604_15356_amd.rotary import Rotary
        rotary = st["rotary"] = Rotary(c["d"], r=c["r"], base=c["base"], interleaved=c["interleaved"], **_scaling(c))
    if op == "rotate" and c["form"] == "back":
        x = st["x"]
        return rotary.rotate(x.view(x.shape[0], -1, c["d"]), st["positions"], inverse=True).view(x.shape)
    cache = st.get("cache")
    if cache is None:
        from paper_2604_15356_amd.paged import PagedKVCache
        cache = st["cache"] = PagedKVCache(st["k"], st["v"], st["table"], st["lens"], st["refs"])
    if op == "rotate":
        if c["form"] == "restore":
            cache.store_rotated(st["new_k"], st["new_v"], st["off"], rotary, base=st["base"])
            return st["k"], st["v"]
        return cache.store_rotated(st["new_k"], st["new_v"], st["off"], rotary, q=st["q"], base=st["base"], rel=st["rel"]), \
            st["k"], st["v"]
    if op == "weigh":
        if c["decay"]:
            st["weights"].copy_(st["weights_start"])
        cache.add_weights(st["q"], st["off"], st["lse"], st["weights"], decay=c["decay"], max_nodes=c["T"], max_len=c["n"] + c["T"])
        return st["weights"]
    st["meta"].copy_(st["start"])
    st["weights"].copy_(st["weights_start"])
    _, first, last = _kept(c)
    cache.evict(st["keep"], st["weights"], st["kept"], first=first, last=last, max_len=c["n"])
    return st["k"], st["v"], st["table"], st["lens"], st["refs"], st["weights"], st["kept"]


def _session_of(off, rows):
    """Of packed rows: the session, and the row's number in it."""
    x = torch.arange(rows, device=off.device)
    s = torch.searchsorted(off[1:].contiguous(), x.to(torch.int32), right=True)
    return s, x - off.long()[s]


def _place(st, s, pos):
    """Page and row of position `pos` of session `s`."""
    B = st["case"]["B"]
    return st["table"].long()[s, pos // B], pos % B


def _rotated(x, positions, c, sign=1.0):
    """x [rows, ..., d] at positions [rows], in 32 bits; the angles in 64.  sign -1: back."""
    theta, magnitude = _angles(c)
    theta = torch.tensor(theta, dtype=torch.float64, device=x.device)
    angle = sign * positions.double()[:, None] * theta
    shape = (x.shape[0],) + (1,) * (x.dim() - 2) + (-1,)
    cos, sin = ((f(angle) * magnitude ** sign).float().view(shape) for f in (torch.cos, torch.sin))
    r, y = c["r"], x.float()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., : r // 2], y[..., r // 2:r])
    pairs = torch.stack((a * cos - b * sin, b * cos + a * sin), -1 if c["interleaved"] else -2)
    return torch.cat((pairs.flatten(-2), y[..., r:]), -1).to(x.dtype)


def _plain_rotate(st):
    c = st["case"]
    if c["form"] == "back":
        return _rotated(st["x"], st["positions"], c, sign=-1.0)
    new_k, new_v, off, lens = st["new_k"], st["new_v"], st["off"].long(), st["lens"].long()
    counts = off[1:] - off[:-1]
    before = lens - counts
    base = before if st["base"] is None else st["base"].long()
    if c["form"] == "restore":
        s, i = torch.nonzero(torch.arange(new_k.shape[3], device=new_k.device)[None] < counts[:, None], as_tuple=True)
        k, v = new_k[s, :, :, i], new_v[s, :, :, i]
    else:
        s, i = _session_of(st["off"], new_k.shape[0])
        k, v = new_k, new_v
    positions = base[s] + (i if st.get("rel") is None else st["rel"].long())
    page, row = _place(st, s, before[s] + i)
    st["k"][page, :, :, row] = _rotated(k, positions, c)
    st["v"][page, :, :, row] = v
    if c["form"] == "restore":
        return st["k"], st["v"]
    return _rotated(st["q"], positions, c), st["k"], st["v"]


def _scores(st):
    """Scaled products of all sessions, padded: [S, H, T G, M B], minus infinity where a row does not see a position, and what takes a
    value for each of its rows back to [nodes, H G]."""
    c = st["case"]
    S, H, G, d, B = (c[x] for x in ("S", "H", "G", "d", "B"))
    q, off, T = st["q"], st["off"].long(), c["T"]
    N, M = q.shape[0], st["table"].shape[1]
    counts, lens = off[1:] - off[:-1], st["lens"].long()
    k = st["k"][st["table"].long().clamp(min=0), 0].float().permute(0, 2, 1, 3, 4).reshape(S, H, M * B, d)
    s, i = _session_of(st["off"], N)
    padded = torch.zeros((S, T, H * G, d), device=q.device)
    padded[s, i] = q.float()
    padded = padded.view(S, T, H, G, d).permute(0, 2, 1, 3, 4).reshape(S, H, T * G, d)
    score = torch.matmul(padded, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    pos, node = torch.arange(M * B, device=q.device), torch.arange(T, device=q.device)
    last = (lens - counts)[:, None] + node  # [S, T]: the last position that a node sees
    hidden = (pos > last[:, :, None]) | (node >= counts[:, None])[:, :, None]
    score.view(S, H, T, G, M * B).masked_fill_(hidden[:, None, :, None], -math.inf)
    back = lambda x: x.view(S, H, T, G).permute(0, 2, 1, 3).reshape(S, T, H * G)[s, i]  # noqa: E731
    return score, back


def _plain_weigh(st):
    c = st["case"]
    S, H, G, T = (c[x] for x in ("S", "H", "G", "T"))
    if c["decay"]:
        st["weights"].copy_(st["weights_start"])
    score, _ = _scores(st)
    lens, off = st["lens"].long(), st["off"].long()
    counts = off[1:] - off[:-1]
    s, i = _session_of(st["off"], st["q"].shape[0])
    lse = torch.zeros((S, T, H * G), device=score.device)
    lse[s, i] = st["lse"]
    lse = lse.view(S, T, H, G).permute(0, 2, 1, 3).reshape(S, H, T * G, 1)
    sums = (score - lse).exp_().sum(2)
    pos = torch.arange(score.shape[3], device=score.device)
    w = st["weights"][:, 0]
    if c["decay"]:  # the call's own positions begin with nothing
        sums = torch.where((pos < (lens - counts)[:, None])[:, None], c["decay"] * w + sums, sums)
    w.copy_(torch.where((pos < lens[:, None])[:, None], sums, w))
    return st["weights"]


def _count_refs(st):
    """A page's references are the entries that name it."""
    entries = st["table"][st["table"] >= 0].long()
    st["refs"].copy_(torch.bincount(entries, minlength=st["refs"].shape[0]))


def _plain_evict(st):
    st["meta"].copy_(st["start"])
    st["weights"].copy_(st["weights_start"])
    c = st["case"]
    L, H, B = c["L"], c["H"], c["B"]
    _, first, last = _kept(c)
    layer, head = torch.arange(L, device="cuda")[:, None, None], torch.arange(H, device="cuda")[None, :, None]
    for s, (n, keep) in enumerate(zip(st["lens"].tolist(), st["keep"].tolist())):
        pos = torch.arange(n, device="cuda")
        if n <= keep:
            st["kept"][s, :, :, :n] = pos.to(torch.int32)
            continue
        w = st["weights"][s, :, :, :n].clone()
        rank = w.clone()
        rank[..., :first] = math.inf
        rank[..., n - last:] = math.inf
        # the largest, of equal ones the lowest positions
        stay = torch.sort(torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep], dim=-1).values
        page, row = _place(st, s, stay)
        k, v = st["k"][page, layer, head, row], st["v"][page, layer, head, row]
        page, row = _place(st, s, pos[:keep].expand(L, H, keep))
        st["k"][page, layer, head, row] = k
        st["v"][page, layer, head, row] = v
        st["weights"][s, :, :, :keep] = torch.gather(w, 2, stay)
        st["kept"][s, :, :, :keep] = stay.to(torch.int32)
    st["lens"].copy_(st["keep"])
    slots = torch.arange(st["table"].shape[1], device="cuda")
    st["table"].masked_fill_(slots[None] * B >= st["lens"][:, None], -1)
    _count_refs(st)
    return st["k"], st["v"], st["table"], st["lens"], st["refs"], st["weights"], st["kept"]


_ROWS = 512  # at a time


def _plain_score(st):
    c = st["case"]
    parts = []
    for at in range(0, c["N"], _ROWS):
        raw, token = st["logits"][at:at + _ROWS].float(), st["tokens"][at:at + _ROWS].long()
        x = raw / c["temperature"]
        top = x.amax(1, keepdim=True)
        e = (x - top).exp()
        total = e.sum(1, keepdim=True)
        lse = (top + total.log())[:, 0]
        seen = x.gather(1, token.clamp(min=0)[:, None])[:, 0]
        logprob = torch.where(token >= 0, seen - lse, torch.zeros_like(lse))
        entropy = total.log()[:, 0] - (e * torch.where(e > 0, x - top, torch.zeros_like(x))).sum(1) / total[:, 0]
        part = [logprob, entropy, lse]
        if c["k"]:
            # by the logits, of equal ones the lowest tokens: both in one whole number
            bits = (raw + 0.0).view(torch.int32)
            bits = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
            key = bits * 2 ** 32 + (c["V"] - 1 - torch.arange(c["V"], device=raw.device))
            ids = torch.topk(key, c["k"], 1).indices
            logprobs = x.gather(1, ids) - lse[:, None]
            hit = (ids == token[:, None])
            chosen = torch.where(hit.any(1), hit.float().argmax(1), torch.full_like(token, -1))
            part += [ids.to(torch.int32), logprobs, logprobs.exp(), chosen.to(torch.int32)]
        parts.append(part)
    return tuple(torch.cat(p) for p in zip(*parts))


_PLAIN = {"rotate": _plain_rotate, "weigh": _plain_weigh, "evict": _plain_evict, "score": _plain_score}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def _turned(x, positions, c, sign=1):
    """Rotated by complex multiplication."""
    theta, magnitude = _angles(c)
    angle = sign * positions.double()[:, None] * torch.tensor(theta, dtype=torch.float64, device=x.device)
    by = torch.polar(torch.full_like(angle, magnitude ** sign), angle)
    r, out = c["r"], x.double()
    at = torch.arange(r // 2, device=x.device)
    re, im = (2 * at, 2 * at + 1) if c["interleaved"] else (at, at + r // 2)
    for j in range(x.shape[1]):  # a head at a time
        z = torch.complex(out[:, j, re], out[:, j, im]) * by
        out[:, j, re], out[:, j, im] = z.real, z.imag
    return out


def _exact_rotate(c, st):
    if c["form"] == "back":
        x = st["x"]
        return _turned(x.view(x.shape[0], -1, c["d"]), st["positions"], c, sign=-1).view(x.shape)
    pool = st["k"].double()
    off, lens = st["off"].tolist(), st["lens"].tolist()
    q = []
    for s in range(c["S"]):
        t, n = off[s + 1] - off[s], lens[s]
        first = n - t if st["base"] is None else int(st["base"][s])
        rel = torch.arange(t, device="cuda") if st.get("rel") is None else st["rel"][off[s]:off[s + 1]].long()
        k = st["new_k"][s, :, :, :t].permute(2, 0, 1, 3) if c["form"] == "restore" else st["new_k"][off[s]:off[s + 1]]
        k = _turned(k.reshape(t, c["L"] * c["H"], c["d"]), first + rel, c).view(t, c["L"], c["H"], c["d"])
        pos = torch.arange(n - t, n, device="cuda")
        pool[st["table"].long()[s, pos // c["B"]], :, :, pos % c["B"]] = k
        if c["form"] == "step":
            q.append(_turned(st["q"][off[s]:off[s + 1]], first + rel, c))
    return (pool, None) if c["form"] == "restore" else (torch.cat(q), pool, None)


def _exact_weigh(c, st):
    H, G, d, B = (c[x] for x in ("H", "G", "d", "B"))
    off, lens, table = st["off"].tolist(), st["lens"].tolist(), st["table"].tolist()
    out = st["weights_start"].double()
    for s in range(c["S"]):
        t, n = off[s + 1] - off[s], lens[s]
        k = torch.cat([st["k"][p, 0] for p in table[s][: _pages_of(n, B)]], dim=1)[:, :n].double()
        q, lse = st["q"][off[s]: off[s + 1]].double(), st["lse"][off[s]: off[s + 1]].double()
        pos = torch.arange(n, device="cuda")
        node = torch.arange(t, device="cuda").repeat_interleave(G)
        hidden = pos[None] > (n - t + node)[:, None]
        for h in range(H):
            score = (q[:, h * G: (h + 1) * G].reshape(t * G, d) @ k[h].T) * d ** -0.5
            sums = (score - lse[:, h * G: (h + 1) * G].reshape(t * G, 1)).exp().masked_fill(hidden, 0.0).sum(0)
            before = c["decay"] * out[s, 0, h, : n - t]
            out[s, 0, h, :n] = sums
            out[s, 0, h, : n - t] += before
    return out


def _exact_score(c, st):
    parts = []
    for at in range(0, c["N"], _ROWS):
        raw, token = st["logits"][at:at + _ROWS], st["tokens"][at:at + _ROWS].long()
        logs = torch.log_softmax(raw.double() / c["temperature"], 1)
        lse = torch.logsumexp(raw.double() / c["temperature"], 1)
        p = logs.exp()
        entropy = -(p * logs.masked_fill(p == 0, 0.0)).sum(1)
        logprob = logs.gather(1, token.clamp(min=0)[:, None])[:, 0].masked_fill(token < 0, 0.0)
        part = [logprob, entropy, lse]
        if c["k"]:
            best = torch.topk(logs, c["k"], 1).values  # (equal logits have equal ones)
            part += [best, best.exp()]
        parts.append(part)
    out = [torch.cat(p) for p in zip(*parts)]
    return (*out[:3], None, *out[3:], None) if c["k"] else tuple(out)


def exact(case, seed):
    """The other operators move values and count."""
    c = {**_BASE, **case}
    if c["op"] == "evict":
        return None
    return {"rotate": _exact_rotate, "weigh": _exact_weigh, "score": _exact_score}[c["op"]](c, prepare(case, seed))
