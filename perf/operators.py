"""Workloads for the paged cache and the attention over it: what a serving loop does around the codec of this package.

A case names the operator ("attend": the attention of drafted tokens over a paged cache, one layer; "beam": a step of beam
search, which forks the beams, makes room for a token each and stores it; "accept": a step of speculative decoding, which
stores the drafted nodes and keeps the accepted ones; "compact": the pages in use moved to the pool's front; "restore" and
"evict": the rows of whole caches into pages, out of the codec's [S, L, H, n, d], and out of pages, packed) and its shape:
S sessions, L layers, H KV heads, G query heads a KV head, d components, pages of B rows, contexts of up to n rows, trees of
up to T nodes.  With `ragged`, the sessions' lengths lie evenly between one row and n, and their trees between half of T and
T nodes; a `chain` is a tree whose nodes follow one another, as the tokens of a prompt's next piece do.

The plain forms are the definitions in elementary torch operations.  A cache's tables, lengths and reference counts are put
back at the start of a pass that changes them, so that a pass can follow another.
"""
import math
import random

import torch

own = False

_BASE = dict(S=1, L=1, H=8, G=1, d=128, B=16, n=1024, T=1, dtype="fp16", ragged=False, chain=False)
_DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _case(**kw):
    return {**_BASE, **kw}


def listed():
    return [
        # one token of one short session of a small model: latency
        _case(name="decode_tiny", op="attend", H=4, d=64, n=512),
        # a serving batch, one token a session, contexts of all lengths
        _case(name="decode_batched", op="attend", S=64, G=4, n=4096, ragged=True),
        # drafted trees of a few sessions, odd counts
        _case(name="tree_sessions", op="attend", S=5, G=4, n=4095, T=27, dtype="bf16", ragged=True),
        # a large tree at the end of a long context
        _case(name="tree_long", op="attend", G=4, n=32768, T=64, dtype="bf16"),
        # a step of beam search of a small model
        _case(name="beam_tiny", op="beam", S=4, L=2, H=4, d=64, n=130),
        # 64 beams of 16 prompts
        _case(name="beam_batched", op="beam", S=64, L=8, n=1000),
        # the accepted path of a drafted tree, small and with every layer of a serving batch
        _case(name="accept_tiny", op="accept", L=2, H=4, d=64, n=100, T=8),
        _case(name="accept_batched", op="accept", S=64, L=32, n=40, T=32, ragged=True),
        # a pool of which half is in use
        _case(name="compact_tiny", op="compact", S=4, L=2, H=4, d=64, n=512),
        _case(name="compact_pool", op="compact", S=8, L=32, n=500, ragged=True, dtype="bf16"),
        # a decoded cache into pages, and sessions of odd lengths out of them
        _case(name="restore_llama8b", op="restore", L=32, n=4096),
        _case(name="evict_ragged", op="evict", S=3, L=7, H=5, d=80, n=777, B=64, ragged=True),
    ]


_MOST_BYTES = 1.07e9   # of one pass: that of "restore_llama8b"
_MOST_FLOPS = 3.4e10   # of one pass: that of "tree_long"
_MOST_STATE = 3.0e9    # bytes of the pool's two halves


def draw(rng):
    log_uniform = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        op = rng.choice(["attend", "attend", "attend", "beam", "accept", "compact", "restore", "evict"])
        c = _case(op=op, H=rng.choice([1, 2, 4, 5, 8, 16, 64]), d=rng.choice([64, 80, 96, 128, 128, 256]),
                  B=rng.choice([16, 16, 32, 64, 128]), S=log_uniform(1, 64), dtype=rng.choice(["fp16", "bf16"]),
                  ragged=rng.random() < 0.5)
        if op == "attend":
            c.update(G=rng.choice([1, 2, 3, 4, 7, 8]), n=log_uniform(65, 32768), T=rng.choice([1, 1, log_uniform(2, 64)]),
                     chain=rng.random() < 0.25)
        elif op == "beam":
            c.update(S=4 * log_uniform(1, 16), L=log_uniform(2, 32), n=log_uniform(10, 4000))
        elif op == "accept":
            c.update(L=log_uniform(2, 32), n=log_uniform(2, 400), T=log_uniform(2, 64))
        else:
            c.update(L=log_uniform(2, 32), n=log_uniform(2, 4096))
        w = work(c)
        pool = 4.0 * _pages(c) * c["B"] * c["L"] * c["H"] * c["d"]
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS and pool <= _MOST_STATE:
            return c


# ---- shapes of a case ---------------------------------------------------------------------------------------------

_BEAMS = 4  # beams of a prompt


def _contexts(c):
    """Rows of each session before a call: by the case alone, so that every seed does the same work."""
    if c["op"] == "beam":
        return [c["n"]] * c["S"]
    return [max(1, c["n"] * (i + 1) // c["S"]) if c["ragged"] else c["n"] for i in range(c["S"])]


def _nodes(c):
    """Nodes of each session's tree."""
    half = c["T"] // 2 + 1
    return [c["T"] - (7 * i) % half if c["ragged"] else c["T"] for i in range(c["S"])]


def _accepted(c):
    return [max(1, t // 4) for t in _nodes(c)]


def _pages_of(rows, B):
    return -(-rows // B)


def _slots(c):
    """Width of the table."""
    return _pages_of(c["n"] + c["T"], c["B"]) + 1


def _pages(c):
    """Pages of the pool."""
    ctx, nodes = _contexts(c), _nodes(c)
    if c["op"] == "beam":  # each prompt's pages once, and of every beam a tail of its own, and one to come
        return (c["S"] // _BEAMS) * _pages_of(c["n"], c["B"]) + 3 * c["S"]
    used = sum(_pages_of(r + (t if c["op"] in ("attend", "accept") else 0), c["B"]) for r, t in zip(ctx, nodes))
    return 2 * used if c["op"] == "compact" else used + 3


def work(case):
    c = {**_BASE, **case}
    ctx, nodes = _contexts(c), _nodes(c)
    row = 2 * 2 * c["L"] * c["H"] * c["d"]  # bytes of a row's K and V in all layers
    if c["op"] == "attend":
        q_rows = sum(nodes) * c["H"] * c["G"]
        rows = sum(r + t for r, t in zip(ctx, nodes))
        return {"bytes": row * rows + q_rows * (2 * 2 * c["d"] + 4),
                "flops": 4.0 * c["d"] * c["H"] * c["G"] * sum(t * (r + t) for r, t in zip(ctx, nodes))}
    table = 4 * c["S"] * _slots(c)
    if c["op"] == "beam":  # of the two children of a beam, one copies the rows of a tail page that is begun
        return {"bytes": 2 * table + 4 * _pages(c) + 2 * row * (c["S"] + (c["S"] // 2) * (c["n"] % c["B"])), "flops": 0.0}
    if c["op"] == "accept":
        return {"bytes": 2 * row * (sum(nodes) + sum(_accepted(c))), "flops": 0.0}
    used = sum(_pages_of(r, c["B"]) for r in ctx)
    if c["op"] == "compact":  # half of the pages in use lie in the pool's upper half
        return {"bytes": 2 * table + 8 * _pages(c) + row * c["B"] * used, "flops": 0.0}
    return {"bytes": 2 * row * sum(ctx), "flops": 0.0}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _pool(c, gen):
    """K and V pages.  Keys have a few strong channels, as those of a model have."""
    shape = (_pages(c), c["L"], c["H"], c["B"], c["d"])
    dt = _DTYPES[c["dtype"]]
    k = torch.randn(shape, generator=gen, device="cuda", dtype=dt)
    k[..., : c["d"] // 16] *= 3
    return k, torch.randn(shape, generator=gen, device="cuda", dtype=dt)


def _tree(rng, t):
    """Parents of t drafted nodes: the first ones are the context's children, the others hang on earlier nodes."""
    return [-1 if i < max(1, t // 8) else rng.randrange(max(0, i - 12), i) for i in range(t)]


def _path(rng, t, m):
    return sorted(rng.sample(range(t), m))


def prepare(case, seed):
    c = {**_BASE, **case}
    rng = random.Random(seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    S, L, H, G, d, B, op = (c[x] for x in ("S", "L", "H", "G", "d", "B", "op"))
    ctx, nodes, P, M, dt = _contexts(c), _nodes(c), _pages(c), _slots(c), _DTYPES[c["dtype"]]
    order = rng.sample(range(S), S) if op not in ("beam", "restore") else list(range(S))
    ctx, nodes, taken = ([v[i] for i in order] for v in (ctx, nodes, _accepted(c)))
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    offsets = lambda v: ints([sum(v[:i]) for i in range(len(v) + 1)])  # noqa: E731
    k, v = _pool(c, gen)
    st = {"case": c, "k": k, "v": v}

    free = list(range(P))
    if op == "compact":  # pages in use all over the pool, as many in its upper half as in its lower one
        used = P // 2
        free = rng.sample(range(P // 2), used - used // 2) + rng.sample(range(P // 2, P), used // 2)
    rng.shuffle(free)
    table, lens = [], []
    if op == "beam":
        for s in range(S):
            if s % _BEAMS == 0:
                prompt = [free.pop() for _ in range(_pages_of(c["n"], B))]
            table.append(prompt[:-1] + [free.pop()] if c["n"] % B else list(prompt))
            lens.append(c["n"])
    else:
        for s in range(S):
            lens.append(ctx[s] + (nodes[s] if op in ("attend", "accept") else 0))
            table.append([free.pop() for _ in range(_pages_of(lens[s], B))])
    refs = [0] * P
    for row in table:
        for page in row:
            refs[page] += 1
    flat = [p for row in table for p in row + [-1] * (M - len(row))]
    meta = ints(lens + flat + refs)  # lengths, table and reference counts in one piece: put back by one copy
    st["start"], st["meta"] = meta, meta.clone()
    st["lens"] = st["meta"][:S]
    st["table"] = st["meta"][S:S + S * M].view(S, M)
    st["refs"] = st["meta"][S + S * M:]

    if op == "attend":
        st["off"] = offsets(nodes)
        st["q"] = torch.randn((sum(nodes), H * G, d), generator=gen, device="cuda", dtype=dt) * 1.5
        st["parents"] = ints([p for t in nodes for p in _tree(rng, t)]) if c["T"] > 1 and not c["chain"] else None
    elif op == "beam":
        src = []  # half of each prompt's beams go on, with two children each
        for g in range(0, S, _BEAMS):
            src += [g + b for b in sorted(rng.sample(range(_BEAMS), _BEAMS // 2)) for _ in range(2)]
        st["src"], st["grow"], st["off"] = ints(src), ints([1] * S), offsets([1] * S)
    elif op == "accept":
        st["off"], st["path_off"] = offsets(nodes), offsets(taken)
        st["path"] = ints([x for t, m in zip(nodes, taken) for x in _path(rng, t, m)])
    if op in ("beam", "accept"):
        rows = S if op == "beam" else sum(nodes)
        st["new_k"], st["new_v"] = (torch.randn((rows, L, H, d), generator=gen, device="cuda", dtype=dt) for _ in range(2))
    elif op == "restore":
        st["off"] = offsets(ctx)
        st["new_k"], st["new_v"] = (torch.randn((S, L, H, c["n"], d), generator=gen, device="cuda", dtype=dt) for _ in range(2))
    elif op == "evict":
        st["off"] = offsets(ctx)
        st["out_k"], st["out_v"] = (torch.zeros((sum(ctx), L, H, d), device="cuda", dtype=dt) for _ in range(2))
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state)


def _run_own(st):
    cache = st.get("cache")
    if cache is None:  # the handle that a user's program makes once for its buffers
        from paper_2604_15356_amd.paged import PagedKVCache
        cache = st["cache"] = PagedKVCache(st["k"], st["v"], st["table"], st["lens"], st["refs"])
    c = st["case"]
    op = c["op"]
    if op == "attend":
        return cache.attend(st["q"], st["off"], parents=st["parents"], max_nodes=c["T"], max_len=c["n"] + c["T"])
    if op == "evict":
        cache.load(st["out_k"], st["out_v"], st["off"])
        return st["out_k"], st["out_v"]
    if op == "restore":
        cache.store(st["new_k"], st["new_v"], st["off"])
        return st["k"], st["v"]
    st["meta"].copy_(st["start"])
    if op == "beam":
        cache.fork(st["src"])
        cache.extend(st["grow"])
        cache.store(st["new_k"], st["new_v"], st["off"])
    elif op == "accept":
        cache.store(st["new_k"], st["new_v"], st["off"])
        cache.accept(st["off"], st["path"], st["path_off"])
    else:
        cache.compact()
    return st["k"], st["v"], st["table"], st["lens"], st["refs"]


def _session_of(off, rows):
    """Of packed rows: the session, and the row's number in it."""
    x = torch.arange(rows, device=off.device)
    s = torch.searchsorted(off[1:].contiguous(), x.to(torch.int32), right=True)
    return s, x - off.long()[s]


def _place(st, s, pos):
    """Page and row of position `pos` of session `s`."""
    B = st["case"]["B"]
    return st["table"].long()[s, pos // B], pos % B


def _plain_attend(st):
    c = st["case"]
    S, H, G, d, B = (c[x] for x in ("S", "H", "G", "d", "B"))
    q, off, T = st["q"], st["off"].long(), c["T"]
    N, M = q.shape[0], st["table"].shape[1]
    counts, lens = off[1:] - off[:-1], st["lens"].long()
    ctx = lens - counts
    pages = st["table"].long().clamp(min=0)
    rows = lambda x: x[pages, 0].float().permute(0, 2, 1, 3, 4).reshape(S, H, M * B, d)  # noqa: E731
    k, v = rows(st["k"]), rows(st["v"])
    s, i = _session_of(st["off"], N)
    padded = torch.zeros((S, T, H * G, d), device=q.device)
    padded[s, i] = q.float()
    padded = padded.view(S, T, H, G, d).permute(0, 2, 1, 3, 4).reshape(S, H, T * G, d)
    # who is whose ancestor: powers of the relation "is, or is the child of"
    step = torch.zeros((S, T, T + 1), dtype=torch.float64, device=q.device)
    step[:, :, 1:] = torch.eye(T, dtype=torch.float64, device=q.device)
    step[s, i, i if st["parents"] is None else st["parents"].long() + 1] = 1
    sees = torch.matrix_power(step[:, :, 1:], T) > 0.5
    node = torch.arange(M * B, device=q.device) - ctx[:, None]  # [S, M B]: the position as a node's number
    in_tree = (node >= 0) & (node < counts[:, None])
    visible = torch.gather(sees, 2, node.clamp(0, T - 1)[:, None].expand(S, T, M * B)) & in_tree[:, None]
    visible |= (node < 0)[:, None]
    scores = torch.matmul(padded, k.transpose(2, 3)) / math.sqrt(d)
    scores.view(S, H, T, G, M * B).masked_fill_(~visible[:, None, :, None], -math.inf)
    top = scores.amax(3, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = scores.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, v) / total
    lse = (top + total.log())[..., 0]
    unpack = lambda x: x.reshape(S, H, T, G, -1).permute(0, 2, 1, 3, 4).reshape(S, T, H * G, -1)[s, i]  # noqa: E731
    return unpack(out).to(q.dtype), unpack(lse)[..., 0]


def _plain_put(st):
    """Rows into the last positions of their sessions."""
    s, i = _session_of(st["off"], st["new_k"].shape[0])
    counts = st["off"][1:] - st["off"][:-1]
    page, row = _place(st, s, (st["lens"] - counts).long()[s] + i)
    st["k"][page, :, :, row] = st["new_k"]
    st["v"][page, :, :, row] = st["new_v"]


def _plain_restore(st):
    new_k, new_v = st["new_k"], st["new_v"]
    s, i = torch.nonzero(torch.arange(new_k.shape[3], device=new_k.device)[None] < st["lens"][:, None], as_tuple=True)
    page, row = _place(st, s, i)
    st["k"][page, :, :, row] = new_k[s, :, :, i]
    st["v"][page, :, :, row] = new_v[s, :, :, i]
    return st["k"], st["v"]


def _plain_evict(st):
    s, i = _session_of(st["off"], st["out_k"].shape[0])
    page, row = _place(st, s, i)
    st["out_k"].copy_(st["k"][page, :, :, row])
    st["out_v"].copy_(st["v"][page, :, :, row])
    return st["out_k"], st["out_v"]


def _count_refs(st):
    """A page's references are the entries that name it."""
    entries = st["table"][st["table"] >= 0].long()
    st["refs"].copy_(torch.bincount(entries, minlength=st["refs"].shape[0]))


def _plain_beam(st):
    st["meta"].copy_(st["start"])
    B, src, table, lens = st["case"]["B"], st["src"].long(), st["table"], st["lens"]
    table.copy_(table[src])
    lens.copy_(lens[src])
    _count_refs(st)
    # room for `grow` rows: a tail page that others hold too is copied, unless they all leave it in this call
    S, M = table.shape
    each = torch.arange(S, device=table.device)
    length, grow = lens.long(), st["grow"].long()
    slot = length // B
    tail = table.long()[each, slot.clamp(max=M - 1)]
    begun = (length % B > 0) & (grow > 0)
    before = ((tail[:, None] == tail[None]) & begun[None] & (each[None] < each[:, None])).sum(1)
    copies = begun & (st["refs"].long()[tail.clamp(min=0)] - before > 1)
    first = torch.where(copies, slot, -(-length // B))
    need = -(-(length + grow) // B) - first
    start = torch.cumsum(need, 0) - need
    taken = torch.nonzero(st["refs"] == 0)[:, 0]
    s = torch.repeat_interleave(each, need)
    j = torch.arange(s.shape[0], device=s.device) - start[s]
    fresh = taken[: s.shape[0]]
    table[s, first[s] + j] = fresh.to(torch.int32)
    _count_refs(st)
    at = start[copies]
    rows = torch.arange(B, device=s.device)[None] < (length % B)[copies][:, None]
    which, row = torch.nonzero(rows, as_tuple=True)
    to, frm = fresh[at][which], tail[copies][which]
    st["k"][to, :, :, row] = st["k"][frm, :, :, row]
    st["v"][to, :, :, row] = st["v"][frm, :, :, row]
    lens.add_(st["grow"])
    _plain_put(st)
    return st["k"], st["v"], table, lens, st["refs"]


def _plain_accept(st):
    st["meta"].copy_(st["start"])
    _plain_put(st)
    B, table, lens = st["case"]["B"], st["table"], st["lens"]
    path_off = st["path_off"]
    s, r = _session_of(path_off, st["path"].shape[0])
    ctx = lens.long() - (st["off"][1:] - st["off"][:-1]).long()
    page, row = _place(st, s, ctx[s] + st["path"].long())
    k, v = st["k"][page, :, :, row], st["v"][page, :, :, row]
    page, row = _place(st, s, ctx[s] + r)
    st["k"][page, :, :, row] = k
    st["v"][page, :, :, row] = v
    lens.copy_(ctx + (path_off[1:] - path_off[:-1]))
    slots = torch.arange(table.shape[1], device=table.device)
    table.masked_fill_(slots[None] * B >= lens[:, None], -1)
    _count_refs(st)
    return st["k"], st["v"], table, lens, st["refs"]


def _plain_compact(st):
    st["meta"].copy_(st["start"])
    refs, table = st["refs"], st["table"]
    used = int((refs > 0).sum())
    frm = used + torch.nonzero(refs[used:] > 0)[:, 0]
    to = torch.nonzero(refs[:used] == 0)[:, 0]
    st["k"][to] = st["k"][frm]
    st["v"][to] = st["v"][frm]
    home = torch.arange(refs.shape[0], device=refs.device, dtype=torch.int32)
    home[frm] = to.to(torch.int32)
    table.copy_(torch.where(table >= 0, home[table.long().clamp(min=0)], table))
    _count_refs(st)
    return st["k"], st["v"], table, st["lens"], refs


_PLAIN = {"attend": _plain_attend, "beam": _plain_beam, "accept": _plain_accept, "compact": _plain_compact,
          "restore": _plain_restore, "evict": _plain_evict}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    """Attention session by session, node by node along its ancestors.  The other operators move values and count."""
    c = {**_BASE, **case}
    if c["op"] != "attend":
        return None
    st = prepare(case, seed)
    H, G, d, B = (c[x] for x in ("H", "G", "d", "B"))
    off, lens, table = st["off"].tolist(), st["lens"].tolist(), st["table"].tolist()
    parents = st["parents"].tolist() if st["parents"] is not None else [i - 1 for s in range(c["S"]) for i in range(off[s + 1] - off[s])]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["q"].shape[:2], dtype=torch.float64, device="cuda")
    for s in range(c["S"]):
        t, n = off[s + 1] - off[s], lens[s]
        pages = table[s][: _pages_of(n, B)]
        k, v = (torch.cat([x[p, 0] for p in pages], dim=1)[:, :n].double() for x in (st["k"], st["v"]))
        hidden = torch.ones((t, n), dtype=torch.bool)
        hidden[:, : n - t] = False
        for i in range(t):
            a = i
            while a >= 0:
                hidden[i, n - t + a] = False
                a = parents[off[s] + a]
        q = st["q"][off[s]: off[s + 1]].double()
        for h in range(H):
            rows = q[:, h * G: (h + 1) * G].reshape(t * G, d)
            score = (rows @ k[h].T) * d ** -0.5
            score[hidden.to("cuda").repeat_interleave(G, 0)] = -math.inf
            total = torch.logsumexp(score, 1)
            out[off[s]: off[s + 1], h * G: (h + 1) * G] = ((score - total[:, None]).exp() @ v[h]).view(t, G, d)
            lse[off[s]: off[s + 1], h * G: (h + 1) * G] = total.view(t, G)
    return out, lse
