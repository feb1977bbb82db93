"""A coded cache put to work: a prompt's KV rows are stored coded, decoded into pages, shared by the sessions that start with
the same tokens, and grown by speculative decoding with trees of drafted tokens.

    python examples/speculative_decoding.py [--steps 12] [--sessions 4]

The model is a toy with random weights (two layers of grouped-query attention, no feed-forward part); every call of the cache
and of the codec is the one that a real model's serving loop makes.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_15356_amd.codec import KVDeltaCodec  # noqa: E402
from paper_2604_15356_amd.paged import PagedKVCache  # noqa: E402
from paper_2604_15356_amd.plc import PrefixTrie  # noqa: E402

L, H, G, D, WIDTH, VOCAB, MAX_LEN = 2, 2, 4, 64, 256, 512, 512
CANDIDATES, DELTA = 4, 0.002


class Toy:
    """x = embedding of token and position; x += attention(x) Wo, layer after layer; logits = x embedding^T."""

    def __init__(self, device, seed=0):
        gen = torch.Generator(device).manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=gen, device=device)  # noqa: E731
        self.tokens, self.positions = randn(VOCAB, WIDTH), 0.5 * randn(MAX_LEN, WIDTH)
        self.wq = [randn(WIDTH, H * G * D) / WIDTH ** 0.5 for _ in range(L)]
        self.wk, self.wv = ([randn(WIDTH, H * D) / WIDTH ** 0.5 for _ in range(L)] for _ in range(2))
        self.wo = [0.4 * randn(H * G * D, WIDTH) / (H * G * D) ** 0.5 for _ in range(L)]
        # what the drafts are taken from: the two tokens that the model would say next without attention
        self.follow = (self.tokens @ self.tokens.T - 1e9 * torch.eye(VOCAB, device=device)).topk(2).indices

    def embed(self, tokens, positions):
        return self.tokens[tokens] + self.positions[positions]

    def logits(self, x, tokens):
        out = x @ self.tokens.T
        return out.scatter(1, tokens[:, None], -1e9)  # it does not repeat itself


def forward(model, cache, tokens, positions, off, parents=None, max_nodes=None):
    """Logits of the sessions' last positions, for which there is room in the cache: their rows go in, layer by layer."""
    x = model.embed(tokens, positions)
    rows = x.shape[0]
    for layer in range(L):
        k, v = ((x @ w[layer]).half().view(rows, H, D) for w in (model.wk, model.wv))
        cache.store(k, v, off, layer=layer)
        q = (x @ model.wq[layer]).half().view(rows, H * G, D)
        out, _ = cache.attend(q, off, parents=parents, layer=layer, max_nodes=max_nodes, max_len=MAX_LEN)
        x = x + out.view(rows, H * G * D).float() @ model.wo[layer]
    return model.logits(x, tokens)


def through_the_codec(k, v):
    """What a cache is after it was stored in coded form.  The candidates stand for what a model expects the rows to be."""
    S, _, _, n, _ = k.shape
    codec = KVDeltaCodec(S, L, H, n, CANDIDATES, D, DELTA, device=k.device)
    cand_k, cand_v = ((x[:, :, :, :, None] + 0.05 * torch.randn((S, L, H, n, CANDIDATES, D), device=x.device)).half() for x in (k, v))
    probs = torch.full((S, n, CANDIDATES), 1.0 / CANDIDATES, device=k.device)
    coded = codec.encode(cand_k, cand_v, probs, k, v)
    out_k, out_v = torch.empty_like(k), torch.empty_like(v)
    codec.decode(cand_k, cand_v, probs, out_k, out_v)
    codec.check_status()
    return out_k, out_v, 16 * int(coded.n_words.sum()) / (2 * k.numel())


def drafted_tree(model, last):
    """Seven nodes for each session: the token that is certain, what may follow it (two), and what may follow those."""
    parents = [-1, 0, 0, 1, 1, 2, 2]
    first = model.follow[last]                       # [S, 2]
    second = model.follow[first].flatten(1)          # [S, 4]
    return torch.cat([last[:, None], first, second], 1), parents


def run(sessions=4, steps=12, device="cuda", seed=0, quiet=False):
    say = (lambda *a: None) if quiet else print
    torch.manual_seed(seed)
    rng = torch.Generator().manual_seed(seed)
    model = Toy(device, seed)
    ints = lambda x: torch.as_tensor(x, dtype=torch.int32, device=device)  # noqa: E731
    offsets = lambda counts: ints([sum(counts[:i]) for i in range(len(counts) + 1)])  # noqa: E731

    # prompts: all sessions begin like the first
    S, n = sessions, 120
    first = torch.randint(VOCAB, (n,), generator=rng)
    prompts = [first] + [torch.cat([first[: 100 - 7 * s], torch.randint(VOCAB, (5 + 3 * s,), generator=rng)]) for s in range(1, S)]
    cache = PagedKVCache.create(P=S * 40, L=L, H=H, d=D, S=S, max_len=MAX_LEN, device=device)

    # the first prompt, all but its last token, as one chain; its rows coded, decoded and put back
    counts = [n - 1] + [0] * (S - 1)
    off = offsets(counts)
    cache.extend(ints(counts))
    forward(model, cache, first[:-1].to(device), torch.arange(n - 1, device=device), off, max_nodes=n - 1)
    k, v = (torch.zeros((S, L, H, n - 1, D), dtype=torch.float16, device=device) for _ in range(2))
    cache.load(k, v, off)
    k[:1], v[:1], bits = through_the_codec(k[:1].contiguous(), v[:1].contiguous())
    cache.store(k, v, off)
    say(f"prompt of {n} tokens: {bits:.2f} coded bits a component")

    # the others share the pages of what they have in common with it
    trie = PrefixTrie()
    trie.insert(first[:-1].numpy(), 0)
    common = [n - 1] + [min(trie.best_match(p[:-1].numpy())[1], len(p) - 1) for p in prompts[1:]]
    cache.fork(ints([0] * S))
    cache.trim(ints(common))
    rest = [len(p) - 1 - c for p, c in zip(prompts, common)]
    cache.extend(ints(rest))
    tokens = torch.cat([p[c:-1] for p, c in zip(prompts, common)]).to(device)
    positions = torch.cat([torch.arange(c, len(p) - 1) for p, c in zip(prompts, common)]).to(device)
    forward(model, cache, tokens, positions, offsets(rest), max_nodes=max(rest))
    say("sessions begin with", common, "shared positions;", int((cache.refs > 0).sum()), "pages in use")

    # speculative decoding: a tree for each session, of which the path that the model itself would have taken stays
    said = [p.tolist() for p in prompts]
    lens = [len(p) - 1 for p in prompts]
    taken = 0
    for _ in range(steps):
        last = torch.tensor([s[-1] for s in said], device=device)
        nodes, parents = drafted_tree(model, last)
        t = nodes.shape[1]
        depth = torch.tensor([0, 1, 1, 2, 2, 2, 2], device=device)
        off = ints([t * s for s in range(S + 1)])
        cache.extend(ints([t] * S))
        positions = (torch.tensor(lens, device=device)[:, None] + depth).flatten()
        logits = forward(model, cache, nodes.flatten(), positions, off, parents=ints(parents * S), max_nodes=t)
        best = logits.argmax(1).view(S, t).tolist()
        drafted = nodes.tolist()
        paths = []
        for s in range(S):
            path = [0]
            while True:
                said[s].append(best[s][path[-1]])
                child = [i for i in range(t) if parents[i] == path[-1] and drafted[s][i] == said[s][-1]]
                if not child:
                    break
                path.append(child[0])
            paths.append(path)
            lens[s] += len(path)
        taken += sum(len(p) for p in paths)
        cache.accept(off, ints([x for p in paths for x in p]), offsets([len(p) for p in paths]))
    used = int(cache.compact())
    cache.check_status()
    say(f"{taken} tokens in {steps} steps of {S} sessions: {taken / steps / S:.2f} a step; {used} pages in use after compaction")
    return model, cache, prompts, said, lens


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=12)
    parser.add_argument("--sessions", type=int, default=4)
    args = parser.parse_args()
    run(args.sessions, args.steps)
