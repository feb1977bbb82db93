"""The example's speculative decoding against the toy model's own definition, computed in 64 bits over whole sequences."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def definition(model, said):
    """Logits after each token, without a cache."""
    import speculative_decoding as ex
    tokens = torch.tensor(said, device="cuda")
    n = len(said)
    x = model.embed(tokens, torch.arange(n, device="cuda")).double()
    later = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
    for layer in range(ex.L):
        q, k, v = (x @ w[layer].double() for w in (model.wq, model.wk, model.wv))
        out = torch.empty_like(q)
        for h in range(ex.H * ex.G):
            one, kv = slice(h * ex.D, (h + 1) * ex.D), slice(h // ex.G * ex.D, (h // ex.G + 1) * ex.D)
            score = (q[:, one] @ k[:, kv].T / ex.D ** 0.5).masked_fill(later, -torch.inf)
            out[:, one] = torch.softmax(score, 1) @ v[:, kv]
        x = x + out @ model.wo[layer].double()
    return (x @ model.tokens.double().T).scatter(1, tokens[:, None], -1e9)


@pytest.mark.parametrize("sessions,seed", [(1, 0), (4, 1), (3, 2)])
def test_every_token_is_the_models_own(sessions, seed):
    """The tokens that were said are those of the largest logit, but for what rounding to 16 bits (2^-11 of a row, in two
    layers' queries, keys, values and outputs) and the codec's step of 0.002 may shift: a few thousandths of the logits' size,
    allowed 2 %."""
    import speculative_decoding as ex
    steps = 10
    model, cache, prompts, said, lens = ex.run(sessions, steps, seed=seed, quiet=True)
    assert cache.lens.tolist() == lens == [len(s) - 1 for s in said]
    for prompt, s in zip(prompts, said):
        assert len(s) >= len(prompt) + steps and s[: len(prompt)] == prompt.tolist()
        logits = definition(model, s)[len(prompt) - 1: -1]
        chosen = torch.tensor(s[len(prompt):], device="cuda")
        best = logits.amax(1)
        assert bool((logits.gather(1, chosen[:, None])[:, 0] >= best - 0.02 * best.abs()).all())
    # no page is lost: what the tables name is in use, as often as it is named
    named = cache.table[cache.table >= 0].long()
    assert torch.equal(torch.bincount(named, minlength=cache.P).int(), cache.refs)
    assert all(int((row >= 0).sum()) == -(-n // cache.B) for row, n in zip(cache.table, lens))
