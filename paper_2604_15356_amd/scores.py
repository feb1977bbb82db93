"""What a model's logits say of tokens: buffer management around plc_score_tokens.

`probs` and `chosen` are what the codec takes (KVDeltaCodec.encode, encode_cond), with logits of the positions' predictions
[S, n, V]; the log-probabilities, as surprisals, are what PrefixTrie.insert takes."""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import plc


class Scores(NamedTuple):
    """Of each row; ids, logprobs and probs have a last dimension of k alternatives, the most probable first."""
    logprob: Optional[torch.Tensor]   # float32: of the given token; 0 where that is -1; None without tokens
    entropy: torch.Tensor             # float32, nats
    lse: torch.Tensor                 # float32: the logarithm of the sum of exponentials
    ids: Optional[torch.Tensor]       # int32; None with k = 0, as what follows
    logprobs: Optional[torch.Tensor]  # float32
    probs: Optional[torch.Tensor]     # float32
    chosen: Optional[torch.Tensor]    # int32: the given token's place among the alternatives, or -1; None without tokens


class TokenScorer:
    """Over a vocabulary of V tokens, with k <= 32 alternatives.  Used from one stream at a time: its workspace is its own."""

    def __init__(self, V, k=0, device="cuda"):
        ws_bytes = plc.plc_score_workspace_bytes(V, k)
        if ws_bytes == 0:
            raise plc.PlcError(plc.PLC_ERR_INVALID, "plc_score_workspace_bytes")
        self.V, self.k = V, k
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def score(self, logits, tokens=None, temperature=1.0) -> Scores:
        """logits [..., V] (fp16, bf16 or fp32; rows evenly apart), divided by the temperature; tokens int32 [...], -1: none."""
        if logits.dim() < 1 or logits.shape[-1] != self.V:
            raise ValueError(f"logits are [..., {self.V}]")
        if tokens is not None and tokens.shape != logits.shape[:-1]:
            raise ValueError("tokens has a number for each row of logits")
        if not temperature > 0:
            raise ValueError("the temperature is positive")
        shape, k, device = logits.shape[:-1], self.k, self.status.device
        plc._on(logits.get_device(), self.status)
        rows = logits if logits.dim() == 2 else logits.view(-1, self.V) if logits.dim() > 2 else logits.unsqueeze(0)
        logprob = chosen = ids = logprobs = probs = None
        at_logprob = at_chosen = at_ids = at_logprobs = at_probs = None
        # (results of one shape out of one tensor: each that is made costs as much of the host's time as the kernel's launch half)
        sums = torch.empty((2 if tokens is None else 3, *shape), dtype=torch.float32, device=device)
        if tokens is None:
            entropy, lse = sums.unbind()
        else:
            entropy, lse, logprob = sums.unbind()
            at_logprob = logprob.data_ptr()
        if k:
            logprobs = torch.empty((*shape, k), dtype=torch.float32, device=device)
            probs = torch.empty_like(logprobs)
            ids = torch.empty((*shape, k), dtype=torch.int32, device=device)
            at_logprobs, at_probs, at_ids = logprobs.data_ptr(), probs.data_ptr(), ids.data_ptr()
            if tokens is not None:
                chosen = torch.empty_like(tokens)
                at_chosen = chosen.data_ptr()
        plc._score_tokens(rows, 1.0 / temperature, tokens, k, at_logprob, entropy.data_ptr(), lse.data_ptr(), at_ids, at_logprobs, at_probs,
                          at_chosen, self.ws.data_ptr(), self.ws.numel(), self.status.data_ptr())
        return Scores(logprob, entropy, lse, ids, logprobs, probs, chosen)

    def check_status(self, where="plc_score_tokens"):
        """Synchronises and raises if a row or a token was none."""
        code = int(self.status.item())
        if code != plc.PLC_OK:
            self.status.zero_()
            raise plc.PlcError(code, where)
