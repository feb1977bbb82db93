"""A live KV cache in pages, and the attention that reads it: buffer management around the plc_pages_* calls and
plc_attend, as codec.py is around the coding path.

A cache that codec.py has decoded is put to work here: `store` takes the decoder's [S, L, H, n, d], `fork` lets sessions go
on from each other's prefix (what PrefixTrie.best_match found, the beams of a search), `extend` makes room for the tokens of
a step or for a tree of drafted ones, `attend` computes their attention, `accept` keeps the verified nodes, and `load` gives
the rows back for the encoder.  Everything works in place, in the order of the current stream, without synchronising;
errors in the data show in `check_status`.  A cache is used from one stream at a time: its workspaces are its own.
examples/speculative_decoding.py has all of it in a serving loop."""
from __future__ import annotations

import torch

from . import plc


class PagedKVCache:
    """Over buffers of the caller's: k, v [P, L, H, B, d] (pages, layers, KV heads, rows of a page, components; fp16 or
    bf16), table int32 [S, M] (pages of each session, -1 behind them), lens int32 [S], refs int32 [P] (entries that name
    each page).  `create` makes them, empty.

    The host does not know the sessions' lengths; where a call's launch depends on them (`attend`), `max_len` bounds them."""

    def __init__(self, k, v, table, lens, refs):
        self.k, self.v, self.table, self.lens, self.refs = k, v, table, lens, refs
        self.device, self.dtype = k.device, k.dtype
        self.pages = plc.make_pages(k, v, table, lens, refs)
        self.P, self.L, self.H, self.B, self.d = k.shape
        self.S, self.M = table.shape
        ws_bytes = plc.plc_pages_workspace_bytes(self.pages)
        if ws_bytes == 0:
            raise plc.PlcError(plc.PLC_ERR_INVALID, "plc_pages_workspace_bytes")
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.used = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._attend_need = {}
        self._attend_ws = [torch.empty(256, dtype=torch.uint8, device=self.device)]

    @classmethod
    def create(cls, P, L, H, d, S, max_len, B=16, dtype=torch.float16, device="cuda"):
        """An empty cache of P pages of B rows for S sessions of up to max_len positions."""
        k, v = (torch.zeros((P, L, H, B, d), dtype=dtype, device=device) for _ in range(2))
        return cls(k, v, torch.full((S, -(-max_len // B)), -1, dtype=torch.int32, device=device),
                   torch.zeros(S, dtype=torch.int32, device=device), torch.zeros(P, dtype=torch.int32, device=device))

    def _per_session(self, t, n, what):
        if t.dim() != 1 or t.numel() != n:
            raise ValueError(f"{what} has {n} entries")
        return t

    # -- pages ----------------------------------------------------------------------------
    def fork(self, src):
        """Session s becomes what session src[s] was (int32 [S]; -1: empty).  Pages are shared."""
        plc.plc_pages_fork(self.pages, self._per_session(src, self.S, "src"), self.status)

    def extend(self, grow):
        """Room for grow[s] more positions (int32 [S]); nobody else holds the pages that they lie on."""
        plc.plc_pages_extend(self.pages, self._per_session(grow, self.S, "grow"), self.ws, self.status)

    def trim(self, new_lens):
        """Keeps the first new_lens[s] positions (int32 [S])."""
        plc.plc_pages_trim(self.pages, self._per_session(new_lens, self.S, "new_lens"), self.status)

    def accept(self, off, path, path_off):
        """Of the drafted nodes, the sessions' last off[s+1] - off[s] positions, keeps the numbers
        path[path_off[s] : path_off[s+1]], ascending (int32)."""
        if path.dim() != 1:
            raise ValueError("path is a list of node numbers")
        plc.plc_pages_accept(self.pages, self._per_session(off, self.S + 1, "off"), path,
                             self._per_session(path_off, self.S + 1, "path_off"), self.status)

    def compact(self):
        """Moves the pages in use to the pool's front; their number, int32 [1], on the device, until the
        next call of it."""
        plc.plc_pages_compact(self.pages, self.used, self.ws, self.status)
        return self.used

    # -- rows -------------------------------------------------------------------------------
    def _rows(self, k, v, layer):
        if k.dim() == 3:  # [rows, H, d]: a single layer's
            k, v = k.unsqueeze(1), v.unsqueeze(1)
        if k.dtype is not self.dtype or v.dtype is not self.dtype:
            raise TypeError(f"expected {self.dtype}, got {k.dtype} and {v.dtype}")
        return k, v, layer

    def store(self, k, v, off, layer=0):
        """Rows into the last off[s+1] - off[s] positions of each session, layers `layer` and up."""
        k, v, layer = self._rows(k, v, layer)
        plc.plc_pages_store(self.pages, self._per_session(off, self.S + 1, "off"), k, v, layer, self.status)

    def load(self, k, v, off, layer=0):
        """The same rows, into k and v."""
        k, v, layer = self._rows(k, v, layer)
        plc.plc_pages_load(self.pages, self._per_session(off, self.S + 1, "off"), k, v, layer, self.status)

    # -- attention ----------------------------------------------------------------------------
    def reserve(self, G, N, max_nodes, max_len=None):
        """Workspace for attend calls of this size, so that none is made during them (under graph capture).  What was
        handed out before stays, for work in flight and for graphs."""
        max_len = self.M * self.B if max_len is None else max_len
        need = self._attend_need.get((G, N, max_nodes, max_len))
        if need is None:
            need = plc.plc_attend_workspace_bytes(self.pages, G, N, max_nodes, max_len)
            if need == 0:
                raise plc.PlcError(plc.PLC_ERR_INVALID, "plc_attend_workspace_bytes")
            if len(self._attend_need) >= 1024:
                self._attend_need.clear()
            self._attend_need[G, N, max_nodes, max_len] = need
        if need > self._attend_ws[-1].numel():
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("reserve the attention's workspace before the capture")
            self._attend_ws.append(torch.empty(max(need, 2 * self._attend_ws[-1].numel()), dtype=torch.uint8,
                                               device=self.device))
        return self._attend_ws[-1]

    def attend(self, q, off, parents=None, layer=0, scale=None, max_nodes=None, max_len=None, out=None, lse=None):
        """Attention of the sessions' last off[s+1] - off[s] positions, q [N, H*G, d], over all that they see, in one
        layer: a tree with `parents` (int32 [N], numbers within the tree, -1: continues the cache), a chain without.
        Returns out [N, H*G, d] and lse float32 [N, H*G].  No session has more than max_nodes nodes (default: N; of a tree at most
        plc.TREE_NODES) and max_len positions (default: what the table holds).  scale: 1/sqrt(d) by default."""
        if q.dim() != 3 or q.dtype is not self.dtype:
            raise ValueError(f"q is [nodes, heads, d] of {self.dtype}")
        N, heads, _ = q.shape
        self._per_session(off, self.S + 1, "off")
        if parents is not None:
            self._per_session(parents, N, "parents")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        if lse is None:
            lse = torch.empty(N, heads, dtype=torch.float32, device=self.device)
        elif lse.shape != (N, heads):
            raise ValueError("lse is [nodes, heads]")
        if N == 0:
            return out, lse
        if max_nodes is None:
            max_nodes = N if parents is None else min(N, plc.TREE_NODES)
        if max_len is None:
            max_len = self.M * self.B
        ws = self.reserve(heads // self.H, N, max_nodes, max_len)
        plc.plc_attend(self.pages, layer, q, off, parents, max_nodes, max_len, self.d ** -0.5 if scale is None else scale, out,
                       lse, ws, self.status)
        return out, lse

    def check_status(self, where="plc_pages"):
        """Synchronises and raises if a kernel reported a data-dependent error."""
        code = int(self.status.item())
        if code != plc.PLC_OK:
            self.status.zero_()
            raise plc.PlcError(code, where)
