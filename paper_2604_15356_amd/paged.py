"""A live KV cache in pages, and the attention that reads it: buffer management around the plc_pages_* calls and
plc_attend, as codec.py is around the coding path.

A cache that codec.py has decoded is put to work here: `store` takes the decoder's [S, L, H, n, d], `fork` lets sessions go
on from each other's prefix (what PrefixTrie.best_match found, the beams of a search), `extend` makes room for the tokens of
a step or for a tree of drafted ones, `store_rotated` turns their keys and queries to their positions, `attend` computes their
attention, `accept` keeps the verified nodes, `add_weights` and `evict` keep a cache that may not grow to the positions that attention goes to,
and `load` gives the rows back for the encoder.  Everything works in place, in the order of the current stream, without synchronising;
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
        self._weights_known = None
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

    def store_rotated(self, k, v, off, rotary, q=None, base=None, rel=None, layer=0, q_out=None):
        """`store`, with the keys rotated (rotary.Rotary), and with packed rows the queries q [rows, H*G, d] too: returns them,
        in q_out, which may be q.  Row i of session s is at position base[s] + rel[row] (int32; default: the positions that the
        cache has, and i; a tree's nodes: their depths; a cache that was thinned out: what its session has seen)."""
        k, v, layer = self._rows(k, v, layer)
        if rotary.d != self.d:
            raise ValueError(f"a rotation of {rotary.d} components, rows of {self.d}")
        if rotary.turns.device != self.device:
            raise ValueError("the rotation is on another device than the cache")
        if q is not None and q_out is None:
            q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        plc.plc_rotate_store(self.pages, rotary.rotary, self._per_session(off, self.S + 1, "off"), base, rel, k, v, layer, q,
                             q_out if q is not None else None, self.status)
        return q_out if q is not None else None

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

    # -- what positions have received, and eviction by it ---------------------------------------
    def make_weights(self):
        """Zeros for all that positions receive: float32 [S, L, H, positions].  They are the caller's, and nothing but add_weights and evict changes
        them.  Sessions that are forked take theirs along by weights.copy_(weights[src]).  Where rows come to positions n0 and up without
        add_weights (a prefix that is restored, a prompt of which only the last rows are counted, a session's place given to another), what others had received
        there would count for them: weights[s, :, :, n0:] = 0 first."""
        return torch.zeros((self.S, self.L, self.H, self.M * self.B), dtype=torch.float32, device=self.device)

    def _weights(self, w):
        layout = w.shape, w.stride(), w.dtype, w.device
        if self._weights_known is None or self._weights_known[0] != layout:
            if w.device != self.device:
                raise ValueError("the weights are on another device than the cache")
            view = plc.make_weights(self.pages, w)
            self._weights_known = layout, view.stride, view.width
        return plc.plc_weights(w.data_ptr(), *self._weights_known[1:])

    def add_weights(self, q, off, lse, weights, decay=1.0, layer=0, scale=None, max_nodes=None, max_len=None):
        """Adds to weights (make_weights) what `layer`'s positions receive from the sessions' last off[s+1] - off[s] positions, a
        chain: q [N, H*G, d] and lse [N, H*G] as for attend and from it, so many times what was there before (`decay`; the call's own
        positions begin with nothing, others with what is in their places: see make_weights).  Of a drafted tree only what was accepted counts: call it after `accept`, with those rows.
        max_nodes, max_len as for attend; of single tokens of many sessions max_nodes=1 is worth saying, as N sets the launch without."""
        if q.dim() != 3 or q.dtype is not self.dtype:
            raise ValueError(f"q is [nodes, heads, d] of {self.dtype}")
        N = q.shape[0]
        self._per_session(off, self.S + 1, "off")
        view = self._weights(weights)
        if N == 0:
            return
        plc.plc_attend_weights(self.pages, layer, q, off, N if max_nodes is None else max_nodes,
                               self.M * self.B if max_len is None else max_len, self.d ** -0.5 if scale is None else scale, lse,
                               decay, view, self.status)

    def evict(self, keep, weights, kept=None, first=0, last=0, max_len=None):
        """Every session of more than keep[s] positions (int32 [S]) is shortened to that, in each layer and head to its first and
        last positions and those with the largest weights, which move along.  Returns kept, int32 [S, L, H, W]: the positions
        that stayed, in front; W is at least what a session has afterwards (default: max_len), and the launch goes by it.  The pages from position `first` on have to be
        the sessions' own: what others share can stay as the first positions.  A row is another position in each layer and head then (store_rotated
        has one for all): what `load` gives goes back to where it was rotated from, and there again, as rows of one head, rotary.rotate(k.view(-1, 1, d),
        positions), by the positions that `kept` names.  max_len: no session has more (default: what the table holds)."""
        self._per_session(keep, self.S, "keep")
        max_len = self.M * self.B if max_len is None else max_len
        if kept is None:
            kept = torch.empty((self.S, self.L, self.H, max_len), dtype=torch.int32, device=self.device)
        plc.plc_pages_evict(self.pages, keep, first, last, self._weights(weights), kept, max_len, self.ws, self.status)
        return kept

    def check_status(self, where="plc_pages"):
        """Synchronises and raises if a kernel reported a data-dependent error."""
        code = int(self.status.item())
        if code != plc.PLC_OK:
            self.status.zero_()
            raise plc.PlcError(code, where)
