"""What the paged cache's calls refuse on the host, before anything is enqueued: no GPU is needed, and no pointer here is
one."""
import ctypes as C

import pytest
import torch

from paper_2604_15356_amd import plc

P = C.c_void_p(4096)
ODD = C.c_void_p(4098)


def _pages(**over):
    g = plc.plc_pages()
    g.k = g.v = 4096
    g.P, g.L, g.H, g.B, g.d, g.S, g.M = 10, 2, 2, 16, 64, 3, 4
    g.stride = (C.c_int64 * 4)(2 * 2 * 16 * 64, 2 * 16 * 64, 16 * 64, 64)
    g.table = g.lens = g.refs = 4096
    for name, value in over.items():
        if name.startswith("stride"):
            g.stride[int(name[6:])] = value
        else:
            setattr(g, name, value)
    return g


def _rows(**over):
    r = plc.plc_rows()
    r.layer, r.layers, r.packed, r.rows = 0, 2, 1, 5
    r.stride = (C.c_int64 * 4)(0, 128, 64, 256)
    for name, value in over.items():
        if name.startswith("stride"):
            r.stride[int(name[6:])] = value
        else:
            setattr(r, name, value)
    return r


BIG = 1 << 24


def _calls(g):
    L, b, r = plc.lib(), C.byref(g), C.byref(_rows())
    st = (C.c_int64 * 2)(8 * 64, 64)
    return [L.plc_pages_fork(b, P, P, None), L.plc_pages_extend(b, P, P, BIG, P, None), L.plc_pages_trim(b, P, P, None),
            L.plc_pages_accept(b, P, P, 5, P, P, None), L.plc_pages_compact(b, P, P, BIG, P, None),
            L.plc_pages_store(b, r, P, P, P, P, None), L.plc_pages_load(b, r, P, P, P, P, None),
            L.plc_attend(b, 0, 0, P, st, 2, 5, P, None, 5, 64, 1.0, P, st, P, P, BIG, P, None)]


@pytest.mark.parametrize("over", [
    dict(k=None), dict(v=4104), dict(table=None), dict(lens=4098), dict(refs=None), dict(P=0), dict(L=0), dict(H=-1),
    dict(B=8), dict(B=24), dict(B=2048), dict(d=0), dict(d=12), dict(S=0), dict(S=1025), dict(M=0), dict(M=1 << 27),
    dict(stride0=4), dict(stride1=-8), dict(stride2=12), dict(stride3=56), dict(stride3=1 << 27), dict(L=1 << 14, H=1 << 14)])
def test_descriptions_that_are_refused(over):
    g = _pages(**over)
    assert plc.plc_pages_workspace_bytes(g) == 0
    assert plc.plc_attend_workspace_bytes(g, 2, 5, 5, 64) == 0
    assert _calls(g) == [plc.PLC_ERR_INVALID] * 8
    assert plc.lib().plc_pages_fork(None, P, P, None) == plc.PLC_ERR_INVALID


def test_arguments_that_are_refused():
    L, g = plc.lib(), _pages()
    b, st = C.byref(g), (C.c_int64 * 2)(8 * 64, 64)
    assert plc.plc_pages_workspace_bytes(g) % 256 == 0 and plc.plc_pages_workspace_bytes(g) >= 4 * 3 * 10
    bad = plc.PLC_ERR_INVALID
    assert L.plc_pages_fork(b, None, P, None) == bad and L.plc_pages_fork(b, ODD, P, None) == bad
    assert L.plc_pages_fork(b, P, None, None) == bad
    assert L.plc_pages_extend(b, None, P, BIG, P, None) == bad
    assert L.plc_pages_extend(b, P, P, 16, P, None) == bad and L.plc_pages_extend(b, P, ODD, BIG, P, None) == bad
    assert L.plc_pages_extend(b, P, P, BIG, None, None) == bad
    assert L.plc_pages_trim(b, None, P, None) == bad and L.plc_pages_trim(b, P, None, None) == bad
    for hole in (1, 2, 4, 5):
        args = [b, P, P, 5, P, P, None]
        args[hole] = None
        assert L.plc_pages_accept(*args) == bad, hole
    assert L.plc_pages_accept(b, P, P, -1, P, P, None) == bad
    assert L.plc_pages_compact(b, P, P, 16, P, None) == bad and L.plc_pages_compact(b, P, None, BIG, P, None) == bad
    assert L.plc_pages_compact(b, P, P, BIG, None, None) == bad
    for call in (L.plc_pages_store, L.plc_pages_load):
        for over in (dict(layer=-1), dict(layer=1), dict(layers=0), dict(layers=3), dict(packed=2), dict(rows=-1),
                     dict(rows=1 << 31), dict(stride1=4), dict(stride2=-8), dict(stride3=1), dict(packed=0, stride0=4)):
            assert call(b, C.byref(_rows(**over)), P, P, P, P, None) == bad, over
        for hole in (1, 2, 3, 4, 5):
            args = [b, C.byref(_rows()), P, P, P, P, None]
            args[hole] = None
            assert call(*args) == bad, hole
        assert call(b, C.byref(_rows()), P, C.c_void_p(4104), P, P, None) == bad
        assert call(b, C.byref(_rows(rows=0)), P, P, P, P, None) == plc.PLC_OK  # nothing to move: nothing is enqueued

    def attend(**over):
        a = dict(pages=b, layer=0, type=0, q=P, qs=st, G=2, N=5, off=P, parents=None, nodes=5, len=64, scale=1.0, out=P, os=st,
                 lse=P, ws=P, bytes=BIG, status=P)
        a.update(over)
        return L.plc_attend(*a.values(), None)

    odd_strides = (C.c_int64 * 2)(8 * 64, 60)
    for over in (dict(layer=-1), dict(layer=2), dict(type=2), dict(q=None), dict(q=C.c_void_p(4104)), dict(qs=None),
                 dict(qs=odd_strides), dict(os=odd_strides), dict(os=None), dict(G=0), dict(G=1 << 16), dict(N=-1),
                 dict(N=1 << 31), dict(off=None), dict(off=ODD), dict(parents=ODD), dict(parents=P, nodes=257), dict(nodes=0),
                 dict(nodes=1 << 30), dict(len=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                 dict(scale=float("inf")), dict(out=None), dict(lse=ODD), dict(ws=None), dict(ws=C.c_void_p(4096 + 128)),
                 dict(len=1 << 20, bytes=256), dict(status=None)):
        assert attend(**over) == bad, over
    assert attend(N=0) == plc.PLC_OK
    assert L.plc_attend(C.byref(_pages(d=264, stride3=264)), 0, 0, P, st, 2, 5, P, None, 5, 64, 1.0, P, st, P, P, BIG, P,
                        None) == bad
    # the workspace: partial results of every chunk where positions are cut, and that not without end
    assert plc.plc_attend_workspace_bytes(_pages(), 2, 5, 5, 64) == 256
    assert plc.plc_attend_workspace_bytes(_pages(), 2, 5, 5, 1 << 20) >= 2 * 2 * 3 * 32 * 66 * 4
    for S in (1, 3, 64, 1024):
        for nodes in (1, 40, 256, 5000):
            n = plc.plc_attend_workspace_bytes(_pages(S=S), 2, S * nodes, nodes, 1 << 24)
            assert n % 256 == 0 and 256 <= n <= 2 * 131072 * 66 * 4
    assert plc.plc_attend_workspace_bytes(_pages(S=1024, H=1024), 2, 1 << 20, 1 << 20, 64) == 0  # tiles beyond 32 bits
    assert attend(pages=C.byref(_pages(S=1024, H=1024)), N=1 << 20, nodes=1 << 20, G=2) == bad


def test_tensors_that_the_binding_refuses():
    k = torch.zeros(4, 2, 2, 16, 64, dtype=torch.float16)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="device tensors"):
        plc.make_pages(k, k, ints(3, 2), ints(3), ints(4))
    for args in ((k, k[:, :1], ints(3, 2), ints(3), ints(4)), (k, k.transpose(3, 4), ints(3, 2), ints(3), ints(4)),
                 (k[0], k[0], ints(3, 2), ints(3), ints(4)), (k, k, ints(3, 2), ints(2), ints(4)),
                 (k, k, ints(3, 2), ints(3), ints(5))):
        with pytest.raises(ValueError):
            plc.make_pages(*args)
    with pytest.raises(TypeError):
        plc.make_pages(k.float(), k.float(), ints(3, 2), ints(3), ints(4))
    g, rows = _pages(), torch.zeros(5, 2, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        plc.plc_pages_store(g, ints(4), rows, rows[:4], 0, ints(1))
    with pytest.raises(ValueError):
        plc.plc_pages_load(g, ints(4), rows[0], rows[0], 0, ints(1))
    q = torch.zeros(5, 4, 64, dtype=torch.float16)
    for bad_q in (q[:, :3], q[:, :, :32], q.permute(0, 2, 1)):
        with pytest.raises(ValueError):
            plc.plc_attend(g, 0, bad_q, ints(4), None, 5, 64, 1.0, bad_q, None, ints(256), ints(1))
    with pytest.raises(TypeError):
        plc.plc_attend(g, 0, q.float(), ints(4), None, 5, 64, 1.0, q.float(), None, ints(256), ints(1))


class Elsewhere:
    """What the binding looks at of a tensor on device 1."""
    is_cuda, device = True, torch.device("cuda", 1)

    def __init__(self, dtype=torch.int32, shape=(4,)):
        self.dtype, self.shape = dtype, torch.Size(shape)
        self.stride = torch.empty(shape).stride

    is_contiguous = lambda self: True  # noqa: E731
    data_ptr = lambda self: 4096  # noqa: E731
    get_device = lambda self: 1  # noqa: E731
    numel = lambda self: self.shape.numel()  # noqa: E731


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The stream that a call takes is the current device's, as is the launch."""
    monkeypatch.setattr(plc, "_current_device", lambda: 0, raising=False)
    i, g = Elsewhere(), _pages()
    rows, q = Elsewhere(torch.float16, (5, 2, 2, 64)), Elsewhere(torch.float16, (5, 4, 64))
    ws = Elsewhere(torch.uint8, (1 << 20,))
    for call in (lambda: plc.plc_pages_fork(g, i, i), lambda: plc.plc_pages_extend(g, i, ws, i), lambda: plc.plc_pages_trim(g, i, i),
                 lambda: plc.plc_pages_accept(g, i, i, i, i), lambda: plc.plc_pages_compact(g, None, ws, i),
                 lambda: plc.plc_pages_store(g, i, rows, rows, 0, i), lambda: plc.plc_pages_load(g, i, rows, rows, 0, i),
                 lambda: plc.plc_attend(g, 0, q, i, None, 5, 64, 1.0, q, None, ws, i)):
        with pytest.raises(ValueError, match="current device"):
            call()
    k, ints = Elsewhere(torch.float16, (4, 2, 2, 16, 64)), lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    k.dim, table = lambda: 5, ints(3, 2)
    with pytest.raises(ValueError, match="one device"):
        plc.make_pages(k, k, table, ints(3), ints(4))


def test_rows_of_another_shape_or_type_than_the_pools_are_refused(monkeypatch):
    monkeypatch.setattr(plc, "_current_device", lambda: 0, raising=False)
    g, i = _pages(), Elsewhere()
    for shape in ((5, 2, 3, 64), (5, 2, 2, 72), (5, 2, 2, 32), (4, 2, 2, 5, 64), (3, 2, 4, 5, 64), (3, 2, 2, 5, 80), (5, 2, 64)):
        rows = Elsewhere(torch.float16, shape)
        for call in (plc.plc_pages_store, plc.plc_pages_load):
            with pytest.raises(ValueError, match="rows"):
                call(g, i, rows, rows, 0, i)
    rows = Elsewhere(torch.float32, (5, 2, 2, 64))
    for call in (plc.plc_pages_store, plc.plc_pages_load):
        with pytest.raises(TypeError):
            call(g, i, rows, rows, 0, i)
