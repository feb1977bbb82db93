"""What the calls around a model's step (rotary positions, weights, eviction, scores) refuse on the host, before anything is
enqueued: no GPU is needed, and no pointer here is one.  And the angles of rotary positions, which are worked out there."""
import ctypes as C
import math
from fractions import Fraction

import pytest
import torch

from paper_2604_15356_amd import plc

P = C.c_void_p(4096)
ODD = C.c_void_p(4098)
BIG = 1 << 24
INF, NAN = float("inf"), float("nan")
INVALID = plc.PLC_ERR_INVALID


def pages(**over):
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


def rows(**over):
    r = plc.plc_rows()
    r.layer, r.layers, r.packed, r.rows = 0, 2, 1, 5
    r.stride = (C.c_int64 * 4)(0, 128, 64, 256)
    for name, value in over.items():
        if name.startswith("stride"):
            r.stride[int(name[6:])] = value
        else:
            setattr(r, name, value)
    return r


def two(a, b):
    return (C.c_int64 * 2)(a, b)


def rotary(**over):
    y = plc.plc_rotary(4096, 32, 0, 1.0)
    for name, value in over.items():
        setattr(y, name, value)
    return y


def weights(**over):
    w = plc.plc_weights(4096, (256, 128, 64), 64)
    for name, value in over.items():
        if name.startswith("stride"):
            w.stride[int(name[6:])] = value
        else:
            setattr(w, name, value)
    return w


def rotate(y=None, type=0, x=P, xs=(128, 64), n=5, heads=2, d=64, pos=P, inverse=0, out=ODD, os=(128, 64)):
    out = C.c_void_p(8192) if out is ODD else out
    return plc.lib().plc_rotate(C.byref(y or rotary()), type, x, two(*xs), n, heads, d, pos, inverse, out, two(*os), None)


ROTARIES = [dict(turns=None), dict(turns=4100), dict(r=0), dict(r=31), dict(r=66), dict(r=-2), dict(interleaved=2), dict(interleaved=-1),
            dict(magnitude=0.0), dict(magnitude=-1.0), dict(magnitude=NAN), dict(magnitude=INF), dict(magnitude=1e-45)]


@pytest.mark.parametrize("over", ROTARIES)
def test_rotations_that_are_refused(over):
    assert rotate(rotary(**over)) == INVALID
    assert store(y=rotary(**over)) == INVALID


@pytest.mark.parametrize("over", [
    dict(type=2), dict(type=-1), dict(x=None), dict(x=ODD), dict(x=C.c_void_p(4104)), dict(out=None), dict(out=C.c_void_p(8200)), dict(pos=None), dict(pos=ODD),
    dict(xs=(60, 64)), dict(xs=(-8, 64)), dict(os=(128, 4)), dict(n=-1), dict(n=1 << 31), dict(heads=0), dict(heads=1 << 26), dict(d=60), dict(d=2056),
    dict(inverse=2), dict(out=P, os=(256, 64)), dict(out=P, os=(128, 128)),
    dict(os=(0, 64)), dict(os=(128, 56))])
def test_rows_that_are_refused(over):
    assert rotate(**over) == INVALID


def test_no_rows_are_nothing_to_do():
    assert rotate(n=0, x=None, out=None, pos=None) == plc.PLC_OK
    assert store(r=rows(rows=0), k=None, v=None, q=None, qo=None) == plc.PLC_OK
    assert weigh(N=0, q=None, lse=None) == plc.PLC_OK
    assert score(N=0, logits=None) == plc.PLC_OK


def store(g=None, r=None, y=None, type=0, off=P, base=None, rel=None, k=P, v=P, q=P, qs=(256, 64), G=2, qo=C.c_void_p(8192), qos=(256, 64), status=P):
    return plc.lib().plc_rotate_store(C.byref(g or pages()), C.byref(r or rows()), C.byref(y or rotary()), type, off, base, rel, k, v, q, two(*qs), G, qo,
                                      two(*qos), status, None)


@pytest.mark.parametrize("over", [
    dict(g=pages(k=None)), dict(g=pages(B=8)), dict(g=pages(d=2056, stride3=2056)), dict(r=rows(layer=1)), dict(r=rows(layers=0)), dict(r=rows(packed=2)),
    dict(r=rows(rows=-1)), dict(r=rows(stride1=4)), dict(r=rows(packed=0)), dict(type=2), dict(off=None), dict(off=ODD), dict(base=ODD), dict(rel=ODD),
    dict(k=None), dict(v=ODD), dict(q=None), dict(qo=None), dict(q=C.c_void_p(4104)), dict(qo=ODD), dict(qs=(4, 64)), dict(qos=(256, -8)), dict(G=0),
    dict(G=1 << 29), dict(qo=P, qos=(512, 64)), dict(qos=(0, 64)), dict(qos=(256, 0)), dict(status=None)])
def test_stores_that_are_refused(over):
    assert store(**over) == INVALID


def weigh(g=None, layer=0, type=0, q=P, qs=(128, 64), G=1, N=5, off=P, max_nodes=5, max_len=64, scale=1.0, lse=P, decay=1.0, w=None, status=P):
    return plc.lib().plc_attend_weights(C.byref(g or pages()), layer, type, q, two(*qs), G, N, off, max_nodes, max_len, scale, lse, decay,
                                        C.byref(w or weights()), status, None)


WEIGHTS = [dict(w=None), dict(w=4104), dict(stride0=130), dict(stride1=0), dict(stride2=60), dict(stride0=-256), dict(width=0), dict(width=62), dict(width=68)]


@pytest.mark.parametrize("over", [
    dict(g=pages(k=None)), dict(g=pages(d=264, stride3=264)), dict(layer=-1), dict(layer=2), dict(type=2), dict(q=None), dict(q=C.c_void_p(4104)), dict(qs=(4, 64)),
    dict(qs=(128, -64)), dict(G=0), dict(G=1 << 15, g=pages(H=4)), dict(N=-1), dict(N=1 << 31), dict(off=None), dict(off=ODD), dict(max_nodes=0),
    dict(max_nodes=1 << 24), dict(max_len=0), dict(scale=0.0), dict(scale=NAN), dict(scale=INF), dict(lse=None), dict(lse=ODD), dict(decay=-0.1),
    dict(decay=1.1), dict(decay=NAN), dict(status=None)] + [dict(w=weights(**o)) for o in WEIGHTS])
def test_weighings_that_are_refused(over):
    assert weigh(**over) == INVALID


def test_scales_beyond_what_their_product_with_log2_e_holds_are_refused():
    """Of a score of 0 and an infinite scale a weight would be NaN."""
    assert weigh(scale=2.4e38) == INVALID and weigh(N=0, q=None, lse=None, scale=2.3e38) == plc.PLC_OK


# Each stride for itself is as large as what it steps over, and together they meet.
@pytest.mark.parametrize("over", [dict(stride0=128, stride1=128), dict(stride0=64, stride1=192), dict(stride0=128, stride1=256, stride2=256),
                                  dict(stride0=192, stride1=128), dict(stride0=1 << 62, stride1=64)])
def test_weights_that_lie_on_each_other_are_refused(over):
    assert weigh(w=weights(**over)) == INVALID
    assert evict(w=weights(**over)) == INVALID


@pytest.mark.parametrize("strides", [(64, 64), (128, 192), (192, 128), (64, 256)])
def test_outputs_that_lie_on_each_other_are_refused(strides):
    assert rotate(heads=3, os=strides) == INVALID
    assert store(qos=strides) == INVALID


def evict(g=None, keep=P, first=1, last=2, w=None, kept=P, W=30, max_len=64, ws=P, ws_bytes=BIG, status=P):
    return plc.lib().plc_pages_evict(C.byref(g or pages()), keep, first, last, C.byref(w or weights()), kept, W, max_len, ws, ws_bytes, status, None)


@pytest.mark.parametrize("over", [
    dict(g=pages(k=None)), dict(keep=None), dict(keep=ODD), dict(first=-1), dict(last=-1), dict(kept=None), dict(kept=ODD), dict(W=-1), dict(max_len=-1),
    dict(max_len=(1 << 30) + 1), dict(ws=None), dict(ws=C.c_void_p(4100)), dict(ws_bytes=100), dict(status=None),
    dict(g=pages(L=1 << 11, H=1 << 11, d=8, S=1), w=weights(stride1=1 << 20))] + [dict(w=weights(**o)) for o in WEIGHTS])
def test_evictions_that_are_refused(over):
    assert evict(**over) == INVALID


def score(type=0, logits=P, stride=100, N=3, V=100, scale=1.0, tokens=P, k=4, logprob=P, entropy=P, lse=P, ids=P, top=P, probs=P, chosen=P, ws=P, ws_bytes=BIG,
          status=P):
    return plc.lib().plc_score_tokens(type, logits, stride, N, V, scale, tokens, k, logprob, entropy, lse, ids, top, probs, chosen, ws, ws_bytes, status, None)


@pytest.mark.parametrize("over", [
    dict(type=3), dict(type=-1), dict(logits=None), dict(logits=C.c_void_p(4097)), dict(type=2, logits=ODD), dict(stride=-1), dict(N=-1), dict(N=1 << 31),
    dict(V=0), dict(V=(1 << 30) + 1), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(scale=3e38), dict(tokens=ODD),
    dict(tokens=None), dict(tokens=None, logprob=None), dict(tokens=None, chosen=None), dict(k=-1), dict(k=33), dict(k=4, V=3), dict(k=0), dict(logprob=ODD),
    dict(entropy=ODD), dict(lse=ODD), dict(ids=ODD), dict(top=ODD), dict(probs=ODD), dict(chosen=ODD), dict(ws=None), dict(ws=C.c_void_p(4100)),
    dict(ws_bytes=100), dict(status=None)])
def test_scores_that_are_refused(over):
    assert score(**over) == INVALID


def test_sizes_of_scores():
    assert plc.plc_score_workspace_bytes(100, 4) > 0 and plc.plc_score_workspace_bytes(100, 4) % 256 == 0
    for V, k in ((0, 0), (100, 33), (3, 4), (100, -1), ((1 << 30) + 1, 0)):
        assert plc.plc_score_workspace_bytes(V, k) == 0


def test_tensors_that_are_refused():
    """On the host: the binding never takes a tensor for what it is not."""
    from paper_2604_15356_amd.scores import TokenScorer
    f = torch.zeros((3, 2, 64), dtype=torch.float16)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises((ValueError, AssertionError, RuntimeError)):
        plc.plc_rotate(rotary(), f, i, False, f)
    with pytest.raises((ValueError, AssertionError, RuntimeError)):
        plc.plc_score_tokens(f[0], 1.0, None, 0, None, None, None, None, None, None, None, i, i)
    w = torch.zeros((3, 2, 2, 64))
    with pytest.raises(ValueError):
        plc.make_weights(pages(), w[:2])
    with pytest.raises(ValueError):
        plc.make_weights(pages(), w.double())
    with pytest.raises(ValueError):
        plc.make_weights(pages(), w.transpose(2, 3))
    with pytest.raises(ValueError):
        plc.make_weights(pages(), w)  # not on a device
    for V, k in ((0, 0), (10, 33), (3, 4)):
        with pytest.raises(plc.PlcError):
            TokenScorer(V, k, device="cpu")
    scorer = TokenScorer(10, 2, device="cpu")
    for logits, kw in ((torch.zeros(2, 9), {}), (torch.zeros(2, 10), dict(tokens=i)), (torch.zeros(2, 10), dict(temperature=0.0)),
                       (torch.zeros(2, 10), dict(temperature=NAN))):
        with pytest.raises(ValueError):
            scorer.score(logits, **kw)


# ---- angles ------------------------------------------------------------------------------------------------------------------

def test_frequencies():
    """The formulas, in 64 bits: powers of the base are off by a few steps of 2^-53."""
    close = lambda a, b: all(abs(x - y) <= 1e-14 * abs(y) for x, y in zip(a, b)) and len(a) == len(b)  # noqa: E731
    r, base, f, trained = 20, 500000.0, 8.0, 4096
    plain = [base ** (-2 * i / r) for i in range(r // 2)]
    assert close(plc.plc_rotary_frequencies(r, base=base), plain)
    assert close(plc.plc_rotary_frequencies(r, "linear", base=base, factor=f), [t / f for t in plain])
    longer = base * f ** (r / (r - 2))
    assert close(plc.plc_rotary_frequencies(r, "stretched", base=base, factor=f), [longer ** (-2 * i / r) for i in range(r // 2)])
    assert plc.plc_rotary_frequencies(2, "stretched", base=base, factor=f) == [1.0]
    parts = []
    for t in plain:
        g = min(1.0, max(0.0, (trained * t / (2 * math.pi) - 1.0) / 3.0))
        parts.append(g * t + (1 - g) * t / f)
    got = plc.plc_rotary_frequencies(r, "parts", base=base, factor=f, low=1.0, high=4.0, trained=trained)
    assert close(got, parts) and got[0] == plain[0] and abs(got[-1] * f / plain[-1] - 1) < 1e-14
    at = lambda n: r * math.log(trained / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
    ramp = []
    for i, t in enumerate(plain):
        g = 1 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
        ramp.append(g * t + (1 - g) * t / f)
    assert 0 < lo < hi < r // 2
    assert close(plc.plc_rotary_frequencies(r, "ramp", base=base, factor=f, low=1.0, high=32.0, trained=trained), ramp)


@pytest.mark.parametrize("kw", [
    dict(r=0), dict(r=3), dict(r=-2), dict(r=2050), dict(r=8, base=0.0), dict(r=8, base=-1.0), dict(r=8, base=NAN), dict(r=8, base=INF),
    dict(r=8, scaling="linear", factor=0.0), dict(r=8, scaling="linear", factor=NAN), dict(r=8, scaling="parts", factor=8.0, low=0.0),
    dict(r=8, scaling="parts", factor=8.0, low=4.0, high=4.0), dict(r=8, scaling="parts", factor=8.0, trained=0), dict(r=8, scaling="ramp", factor=8.0, base=1.0, trained=10),
    dict(r=8, scaling="ramp", factor=8.0, high=INF, trained=10)])
def test_frequencies_that_are_refused(kw):
    with pytest.raises(plc.PlcError):
        plc.plc_rotary_frequencies(**kw)


def test_turns():
    """In whole numbers of 2^-64, against exact arithmetic; a 64-bit theta over 2 pi is held to 2^-64 of itself, by 64-bit fractions."""
    two_pi = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
    theta = [1.0, 0.0, 10000.0 ** -0.5, -1.0, 2 * math.pi, 1e-9, 123.456, 5e-324, 1e6]
    for t, u in zip(theta, plc.plc_rotary_turns(theta)):
        want = Fraction(t) / two_pi * 2 ** 64
        off = (u - want) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= 1 + abs(Fraction(t) / two_pi) * 2
    for bad in ([INF], [1.0, NAN]):
        with pytest.raises(plc.PlcError):
            plc.plc_rotary_turns(bad)
    with pytest.raises(plc.PlcError):
        plc.plc_rotary_turns([])
    with pytest.raises(ValueError):
        plc.plc_rotary_frequencies(8, "other")
