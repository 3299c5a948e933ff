"""CPU-side checks that the gated recurrence's results lie apart from its operands
and from one another, to the element.  No kernel is launched and no pointer is
followed."""
import ctypes

import pytest

F32, BF16 = 0, 1
BASE = 1 << 30
B, T, C = 3, 9, 8


def _lib():
    import paper_2211_06934_amd as P
    return P.diffopt._lib


def _error():
    import paper_2211_06934_amd as P
    return P.last_error()


def _seq(at, sb=T * C, st=C):
    import paper_2211_06934_amd as P
    return ctypes.byref(P.operators._Heads(BASE + at, sb, st, 0))


def far(i):
    return _seq(i << 20)


def block(at):
    return ctypes.c_void_p(BASE + at)


def _call(name, sizes=(B, T, C), dtype=F32, ws=None, nws=0, **change):
    """Refusals alone are called: a call that passes every check would launch."""
    lib = _lib()
    a = dict(lg=far(1), x=far(2), dh=far(3), r=far(4), p=far(5), o=far(6), o1=far(7), o2=far(8), lengths=None, s0=None, ds1=None, dds=None, s1=None, s2=None)
    a.update(change)
    rest = (a["lengths"], a["s0"], *sizes, dtype)
    if name == "fwd":
        return lib.diffopt_gscan_fwd(a["lg"], a["x"], *rest, a["o"], a["s1"], ws, nws, None)
    if name == "bwd":
        return lib.diffopt_gscan_bwd(a["dh"], a["ds1"], a["lg"], a["x"], *rest, a["o"], a["o1"], a["s1"], ws, nws, None)
    if name == "bwd_bwd":
        return lib.diffopt_gscan_bwd_bwd(a["r"], a["p"], a["dds"], a["dh"], a["ds1"], a["lg"], a["x"], *rest, a["o"], a["s1"], a["o1"], a["o2"], a["s2"], ws, nws,
                                         None)
    return lib.diffopt_gscan_step(a["lg"], a["x"], sizes[0], sizes[2], dtype, a["s0"], a["o"], None)


def _refused(word, name, **kw):
    rc = _call(name, **kw)
    assert rc == -1 and word in _error(), (rc, _error())


def test_shifted_views():
    # h = buf[:, :-1] and x = buf[:, 1:], and the other way round; buf[:-1] and buf[1:]
    for by in (C, -C, T * C, 4, -4, (T - 1) * C + C - 1):
        for dtype, size in ((F32, 4), (BF16, 2)):
            _refused("h must lie apart from x", "fwd", dtype=dtype, x=_seq(1 << 19), o=_seq((1 << 19) + by * size))
            _refused("h must lie apart from log_gate", "fwd", dtype=dtype, lg=_seq(1 << 19), o=_seq((1 << 19) + by * size))
    _refused("dx must lie apart from dh", "bwd", dh=_seq(0), o1=_seq(4 * C))
    _refused("dx must lie apart from dlog_gate", "bwd", o=_seq(0), o1=_seq(4 * C))
    _refused("out_x must lie apart from ddx", "bwd_bwd", p=_seq(0), o2=_seq(4 * C))
    _refused("out_log_gate must lie apart from out_dh", "bwd_bwd", o=_seq(0), o1=_seq(4 * C))


def test_other_strides():
    # rows that interleave meet or not by their places; spans that meet at other strides are refused
    wide = dict(sb=T * 3 * C, st=3 * C)
    _refused("h must lie apart from x", "fwd", x=_seq(0, **wide), o=_seq(4 * (C - 1), **wide))
    _refused("h must lie apart from x", "fwd", x=_seq(0, **wide), o=_seq(4 * (3 * C * 5 - C + 1), **wide))
    _refused("h must lie apart from x", "fwd", x=_seq(0, **wide), o=_seq(4 * C))
    _refused("h must lie apart from x", "fwd", x=_seq(4 * C * T * B, sb=-T * C, st=C), o=_seq(0))
    _refused("h must lie apart from x", "fwd", x=_seq(4 * 100, sb=0, st=0), o=_seq(0))


def test_states():
    n = 4 * B * C  # bytes of a state
    for at in (0, 4 * (B * T * C - 1), 4 - n):
        _refused("h must lie apart from state", "fwd", o=_seq(1 << 19), s0=block((1 << 19) + at))
        _refused("state_out must lie apart from h", "fwd", o=_seq(1 << 19), s1=block((1 << 19) + at))
        _refused("state_out must lie apart from x", "fwd", x=_seq(1 << 19), s1=block((1 << 19) + at))
        _refused("dx must lie apart from dstate_out", "bwd", o1=_seq(1 << 19), ds1=block((1 << 19) + at))
        _refused("dstate must lie apart from dh", "bwd", dh=_seq(1 << 19), s1=block((1 << 19) + at))
        _refused("out_state must lie apart from out_x", "bwd_bwd", o2=_seq(1 << 19), s2=block((1 << 19) + at))
        _refused("out_dh must lie apart from ddstate", "bwd_bwd", o=_seq(1 << 19), dds=block((1 << 19) + at))
    _refused("h must lie apart from lengths", "fwd", o=_seq(0), lengths=block(4 * B * T * C - 4))
    _refused("state_out must lie apart from lengths", "fwd", s1=block(0), lengths=block(n - 4))


def test_single_tokens():
    n = 4 * B * C
    one = dict(sb=C, st=0)
    for at in (4, -4, n - 4, 4 - n):
        _refused("out must lie apart from x", "step", x=_seq(1 << 19, **one), o=_seq((1 << 19) + at, **one), s0=block(0))
        _refused("state must lie apart from the operands and out", "step", x=_seq(1 << 19, **one), s0=block((1 << 19) + at))
        _refused("state must lie apart from the operands and out", "step", lg=_seq(1 << 19, **one), s0=block((1 << 19) + at))
        _refused("state must lie apart from the operands and out", "step", o=_seq(1 << 19, **one), s0=block((1 << 19) + at))


@pytest.mark.parametrize("name,used", [("fwd", ("lg", "x", "o")), ("bwd", ("lg", "x", "dh", "o", "o1")), ("bwd_bwd", ("lg", "x", "dh", "r", "p", "o", "o1", "o2"))])
@pytest.mark.parametrize("by", [-4, 4])
def test_neighbours_in_one_buffer(name, used, by):
    # operands and results side by side in one buffer, a result moved by one element into its neighbour's rows (whole rows
    # beside one another are taken: the tests that launch have them)
    wide = dict(sb=T * len(used) * C, st=len(used) * C)
    for i, k in enumerate(used):
        if not k.startswith("o") or (by > 0 and k == used[-1]):
            continue
        change = {n: _seq(4 * C * j + (by if n == k else 0), **wide) for j, n in enumerate(used)}
        rc = _call(name, **change)
        assert rc == -1 and "must lie apart" in _error(), (k, by, rc, _error())
