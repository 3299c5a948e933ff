"""CPU-side checks of the clipping entry points: refusals come before any device
call, with their messages, and the workspaces' sizes.  No kernel is launched and
no pointer is followed."""
import ctypes
import math

import pytest

odd = ctypes.c_void_p((1 << 20) + 2)


def at(i):  # never followed, a megabyte apart
    return ctypes.c_void_p(i << 20)


def _binding():
    import paper_2211_06934_amd as P
    return P.diffopt._lib, P.last_error


def _refused(rc, word):
    assert rc == -1 and word in _binding()[1](), (rc, _binding()[1]())


def _fwd(**change):
    a = dict(g=at(1), n=20000, max=1.0, eps=1e-6, out=at(2), st=at(3), ws=at(4), nws=4096)
    a.update(change)
    return _binding()[0].diffopt_clip_norm_fwd(a["g"], a["n"], a["max"], a["eps"], a["out"], a["st"], a["ws"], a["nws"], None)


def _bwd(**change):
    a = dict(d=at(5), dn=at(6), g=at(1), st=at(3), n=20000, eps=1e-6, dg=at(7), ws=at(4), nws=4096)
    a.update(change)
    return _binding()[0].diffopt_clip_norm_bwd(a["d"], a["dn"], a["g"], a["st"], a["n"], a["eps"], a["dg"], a["ws"], a["nws"], None)


@pytest.mark.parametrize("change,word", [
    (dict(n=-1), "n must be >= 0"), (dict(n=1 << 38), "too many"), (dict(n=1 << 62), "too many"), (dict(eps=-1e-6), "eps"), (dict(eps=math.nan), "eps"),
    (dict(eps=math.inf), "eps"), (dict(g=None), "null grad"), (dict(st=None), "stats"), (dict(g=odd), "aligned"), (dict(st=odd), "aligned"),
    (dict(ws=None), "the workspace has 0 bytes"), (dict(nws=7), "the workspace has 7 bytes"), (dict(ws=ctypes.c_void_p((4 << 20) + 4)), "8-byte"),
])
def test_refusals(change, word):
    _refused(_fwd(**change), word)
    _refused(_bwd(**change), word)


def test_each_directions_own():
    _refused(_fwd(max=-1.0), "max_norm")
    _refused(_fwd(max=math.nan), "max_norm")
    _refused(_fwd(out=odd), "aligned")
    _refused(_fwd(out=ctypes.c_void_p((1 << 20) + 4)), "out must be an operand or lie apart")
    _refused(_fwd(st=ctypes.c_void_p((1 << 20) + 64)), "stats must lie apart")
    _refused(_fwd(st=ctypes.c_void_p((2 << 20) + 64)), "stats must lie apart")
    _refused(_bwd(dg=None), "null grad, stats or dgrad")
    _refused(_bwd(d=odd), "aligned")
    _refused(_bwd(dg=ctypes.c_void_p((5 << 20) + 4)), "dgrad must be an operand or lie apart")
    _refused(_bwd(dg=ctypes.c_void_p((1 << 20) - 4)), "dgrad must be an operand or lie apart")
    _refused(_bwd(st=ctypes.c_void_p((7 << 20) + 64)), "dgrad must lie apart")
    _refused(_bwd(dn=ctypes.c_void_p((7 << 20) + 64)), "dgrad must lie apart")
    assert _bwd(n=0) == 0


def test_tables():
    lib = _binding()[0]
    _refused(lib.diffopt_clip_norm_fwd_tree(None, at(1), 1.0, 1e-6, at(2), at(3), None, 0, None), "table is NULL")
    _refused(lib.diffopt_clip_norm_bwd_tree(None, at(1), None, at(1), at(3), 1e-6, at(2), None, 0, None), "table is NULL")
    assert lib.diffopt_clip_norm_workspace_tree(None) == -1


def test_workspaces():
    size = _binding()[0].diffopt_clip_norm_workspace
    assert size(0) == size(1) == size(1761) == 0 and size(-1) == size(1 << 41) == -1
    last = 0
    for n in (10_000, 1_000_000, 100_000_000, 1_000_000_000):
        assert size(n) % 8 == 0 and last <= size(n) <= 1 << 16
        last = size(n)
