"""CPU-side checks of the log probabilities' entry points: refusals come before
any device call, with their messages, and the workspaces' sizes.  No kernel is
launched and no pointer is followed."""
import ctypes
import math

import pytest

F32, BF16 = 0, 1
odd = ctypes.c_void_p(66)


def at(i):  # never followed
    return ctypes.c_void_p(4096 * (i + 1))


def _binding():
    import paper_2211_06934_amd as P
    return P.diffopt._lib, P.last_error


def _refused(rc, word):
    assert rc == -1 and word in _binding()[1](), (rc, _binding()[1]())


def _call(name, **change):
    lib = _binding()[0]
    a = dict(x=at(0), stride=100, N=3, V=100, dtype=F32, ids=at(1), ib=8, T=1.0, lp=at(2), ent=at(3), st=at(4), top=at(5), ti=at(6), tb=8, K=5, g=at(7),
             h=at(8), c=at(9), dx=at(10), ds=100, a=at(11), as_=100, og=at(12), oh=at(13), oc=at(14), ws=None, nws=0)
    a.update(change)
    rows = (a["x"], a["stride"], a["N"], a["V"], a["dtype"], a["ids"], a["ib"], a["T"])
    if name == "fwd":
        return lib.diffopt_logprob_fwd(*rows, a["lp"], a["ent"], a["st"], a["top"], a["ti"], a["tb"], a["K"], a["ws"], a["nws"], None)
    if name == "bwd":
        return lib.diffopt_logprob_bwd(a["g"], a["h"], a["ent"], a["c"], a["ti"], a["tb"], a["K"], *rows, a["st"], a["dx"], a["ds"], None)
    if name == "fwd_bwd":
        return lib.diffopt_logprob_fwd_bwd(a["g"], a["h"], *rows, a["lp"], a["ent"], a["st"], a["dx"], a["ds"], a["ws"], a["nws"], None)
    return lib.diffopt_logprob_bwd_bwd(a["a"], a["as_"], a["g"], a["h"], a["ent"], a["c"], a["ti"], a["tb"], a["K"], *rows, a["st"], a["og"], a["oh"],
                                       a["oc"], a["dx"], a["ds"], a["ws"], a["nws"], None)


@pytest.mark.parametrize("name", ["fwd", "bwd", "fwd_bwd", "bwd_bwd"])
@pytest.mark.parametrize("change,word", [
    (dict(N=-1), "N must be"), (dict(N=1 << 22), "below 2^22"), (dict(V=0), "V must"), (dict(V=1 << 31), "V must"), (dict(dtype=3), "element type"),
    (dict(ib=2), "id_bytes"), (dict(T=0.0), "temperature"), (dict(T=-1.0), "temperature"), (dict(T=math.nan), "temperature"), (dict(T=math.inf), "temperature"),
    (dict(T=1e-40), "temperature"), (dict(T=1e60), "temperature"), (dict(x=None), "null logits"), (dict(x=odd), "aligned"), (dict(ids=ctypes.c_void_p(68)), "aligned"),
    (dict(st=None), "null"), (dict(st=odd), "aligned"),
])
def test_refusals(name, change, word):
    _refused(_call(name, **change), word)


@pytest.mark.parametrize("name", ["fwd", "bwd", "bwd_bwd"])
def test_alternatives(name):
    _refused(_call(name, K=-1), "K must be in")
    _refused(_call(name, K=129), "K must be in")
    _refused(_call(name, tb=3), "top_id_bytes")
    _refused(_call(name, ti=None), "null")
    _refused(_call(name, ti=ctypes.c_void_p(4100)), "aligned")
    _refused(_call(name, **({"top": None} if name == "fwd" else {"c": None})), "null")


def test_what_goes_together():
    _refused(_call("fwd", lp=None), "null stats or logprob")
    _refused(_call("fwd", ids=None), "logprob without ids")
    _refused(_call("bwd", ent=None), "dentropy without entropy")
    _refused(_call("bwd", ids=None), "dlogprob without ids")
    _refused(_call("fwd_bwd", g=None), "null required")
    _refused(_call("fwd_bwd", ids=None), "null required")
    _refused(_call("bwd_bwd", a=None), "null stats or ddlogits")
    _refused(_call("bwd_bwd", h=None, ent=None), "out_dentropy without")
    _refused(_call("bwd_bwd", g=None, ids=None), "out_dlogprob without")


def test_results_lie_apart():
    _refused(_call("fwd", ent=at(2)), "one array")
    _refused(_call("fwd", top=at(4)), "one array")
    _refused(_call("fwd", lp=at(1)), "operand")
    _refused(_call("fwd_bwd", dx=at(0)), "must not be logits")
    _refused(_call("fwd_bwd", lp=at(7)), "operand")
    _refused(_call("fwd_bwd", dx=None), "null")
    _refused(_call("bwd", dx=at(0), ds=101), "row stride")
    _refused(_call("bwd", ds=99), "overlap")
    _refused(_call("bwd_bwd", dx=at(0)), "neither")
    _refused(_call("bwd_bwd", dx=at(11)), "neither")
    _refused(_call("bwd_bwd", og=at(7)), "operand")
    _refused(_call("bwd_bwd", oh=at(12)), "one array")
    _refused(_call("bwd_bwd", oc=at(6)), "operand")


def test_no_rows():
    for name in ("fwd", "bwd", "fwd_bwd", "bwd_bwd"):
        assert _call(name, N=0) == 0


def test_workspaces():
    size = _binding()[0].diffopt_logprob_workspace
    assert size(0, 50000, F32, 5) == 0 and size(5000, 50000, F32, 5) == 0
    assert size(3, 50000, F32, -1) == size(3, 50000, F32, 129) == size(3, 50000, 9, 5) == size(3, 0, F32, 5) == size(1 << 22, 50, F32, 5) == -1
    need = size(2, 1 << 20, F32, 5)
    assert need > size(2, 1 << 20, F32, 0) > 0
    big = dict(N=2, V=1 << 20, stride=1 << 20, ds=1 << 20, as_=1 << 20)
    for name, n in (("fwd", need), ("fwd_bwd", size(2, 1 << 20, F32, 0)), ("bwd_bwd", size(2, 1 << 20, F32, 0))):
        _refused(_call(name, **big), "the workspace has 0 bytes")
        _refused(_call(name, **big, ws=at(20), nws=n - 1), "the workspace has")
        _refused(_call(name, **big, ws=odd, nws=n), "not 4-byte aligned")


@pytest.mark.parametrize("bad", [(), (8,), (2, 3, 4)])
def test_operands_of_other_axes_are_named(bad):
    import torch

    import paper_2211_06934_amd as P
    for logits in (None, torch.zeros(bad)):
        with pytest.raises(ValueError, match="logits: expected a tensor of 2 axes"):
            P.token_logprobs(logits, top=2)
    for ids in ([1, 2], torch.zeros(2, 1, dtype=torch.int64), torch.zeros((), dtype=torch.int64)):
        with pytest.raises(ValueError, match="ids: expected a tensor of 1 axes"):
            P.token_logprobs(torch.zeros(2, 9), ids)
