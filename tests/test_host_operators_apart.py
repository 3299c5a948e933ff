"""Results of the operators that lie on operands, or on one another, where an entry
point does not allow it: refused before any device call.  No pointer is followed."""
import ctypes

import pytest

from test_host_operators import BF16, F32, _binding, _refused


def _p(at):
    return ctypes.c_void_p(at)


def _h(at, b=1024, t=64, h=8):
    return ctypes.byref(_binding()[2](at, b, t, h))


def _fwd(q=0x10000, k=0x20000, v=0x30000, out=0x40000, state=None, state_out=None, dtype=F32):
    lib, _, _ = _binding()
    return lib.diffopt_linattn_fwd(_h(q), _h(k), _h(v), _p(64), None, _p(state), 2, 9, 4, 2, 8, 8, dtype, 1.0, _h(out), _p(state_out), None, 0, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_linattn_fwd_out_is_no_operand(name, dtype):
    _refused(_fwd(**{name: 0x40000}, dtype=dtype), "must not be an operand")


@pytest.mark.parametrize("shift", [4, 512, 2 * 2 * 8 * 8 * 4 - 4])
@pytest.mark.parametrize("sign", [-1, 1])
def test_linattn_fwd_states_are_one_or_apart(shift, sign):
    _refused(_fwd(state=0x50000, state_out=0x50000 + sign * shift), "state_out must be state or lie apart")


def _bwd(dq=0x50000, dk=0x60000, dv=0x70000, dout=0x40000, state=None, ds1=None, ds=None):
    lib, _, _ = _binding()
    return lib.diffopt_linattn_bwd(_h(dout), _p(ds1), _h(0x10000), _h(0x20000), _h(0x30000), _p(64), None, _p(state), 2, 9, 4, 2, 8, 8, F32, 1.0,
                                   _h(dq), _h(dk), _h(dv), _p(ds), None, 0, None)


@pytest.mark.parametrize("result", ["dq", "dk", "dv"])
@pytest.mark.parametrize("operand", [0x10000, 0x20000, 0x30000, 0x40000])
def test_linattn_bwd_results_are_no_operands(result, operand):
    _refused(_bwd(**{result: operand}), "must not be an operand")


def test_linattn_bwd_results_are_apart():
    _refused(_bwd(dq=0x60000), "two results")
    _refused(_bwd(dv=0x60000), "two results")
    _refused(_bwd(dv=0x50000), "two results")
    for shift in (-4, 0, 4):
        _refused(_bwd(state=0x80000, ds=0x80000 + shift), "dstate must")
        _refused(_bwd(ds1=0x80000, ds=0x80000 + shift), "dstate must")


@pytest.mark.parametrize("operand", [0x10000, 0x20000, 0x30000])
def test_linattn_step_out_is_no_operand(operand):
    lib, _, _ = _binding()
    rc = lib.diffopt_linattn_step(_h(0x10000), _h(0x20000), _h(0x30000), _p(64), 2, 4, 2, 8, 8, F32, 1.0, _p(0x80000), _h(operand), None)
    _refused(rc, "must not be an operand")


def _distill(name, **change):
    lib, _, _ = _binding()
    a = dict(logits=0x100000, stride=64, ids=0x200000, teacher=0x210000, dloss=0x220000, loss=0x230000, stats=0x240000, dlogits=0x300000, dstride=64,
             dteacher=0x250000, ddlogits=0x400000, ddteacher=0x260000, out_dloss=0x270000, out_logits=0x500000, out_teacher=0x280000)
    a.update(change)
    p = {k: v if k in ("stride", "dstride") else _p(v) for k, v in a.items()}
    rows = (p["logits"], p["stride"], 3, 50, F32, p["ids"], 4, p["teacher"], 5, 1.0)
    if name == "fwd":
        return lib.diffopt_distill_fwd(*rows, p["loss"], p["stats"], None, 0, None)
    if name == "bwd":
        return lib.diffopt_distill_bwd(p["dloss"], *rows, p["stats"], p["dlogits"], p["dstride"], p["dteacher"], None)
    if name == "fwd_bwd":
        return lib.diffopt_distill_fwd_bwd(p["dloss"], *rows, p["loss"], p["stats"], p["dlogits"], p["dstride"], p["dteacher"], None, 0, None)
    return lib.diffopt_distill_bwd_bwd(p["ddlogits"], 64, p["ddteacher"], p["dloss"], *rows, p["stats"], p["out_dloss"], p["out_logits"], 64,
                                       p["out_teacher"], None, 0, None)


@pytest.mark.parametrize("name,change,word", [
    ("bwd", dict(dlogits=0x100000, dstride=128), "row stride"), ("bwd", dict(dlogits=0x100000, stride=50), "row stride"),
    ("fwd", dict(loss=0x210000), "an operand"), ("fwd", dict(stats=0x210000 + 4 * 14), "an operand"), ("fwd", dict(loss=0x240000 + 20), "two results"),
    ("bwd", dict(dteacher=0x210000), "an operand"), ("bwd", dict(dteacher=0x220008), "an operand"), ("bwd", dict(dteacher=0x240000), "an operand"),
    ("fwd_bwd", dict(loss=0x220000), "an operand"), ("fwd_bwd", dict(dteacher=0x210000), "an operand"),
    ("fwd_bwd", dict(stats=0x230000), "two results"), ("fwd_bwd", dict(dteacher=0x230004), "two results"),
    ("bwd_bwd", dict(out_dloss=0x220000), "an operand"), ("bwd_bwd", dict(out_teacher=0x260000), "an operand"),
    ("bwd_bwd", dict(out_teacher=0x210000), "an operand"), ("bwd_bwd", dict(out_dloss=0x280000), "two results"),
])
def test_distill_results_are_apart(name, change, word):
    _refused(_distill(name, **change), word)


def _qknorm(name, **change):
    lib, _, Heads = _binding()
    # q [2, 9, 4, 16], k [2, 9, 2, 16], every operand and result in a place of its own
    names = ("q", "k", "q_out", "k_out", "dq_out", "dk_out", "dq", "dk", "ddq", "ddk", "out_dq_out", "out_dk_out", "out_q", "out_k")
    a = {n: Heads((i + 1) << 16, 9 * 16 * (2 if "k" in n else 4), 16 * (2 if "k" in n else 4), 16) for i, n in enumerate(names)}
    a["dwq"], a["dwk"] = 0x800000, 0x810000
    for n, v in change.items():
        a[n] = v if isinstance(v, int) else a[v] if isinstance(v, str) else Heads(*v)
    h = lambda n: ctypes.byref(a[n])  # noqa: E731
    shape = (None, None, _p(64), _p(64), 32, None, 0, 0, 2, 9, 4, 2, 16, 8, 0, F32, 1e-6)
    ws = (_p(0x900000), lib.diffopt_qknorm_rope_workspace(2, 9, 4, 2, 16), None)
    if name == "fwd":
        return lib.diffopt_qknorm_rope_fwd(h("q"), h("k"), *shape, h("q_out"), h("k_out"), None)
    if name == "bwd":
        return lib.diffopt_qknorm_rope_bwd(h("dq_out"), h("dk_out"), h("q"), h("k"), *shape, h("dq"), h("dk"), _p(a["dwq"]), _p(a["dwk"]), *ws)
    return lib.diffopt_qknorm_rope_bwd_bwd(h("ddq"), h("ddk"), None, None, h("dq_out"), h("dk_out"), h("q"), h("k"), *shape, h("out_dq_out"),
                                           h("out_dk_out"), h("out_q"), h("out_k"), _p(a["dwq"]), _p(a["dwk"]), *ws)


Q = 1 << 16  # q's address; its strides are 576, 64, 16


@pytest.mark.parametrize("name,change,word", [
    ("fwd", dict(q_out=(Q, 576, 16, 144)), "an operand"), ("fwd", dict(q_out=(Q, 1152, 64, 16)), "an operand"), ("fwd", dict(q_out="k"), "an operand"),
    ("fwd", dict(k_out="q"), "an operand"), ("fwd", dict(k_out="q_out"), "two results"),
    ("bwd", dict(dq="dk_out"), "an operand"), ("bwd", dict(dk="q"), "an operand"), ("bwd", dict(dk="dq"), "two results"),
    ("bwd", dict(dwk=0x800000 + 60), "two results"),
    ("bwd_bwd", dict(out_q="ddk"), "an operand"), ("bwd_bwd", dict(out_dk_out="q"), "an operand"), ("bwd_bwd", dict(out_q="out_dq_out"), "two results"),
    ("bwd_bwd", dict(out_k="out_dq_out"), "two results"),
])
def test_qknorm_rope_results_are_apart(name, change, word):
    _refused(_qknorm(name, **change), word)
