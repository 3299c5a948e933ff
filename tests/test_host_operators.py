"""CPU-side checks of the language-model operators' entry points: every refusal
comes before any device call, with its message, and the workspaces' sizes.  No
kernel is launched and no pointer is followed."""
import ctypes
import math

import pytest
import torch

F32, BF16 = 0, 1
f = ctypes.c_void_p(64)  # never followed
odd = ctypes.c_void_p(66)


def _binding():
    import paper_2211_06934_amd as P
    return P.diffopt._lib, P.last_error, P.operators._Heads


def _refused(rc, word):
    _, last_error, _ = _binding()
    assert rc == -1 and word in last_error(), (rc, last_error())


def _head(Heads, at=64):
    return ctypes.byref(Heads(at, 64, 16, 8))


def _linattn(**change):
    lib, _, Heads = _binding()
    a = dict(q=_head(Heads), k=_head(Heads), v=_head(Heads), lg=f, lengths=None, state=None, B=2, T=9, H=4, Hk=2, Dk=8, Dv=8, dtype=F32,
             scale=1.0, out=_head(Heads), state_out=None, ws=None, nws=0)
    a.update(change)
    return lib.diffopt_linattn_fwd(a["q"], a["k"], a["v"], a["lg"], a["lengths"], a["state"], a["B"], a["T"], a["H"], a["Hk"], a["Dk"],
                                   a["Dv"], a["dtype"], a["scale"], a["out"], a["state_out"], a["ws"], a["nws"], None)


@pytest.mark.parametrize("change,word", [
    (dict(B=-1), "must be >= 0"), (dict(T=-5), "must be >= 0"), (dict(H=3), "multiple"), (dict(H=0), "multiple"), (dict(Hk=0), "multiple"),
    (dict(Dk=0), "Dk and Dv"), (dict(Dv=257), "Dk and Dv"), (dict(dtype=7), "element type"), (dict(scale=math.nan), "scale"),
    (dict(scale=math.inf), "scale"), (dict(scale=1e300), "scale"), (dict(lg=None), "null log_decay"), (dict(lg=odd), "aligned"),
    (dict(lengths=odd), "aligned"), (dict(state=odd), "aligned"), (dict(state_out=odd), "aligned"), (dict(q=None), "null q"),
    (dict(out=None), "null out"), (dict(T=1 << 36), "too many"), (dict(H=1 << 17, Hk=1), "too many"), (dict(B=1 << 25), "too many"),
    (dict(B=1 << 18, H=64, Hk=64, Dk=8, Dv=8), "too many"), (dict(B=1 << 17, H=64, Hk=64, Dk=8, Dv=64), "too many"),
])
def test_linattn_fwd_refuses(change, word):
    _refused(_linattn(**change), word)


def test_linattn_alignment_of_elements():
    _, _, Heads = _binding()
    _refused(_linattn(k=_head(Heads, 66)), "k is not aligned")
    _refused(_linattn(v=_head(Heads, 65), dtype=BF16), "v is not aligned")


def test_linattn_workspace():
    lib, _, _ = _binding()
    size = lib.diffopt_linattn_workspace
    assert size(1, 0, 4, 4, 64, 64, F32, 0) == 0
    assert size(0, 100000, 4, 4, 64, 64, F32, 1) == 0
    assert size(1, 4, 4, 4, 64, 64, F32, 0) == 0  # single tokens take none
    assert size(1, 16384, 4, 4, 64, 64, BF16, 0) > 0
    assert size(1, 16384, 4, 4, 64, 64, BF16, 0) % 256 == 0
    assert size(1, 16384, 4, 3, 64, 64, BF16, 0) == -1
    assert size(1, 16384, 4, 4, 64, 300, BF16, 0) == -1
    need = size(1, 16384, 4, 4, 64, 64, F32, 0)
    _refused(_linattn(B=1, T=16384, Hk=4, Dk=64, Dv=64), "the workspace has 0 bytes")
    _refused(_linattn(B=1, T=16384, Hk=4, Dk=64, Dv=64, ws=f, nws=need - 1), "the workspace has")
    _refused(_linattn(B=1, T=16384, Hk=4, Dk=64, Dv=64, ws=ctypes.c_void_p(72), nws=need), "16-byte")


def test_linattn_bwd_and_step_refuse():
    lib, _, Heads = _binding()
    h = _head(Heads)

    def bwd(B=1, T=9, state=None, ds1=None, ds=None, dout=h, dq=h):
        return lib.diffopt_linattn_bwd(dout, ds1, h, h, h, f, None, state, B, T, 2, 2, 8, 8, F32, 1.0, dq, None, None, ds, None, 0, None)

    _refused(bwd(dout=None), "null dout")
    _refused(bwd(state=f, ds=f), "dstate")
    _refused(bwd(ds1=f, ds=f), "dstate")
    _refused(bwd(ds=odd), "aligned")
    _refused(bwd(dq=_head(Heads, 66)), "dq is not aligned")
    assert bwd(B=0) == 0 and bwd(dq=None) == 0  # nothing wanted

    def step(state=f, out=h, lg=f, Dk=8):
        return lib.diffopt_linattn_step(h, h, h, lg, 1, 2, 2, Dk, 8, F32, 1.0, state, out, None)

    _refused(step(state=None), "null state")
    _refused(step(out=None), "null out")
    _refused(step(lg=None), "null log_decay")
    _refused(step(Dk=300), "Dk and Dv")


def _qknorm(**change):
    lib, _, Heads = _binding()
    a = dict(q=_head(Heads), k=_head(Heads), qw=None, kw=None, cos=f, sin=f, rows=32, pos=None, pb=0, first=0, B=2, T=9, H=4, Hk=2, D=16, rot=8,
             inter=0, dtype=F32, eps=1e-6, qo=_head(Heads), ko=_head(Heads))
    a.update(change)
    return lib.diffopt_qknorm_rope_fwd(a["q"], a["k"], a["qw"], a["kw"], a["cos"], a["sin"], a["rows"], a["pos"], a["pb"], a["first"], a["B"],
                                       a["T"], a["H"], a["Hk"], a["D"], a["rot"], a["inter"], a["dtype"], a["eps"], a["qo"], a["ko"], None)


@pytest.mark.parametrize("change,word", [
    (dict(T=-1), "sizes"), (dict(D=0), "sizes"), (dict(D=1025), "sizes"), (dict(H=70000), "sizes"), (dict(rot=7), "rot"), (dict(rot=18), "rot"),
    (dict(rot=-2), "rot"), (dict(dtype=2), "element type"), (dict(eps=-1e-6), "eps"), (dict(eps=math.nan), "eps"), (dict(cos=None), "null cos"),
    (dict(sin=None), "null cos or sin"), (dict(cos=odd), "aligned"), (dict(rows=-1), "rows"), (dict(rows=8), "outside"),
    (dict(first=30), "outside"), (dict(first=-1), "outside"), (dict(first=(1 << 63) - 1), "outside"), (dict(pos=f, pb=2), "position_bytes"),
    (dict(pos=ctypes.c_void_p(68), pb=8), "positions"), (dict(q=None), "null q"), (dict(ko=None), "null q_out or k_out"),
    (dict(qw=odd), "aligned"),
])
def test_qknorm_rope_refuses(change, word):
    _refused(_qknorm(**change), word)


def test_qknorm_rope_workspace():
    lib, _, Heads = _binding()
    size = lib.diffopt_qknorm_rope_workspace
    assert size(2, 9, 4, 0, 16) > 0 and size(0, 9, 4, 2, 16) == 0 and size(2, 9, 4, 2, 1025) == -1
    h = _head(Heads)
    call = lambda ws, n: lib.diffopt_qknorm_rope_bwd(h, h, h, h, None, None, f, f, 32, None, 0, 0, 2, 9, 4, 2, 16, 8, 0, F32, 1e-6, h, h, f,  # noqa: E731
                                                     None, ws, n, None)
    _refused(call(None, 0), "the workspace has 0 bytes")
    _refused(call(f, 4), "the workspace has 4 bytes")


def _distill(**change):
    lib, _, _ = _binding()
    a = dict(x=f, stride=100, N=3, V=100, dtype=F32, ids=f, ib=4, t=f, K=5, T=1.0, loss=f, stats=f, ws=None, nws=0)
    a.update(change)
    return lib.diffopt_distill_fwd(a["x"], a["stride"], a["N"], a["V"], a["dtype"], a["ids"], a["ib"], a["t"], a["K"], a["T"], a["loss"],
                                   a["stats"], a["ws"], a["nws"], None)


@pytest.mark.parametrize("change", [dict(N=-1), dict(N=1 << 22), dict(V=-1), dict(K=0), dict(K=1025), dict(dtype=5), dict(ib=3), dict(T=0.0), dict(T=-1.0),
                                    dict(T=math.nan), dict(T=math.inf), dict(x=None), dict(ids=None), dict(t=None), dict(loss=None),
                                    dict(stats=None), dict(x=odd), dict(t=odd), dict(ids=ctypes.c_void_p(68), ib=8), dict(stats=odd)])
def test_distill_refuses(change):
    assert _distill(**change) == -1
    assert "diffopt_distill_fwd" in _binding()[1]()


def test_distill_workspace():
    lib, _, _ = _binding()
    size = lib.diffopt_distill_workspace
    assert size(0, 50000, F32, 8) == 0 and size(3, 50000, F32, 0) == -1 and size(3, 50000, 9, 8) == -1
    assert size(2, 1 << 20, F32, 8) > 0  # few long rows are split
    _refused(_distill(N=2, V=1 << 20, stride=1 << 20), "the workspace has 0 bytes")


def test_constants_that_ask_for_gradients_are_refused():
    import paper_2211_06934_amd as P
    q, lg = torch.zeros(1, 3, 2, 8), torch.zeros(2, requires_grad=True)
    with pytest.raises(ValueError, match="log_decay"):
        P.linear_attention(q, q, q, lg)
    with pytest.raises(ValueError, match="sin"):
        P.qknorm_rope(q, q, cos=torch.ones(3, 4), sin=torch.ones(3, 4, requires_grad=True))
