"""The gated recurrence: forward, gradients, the gradients' own VJP and single
tokens against a token-after-token fp64 loop and its autograd."""
import math

import pytest
import torch

from lm_reference import F32, assert_close, tol

pytestmark = pytest.mark.gpu

# The tolerances are those of the other operators: a state sums at most a few
# thousand terms whose fp32 roundings (2^-24 each, decaying with the state) add
# like a random walk, and results in bf16 are rounded once.


def _recurrence(lg, x, state, lengths):
    """fp64 (h, state_out), differentiable."""
    B, T, C = x.shape
    h = torch.zeros(B, C, dtype=torch.float64) if state is None else state
    n = torch.full((B,), T) if lengths is None else lengths.long().clamp(0, T)
    outs = []
    for t in range(T):
        live = (t < n)[:, None]
        nought = torch.zeros((), dtype=torch.float64)
        gate, new = torch.where(live, lg[:, t], nought), torch.where(live, x[:, t], nought)
        h = torch.where(live, torch.exp(gate) * h + new, h)
        outs.append(torch.where(live, h, nought))
    return (torch.stack(outs, 1) if T else x), h


def _inputs(B, T, C, dtype, seed=0, state=True, lengths=True, resets=True):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    rate = torch.exp2(-8.0 * torch.rand(C, generator=gen))
    lg = -rate * torch.rand(B, T, C, generator=gen)
    if resets:
        lg = torch.where(torch.rand(B, T, 1, generator=gen) < 0.05, -math.inf, lg)
    I = dict(lg=lg.to(dtype), x=r(B, T, C).to(dtype), dh=r(B, T, C).to(dtype), r=r(B, T, C).to(dtype), p=r(B, T, C).to(dtype))
    I["lengths"] = torch.randint(0, T + 1, (B,), generator=gen).to(torch.int32) if lengths else None
    if lengths and B > 1:
        I["lengths"][0] = T
    for k in ("s0", "ds1", "s"):
        I[k] = r(B, C) if state else None
    return I


def _reference(I):
    d = lambda t: None if t is None else t.double().requires_grad_()  # noqa: E731
    lg, x, s0, dh, ds1 = (d(I[k]) for k in ("lg", "x", "s0", "dh", "ds1"))
    h, s1 = _recurrence(lg, x, s0, I["lengths"])
    outs, cots, leaves = ([h], [dh], [lg, x]) if s0 is None else ([h, s1], [dh, ds1], [lg, x, s0])
    grads = torch.autograd.grad(outs, leaves, cots, create_graph=True)
    seconds = [I["r"].double(), I["p"].double()] + ([I["s"].double()] if s0 is not None else [])
    back = torch.autograd.grad(grads, cots + leaves, seconds, allow_unused=True)
    back = [torch.zeros_like(of) if b is None else b for b, of in zip(back, cots + leaves)]
    ref = dict(h=h, s1=s1, dlg=grads[0], dx=grads[1], out_dh=back[0], out_lg=back[len(cots)], out_x=back[len(cots) + 1])
    if s0 is not None:
        ref |= dict(ds0=grads[2], out_ds1=back[1], out_s0=back[-1])
    return ref


def _run(I, wrap=lambda t: t.cuda(), new=None):
    import paper_2211_06934_amd as P
    lg, x, dh, r, p = (wrap(I[k]) for k in ("lg", "x", "dh", "r", "p"))
    n = None if I["lengths"] is None else I["lengths"].cuda()
    s0, ds1, s = (None if I[k] is None else I[k].cuda() for k in ("s0", "ds1", "s"))
    nan = new or (lambda: torch.full(x.shape, math.nan, dtype=x.dtype, device="cuda"))
    st = lambda: torch.full((x.shape[0], x.shape[2]), math.nan, device="cuda")  # noqa: E731
    got = dict(h=nan(), s1=st(), dlg=nan(), dx=nan(), out_dh=nan(), out_lg=nan(), out_x=nan())
    if s0 is not None:
        got |= dict(ds0=st(), out_ds1=st(), out_s0=st())
    P.gscan_fwd(lg, x, got["h"], s0, got["s1"], n)
    P.gscan_bwd(dh, lg, x, got["dlg"], got["dx"], s0, ds1, got.get("ds0"), n)
    P.gscan_bwd_bwd(r, p, dh, lg, x, got["out_dh"], got["out_lg"], got["out_x"], s0, ds1, s, got.get("out_ds1"), got.get("out_s0"), n)
    return got


_STATES = ("s1", "ds0", "out_ds1", "out_s0")


def _compare(got, ref, dtype, what=""):
    assert set(got) == set(ref)
    for k in ref:
        assert_close(got[k], ref[k], F32 if k in _STATES else tol(dtype), "%s %s" % (what, k))


def _check(B, T, C, dtype, seed=0, wrap=lambda t: t.cuda(), **kw):
    I = _inputs(B, T, C, dtype, seed, **kw)
    _compare(_run(I, wrap), _reference(I), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 63, 64, 65, 128, 129, 509, 513, 577, 1030])
def test_lengths_of_sequences(T, dtype):
    _check(3, T, 37, dtype, seed=T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C", [1, 2, 3, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 517, 1024])
def test_channels(C, dtype):
    _check(2, 70, C, dtype, seed=C)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("state,lengths,resets", [(False, False, False), (True, False, False), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("T", [5, 200, 1500])
def test_what_may_be_left_out(T, state, lengths, resets, dtype):
    _check(2, T, 130, dtype, seed=T, state=state, lengths=lengths, resets=resets)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,C", [(200, 260, 3), (193, 512, 5), (210, 1100, 2), (97, 300, 67), (66, 1100, 1), (3, 257, 4100), (4, 1030, 517), (130, 60, 129)])
@pytest.mark.parametrize("rest", [False, True])
def test_many_channels(B, T, C, rest, dtype):
    # enough columns of channels for both directions to take a sequence in one sweep; whole steps and a rest
    _check(B, T, C, dtype, seed=T, state=rest, lengths=rest, resets=rest)


@pytest.mark.parametrize("lengths", [[0, 0, 0], [1, 0, 64], [65, 130, 129], [-5, 1000, 8]])
def test_ends_of_sequences(lengths):
    I = _inputs(3, 130, 70, torch.float32)
    I["lengths"] = torch.tensor(lengths, dtype=torch.int32)
    ref = _reference(I)
    for k in ("lg", "x", "dh", "r", "p"):  # padding may hold anything
        for b, n in enumerate(I["lengths"].clamp(0, 130).tolist()):
            I[k][b, n:] = math.nan
    _compare(_run(I), ref, torch.float32)


def test_long_memory():
    # gates near one, constant over time: a product of roundings of exp(log_gate) would drift by T 2^-25 = 1e-4 of the state
    T = 4096
    I = _inputs(1, T, 64, torch.float32, lengths=False, resets=False)
    I["lg"] = (-torch.exp2(-6.0 - 8.0 * torch.arange(64) / 64))[None, None].expand(1, T, 64).contiguous()
    _compare(_run(I), _reference(I), torch.float32)


def test_gates_above_zero_and_strong_ones():
    I = _inputs(2, 140, 70, torch.float32, resets=False)
    I["lg"] = 0.2 * torch.randn(I["lg"].shape, generator=torch.Generator().manual_seed(8)) - 0.02
    _compare(_run(I), _reference(I), torch.float32)
    I["lg"] = -30.0 * torch.rand(I["lg"].shape, generator=torch.Generator().manual_seed(9))
    _compare(_run(I), _reference(I), torch.float32)


@pytest.mark.parametrize("T", [60, 300, 900, 1500])
def test_values_that_are_not_finite(T):
    # finite exactly where the recurrence's results are: before the token, in other channels
    I = _inputs(2, T, 70, torch.float32, resets=False, lengths=False)
    I["x"][0, T // 3, 4] = math.nan
    I["x"][1, T // 2, 9] = math.inf
    I["lg"][1, T // 2 + 9, 9] = -0.1
    got, ref = _run(I), _reference(I)
    for k in ("h", "s1"):
        assert torch.equal(torch.isfinite(got[k]).cpu(), torch.isfinite(ref[k])), k
    h, r = got["h"].cpu(), ref["h"].detach()
    fine = torch.isfinite(r)
    assert_close(torch.where(fine, h, 0.0), torch.where(fine, r, 0.0), F32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["wide tokens", "odd tokens", "time first", "backwards"])
def test_strides(kind, dtype):
    def wrap(t):
        B, T, C = t.shape
        if kind == "time first":
            return torch.full((T, B, C), math.nan, dtype=t.dtype, device="cuda").transpose(0, 1).copy_(t)
        pad, off = (8, 0) if kind == "wide tokens" else (3, 1) if kind == "odd tokens" else (0, 0)
        buf = torch.full((B * T * (C + pad) + 1,), math.nan, dtype=t.dtype, device="cuda")
        return buf.as_strided((B, T, C), (T * (C + pad), C + pad, 1), off).copy_(t)
    for B, T, C in ((2, 70, 131), (2, 700, 131), (2, 1100, 131), (64, 300, 131)):
        I = _inputs(B, T, C, dtype, seed=T)
        results = lambda: wrap(torch.zeros(B, T, C, dtype=dtype))  # noqa: E731
        _compare(_run(I, wrap, None if kind == "backwards" else results), _reference(I), dtype)


def test_broadcast_operands():
    # one gate for all sequences, one input for all tokens
    I = _inputs(3, 90, 70, torch.float32)
    I["lg"], I["x"] = I["lg"][:1].expand(3, -1, -1), I["x"][:, :1].expand(-1, 90, -1)
    wrap = lambda t: t.cuda() if t.stride(0) and t.stride(1) else t[:1, :].cuda().expand(3, -1, -1) if t.stride(0) == 0 else t[:, :1].cuda().expand(-1, 90, -1)  # noqa: E731
    _compare(_run(I, wrap), _reference(I), torch.float32)


@pytest.mark.parametrize("T", [1, 64, 100, 700, 1500])
def test_state_in_place(T):
    import paper_2211_06934_amd as P
    I = _inputs(2, T, 300, torch.float32)
    want = _run(I)
    state, h = I["s0"].cuda(), torch.empty(2, T, 300, device="cuda")
    P.gscan_fwd(I["lg"].cuda(), I["x"].cuda(), h, state, state, I["lengths"].cuda())
    assert_close(h, want["h"].double(), 1e-6)
    assert_close(state, want["s1"].double(), 1e-6)


@pytest.mark.parametrize("T,C", [(60, 70), (300, 70), (900, 70), (300, 6300)])
def test_results_that_are_not_wanted(T, C):
    import paper_2211_06934_amd as P
    I = {k: None if v is None else v.cuda() for k, v in _inputs(2, T, C, torch.float32).items()}
    want = _run(I)
    new = lambda: torch.empty_like(I["x"])  # noqa: E731
    for keep in range(8):
        dlg, dx, ds = (new() if keep & 1 else None), (new() if keep & 2 else None), (torch.empty_like(I["s0"]) if keep & 4 else None)
        P.gscan_bwd(I["dh"], I["lg"], I["x"], dlg, dx, I["s0"], I["ds1"], ds, I["lengths"])
        for o, k in ((dlg, "dlg"), (dx, "dx"), (ds, "ds0")):
            assert o is None or torch.equal(o, want[k])
    h = new()
    P.gscan_fwd(I["lg"], I["x"], h, I["s0"], None, I["lengths"])
    assert torch.equal(h, want["h"])
    oh, og, ox = new(), new(), new()
    P.gscan_bwd_bwd(I["r"], I["p"], I["dh"], I["lg"], I["x"], oh, og, ox, I["s0"], I["ds1"], I["s"], None, None, I["lengths"])
    assert torch.equal(oh, want["out_dh"]) and torch.equal(og, want["out_lg"]) and torch.equal(ox, want["out_x"])


def test_nothing_to_do():
    import paper_2211_06934_amd as P
    e = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    P.gscan_fwd(e(0, 5, 3), e(0, 5, 3), e(0, 5, 3))
    P.gscan_fwd(e(2, 5, 0), e(2, 5, 0), e(2, 5, 0), state_out=e(2, 0))
    s0, s1 = torch.randn(2, 3, device="cuda"), e(2, 3)
    P.gscan_fwd(e(2, 0, 3), e(2, 0, 3), e(2, 0, 3), s0, s1)
    assert torch.equal(s0, s1)
    P.gscan_bwd(e(2, 0, 3), e(2, 0, 3), e(2, 0, 3), e(2, 0, 3), e(2, 0, 3), s0, s1, s2 := e(2, 3))
    assert torch.equal(s2, s1)
    P.gscan_bwd_bwd(*[e(2, 0, 3)] * 5, e(2, 0, 3), e(2, 0, 3), e(2, 0, 3), s0, s1, s0, o1 := e(2, 3), o0 := e(2, 3))
    assert torch.equal(o1, s0) and not o0.any()
    P.gscan_step(e(0, 3), e(0, 3), e(0, 3), e(0, 3))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C", [(1, 1), (3, 4), (2, 2048), (5, 517), (300, 130)])
def test_step_goes_on_where_the_scan_ends(B, C, dtype):
    import paper_2211_06934_amd as P
    I = _inputs(B, 9, C, dtype, lengths=False)
    lg, x, state = I["lg"].cuda(), I["x"].cuda(), I["s0"].cuda()
    ref_h, ref_s = _recurrence(I["lg"].double(), I["x"].double(), I["s0"].double(), None)
    for t in range(9):
        out = torch.full((B, C), math.nan, dtype=dtype, device="cuda")
        P.gscan_step(lg[:, t], x[:, t], state, out)
        assert_close(out, ref_h[:, t], tol(dtype))
    assert_close(state, ref_s, F32)


def test_gradients_against_differences():
    import paper_2211_06934_amd as P
    I = {k: None if v is None else v.cuda() for k, v in _inputs(2, 150, 70, torch.float32, resets=False).items()}

    def at(e):
        lg, x, s0 = I["lg"] + e * I["r"], I["x"] + e * I["p"], I["s0"] + e * I["s"]
        h, s1, dlg, dx, ds0 = torch.empty_like(x), torch.empty_like(s0), torch.empty_like(x), torch.empty_like(x), torch.empty_like(s0)
        P.gscan_fwd(lg, x, h, s0, s1, I["lengths"])
        P.gscan_bwd(I["dh"], lg, x, dlg, dx, s0, I["ds1"], ds0, I["lengths"])
        value = (h.double() * I["dh"].double()).sum() + (s1.double() * I["ds1"].double()).sum()
        return value, [t.double() for t in (dlg, dx, ds0, h, s1)]

    got, d = _run(I), 2.0 ** -10
    (v2, g2), (v1, g1), (w1, k1), (w2, k2) = (at(e) for e in (2 * d, d, -d, -2 * d))
    slope = float((8 * (v1 - w1) - (v2 - w2)) / (12 * d))
    _, (dlg, dx, ds0, _, _) = at(0.0)
    live = torch.arange(150, device="cuda")[None, :, None] < I["lengths"][:, None, None]
    along = sum(float((torch.where(live, a, 0.0) * b.double()).sum()) for a, b in ((dlg, I["r"]), (dx, I["p"]))) + float((ds0 * I["s"].double()).sum())
    size = float(sum(torch.where(live, a * b.double(), 0.0).square().sum() for a, b in ((dlg, I["r"]), (dx, I["p"]))).sqrt())
    assert abs(slope - along) <= 1e-3 * size  # d^4 of the fifth derivative, 2^-24 / d of the values
    # <r, dlog_gate> + <p, dx> + <s, dstate> has the second operator's results as its gradient: symmetric in the inputs, so these
    # are the differences of the gradient along (r, p, s)
    names = ("out_lg", "out_x", "out_s0", "out_dh", "out_ds1")
    for k, a2, a1, b1, b2 in zip(names, g2, g1, k1, k2):
        assert_close(got[k], (8 * (a1 - b1) - (a2 - b2)) / (12 * d), 2e-3, k)


def test_streams_workspaces_and_repeats():
    import paper_2211_06934_amd as P
    I = {k: None if v is None else v.cuda() for k, v in _inputs(2, 1900, 300, torch.bfloat16).items()}
    ref = _run(I)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for st in streams:
        with torch.cuda.stream(st):
            got.append(_run(I))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(g[k], ref[k]) for k in ref)
    need = P.gscan_workspace(2, 1900, 300, torch.bfloat16)
    assert need > 0
    h, ws = torch.empty_like(I["x"]), torch.full((need // 4,), math.nan, device="cuda").view(torch.uint8)
    P.gscan_fwd(I["lg"], I["x"], h, I["s0"], None, I["lengths"], workspace=ws, stream=torch.cuda.current_stream())
    assert torch.equal(h, ref["h"])
    with pytest.raises(ValueError, match="workspace"):
        P.gscan_fwd(I["lg"], I["x"], h, I["s0"], None, I["lengths"], workspace=ws[:-1])


def test_captured_and_replayed():
    import paper_2211_06934_amd as P
    I = {k: None if v is None else v.cuda() for k, v in _inputs(2, 700, 130, torch.float32).items()}
    x, lg, state, n = I["x"], I["lg"], I["s0"].clone(), I["lengths"]
    h, dlg, dx = (torch.empty_like(x) for _ in range(3))
    one, out = torch.empty(2, 130, device="cuda"), torch.empty(2, 130, device="cuda")
    ws = torch.empty(P.gscan_workspace(2, 700, 130, torch.float32, 1), dtype=torch.uint8, device="cuda")

    def step():
        P.gscan_fwd(lg, x, h, state, one, n, workspace=ws)
        P.gscan_bwd(I["dh"], lg, x, dlg, dx, state, None, None, n, workspace=ws)
        P.gscan_step(lg[:, 0], x[:, 0], state, out)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    state.copy_(I["s0"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    state.copy_(I["s0"])
    for _ in range(3):
        before = state.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (h, one, dlg, dx, out, state)]
        state.copy_(before)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (h, one, dlg, dx, out, state)))
        x.mul_(0.5)


def test_refusals():
    import paper_2211_06934_amd as P
    x, s = torch.randn(2, 5, 8, device="cuda"), torch.randn(2, 8, device="cuda")
    h, n = torch.empty_like(x), torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    for bad, err, word in (((x, x, x), P.DiffoptError, "h must not be"), ((x.half(), x, h), ValueError, "log_gate"), ((x, x.half(), h), ValueError, "float16"),
                           ((x[:, :4], x, h), ValueError, "log_gate"), ((x, x, h[:1].expand(2, -1, -1)), ValueError, "overlap"),
                           ((x, x.transpose(1, 2).contiguous().transpose(1, 2), h), ValueError, "contiguous"), ((x, x[0], h), ValueError, "3 axes"),
                           ((x, x.cpu(), h), ValueError, "device memory"), ((None, x, h), TypeError, "log_gate"),
                           ((x, x, h, s[:1]), ValueError, "state"), ((x, x, h, s.bfloat16()), ValueError, "state"),
                           ((x, x, h, None, None, n.long()), ValueError, "lengths"), ((x, x, h, None, None, n[:1]), ValueError, "lengths")):
        with pytest.raises(err, match=word):
            P.gscan_fwd(*bad)
    with pytest.raises(P.DiffoptError, match="dstate must lie apart"):
        P.gscan_bwd(x, x, x, h, torch.empty_like(x), s, None, s)
    with pytest.raises(P.DiffoptError, match="dx must not be dlog_gate"):
        P.gscan_bwd(x, x, x, h, h)
    with pytest.raises(P.DiffoptError, match="out"):
        P.gscan_step(x[:, 0], x[:, 0], s, x[:, 0])
    with pytest.raises(ValueError, match="state"):
        P.gscan_step(x[:, 0], x[:, 0], s.t().contiguous().t(), h[:, 0])
