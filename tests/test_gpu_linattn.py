"""Linear attention with a decay per head: forward, gradients and single tokens
against the recurrence in fp64, at the sizes and values where it can go wrong."""
import math

import pytest
import torch

from lm_reference import F32, assert_close, linattn, tol

pytestmark = pytest.mark.gpu


def _inputs(B, T, H, Hk, Dk, Dv, dtype, seed=0, decays=None):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q, k, v, do = (r(B, T, h, d).to(dtype) for h, d in ((H, Dk), (Hk, Dk), (Hk, Dv), (H, Dv)))
    lg = torch.log1p(-torch.exp2(-1.0 - 8.0 * torch.rand(Hk, generator=g))) if decays is None else torch.tensor(decays)
    return q, k, v, do, lg, r(B, Hk, Dk, Dv), r(B, Hk, Dk, Dv)


def _check(q, k, v, do, lg, s0, ds1, lengths=None, scale=None, warm=True, wrap=lambda x: x.cuda()):
    """One call of the forward and of the backward against the reference and its autograd."""
    import paper_2211_06934_amd as P
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    B, T, H, Dk = q.shape
    Hk, Dv = k.shape[2], v.shape[3]
    ref = [x.double().requires_grad_() for x in (q, k, v)] + ([s0.double().requires_grad_()] if warm else [])
    out, s1 = linattn(*ref[:3], lg, ref[3] if warm else None, lengths, scale)
    grads = torch.autograd.grad((out, s1), ref, (do.double(), ds1.double() if warm else torch.zeros_like(s1)), allow_unused=True)
    grads = [torch.zeros_like(x) if g is None else g for x, g in zip(ref, grads)]
    dev = [wrap(x) for x in (q, k, v, do)]
    lgd, n = lg.cuda(), None if lengths is None else lengths.to(torch.int32).cuda()
    nan = lambda *s, dt=q.dtype: torch.full(s, math.nan, dtype=dt, device="cuda")  # noqa: E731
    o, so = nan(B, T, H, Dv), nan(B, Hk, Dk, Dv, dt=torch.float32)
    d_s0, d_ds1 = (s0.cuda(), ds1.cuda()) if warm else (None, None)
    P.linattn_fwd(*dev[:3], lgd, o, state=d_s0, state_out=so, lengths=n, scale=scale)
    b = tol(q.dtype, products=True)
    assert_close(o, out, b, "out")
    assert_close(so, s1, F32, "state_out")
    dq, dk, dv, ds0 = nan(B, T, H, Dk), nan(B, T, Hk, Dk), nan(B, T, Hk, Dv), nan(B, Hk, Dk, Dv, dt=torch.float32)
    P.linattn_bwd(dev[3], *dev[:3], lgd, dq, dk, dv, state=d_s0, dstate_out=d_ds1, dstate=ds0, lengths=n, scale=scale)
    for got, r, what in zip((dq, dk, dv), grads, ("dq", "dk", "dv")):
        assert_close(got, r, b, what)
    if warm:
        assert_close(ds0, grads[3], F32, "dstate")
    # without a final state, each result alone: the same values
    o2, dk2 = nan(B, T, H, Dv), nan(B, T, Hk, Dk)
    P.linattn_fwd(*dev[:3], lgd, o2, state=d_s0, lengths=n, scale=scale)
    assert_close(o2, out, b, "out alone")
    P.linattn_bwd(dev[3], *dev[:3], lgd, None, dk2, None, state=d_s0, dstate_out=d_ds1, lengths=n, scale=scale)
    assert_close(dk2, grads[1], b, "dk alone")
    return o, so


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 200, 321])
def test_lengths(T, dtype):
    _check(*_inputs(2, T, 2, 2, 32, 32, dtype, seed=T))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Dk,Dv", [(1, 1), (3, 5), (8, 16), (16, 64), (40, 40), (64, 128), (100, 36), (128, 128), (130, 70), (256, 32),
                                   (32, 256), (200, 256)])
def test_widths(Dk, Dv, dtype):
    _check(*_inputs(1, 77, 2, 1, Dk, Dv, dtype, seed=Dk + Dv))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 4), (4, 2), (6, 2), (8, 1), (5, 1)])
def test_shared_heads(H, Hk, dtype):
    _check(*_inputs(2, 90, H, Hk, 32, 64, dtype, seed=H * 10 + Hk))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [70, 300])
def test_padded_sequences(T, dtype):
    # lengths of zero and one, whole, ends inside and at tiles; what lies beyond is not read
    n = torch.tensor([0, 1, T, 64, 65, 63, T - 1, 17])
    q, k, v, do, lg, s0, ds1 = _inputs(8, T, 2, 2, 32, 32, dtype, seed=5)
    clean = [x.clone() for x in (q, k, v, do)]
    for b in range(8):
        for i, x in enumerate((q, k, v, do)):
            x[b, n[b]:] = math.nan if i % 2 else math.inf
            clean[i][b, n[b]:] = 0.0
    import paper_2211_06934_amd as P
    scale = 0.25
    ref = [x.double().requires_grad_() for x in clean[:3]]
    out, s1 = linattn(*ref, lg, s0, n, scale)
    grads = torch.autograd.grad((out, s1), ref, (clean[3].double(), ds1.double()))
    o = torch.full(do.shape, math.nan, dtype=dtype, device="cuda")
    so = torch.empty(s0.shape, device="cuda")
    dev, lens = [x.cuda() for x in (q, k, v, do)], n.to(torch.int32).cuda()
    P.linattn_fwd(*dev[:3], lg.cuda(), o, state=s0.cuda(), state_out=so, lengths=lens, scale=scale)
    b = tol(dtype, products=True)
    assert_close(o, out, b, "out")
    assert_close(so, s1, F32, "state_out")
    assert torch.equal(so[0].cpu(), s0[0])  # no token: the state as it was
    got = [torch.full(x.shape, math.nan, dtype=dtype, device="cuda") for x in clean[:3]]
    P.linattn_bwd(dev[3], *dev[:3], lg.cuda(), *got, state=s0.cuda(), dstate_out=ds1.cuda(), lengths=lens, scale=scale)
    for x, r, what in zip(got, grads, ("dq", "dk", "dv")):
        assert_close(x, r, b, what)
        for i in range(8):
            assert not x[i, n[i]:].any(), (what, i)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decays_at_their_ends(dtype):
    # no decay, decay to nothing at once, so strong that powers underflow, and so weak that its rounding would show
    _check(*_inputs(1, 333, 5, 5, 32, 32, dtype, seed=3, decays=[0.0, -math.inf, -40.0, -1e-3, -1.0]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,Dk,Dv", [(1100, 64, 64), (2500, 32, 32), (1500, 128, 128)])
def test_long_sequences(T, Dk, Dv, dtype):
    # one head alone, so that the tokens have to be split over the card
    _check(*_inputs(1, T, 1, 1, Dk, Dv, dtype, seed=T))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decay_is_not_rounded_along_the_way(dtype):
    # a state carried over 20,000 tokens that add nothing: g^20000 to fp32's accuracy, not 20,000 roundings of g
    import paper_2211_06934_amd as P
    T, lg = 20000, torch.tensor([-1.0 / 8000, -1e-5], dtype=torch.float32)
    z = torch.zeros(1, T, 2, 32, dtype=dtype, device="cuda")
    s0 = torch.randn(1, 2, 32, 32, generator=torch.Generator().manual_seed(1))
    so, o = torch.empty(1, 2, 32, 32, device="cuda"), torch.empty_like(z)
    P.linattn_fwd(z, z, z, lg.cuda(), o, state=s0.cuda(), state_out=so)
    ref = s0.double() * torch.exp(lg.double() * T)[None, :, None, None]
    assert float((so.double().cpu() - ref).norm() / ref.norm()) < 2e-6


def _strided(kind):
    def wrap(x):
        B, T, H, D = x.shape
        if kind == "heads first":
            return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
        if kind == "odd rows":  # rows of odd length at an odd offset: no wide access is aligned
            buf = torch.zeros(B, T, H * (D + 1) + 3, dtype=x.dtype, device="cuda")
            y = buf.as_strided((B, T, H, D), (buf.stride(0), buf.stride(1), D + 1, 1), 1)
            return y.copy_(x)
        if kind == "time first":
            return x.permute(1, 0, 2, 3).contiguous().cuda().permute(1, 0, 2, 3)
        raise AssertionError(kind)
    return wrap


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["heads first", "odd rows", "time first"])
@pytest.mark.parametrize("D", [32, 33, 64])
def test_strides(kind, D, dtype):
    _check(*_inputs(2, 100, 2, 2, D, D, dtype, seed=7), wrap=_strided(kind))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_broadcast_inputs_and_strided_results(dtype):
    import paper_2211_06934_amd as P
    q, k, v, do, lg, s0, _ = _inputs(3, 70, 2, 2, 32, 32, dtype, seed=11)
    one = k[:1].cuda().expand(3, -1, -1, -1)  # keys shared by the batch: stride 0
    out, _ = linattn(q, k[:1].expand(3, -1, -1, -1), v, lg)
    both = torch.full((3, 70, 4, 32), math.nan, dtype=dtype, device="cuda")
    P.linattn_fwd(q.cuda(), one, v.cuda(), lg.cuda(), both[:, :, 1:3])
    assert_close(both[:, :, 1:3], out, tol(dtype, products=True))
    assert torch.isnan(both[:, :, 0]).all() and torch.isnan(both[:, :, 3]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nan_and_inf_stay_in_their_head(dtype):
    import paper_2211_06934_amd as P
    q, k, v, do, lg, _, _ = _inputs(1, 150, 3, 3, 32, 32, dtype, seed=2)
    v[0, 100, 1, 4] = math.inf
    q[0, 50, 2, 0] = math.nan
    out = torch.empty(1, 150, 3, 32, dtype=dtype, device="cuda")
    P.linattn_fwd(q.cuda(), k.cuda(), v.cuda(), lg.cuda(), out)
    ref, _ = linattn(q, k, v, lg)
    assert torch.isfinite(out[:, :, 0]).all()
    bad = ~torch.isfinite(out[0, :, 1]).cpu()
    assert not bad[:100].any() and bad[100, 4]  # nothing before the token is touched
    assert torch.isnan(out[0, 50, 2]).all() and torch.isfinite(out[0, :50, 2]).all() and torch.isfinite(out[0, 51:, 2]).all()
    assert_close(out[:, :100], torch.where(torch.isnan(ref[:, :100]), ref[:, :100], ref[:, :100]), tol(dtype, products=True))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,H,Hk,Dk,Dv", [(1, 1, 1, 1, 1), (1, 4, 4, 64, 64), (3, 8, 2, 128, 128), (2, 6, 3, 100, 36), (5, 2, 2, 256, 256),
                                          (70, 4, 4, 32, 32), (1, 16, 1, 128, 64), (2, 3, 3, 33, 130)])
def test_single_tokens_continue_a_prompt(B, H, Hk, Dk, Dv, dtype):
    import paper_2211_06934_amd as P
    q, k, v, do, lg, s0, _ = _inputs(B, 4, H, Hk, Dk, Dv, dtype, seed=B + Dk)
    ref, s1 = linattn(q, k, v, lg, s0, None, 0.5)
    state = s0.cuda()
    for t in range(4):
        out = torch.full((B, H, Dv), math.nan, dtype=dtype, device="cuda")
        P.linattn_step(q[:, t].cuda(), k[:, t].cuda(), v[:, t].cuda(), lg.cuda(), state, out, scale=0.5)
        assert_close(out, ref[:, t], tol(dtype), "token %d" % t)
    assert_close(state, s1, F32, "state")


def test_single_token_strides():
    import paper_2211_06934_amd as P
    q, k, v, do, lg, s0, _ = _inputs(3, 2, 4, 2, 64, 64, torch.bfloat16, seed=8)
    qkv = torch.cat([x[:, 1].reshape(3, -1) for x in (q, k, v)], 1).cuda()  # one projection's output
    cut = qkv.split([256, 128, 128], 1)
    views = [c.unflatten(1, (-1, 64)) for c in cut]
    ref, s1 = linattn(q[:, 1:], k[:, 1:], v[:, 1:], lg, s0)
    out, state = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda"), s0.cuda()
    P.linattn_step(*views, lg.cuda(), state, out)
    assert_close(out, ref[:, 0], tol(torch.bfloat16))
    assert_close(state, s1, F32)


@pytest.mark.parametrize("shape", [(0, 5, 2, 2), (2, 0, 2, 2)])
def test_empty(shape):
    import paper_2211_06934_amd as P
    B, T, H, Hk = shape
    q, k, v, do, lg, s0, ds1 = (x.cuda() for x in _inputs(B, T, H, Hk, 32, 32, torch.float32))
    so, out = torch.full_like(s0, math.nan), torch.empty_like(do)
    P.linattn_fwd(q, k, v, lg, out, state=s0, state_out=so)
    assert torch.equal(so, s0)
    ds0 = torch.full_like(s0, math.nan)
    P.linattn_bwd(do, q, k, v, lg, torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), state=s0, dstate_out=ds1, dstate=ds0)
    assert torch.equal(ds0, ds1)


def test_gradient_against_differences():
    # the directional derivative of the operator itself, by central differences of fp32 results of a loss summed in fp64
    import paper_2211_06934_amd as P
    q, k, v, do, lg, s0, _ = (x.cuda() for x in _inputs(1, 80, 2, 1, 16, 16, torch.float32, seed=4))
    gen = torch.Generator(device="cuda").manual_seed(9)
    d = [torch.randn(x.shape, device="cuda", generator=gen) for x in (q, k, v, s0)]

    def loss(e):
        out = torch.empty_like(do)
        P.linattn_fwd(q + e * d[0], k + e * d[1], v + e * d[2], lg, out, state=s0 + e * d[3])
        return float((out.double() * do.double()).sum())

    g = [torch.empty_like(x) for x in (q, k, v, s0)]
    P.linattn_bwd(do, q, k, v, lg, *g[:3], state=s0, dstate=g[3])
    exact = sum(float((a.double() * b.double()).sum()) for a, b in zip(g, d))
    # the loss is cubic along the line: the difference is off by h^2 times the cubic term, and by 1e-7 |loss| / h
    h = 2.0 ** -7
    want = (8 * (loss(h) - loss(-h)) - (loss(2 * h) - loss(-2 * h))) / (12 * h)
    assert abs(want - exact) <= 1e-3 * abs(exact) + 1e-3 * sum(float((a * b).double().norm()) for a, b in zip(g, d))


def test_streams_and_repeats():
    # results do not depend on the stream or on earlier calls, bit for bit
    import paper_2211_06934_amd as P
    q, k, v, do, lg, s0, ds1 = (x.cuda() for x in _inputs(2, 700, 4, 2, 64, 64, torch.bfloat16, seed=6))

    def both():
        out, so = torch.empty_like(do), torch.empty_like(s0)
        g = [torch.empty_like(x) for x in (q, k, v, s0)]
        P.linattn_fwd(q, k, v, lg, out, state=s0, state_out=so)
        P.linattn_bwd(do, q, k, v, lg, *g[:3], state=s0, dstate_out=ds1, dstate=g[3])
        return [out, so, *g]

    ref = both()
    torch.cuda.synchronize()
    for _ in range(2):
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        with torch.cuda.stream(s1):
            a = both()
        with torch.cuda.stream(s2):
            b = both()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(ref, a, b))


def test_refusals():
    import paper_2211_06934_amd as P
    q, k, v, do, lg, s0, _ = (x.cuda() for x in _inputs(2, 8, 4, 2, 32, 32, torch.float32))
    out = torch.empty_like(do)
    ok = dict(state=s0)
    P.linattn_fwd(q, k, v, lg, out, **ok)
    for bad, err in (((q.half(), k, v, lg, out), ValueError), ((q, k.bfloat16(), v, lg, out), ValueError), ((q.cpu(), k, v, lg, out), ValueError),
                     ((q[:, :, :3], k, v, lg, out[:, :, :3]), P.DiffoptError), ((q, k[:, :7], v, lg, out), ValueError),
                     ((q.transpose(2, 3).contiguous().transpose(2, 3), k, v, lg, out), ValueError), ((q, k, v, lg[:1], out), ValueError),
                     ((q, k, v, lg, out[:1].expand(2, -1, -1, -1)), ValueError), ((q, k, v, lg.double(), out), ValueError),
                     ((None, k, v, lg, out), TypeError), ((q[0], k, v, lg, out), ValueError)):
        with pytest.raises(err):
            P.linattn_fwd(*bad, **ok)
    for kw, err in ((dict(state=s0[:1]), ValueError), (dict(state=s0.double()), ValueError), (dict(lengths=torch.zeros(2, device="cuda")), ValueError),
                    (dict(scale=math.inf), P.DiffoptError), (dict(state=s0.transpose(2, 3)), ValueError),
                    (dict(workspace=torch.zeros(4, device="cuda")), ValueError)):
        with pytest.raises(err):
            P.linattn_fwd(q, k, v, lg, out, **kw)
    with pytest.raises(P.DiffoptError, match="dstate"):
        P.linattn_bwd(do, q, k, v, lg, None, None, torch.empty_like(v), state=s0, dstate=s0)
    wide = torch.zeros(1, 1, 1, 257, device="cuda")
    with pytest.raises(P.DiffoptError, match="256"):
        P.linattn_fwd(wide, wide, wide, lg[:1], torch.empty_like(wide))
    with pytest.raises(ValueError):
        P.linattn_step(q[:, 0], k[:, 0], v[:, 0], lg, s0[:1], out[:, 0])
    with pytest.raises(ValueError):
        P.linattn_workspace(1, 1, 3, 2, 32, 32)
