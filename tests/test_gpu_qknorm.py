"""Norms of queries and keys with the rotation: forward, VJP and the VJP's own
VJP against autograd of the definition in fp64."""
import math

import pytest
import torch

from lm_reference import F32, assert_close, qknorm_rope, tol

pytestmark = pytest.mark.gpu


def _tables(rows, rot):
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * torch.pow(torch.tensor(10000.0, dtype=torch.float64),
                                                                       -torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    return angle.cos().float(), angle.sin().float()


def _check(B, T, H, Hk, D, rot, dtype, interleaved=False, places=None, weights=True, first=0, seed=0, wrap=lambda x: x.cuda(), eps=1e-6):
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    heads = {"q": H, "k": Hk}
    x = {n: (1.5 * r(B, T, h, D)).to(dtype) for n, h in heads.items()}
    dy, a = ({n: r(B, T, h, D).to(dtype) for n, h in heads.items()} for _ in range(2))
    w = {n: 1.0 + 0.2 * r(D) if weights else None for n in heads}
    b = {n: 0.3 * r(D) for n in heads}
    rows = max(T + first, 50)
    cos, sin = _tables(rows, rot) if rot else (None, None)
    where = torch.arange(T).expand(B, T) + first
    if places is not None:
        where = torch.randint(0, rows, (B, T), generator=gen)
    pos = None if places is None else where.to(places).cuda()
    dev = lambda d: {n: None if t is None else t.cuda() for n, t in d.items()}  # noqa: E731
    X, DY, A = ({n: wrap(t) for n, t in d.items()} for d in (x, dy, a))
    W, Bw = dev(w), dev(b)
    C, S = (None, None) if cos is None else (cos.cuda(), sin.cuda())
    kw = dict(positions=pos, first=first, eps=eps, interleaved=interleaved)
    nan = lambda n: torch.full((B, T, heads[n], D), math.nan, dtype=dtype, device="cuda")  # noqa: E731
    wnan = lambda: torch.full((D,), math.nan, device="cuda")  # noqa: E731
    Y, DX, O1, O2 = ({n: nan(n) for n in heads} for _ in range(4))
    DW, OW = ({n: wnan() for n in heads} for _ in range(2))
    P.qknorm_rope_fwd(X["q"], X["k"], W["q"], W["k"], C, S, Y["q"], Y["k"], **kw)
    P.qknorm_rope_bwd(DY["q"], DY["k"], X["q"], X["k"], W["q"], W["k"], C, S, DX["q"], DX["k"], DW["q"], DW["k"], **kw)
    P.qknorm_rope_bwd_bwd(A["q"], A["k"], Bw["q"], Bw["k"], DY["q"], DY["k"], X["q"], X["k"], W["q"], W["k"], C, S, O1["q"], O1["k"],
                          O2["q"], O2["k"], OW["q"], OW["k"], **kw)
    t = tol(dtype)
    for n in heads:
        xr, dyr = x[n].double().requires_grad_(), dy[n].double().requires_grad_()
        wr = (torch.ones(D) if w[n] is None else w[n]).double().requires_grad_()
        y = qknorm_rope(xr, wr, cos, sin, where, eps, interleaved)
        assert_close(Y[n], y, t, n)
        if heads[n] == 0 or B * T == 0:
            assert not DW[n].any() and not OW[n].any()
            continue
        dx, dw = torch.autograd.grad(y, (xr, wr), dyr, create_graph=True)
        assert_close(DX[n], dx, t, "d" + n)
        assert_close(DW[n], dw, F32, "d%s_weight" % n)
        second = torch.autograd.grad((dx, dw), (dyr, xr, wr), (a[n].double(), b[n].double()))
        for got, ref, what, bound in zip((O1[n], O2[n], OW[n]), second, ("dy", "x", "w"), (t, t, F32)):
            assert_close(got, ref, bound, "second %s %s" % (n, what))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(2, 2), (3, 2), (8, 8), (16, 4), (32, 32), (64, 32), (64, 64), (80, 80), (96, 96), (100, 50), (128, 128),
                                   (128, 0), (129, 128), (200, 64), (256, 256), (384, 384), (1000, 500), (1024, 1024)])
def test_widths(D, rot, interleaved, dtype):
    _check(2, 5, 4, 2, D, rot, dtype, interleaved=interleaved, seed=D + rot)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,H,Hk", [(1, 1, 1, 1), (1, 1, 16, 4), (3, 1, 5, 1), (2, 77, 8, 8), (1, 700, 3, 1), (4, 33, 1, 0), (40, 60, 6, 2)])
def test_shapes(B, T, H, Hk, dtype):
    _check(B, T, H, Hk, 64, 64, dtype, seed=T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("places", [torch.int32, torch.int64])
def test_positions(places, dtype):
    _check(3, 40, 4, 2, 64, 64, dtype, places=places)


@pytest.mark.parametrize("weights,first,eps", [(False, 0, 1e-6), (True, 17, 1e-6), (True, 0, 0.0), (True, 3, 0.5)])
def test_options(weights, first, eps):
    _check(2, 20, 4, 2, 128, 128, torch.float32, weights=weights, first=first, eps=eps)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D,rot", [(64, 64), (33, 32), (128, 64)])
@pytest.mark.parametrize("kind", ["projection", "heads first", "odd rows"])
def test_strides(kind, D, rot, dtype):
    def wrap(x):
        B, T, H, D = x.shape
        if kind == "projection":
            buf = torch.zeros(B, T, H + 3, D, dtype=x.dtype, device="cuda")
            return buf[:, :, 2:2 + H].copy_(x)
        if kind == "heads first":
            return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
        buf = torch.zeros(B, T, H * (D + 1) + 3, dtype=x.dtype, device="cuda")
        return buf.as_strided((B, T, H, D), (buf.stride(0), buf.stride(1), D + 1, 1), 1).copy_(x)
    _check(2, 30, 4, 2, D, rot, dtype, wrap=wrap)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place_and_some_results(dtype):
    import paper_2211_06934_amd as P
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, dq, dk = (torch.randn(2, 9, h, 64, device="cuda", generator=gen).to(dtype) for h in (4, 2, 4, 2))
    w = torch.randn(64, device="cuda", generator=gen)
    c, s = (t.cuda() for t in _tables(9, 64))
    y, g = [torch.empty_like(q), torch.empty_like(k)], [torch.empty_like(q), torch.empty_like(k)]
    P.qknorm_rope_fwd(q, k, w, None, c, s, *y)
    dw = torch.empty(64, device="cuda")
    P.qknorm_rope_bwd(dq, dk, q, k, w, None, c, s, *g, dw)
    a, b = dq.clone(), dk.clone()
    P.qknorm_rope_bwd(a, b, q, k, w, None, c, s, a, b)
    assert torch.equal(a, g[0]) and torch.equal(b, g[1])
    q2, k2 = q.clone(), k.clone()
    P.qknorm_rope_fwd(q2, k2, w, None, c, s, q2, k2)
    assert torch.equal(q2, y[0]) and torch.equal(k2, y[1])
    z = torch.empty_like(q), torch.empty_like(k)
    x = torch.empty_like(q), torch.empty_like(k)
    zero = torch.zeros_like(q), torch.zeros_like(k)
    P.qknorm_rope_bwd_bwd(None, None, w, None, dq, dk, q, k, w, None, c, s, *z, *x)
    z2, x2 = (tuple(torch.empty_like(t) for t in zero) for _ in range(2))
    P.qknorm_rope_bwd_bwd(*zero, w, torch.zeros_like(w), dq, dk, q, k, w, torch.ones_like(w), c, s, *z2, *x2)
    assert all(torch.equal(m, n) for m, n in zip(z + x, z2 + x2))


def test_zero_rows_large_values_and_unknown_positions():
    import paper_2211_06934_amd as P
    c, s = (t.cuda() for t in _tables(10, 64))
    q = torch.zeros(1, 4, 2, 64, device="cuda")
    q[0, 1] = 1e18  # the mean square stays finite in fp32
    q[0, 2, 0, 3] = math.inf
    out = torch.empty_like(q)
    pos = torch.tensor([[0, 1, 2, 3]], device="cuda", dtype=torch.int32)
    P.qknorm_rope_fwd(q, None, None, None, c, s, out, None, positions=pos)
    assert not out[0, 0].any() and torch.isfinite(out[0, 1]).all() and torch.isfinite(out[0, 2, 1]).all() and torch.isnan(out[0, 2, 0]).any()
    for bad in (-1, 10, 2 ** 31 - 1):  # outside the table: that token alone is NaN, nothing else is read
        x = torch.randn(1, 4, 2, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
        pos[0, 2] = bad
        P.qknorm_rope_fwd(x, None, None, None, c, s, out, None, positions=pos)
        assert torch.isnan(out[0, 2]).all() and torch.isfinite(out[0, [0, 1, 3]]).all()


def test_refusals():
    import paper_2211_06934_amd as P
    q, k = torch.randn(2, 6, 4, 64, device="cuda"), torch.randn(2, 6, 2, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    c, s = (t.cuda() for t in _tables(6, 64))
    y = torch.empty_like(q), torch.empty_like(k)
    P.qknorm_rope_fwd(q, k, w, w, c, s, *y)
    for bad, kw, err in (((q, k, w[:3], w, c, s, *y), {}, ValueError), ((q, k, w, w, c[:5], s[:5], *y), {}, P.DiffoptError),
                         ((q, k, w, w, c, s, *y), dict(first=1), P.DiffoptError), ((q, k, w, w, c, s[:, :3], *y), {}, ValueError),
                         ((q, k.bfloat16(), w, w, c, s, *y), {}, ValueError), ((q.half(), k, w, w, c, s, *y), {}, ValueError),
                         ((q, k, w, w, c, s, *y), dict(eps=-1.0), P.DiffoptError), ((q, k, w, w, c, s, y[0][:1].expand(2, -1, -1, -1), y[1]), {}, ValueError),
                         ((q, k, w, w, c, s, *y), dict(positions=torch.zeros(2, 6, device="cuda")), ValueError),
                         ((q, k, w, w, c, s, *y), dict(positions=torch.zeros(2, 5, device="cuda", dtype=torch.int32)), ValueError),
                         ((q, k, w, w, torch.zeros(6, 40, device="cuda"), torch.zeros(6, 40, device="cuda"), *y), {}, P.DiffoptError),
                         ((q, None, w, w, c, s, y[0], None), dict(eps=math.nan), P.DiffoptError), ((q, k, w, w, c, None, *y), {}, TypeError)):
        with pytest.raises(err):
            P.qknorm_rope_fwd(*bad, **kw)
    with pytest.raises(ValueError, match="workspace"):
        P.qknorm_rope_bwd(*y, q, k, w, w, c, s, *y, w.clone(), None, workspace=torch.zeros(3, dtype=torch.uint8, device="cuda"))
