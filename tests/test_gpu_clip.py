"""The global norm of a gradient and clipping to it, over buffers and trees,
against fp64 autograd of the definition; inside the meta-optimizers."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

# The norm is a sum in fp64, rounded once: 2^-24 of it.  c is rounded once and
# multiplies a gradient with one more rounding: 2^-23 of each element.  The
# gradient's gradient is c dout + s grad with c, s and the two terms rounded
# once each: 3 * 2^-24 of the sum of the two terms' sizes; s itself is a
# difference of dnorm and c <dout, grad> / (norm + eps), known to 2^-23 of the
# two (c and the norm it takes are rounded).
E24 = 2.0 ** -24


def _numbers(shapes, seed, norm, offset=0):
    """Leaves of these shapes (offset elements into their buffers) with about this global norm."""
    gen = torch.Generator().manual_seed(seed)
    n = max(1, sum(math.prod(s) for s in shapes))
    return [torch.randn(s, generator=gen) * (norm / math.sqrt(n)) for s in shapes]


def _place(x, offset):
    buf = torch.full((x.numel() + offset + 5,), math.nan, device="cuda")
    return buf[offset:offset + x.numel()].view(x.shape).copy_(x)


def _reference(g, dout, dnorm, max_norm, eps):
    """fp64: norm, c, out, dgrad and the sizes of dgrad's terms."""
    flat = torch.cat([x.reshape(-1).double() for x in g])
    norm = flat.norm()
    c = torch.clamp(max_norm / (norm + eps), max=1.0) if float(norm + eps) > 0 else torch.ones((), dtype=torch.float64)
    d = torch.cat([x.reshape(-1).double() for x in dout])
    dot = (flat * d).sum()
    if float(norm) == 0:
        slope = slope_size = torch.zeros((), dtype=torch.float64)
    else:
        pull = c * dot / (norm + eps) if float(c) < 1 else torch.zeros((), dtype=torch.float64)
        slope, slope_size = (dnorm.double() - pull) / norm, (dnorm.double().abs() + pull.abs()) / norm
    return norm, c, c * flat, c * d + slope * flat, (c * d).abs() + (slope_size * flat).abs()


def _run(g, dout, dnorm, max_norm, eps, flat, offset, alias=False):
    import paper_2211_06934_amd as P
    G, D = ([_place(x, offset + i) for i, x in enumerate(t)] for t in (g, dout))
    new = lambda t: [_place(torch.full_like(x, math.nan), (offset + 2 * i) % 7) for i, x in enumerate(t)]  # noqa: E731
    stats, dn = torch.full((2,), math.nan, device="cuda"), dnorm.cuda()
    if flat:
        out = [G[0].clone()] if alias else new(g)
        P.clip_norm_fwd(out[0] if alias else G[0], max_norm, out[0], stats, eps)
        dg = [D[0].clone()] if alias else new(g)
        P.clip_norm_bwd(dg[0] if alias else D[0], dn, G[0], stats, dg[0], eps)
        return stats, out, dg
    table = P.segtable_create([x.numel() for x in g])
    ptr = lambda t: P.tree.leaf_pointer_tensor(t, "cuda")  # noqa: E731
    out = [x.clone() for x in G] if alias else new(g)
    at = ptr(out)
    P.clip_norm_fwd_tree(table, at if alias else ptr(G), max_norm, at, stats, eps)
    dg = [x.clone() for x in D] if alias else new(g)
    at = ptr(dg)
    P.clip_norm_bwd_tree(table, at if alias else ptr(D), dn, ptr(G), stats, at, eps)
    torch.cuda.synchronize()
    return stats, out, dg


def _check(shapes, norm=3.0, max_norm=1.0, eps=1e-6, seed=0, flat=False, offset=0, alias=False):
    g, dout = _numbers(shapes, seed, norm), _numbers(shapes, seed + 1, 1.0)
    dnorm = torch.tensor([0.7])
    stats, out, dg = _run(g, dout, dnorm, max_norm, eps, flat, offset, alias)
    n, c, o, d, size = _reference(g, dout, dnorm, max_norm, eps)
    assert abs(float(stats[0]) - float(n)) <= E24 * float(n)
    assert abs(float(stats[1]) - float(c)) <= E24 * float(c)
    got = torch.cat([x.reshape(-1).double().cpu() for x in out])
    assert bool(((got - o).abs() <= 2 * E24 * o.abs() + 2.0 ** -149).all())
    got = torch.cat([x.reshape(-1).double().cpu() for x in dg])
    assert bool(((got - d).abs() <= 8 * E24 * size + 2.0 ** -149).all())


_SIZES = [1, 2, 3, 4, 5, 31, 1000, 1761, 8191, 8192, 8193, 8200, 20001, 100_003, 3_000_001]


@pytest.mark.parametrize("n", _SIZES)
@pytest.mark.parametrize("offset", [0, 1, 6])
def test_buffers(n, offset):
    _check([(n,)], flat=True, offset=offset, seed=n)


@pytest.mark.parametrize("n", [7, 9000, 200_003])
@pytest.mark.parametrize("norm,max_norm,eps", [(0.4, 1.0, 1e-6), (3.0, 1.0, 0.0), (1e-3, 1e-3, 1e-4), (3.0, 0.0, 1e-6), (3.0, math.inf, 1e-6), (1e-30, 1e-31, 0.0),
                                               (1e25, 1.0, 1e-6)])
def test_norms(n, norm, max_norm, eps):
    # squares that fp32 does not hold among them
    _check([(n,)], norm, max_norm, eps, flat=True)
    _check([(n // 3, 2), (n - n // 3 * 2,)], norm, max_norm, eps)


def _many(count, hi, seed):
    gen = torch.Generator().manual_seed(seed)
    return [(int(s),) for s in torch.exp(torch.rand(count, generator=gen) * math.log(hi)).round()]


_TREES = {
    "one": [(5,)], "tiny MLP": [(40, 1), (40,), (40, 40), (40,), (1, 40), (1,)], "scalars": [()] * 40, "threes": [(3,)] * 700,
    "empty among them": [(0,), (7,), (0, 3), (9000,), (0,)], "one large": [(300_007,)], "two large": [(70_001, 3), (13, 7001)],
    "small": _many(300, 60, 1), "mixed": _many(400, 20_000, 2), "32 leaves": [(300,)] * 32, "33 leaves": [(300,)] * 33,
    "at tiles' ends": [(2016,), (2015,), (1,), (2017,), (4064,), (2048,), (1,)], "all at once": _many(60, 100_000, 3) + [(1,)] * 40 + [(2,), (3,), (4,), (5,)],
}


@pytest.mark.parametrize("alias", [False, True])
@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("name", sorted(_TREES))
def test_trees(name, offset, alias):
    _check(_TREES[name], offset=offset, alias=alias, seed=len(name))


@pytest.mark.parametrize("n", [100, 50_001])
@pytest.mark.parametrize("norm", [0.4, 3.0])
def test_in_place(n, norm):
    _check([(n,)], norm, flat=True, alias=True)
    _check([(n,), (n, 2)], norm, alias=True)


def test_many_tiles():
    # more tiles than the workgroups of sums take at once
    _check(_many(3000, 65_536, 5), seed=9)
    _check([(40_000_003,)], flat=True, offset=1)


@pytest.mark.parametrize("n", [50, 20_000])
def test_what_is_not_finite(n):
    import paper_2211_06934_amd as P
    for bad, want in ((math.inf, 0.0), (math.nan, math.nan)):
        g = torch.ones(n, device="cuda")
        g[n // 2] = bad
        out, stats = torch.empty_like(g), torch.empty(2, device="cuda")
        P.clip_norm_fwd(g, 1.0, out, stats)
        torch.cuda.synchronize()
        assert stats[0].isnan() if math.isnan(bad) else stats[0] == math.inf
        rest = torch.cat((out[:n // 2], out[n // 2 + 1:]))
        assert rest.isnan().all() if math.isnan(want) else not rest.any()
        assert out[n // 2].isnan()


@pytest.mark.parametrize("n", [50, 20_000])
def test_no_gradient_at_all(n):
    import paper_2211_06934_amd as P
    g, stats = torch.zeros(n, device="cuda"), torch.empty(2, device="cuda")
    out, d, dg = torch.full_like(g, 9.0), torch.randn(n, device="cuda"), torch.empty_like(g)
    for max_norm, eps in ((1.0, 1e-6), (0.0, 0.0), (1.0, 0.0)):
        P.clip_norm_fwd(g, max_norm, out, stats, eps)
        P.clip_norm_bwd(d, torch.ones(1, device="cuda"), g, stats, dg, eps)
        assert stats.tolist() == [0.0, 1.0] and not out.any() and torch.equal(dg, d)


@pytest.mark.parametrize("n", [50, 20_000])
def test_what_may_be_left_out(n):
    import paper_2211_06934_amd as P
    g, d = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    out, dn, zero = torch.empty_like(g), torch.tensor([0.3], device="cuda"), torch.zeros(1, device="cuda")
    stats, alone = torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    P.clip_norm_fwd(g, 1.0, out, stats)
    P.clip_norm_fwd(g, 1.0, None, alone)
    assert torch.equal(stats, alone)
    a, b = torch.empty_like(g), torch.empty_like(g)
    for pair in (((d, None), (d, zero)), ((None, dn), (torch.zeros_like(d), dn)), ((None, None), (torch.zeros_like(d), zero))):
        P.clip_norm_bwd(*pair[0], g, stats, a)
        P.clip_norm_bwd(*pair[1], g, stats, b)
        assert torch.equal(a, b)
    table = P.segtable_create([n])
    at = [P.tree.leaf_pointer_tensor([x], "cuda") for x in (g, out)]
    P.clip_norm_fwd_tree(table, at[0], 1.0, None, alone)
    assert float((stats - alone).abs().max()) <= 2 * E24 * float(stats.max())
    P.clip_norm_bwd_tree(table, None, dn, at[0], stats, at[1])
    P.clip_norm_bwd(None, dn, g, stats, a)
    assert torch.equal(a, out)


def test_nothing():
    import paper_2211_06934_amd as P
    e, stats = torch.empty(0, device="cuda"), torch.full((2,), 7.0, device="cuda")
    P.clip_norm_fwd(e, 1.0, e, stats)
    assert stats.tolist() == [0.0, 1.0]
    P.clip_norm_bwd(e, None, e, stats, e)
    table = P.segtable_create([0, 0])
    at = torch.zeros(2, dtype=torch.int64, device="cuda")
    stats.fill_(7.0)
    P.clip_norm_fwd_tree(table, at, 1.0, at, stats)
    assert stats.tolist() == [0.0, 1.0]
    P.clip_norm_bwd_tree(table, at, None, at, stats, at)


def test_gradient_against_differences():
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(3)
    g, d, v = (torch.randn(300, generator=gen, dtype=torch.float64) for _ in range(3))
    dn, stats, out = torch.tensor([0.7]), torch.empty(2, device="cuda"), torch.empty(300, device="cuda")

    def value(e):
        P.clip_norm_fwd((g + e * v).float().cuda(), 5.0, out, stats)
        return float((out.double().cpu() * d).sum() + 0.7 * stats[0].double().cpu())

    h, dg = 2.0 ** -7, torch.empty(300, device="cuda")
    slope = (8 * (value(h) - value(-h)) - (value(2 * h) - value(-2 * h))) / (12 * h)
    value(0.0)
    P.clip_norm_bwd(d.float().cuda(), dn.cuda(), g.float().cuda(), stats, dg)
    # 300 roundings of 2^-23 of the products over 12 h, and the inputs' own
    assert abs(slope - float((dg.double().cpu() * v).sum())) <= 2e-3


def test_streams_workspaces_and_repeats():
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(1)
    g, d = (torch.randn(1_000_003, generator=gen).cuda() for _ in range(2))
    dn = torch.ones(1, device="cuda")

    def run(**kw):
        stats, out, dg = torch.empty(2, device="cuda"), torch.empty_like(g), torch.empty_like(g)
        P.clip_norm_fwd(g, 1.0, out, stats, **kw)
        P.clip_norm_bwd(d, dn, g, stats, dg, **kw)
        return stats, out, dg

    ref = run()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    torch.cuda.synchronize()
    for st in streams:
        with torch.cuda.stream(st):
            got.append(run())
    torch.cuda.synchronize()
    ws = torch.full((P.clip_norm_workspace(1_000_003) // 4,), math.nan, device="cuda").view(torch.uint8)
    got.append(run(workspace=ws, stream=torch.cuda.current_stream()))
    for r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, ref))
    with pytest.raises(ValueError, match="workspace"):
        run(workspace=ws[:-8])


def test_captured_and_replayed():
    import paper_2211_06934_amd as P
    g = [torch.randn(50_001, device="cuda"), torch.randn(17, device="cuda")]
    d, out, dg = ([torch.randn_like(x) for x in g] for _ in range(3))
    table = P.segtable_create([x.numel() for x in g])
    at = [P.tree.leaf_pointer_tensor(t, "cuda") for t in (g, out, d, dg)]
    stats, dn, ws = torch.empty(2, device="cuda"), torch.ones(1, device="cuda"), torch.empty(P.clip_norm_workspace_tree(table), dtype=torch.uint8, device="cuda")

    def step():
        P.clip_norm_fwd_tree(table, at[0], 1.0, at[1], stats, workspace=ws)
        P.clip_norm_bwd_tree(table, at[2], dn, at[0], stats, at[3], workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (stats, *out, *dg)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (stats, *out, *dg)))
        g[0].mul_(0.1)


def test_clip_grad_norm_of_trees():
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(5)
    tree = {"w": torch.randn(30, 40, generator=gen).cuda().requires_grad_(True), "b": [torch.randn(7, generator=gen).cuda().requires_grad_(True), None]}
    clipped, norm = P.clip_grad_norm(tree, 2.0)
    assert set(clipped) == {"w", "b"} and clipped["b"][1] is None and norm.shape == ()
    cw, cb = torch.randn(30, 40, generator=gen).cuda(), torch.randn(7, generator=gen).cuda()
    got = torch.autograd.grad((clipped["w"] * cw).sum() + (clipped["b"][0] * cb).sum() + 0.5 * norm, [tree["w"], tree["b"][0]])
    leaves = [x.detach().double().cpu() for x in (tree["w"], tree["b"][0])]
    n, c, _, d, size = _reference(leaves, [cw.cpu(), cb.cpu()], torch.tensor(0.5), 2.0, 1e-6)
    assert abs(float(norm.detach()) - float(n)) <= E24 * float(n)
    flat = torch.cat([x.reshape(-1).double().cpu() for x in got])
    assert bool(((flat - d).abs() <= 8 * E24 * size).all())
    # one of the results alone
    (only,) = torch.autograd.grad(P.clip_grad_norm(tree, 2.0)[1], [tree["w"]])
    assert float((only.double().cpu() - leaves[0] / n).abs().max()) <= 4 * E24
    first, _ = P.clip_grad_norm(tree, 2.0)
    one = torch.autograd.grad(first["b"][0].sum(), [tree["w"], tree["b"][0]])
    _, _, _, d, size = _reference(leaves, [torch.zeros(30, 40), torch.ones(7)], torch.tensor(0.0), 2.0, 1e-6)
    assert bool(((torch.cat([x.reshape(-1).double().cpu() for x in one]) - d).abs() <= 8 * E24 * size).all())
    with pytest.raises(RuntimeError):  # once differentiable
        (g,) = torch.autograd.grad(P.clip_grad_norm(tree, 2.0)[0]["w"].sum(), [tree["w"]], create_graph=True)
        torch.autograd.grad(g.sum(), [tree["w"]])
    for bad, kw, word in (({}, {}, "no tensor"), ([torch.ones(3)], {}, "device memory"), ([torch.ones(3, device="cuda").bfloat16()], {}, "fp32")):
        with pytest.raises(ValueError, match=word):
            P.clip_grad_norm(bad, 1.0)
    with pytest.raises(P.DiffoptError, match="max_norm"):
        P.clip_grad_norm(tree, -1.0)
    with pytest.raises(P.DiffoptError, match="eps"):
        P.clip_grad_norm(tree, 1.0, math.nan)


@pytest.mark.parametrize("name", ["MetaSGD", "MetaAdam", "MetaRMSProp"])
@pytest.mark.parametrize("max_norm", [0.05, 100.0])
def test_meta_gradient_through_clipped_steps(name, max_norm):
    """The outer gradient through two clipped inner steps against the same loop in fp64."""
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(7)
    x, y = torch.randn(16, 5, generator=gen), torch.randn(16, 3, generator=gen)
    w0, b0 = torch.randn(3, 5, generator=gen), torch.randn(3, generator=gen)
    scale0 = torch.tensor(1.3)

    net = torch.nn.Linear(5, 3)
    with torch.no_grad():
        net.weight.copy_(w0), net.bias.copy_(b0)
    net, scale = net.cuda(), scale0.cuda().requires_grad_(True)
    loss = lambda w, b, s, x, y: ((torch.tanh(x @ w.T + b) * s - y) ** 2).mean()  # noqa: E731
    kw = dict(MetaSGD=dict(lr=0.3, momentum=0.9), MetaAdam=dict(lr=0.05, eps=0.1), MetaRMSProp=dict(lr=0.05, eps=0.1))[name]
    opt = getattr(P, name)(net, max_norm=max_norm, **kw)
    norms = []
    for _ in range(2):
        p = net._parameters
        opt.step(loss(p["weight"], p["bias"], scale, x.cuda(), y.cuda()))
        norms.append(opt.grad_norm)
    p = net._parameters
    (got,) = torch.autograd.grad(loss(p["weight"], p["bias"], scale, x.cuda(), y.cuda()), [scale])

    w, b, s, X, Y = (t.double().requires_grad_(True) for t in (w0, b0, scale0, x, y))
    state = [torch.zeros_like(t) for t in (w, b)]
    mom = [torch.zeros_like(t) for t in (w, b)]
    ps = [w, b]
    for k in range(2):
        g = torch.autograd.grad(loss(*ps, s, X, Y), ps, create_graph=True)
        n = torch.sqrt(sum((t * t).sum() for t in g))
        assert abs(float(n.detach()) - float(norms[k])) <= 1e-4 * float(n.detach())
        g = [t * torch.clamp(max_norm / (n + 1e-6), max=1.0) for t in g]
        if name == "MetaSGD":
            state = [t + 0.9 * u for t, u in zip(g, state)]
            ps = [t - 0.3 * u for t, u in zip(ps, state)]
        elif name == "MetaAdam":
            mom = [0.9 * u + 0.1 * t for u, t in zip(mom, g)]
            state = [0.999 * u + 0.001 * t * t for u, t in zip(state, g)]
            ps = [t - 0.05 * (m / (1 - 0.9 ** (k + 1))) / (torch.sqrt(v / (1 - 0.999 ** (k + 1))) + 0.1) for t, m, v in zip(ps, mom, state)]
        else:
            state = [0.99 * u + 0.01 * t * t for u, t in zip(state, g)]
            ps = [t - 0.05 * u / (torch.sqrt(v) + 0.1) for t, u, v in zip(ps, g, state)]
    (ref,) = torch.autograd.grad(loss(*ps, s, X, Y), [s])
    assert abs(float(got) - float(ref)) <= 1e-3 * abs(float(ref))
    with pytest.raises(ValueError, match="max_norm"):
        getattr(P, name)(torch.nn.Linear(2, 2).cuda(), max_norm=-1.0)


def test_refusals():
    import paper_2211_06934_amd as P
    g, stats = torch.ones(9000, device="cuda"), torch.empty(2, device="cuda")
    out = torch.empty_like(g)
    for args, err, word in (((g, -1.0, out, stats), P.DiffoptError, "max_norm"), ((g, math.nan, out, stats), P.DiffoptError, "max_norm"),
                            ((g, 1.0, out, stats, -1.0), P.DiffoptError, "eps"), ((g, 1.0, out, stats, math.inf), P.DiffoptError, "eps"),
                            ((g, 1.0, out[1:], stats), ValueError, "out"), ((g, 1.0, out.double(), stats), ValueError, "out"),
                            ((g, 1.0, out, stats[:1]), ValueError, "stats"), ((g, 1.0, out, None), TypeError, "stats"), ((None, 1.0, out, stats), TypeError, "grad"),
                            ((g.cpu(), 1.0, out, stats), ValueError, "device memory"), ((g[:4500], 1.0, g[1:4501], stats), P.DiffoptError, "apart"),
                            ((g, 1.0, out, out[:2]), P.DiffoptError, "stats must lie apart")):
        with pytest.raises(err, match=word):
            P.clip_norm_fwd(*args)
    with pytest.raises(P.DiffoptError, match="dgrad must be an operand or lie apart"):
        P.clip_norm_bwd(g[:4500], None, out[:4500], stats, g[1:4501])
    with pytest.raises(ValueError, match="dnorm"):
        P.clip_norm_bwd(g, stats, out, stats, g)
    with pytest.raises(P.DiffoptError, match="elem_bytes"):
        P.clip_norm_fwd_tree(P.segtable_create([4], None, 2), torch.zeros(1, dtype=torch.int64, device="cuda"), 1.0, None, stats)
    table = P.segtable_create([4, 5])
    with pytest.raises(ValueError, match="grad"):
        P.clip_norm_fwd_tree(table, torch.zeros(1, dtype=torch.int64, device="cuda"), 1.0, None, stats)
    with pytest.raises(P.DiffoptError, match="null grad"):
        P.clip_norm_fwd_tree(table, None, 1.0, None, stats)
