"""Log probabilities of tokens: results, alternatives, gradients and the
gradients' own VJP against log_softmax and its autograd in fp64."""
import math

import pytest
import torch

import paper_2211_06934_amd as P
from lm_reference import F32, assert_close, tol

pytestmark = pytest.mark.gpu

# The tolerances are those of distillation, whose sums these are; the entropy's
# terms p log p are of one sign.  A result in bf16 is rounded once.


def _inputs(N, V, K, dtype, seed=0, padded=True, masked=False, ids64=True):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    I = dict(x=(2.5 * r(N, V)).to(dtype), a=r(N, V).to(dtype), ids=torch.randint(0, V, (N,), generator=gen), g=0.5 + torch.rand(N, generator=gen), h=r(N),
             c=r(N, K))
    if masked:
        out = torch.rand(N, V, generator=gen) > torch.rand(N, 1, generator=gen) ** 4
        I["x"] = torch.where(out.scatter(1, I["ids"][:, None], False), -math.inf, I["x"].float()).to(dtype)
    if padded and N > 2:
        I["ids"][1] = -1
        I["x"][1] = math.nan  # padding is not read
    if not ids64:
        I["ids"] = I["ids"].to(torch.int32)
    return I


def _reference(I, T):
    """fp64 results; rows of padding and entries that are no alternatives as the operator gives them."""
    ids, K, V = I["ids"].long(), I["c"].shape[1], I["x"].shape[1]
    there = ids >= 0
    raw = torch.where(there[:, None], I["x"].double(), torch.zeros((), dtype=torch.float64))
    x = raw.clone().requires_grad_()
    g, h, c = (I[k].double().requires_grad_() for k in ("g", "h", "c"))
    gone = raw == -math.inf
    lp = torch.log_softmax(x / T, 1)
    p, safe = torch.softmax(x / T, 1), torch.where(gone, 0.0, lp)
    on = there.double()
    logprob = torch.where(there, lp.gather(1, ids.clamp(min=0)[:, None])[:, 0], 0.0)
    entropy = -(p * safe).sum(1) * on
    by = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :K]
    by = torch.nn.functional.pad(by, (0, K - by.shape[1]), value=0)
    none = (torch.arange(K)[None, :] >= (~gone).sum(1)[:, None]) | ~there[:, None]
    tops = torch.where(none, 0.0, safe.gather(1, by))
    (dx,) = torch.autograd.grad((logprob, entropy, tops), x, (g, h, c), create_graph=True)
    og, oh, oc, ox = torch.autograd.grad(dx, (g, h, c, x), torch.where(there[:, None], I["a"].double(), 0.0))
    return dict(logprob=logprob, entropy=entropy, top=torch.where(none, -math.inf, tops), top_ids=torch.where(none, -1, by), dx=dx, og=og, oh=oh, oc=oc, ox=ox)


def _run(I, T, wrap=lambda t: t.cuda(), top64=True, entropy=True):
    import paper_2211_06934_amd as P
    N, V = I["x"].shape
    K = I["c"].shape[1]
    x, a = wrap(I["x"]), wrap(I["a"])
    ids, g, h, c = (I[k].cuda() for k in ("ids", "g", "h", "c"))
    nan = lambda *s, dt=torch.float32: torch.full(s, math.nan, dtype=dt, device="cuda")  # noqa: E731
    o = dict(logprob=nan(N), entropy=nan(N), dx=nan(N, V, dt=x.dtype), og=nan(N), oh=nan(N), ox=nan(N, V, dt=x.dtype))
    tops = tids = otop = None
    if K:
        tops, tids, otop = nan(N, K), torch.full((N, K), 77, dtype=torch.int64 if top64 else torch.int32, device="cuda"), nan(N, K)
    stats = nan(N, 2)
    P.logprob_fwd(x, ids, o["logprob"], stats, o["entropy"], tops, tids, T)
    given = dict(dlogprob=g, dentropy=h, entropy=o["entropy"], dtop_logprob=c if K else None, top_ids=tids, temperature=T)
    P.logprob_bwd(x, ids, stats, o["dx"], **given)
    P.logprob_bwd_bwd(a, x, ids, stats, o["ox"], out_dlogprob=o["og"], out_dentropy=o["oh"], out_dtop_logprob=otop, **given)
    o |= dict(top=tops if K else torch.zeros(N, 0), top_ids=tids.long() if K else torch.zeros(N, 0, dtype=torch.int64), oc=otop if K else torch.zeros(N, 0))
    both = dict(logprob=nan(N), entropy=nan(N), dx=nan(N, V, dt=x.dtype))
    P.logprob_fwd_bwd(g, x, ids, both["logprob"], nan(N, 2), both["dx"], h, both["entropy"], T)
    return o, both


# With K alternatives the gradient's dense part has the factor g + sum c + h (l + H): one more rounded sum of K terms.
def _compare(o, ref, dtype, what=""):
    assert torch.equal(o["top_ids"].cpu(), ref["top_ids"]), what
    for k in ref:
        if k != "top_ids":
            if k == "top":
                assert torch.equal(torch.isinf(o[k]).cpu(), torch.isinf(ref[k]))
            assert_close(o[k], ref[k], tol(dtype) if k in ("dx", "ox") else F32, "%s %s" % (what, k))


def _check(N, V, K, dtype, T=1.0, seed=0, wrap=lambda t: t.cuda(), top64=True, **kw):
    I = _inputs(N, V, K, dtype, seed, **kw)
    o, both = _run(I, T, wrap, top64)
    _compare(o, _reference(I, T), dtype)
    plain = dict(I, c=torch.zeros(N, 0))
    ref = _reference(plain, T)
    for k in both:
        assert_close(both[k], ref[k], tol(dtype) if k == "dx" else F32, "at once " + k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [2, 7, 64, 255, 1000, 4097, 8192, 20011, 50021])
def test_vocabularies(V, dtype):
    _check(5, V, min(8, V), dtype, seed=V, T=2.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [65536, 131072, 160001])
def test_large_vocabularies(V, dtype):
    _check(3, V, 32, dtype, seed=V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_rows_whole(dtype):
    # as many rows of more than a workgroup's registers as are not cut
    _check(260, 140001, 5, dtype, seed=1)


@pytest.mark.parametrize("K", [0, 1, 2, 20, 63, 64, 65, 128])
@pytest.mark.parametrize("ids64", [False, True])
def test_alternatives(K, ids64):
    _check(4, 2000, K, torch.float32, seed=K, T=1.5, ids64=ids64, top64=ids64)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(1, 150001), (40, 70003), (2, 17000), (300, 10000), (2, 300001)])
def test_most_alternatives(N, V, dtype):
    # cut rows and whole ones, workgroups of each size
    _check(N, V, 128, dtype, seed=N)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N", [1, 2, 9, 300, 2000])
def test_rows(N, dtype):
    _check(N, 501, 5, dtype, seed=N)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,K", [(2100, 1, 1), (2100, 37, 64), (2100, 500, 0), (2100, 500, 64), (2300, 900, 128), (2100, 2049, 5), (2100, 4090, 20), (2100, 4090, 0),
                                   (2049, 8193, 0), (2049, 9001, 128), (2100, 16001, 0), (2100, 30011, 0), (2047, 500, 20), (3, 700, 128),
                                   (300, 1999, 128), (2100, 4090, 128), (2050, 4001, 49)])
@pytest.mark.parametrize("values", ["all", "few", "one"])
def test_many_rows(N, V, K, values, dtype):
    # short rows whose results come from registers; values that many tokens share
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = 2.5 * torch.randn(N, V + 3, generator=gen, device="cuda")
    x = (x.round() if values == "few" else torch.ones_like(x) if values == "one" else x).to(dtype)[:, 1 : V + 1]
    x[5 % N, 1:] = -math.inf
    ids = torch.randint(0, V, (N,), generator=gen, device="cuda")
    ids[1], ids[5 % N] = -1, 0
    lp, en, stats, tops = (torch.full(n, math.nan, device="cuda") for n in ((N,), (N,), (N, 2), (N, K)))
    tids = torch.full((N, K), 77, dtype=torch.int64, device="cuda")
    P.logprob_fwd(x, ids, lp, stats, en, tops if K else None, tids if K else None, 0.8)
    raw = x.double()
    ref = torch.log_softmax(raw / 0.8, 1)
    there = ids >= 0
    assert_close(lp, torch.where(there, ref.gather(1, ids.clamp(min=0)[:, None])[:, 0], 0.0), F32)
    assert_close(en, torch.where(there, -(ref.exp() * torch.where(raw == -math.inf, 0.0, ref)).sum(1), 0.0), F32)
    order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :K]
    value = ref.gather(1, order)
    order = torch.where((value == -math.inf) | ~there[:, None], -1, order)
    n = order.shape[1]
    assert torch.equal(tids[:, :n], order) and bool((tids[:, n:] == -1).all())
    assert torch.equal(tops == -math.inf, tids < 0)
    assert_close(torch.where(order < 0, 0.0, tops[:, :n].double()), torch.where(order < 0, 0.0, value), F32)


@pytest.mark.parametrize("V,K", [(900, 128), (500, 64), (230, 100)])
def test_ranks_of_many_equal_values(V, K):
    # the candidates are counted twice: no wave takes the second count for the first, however late it is
    x, ids = torch.ones(6000, V, device="cuda"), torch.zeros(6000, dtype=torch.int64, device="cuda")
    lp, stats, tops = torch.empty(6000, device="cuda"), torch.empty(6000, 2, device="cuda"), torch.empty(6000, K, device="cuda")
    want = torch.arange(K, device="cuda").expand(6000, K)
    for _ in range(30):
        tids = torch.full((6000, K), -7, dtype=torch.int64, device="cuda")
        P.logprob_fwd(x, ids, lp, stats, None, tops, tids)
        assert torch.equal(tids, want)


@pytest.mark.parametrize("T", [0.25, 1.0, 7.5])
def test_temperatures(T):
    _check(6, 3001, 12, torch.float32, T=T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [-40.0, 40.0])
@pytest.mark.parametrize("N,V", [(4, 1), (4, 9), (300, 700), (40, 33000), (6, 50021)])
def test_values_of_one_sign(N, V, shift, dtype):
    # logits of 8 bits about the shift; the other results have 1 and no token at 0
    I = _inputs(N, V, min(V, 5), dtype, seed=V)
    I["x"] = (I["x"].float() + shift).to(dtype)
    if V > 2:
        I["x"][0, : V // 2] = -math.inf
        I["ids"][0] = V - 1
    o, both = _run(I, 1.0)
    ref = _reference(I, 1.0)
    alone = _reference(dict(I, c=torch.zeros(N, 0)), 1.0)
    for k in ("logprob", "entropy", "top", "dx"):
        if V > 1:
            assert_close(o[k], ref[k], tol(dtype) if k == "dx" else F32, k)
    for k in both:
        if V > 1:
            assert_close(both[k], alone[k], tol(dtype) if k == "dx" else F32, "at once " + k)
    if V == 1:
        assert not both["logprob"].any() and not both["entropy"].any() and not o["logprob"].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_nan_shows(dtype):
    # of either sign, among values of either sign, in a lane's packed pieces and beside them
    for V in (300, 9001):
        x = torch.randn(8, V, generator=torch.Generator().manual_seed(V)).to(dtype).cuda()
        bits = x.view(torch.int16 if dtype == torch.bfloat16 else torch.int32)
        quiet = 0x7FC0 if dtype == torch.bfloat16 else 0x7FC00000
        low = -0x8000 if dtype == torch.bfloat16 else -0x80000000
        x[2:4] = x[2:4].abs().neg()
        for row, at in ((0, 17), (2, 17), (4, V - 1)):
            bits[row, at], bits[row + 1, at] = quiet, quiet + low
        ids = torch.zeros(8, dtype=torch.int64, device="cuda")
        new = lambda *n: torch.zeros(n, device="cuda")  # noqa: E731
        lp, en, dx = new(8), new(8), torch.zeros_like(x)
        P.logprob_fwd_bwd(new(8) + 1.0, x, ids, lp, new(8, 2), dx, new(8), en)
        for t in (lp, en, dx.float().sum(1)):
            assert torch.isnan(t).tolist() == [True] * 6 + [False] * 2
        P.logprob_fwd(x, ids, lp, new(8, 2), en)
        assert torch.isnan(lp).tolist() == torch.isnan(en).tolist() == [True] * 6 + [False] * 2


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [40, 700, 33000, 140001])
def test_masked_vocabularies(V, dtype):
    # from a single token on; fewer than K are left in some rows
    _check(12, V, 30, dtype, seed=V, masked=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,K", [(1, 1), (3, 5), (100, 128)])
def test_more_alternatives_than_tokens(V, K, dtype):
    if V == 1:  # one token: no entropy, no gradient; the references are exact zeros
        I = _inputs(4, V, K, dtype)
        o, both = _run(I, 1.0)
        ref = _reference(I, 1.0)
        assert torch.equal(o["top_ids"].cpu(), ref["top_ids"])
        for k in ("logprob", "entropy", "dx", "og", "oc"):
            assert not o[k].any() and not (k in both and both[k].any())
        # the second derivatives have l + H as the sum of ln 2 d and its negative, d the rounding of a logit's product with
        # log2(e), at most 2^-24 times 16: what is left of them is at most 2^-24 of 2^-20, and a is below 8
        assert float(o["oh"].abs().max()) <= 2.0 ** -40 and float(o["ox"].abs().max()) <= 2.0 ** -40
        return
    _check(4, V, K, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 5000, 70001, 150001])
def test_ties_go_to_the_lowest_id(V, dtype):
    gen = torch.Generator().manual_seed(V)
    I = _inputs(5, V, 100, dtype, padded=False)
    I["x"][0] = 0.5                                                             # all equal
    I["x"][1] = torch.randint(0, 3, (V,), generator=gen).to(dtype)              # few values
    I["x"][2] = torch.where(torch.rand(V, generator=gen) < 0.5, 0.0, -0.0).to(dtype)  # one value of two signs
    I["x"][3, V // 2:] = 9.0                                                    # more than a thousand of the largest, late
    I["x"][4] = torch.arange(V).to(dtype) / 64.0                                # rising
    _compare(_run(I, 1.0)[0], _reference(I, 1.0), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["wide rows", "odd rows", "padded vocabulary"])
def test_strides(kind, dtype):
    def wrap(x):
        N, V = x.shape
        pad = {"wide rows": 8, "odd rows": 1, "padded vocabulary": 51}[kind]
        off = 1 if kind == "odd rows" else 0
        buf = torch.full((N * (V + pad) + 1,), math.nan, dtype=x.dtype, device="cuda")
        return buf.as_strided((N, V), (V + pad, 1), off).copy_(x)
    _check(7, 1003, 9, dtype, wrap=wrap)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(6, 700), (3, 150001)])
def test_strided_results_and_in_place(N, V, dtype):
    import paper_2211_06934_amd as P
    I = _inputs(N, V, 4, dtype)
    o, _ = _run(I, 1.0)
    X, ids = I["x"].cuda(), I["ids"].cuda()
    buf = torch.full((N, V + 5), 3.0, dtype=dtype, device="cuda")
    lp, ent, stats = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, 2, device="cuda")
    tops, tids = torch.empty(N, 4, device="cuda"), torch.empty(N, 4, dtype=torch.int64, device="cuda")
    P.logprob_fwd(X, ids, lp, stats, ent, tops, tids)
    given = dict(dlogprob=I["g"].cuda(), dentropy=I["h"].cuda(), entropy=ent, dtop_logprob=I["c"].cuda(), top_ids=tids)
    P.logprob_bwd(X, ids, stats, buf[:, 2:V + 2], **given)
    assert torch.equal(buf[:, 2:V + 2], o["dx"])
    assert (buf[:, :2] == 3.0).all() and (buf[:, V + 2:] == 3.0).all()
    P.logprob_bwd(X, ids, stats, X, **given)  # over the logits
    assert torch.equal(X, o["dx"])


def test_extreme_logits():
    low = torch.finfo(torch.float32).min
    I = _inputs(8, 100, 6, torch.float32, padded=False)
    x = I["x"]
    x[0, 50:] = -math.inf       # part of the vocabulary ruled out, the token among the rest
    I["ids"][0] = 60            # no: the token itself
    x[1, :] = low               # a row of the lowest value: uniform
    x[2, 10:] = low
    I["ids"][2] = 3
    x[3, 7] = 3e38
    I["ids"][3] = 7
    x[4, :] = -math.inf
    x[4, 5] = 1.0               # one token left
    I["ids"][4] = 5
    x[5, 5] = math.nan
    x[6, :] = -math.inf         # nothing left: no distribution
    x[7, 9] = math.inf
    o, both = _run(I, 1.0)
    ref = _reference({k: v[:5] for k, v in I.items()}, 1.0)
    for k in ("entropy", "dx", "ox", "oh", "og", "oc"):
        assert_close(o[k][:5], ref[k], F32, k)
    assert_close(o["logprob"][:5], ref["logprob"], F32)
    assert o["logprob"][0] == -math.inf
    assert torch.equal(o["top_ids"][:5].cpu(), ref["top_ids"])
    for k in ("logprob", "entropy", "top", "dx", "og", "oh", "oc", "ox"):
        assert torch.isnan(o[k][5:]).all(), k
    assert (o["top_ids"][5:] == -1).all()
    for k in both:
        assert torch.isnan(both[k][5:]).all() and torch.equal(torch.isfinite(both[k][:5]), torch.isfinite(o[k][:5]))


@pytest.mark.parametrize("scale,T", [(1.0, 1.0), (1e6, 1e3), (1e30, 1.0), (1e37, 1e37)])
def test_far_values(scale, T):
    # rows far from zero, and spread further than the exponentials reach
    I = _inputs(4, 5000, 5, torch.float32, padded=False)
    I["x"] = I["x"] * scale + 3.0 * scale
    ref = _reference(I, T)
    o, both = _run(I, T)
    # a logit's rounding does not enter: the reference has the same fp32 logits; the difference to the maximum is rounded once.
    # The sum of exponentials begins with the largest one's 1, so that its logarithm, a part of the entropy and of the log
    # probabilities, is known to 2^-24 absolutely however small it is: 1 + n 2^-24 has that rounding and nothing finer.
    for k in ("logprob", "entropy", "top", "dx"):
        for got in (o, both):
            if k in got and not (k == "dx" and got is both):
                err = (got[k].double().cpu() - ref[k].detach()).abs()
                assert float(err.max()) <= 2 * F32 * float(ref[k].detach().abs().max()) + 2.0 ** -23, k


def test_foreign_tokens():
    I = _inputs(4, 300, 6, torch.float32, padded=False)
    I["ids"][2] = 300
    o, both = _run(I, 1.0)
    for res in (o, both):
        for k, v in res.items():
            if k != "top_ids":
                assert torch.isnan(v[2]).all() and torch.isfinite(v[3]).all() and torch.isfinite(v[:2]).all(), k
    assert (o["top_ids"][2] == -1).all() and (o["top_ids"][3] >= 0).all()


@pytest.mark.parametrize("V", [400, 150001])
def test_what_may_be_left_out(V):
    import paper_2211_06934_amd as P
    I = {k: v.cuda() for k, v in _inputs(5, V, 6, torch.float32, padded=False).items()}
    o, _ = _run(I, 1.0)
    x, ids = I["x"], I["ids"]
    new = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    for given in (False, True):
        for ent in (False, True):
            for top in (False, True):
                lp, e, st = new(5) if given else None, new(5) if ent else None, new(5, 2)
                t, ti = (new(5, 6), new(5, 6, dt=torch.int32)) if top else (None, None)
                P.logprob_fwd(x, ids if given else None, lp, st, e, t, ti)
                for got, k in ((lp, "logprob"), (e, "entropy"), (t, "top")):
                    if got is not None:
                        assert_close(got, o[k].double(), 1e-6)
                assert ti is None or torch.equal(ti.long(), o["top_ids"])
    st, e, lp, ti, t = new(5, 2), new(5), new(5), new(5, 6, dt=torch.int64), new(5, 6)
    P.logprob_fwd(x, ids, lp, st, e, t, ti)

    def grads(g, h, c):
        dx, ox, outs = new(5, V), new(5, V), [None if k is None else torch.empty_like(k) for k in (g, h, c)]
        how = dict(dlogprob=g, dentropy=h, entropy=None if h is None else e, dtop_logprob=c, top_ids=None if c is None else ti)
        P.logprob_bwd(x, ids, st, dx, **how)
        P.logprob_bwd_bwd(I["a"], x, ids, st, ox, out_dlogprob=outs[0], out_dentropy=outs[1], out_dtop_logprob=outs[2], **how)
        return dx, ox, *outs

    zero = [torch.zeros_like(I[k]) for k in "ghc"]
    for keep in range(8):
        some = [I[k] if keep >> i & 1 else None for i, k in enumerate("ghc")]
        full = grads(*[z if s is None else s for s, z in zip(some, zero)])
        for got, want, k in zip(grads(*some), full, ("dx", "ox", "og", "oh", "oc")):
            assert got is None or float((got - want).abs().max()) <= 1e-6 * max(1.0, float(want.abs().max())), (keep, k)
    # the same alternative named twice adds up
    ti[:, 1] = ti[:, 0]
    twice, once = grads(None, None, I["c"])[0], I["c"].clone()
    once[:, 0] += once[:, 1]
    once[:, 1] = 0
    assert_close(twice, grads(None, None, once)[0].double(), 1e-6)
    # and the dx of fwd_bwd is that of bwd, whether or not an entropy is wanted
    a, b = new(5, V), new(5, V)
    P.logprob_fwd_bwd(I["g"], x, ids, lp, st, a)
    P.logprob_fwd_bwd(I["g"], x, ids, lp, st, b, None, e)
    assert_close(a, grads(I["g"], None, None)[0].double(), 1e-6)
    assert_close(b, a.double(), 1e-6)


def test_gradient_against_differences():
    import paper_2211_06934_amd as P
    I = {k: v.cuda() for k, v in _inputs(4, 60, 6, torch.float32, padded=False).items()}
    ids = I["ids"]
    new = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    ti, keep = torch.empty(4, 6, dtype=torch.int64, device="cuda"), torch.empty(4, 6, dtype=torch.int64, device="cuda")

    def at(e):
        x = I["x"] + e * I["a"]
        lp, ent, st, t, dx = new(4), new(4), new(4, 2), new(4, 6), torch.empty_like(x)
        P.logprob_fwd(x, ids, lp, st, ent, t, ti)
        P.logprob_bwd(x, ids, st, dx, I["g"], I["h"], ent, I["c"], ti)
        return (I["g"] * lp).double() + (I["h"] * ent).double() + (I["c"] * t).double().sum(1), dx.double(), ti.clone()

    h = 2.0 ** -8
    (l2, p2, i2), (l1, p1, i1), (m1, n1, j1), (m2, n2, j2) = (at(e) for e in (2 * h, h, -h, -2 * h))
    _, dx, keep = at(0.0)
    same = (i2 == keep).all(1) & (i1 == keep).all(1) & (j1 == keep).all(1) & (j2 == keep).all(1)
    assert same.sum() >= 2  # rows whose alternatives stay the same
    slope = (8 * (l1 - m1) - (l2 - m2)) / (12 * h)
    assert_close(slope[same], (dx * I["a"]).sum(1)[same], 1e-3)
    st, ent, lp, t, ox = new(4, 2), new(4), new(4), new(4, 6), torch.empty_like(I["x"])
    P.logprob_fwd(I["x"], ids, lp, st, ent, t, ti)
    P.logprob_bwd_bwd(I["a"], I["x"], ids, st, ox, I["g"], I["h"], ent, I["c"], ti)
    assert_close(ox[same], ((8 * (p1 - n1) - (p2 - n2)) / (12 * h))[same], 1e-3)


def test_streams_workspaces_and_repeats():
    import paper_2211_06934_amd as P
    I = _inputs(9, 140001, 16, torch.bfloat16)
    ref = [v for res in _run(I, 1.0) for v in res.values()]
    got = []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for st in streams:
        with torch.cuda.stream(st):
            got.append([v for res in _run(I, 1.0) for v in res.values()])
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, ref))
    need = P.logprob_workspace(9, 140001, 16, torch.bfloat16)
    assert need > 0
    lp, st = torch.empty(9, device="cuda"), torch.empty(9, 2, device="cuda")
    t, ti = torch.empty(9, 16, device="cuda"), torch.empty(9, 16, dtype=torch.int64, device="cuda")
    ws = torch.full((need // 4,), math.nan, device="cuda").view(torch.uint8)
    P.logprob_fwd(I["x"].cuda(), I["ids"].cuda(), lp, st, None, t, ti, workspace=ws, stream=torch.cuda.current_stream())
    assert torch.equal(lp, ref[0])
    with pytest.raises(ValueError, match="workspace"):
        P.logprob_fwd(I["x"].cuda(), I["ids"].cuda(), lp, st, None, t, ti, workspace=ws[:-4])


def test_captured_and_replayed():
    import paper_2211_06934_amd as P
    I = {k: v.cuda() for k, v in _inputs(3, 150001, 5, torch.float32).items()}
    x, ids = I["x"], I["ids"]
    new = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    o = [new(3), new(3, 2), new(3), new(3, 5), new(3, 5, dt=torch.int64), torch.zeros_like(x), torch.zeros_like(x)]
    ws = torch.empty(P.logprob_workspace(3, 150001, 5), dtype=torch.uint8, device="cuda")

    def step():
        P.logprob_fwd(x, ids, o[0], o[1], o[2], o[3], o[4], workspace=ws)
        P.logprob_bwd(x, ids, o[1], o[5], I["g"], I["h"], o[2], I["c"], o[4])
        P.logprob_fwd_bwd(I["g"], x, ids, o[0], o[1], o[6], I["h"], o[2], workspace=ws)

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
        got = [t.clone() for t in o]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, o))
        x[0].mul_(0.9)


def test_no_rows_and_refusals():
    import paper_2211_06934_amd as P
    I = {k: v.cuda() for k, v in _inputs(4, 60, 6, torch.float32).items()}
    x, ids, g, h, c = (I[k] for k in ("x", "ids", "g", "h", "c"))
    lp, st, e, dx = torch.empty(4, device="cuda"), torch.empty(4, 2, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(x)
    t, ti = torch.empty(4, 6, device="cuda"), torch.empty(4, 6, dtype=torch.int64, device="cuda")
    P.logprob_fwd(x[:0], ids[:0], lp[:0], st[:0], e[:0], t[:0], ti[:0])
    P.logprob_fwd(x, ids, lp, st, e, t, ti)
    for bad, err, word in (((x.half(), ids, lp, st), ValueError, "float16"), ((x, ids.float(), lp, st), ValueError, "ids"), ((x, ids[:3], lp, st), ValueError, "ids"),
                           ((x, ids, lp, st[:, :1]), ValueError, "stats"), ((x, ids, lp, None), TypeError, "stats"), ((x, None, lp, st), P.DiffoptError, "ids"),
                           ((x, ids, None, st), P.DiffoptError, "logprob"), ((x.cpu(), ids, lp, st), ValueError, "device memory"),
                           ((x.t().contiguous().t(), ids, lp, st), ValueError, "contiguous"), ((x[0], ids, lp, st), ValueError, "2 axes"),
                           ((x, ids, lp, st, e, t, None), ValueError, "top_ids"), ((x, ids, lp, st, e, None, ti), ValueError, "top_logprob"),
                           ((x, ids, lp, st, e, t, ti[:, :5]), ValueError, "top_ids"), ((x, ids, lp, st, e, t, ti.float()), ValueError, "top_ids"),
                           ((x, ids, lp, st, lp), P.DiffoptError, "one array"), ((x, ids, lp, st, e, t, ti, 0.0), P.DiffoptError, "temperature"),
                           ((x, ids, lp, st, e, t, ti, math.nan), P.DiffoptError, "temperature")):
        with pytest.raises(err, match=word):
            P.logprob_fwd(*bad)
    many = torch.zeros(4, 129, device="cuda")
    with pytest.raises(P.DiffoptError, match="128"):
        P.logprob_fwd(x, ids, lp, st, e, many, many.long())
    for kw, err, word in ((dict(dentropy=h), P.DiffoptError, "entropy"), (dict(dtop_logprob=c), ValueError, "top_ids"), (dict(dlogprob=g[:3]), ValueError, "dlogprob")):
        with pytest.raises(err, match=word):
            P.logprob_bwd(x, ids, st, dx, **kw)
    with pytest.raises(P.DiffoptError, match="must not be logits"):
        P.logprob_fwd_bwd(g, x, ids, lp, st, x)
    with pytest.raises(P.DiffoptError, match="neither"):
        P.logprob_bwd_bwd(I["a"], x, ids, st, I["a"], dlogprob=g)
    with pytest.raises(P.DiffoptError, match="out_dentropy without"):
        P.logprob_bwd_bwd(I["a"], x, ids, st, dx, dlogprob=g, out_dentropy=e)
    with pytest.raises(ValueError, match="out_dtop_logprob"):
        P.logprob_bwd_bwd(I["a"], x, ids, st, dx, dlogprob=g, out_dtop_logprob=t)
