"""Clipping's gradient where the norm is so small that the norm's own gradient
per unit of the gradient is no fp32 number, and where the norm is above fp32."""
import math

import pytest
import torch

import paper_2211_06934_amd as P

pytestmark = pytest.mark.gpu


def _tree(values, cuts):
    leaves = [t.clone() for t in values.split(cuts)]
    return P.segtable_create([t.numel() for t in leaves]), leaves


def _gradient(form, grad, dout, dnorm, max_norm, stats):
    """dgrad, with the stats of the forward."""
    n, out, dgrad = grad.numel(), torch.full_like(grad, math.nan), torch.full_like(grad, math.nan)
    if form == "buffer":
        P.clip_norm_fwd(grad, max_norm, out, stats, eps=0.0)
        P.clip_norm_bwd(dout, dnorm, grad, stats, dgrad, eps=0.0)
        return dgrad
    cuts = [1, 2, 33, n - 36]
    table, g = _tree(grad, cuts)
    o, dg = ([t.clone() for t in x.split(cuts)] for x in (out, dgrad))
    d = None if dout is None else [t.clone() for t in dout.split(cuts)]
    at = [None if x is None else P.tree.leaf_pointer_tensor(x, "cuda") for x in (g, o, d, dg)]
    P.clip_norm_fwd_tree(table, at[0], max_norm, at[1], stats, eps=0.0)
    P.clip_norm_bwd_tree(table, at[2], dnorm, at[0], stats, at[3], eps=0.0)
    return torch.cat(dg)


@pytest.mark.parametrize("form", ["buffer", "tree"])
@pytest.mark.parametrize("n", [64, 5000, 30000])
@pytest.mark.parametrize("size", [1e-40, 3e-39, 1e-38, 1e-30, 1e20])
@pytest.mark.parametrize("cotangent", [False, True])
def test_norms_at_the_ends(form, n, size, cotangent):
    # fifty elements, the others 0.  dgrad = c dout + grad (dnorm - [c < 1] c <dout, grad> / norm) / norm: the norm is known to
    # half of fp32's least step, or to 2^-24 of itself, c and the factor's parts to 2^-24 each, and so are the two products and
    # their sum: eight of them, and the norm's error twice.
    gen = torch.Generator().manual_seed(n)
    grad = torch.zeros(n)
    grad[torch.randperm(n, generator=gen)[:50]] = size * (0.5 + torch.rand(50, generator=gen))
    grad = grad.cuda()
    dnorm, dout = torch.tensor([0.3], device="cuda"), torch.randn(n, generator=gen).cuda() if cotangent else None
    norm = float(grad.double().norm())
    for max_norm in (0.5 * norm, math.inf):
        stats = torch.full((2,), math.nan, device="cuda")
        got = _gradient(form, grad, dout, dnorm, max_norm, stats)
        c = min(1.0, max_norm / norm)
        d = torch.zeros(n, dtype=torch.float64, device="cuda") if dout is None else dout.double()
        dot = float((d * grad.double()).sum())
        radial = grad.double() * ((float(dnorm) - (c * dot / norm if c < 1 else 0.0)) / norm)
        ref = c * d + radial
        unit = 2.0 ** -24
        off = 8 * unit + 2 * max(unit, 2.0 ** -150 / norm)
        terms = (c * d).abs() + grad.double() * ((abs(float(dnorm)) + abs(c * dot / norm)) / norm)
        assert bool(torch.isfinite(got).all())
        assert bool(((got.double() - ref).abs() <= off * terms).all()), float(((got.double() - ref).abs() / terms.clamp(min=1e-300)).max())


@pytest.mark.parametrize("form", ["buffer", "tree"])
@pytest.mark.parametrize("n", [5000, 30000])
def test_norms_above_fp32(form, n):
    # finite elements whose norm is not: c is right, the norm's own gradient is gone
    gen = torch.Generator().manual_seed(n)
    grad, dout = (1e37 * (1.0 + torch.rand(n, generator=gen))).cuda(), torch.randn(n, generator=gen).cuda()
    norm, stats = float(grad.double().norm()), torch.empty(2, device="cuda")
    got = _gradient(form, grad, dout, torch.tensor([0.3], device="cuda"), 0.25 * norm, stats)
    assert float(stats[0]) == math.inf and abs(float(stats[1]) - 0.25) <= 0.25 * 2.0 ** -24
    assert torch.equal(got, stats[1] * dout)
