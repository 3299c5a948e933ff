"""The second derivative of token log probabilities where the cotangent of the
gradient lies about a value far from 0: what depends on its differences alone."""
import math

import pytest
import torch

import paper_2211_06934_amd as P
from lm_reference import F32, assert_close, tol

pytestmark = pytest.mark.gpu

# Averages of a cotangent a are sums of exact products in fp64, divided by the
# sum of the same weights, and what is subtracted from a is kept to more than
# fp32: a value common to all of a drops out of out_dlogprob, out_dentropy and
# out_logits.  What is left are the weights' own errors, as without that value:
# the usual tolerances hold, against the same fp32 (or bf16) operands in fp64.


def _reference(x, a, ids, g, h, c, top, T):
    l = torch.log_softmax(x.double() / T, 1)
    p = l.exp()
    l = torch.where(p > 0, l, torch.zeros((), dtype=torch.float64, device=x.device))
    H = -(p * l).sum(1, keepdim=True)
    a, g, h, c = a.double(), g.double()[:, None], h.double()[:, None], c.double()
    mean = (p * a).sum(1, keepdim=True)
    k = (p * (a - mean) * (l + H)).sum(1, keepdim=True)
    G = g + c.sum(1, keepdim=True)
    return dict(og=((a.gather(1, ids[:, None]) - mean) / T)[:, 0], oh=(-k / T)[:, 0], oc=(a.gather(1, top) - mean) / T,
                ox=-p * (G * (a - mean) + h * ((a - mean) * (l + H + 1) - k)) / (T * T))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0.0, -10.0, 100.0, 1000.0])
@pytest.mark.parametrize("N,V", [(6, 700), (5, 8001), (4, 15000), (40, 32003), (260, 70001), (3, 150001)])
@pytest.mark.parametrize("entropy", [True, False])
def test_a_common_value_drops_out(N, V, offset, entropy, dtype):
    # from registers, streamed and cut; in bf16 the cotangent has few values about the offset, exactly
    gen = torch.Generator(device="cuda").manual_seed(V)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, T, K = (2.5 * r(N, V)).to(dtype), 0.8, 4
    a = (offset + (0.1 if dtype == torch.float32 else 4.0) * r(N, V)).to(dtype)
    ids, g, h, c = torch.randint(0, V, (N,), generator=gen, device="cuda"), 0.5 + r(N).abs(), r(N), r(N, K)
    new = lambda *s, dt=torch.float32: torch.full(s, math.nan, dtype=dt, device="cuda")  # noqa: E731
    lp, stats, ent, tops, top = new(N), new(N, 2), new(N), new(N, K), torch.zeros(N, K, dtype=torch.int64, device="cuda")
    P.logprob_fwd(x, ids, lp, stats, ent, tops, top, T)
    got = dict(og=new(N), oh=new(N) if entropy else None, oc=new(N, K), ox=new(N, V, dt=dtype))
    h = h if entropy else torch.zeros(N, device="cuda")
    P.logprob_bwd_bwd(a, x, ids, stats, got["ox"], g, h if entropy else None, ent if entropy else None, c, top, got["og"], got["oh"], got["oc"], T)
    ref = _reference(x, a, ids, g, h, c, top, T)
    for k, v in got.items():
        if v is not None:
            assert_close(v, ref[k], tol(dtype) if k == "ox" else F32, k)


@pytest.mark.parametrize("N,V", [(6, 700), (40, 40000), (3, 150001)])
def test_cotangents_of_tokens_that_are_ruled_out(N, V):
    # whatever they are, they have no weight: with 1e30 there the results are those with 0 there
    gen = torch.Generator(device="cuda").manual_seed(N)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, a, g, h = 2.5 * r(N, V), 3.0 + r(N, V), 0.5 + r(N).abs(), r(N)
    out = torch.rand(N, V, generator=gen, device="cuda") < 0.3
    out[:, 0], out[:, V // 2] = True, False
    x = torch.where(out, -math.inf, x)
    ids = torch.full((N,), V // 2, dtype=torch.int64, device="cuda")
    got = []
    for value in (0.0, 1e30):
        new = lambda *s: torch.full(s, math.nan, device="cuda")  # noqa: E731
        lp, stats, ent, og, oh, ox = new(N), new(N, 2), new(N), new(N), new(N), new(N, V)
        P.logprob_fwd(x, ids, lp, stats, ent)
        P.logprob_bwd_bwd(torch.where(out, value, a), x, ids, stats, ox, g, h, ent, None, None, og, oh)
        got.append((og, oh, ox))
    for one, other in zip(*got):
        assert bool(torch.isfinite(one).all()) and torch.equal(one, other)
