"""Log probabilities of rows with one likely token and a long flat rest: what
the sum of exponentials, a 1 and many numbers far below it, has to keep."""
import math

import pytest
import torch

import paper_2211_06934_amd as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24  # half a step of fp32, relative

# One logit lies D above V - 1 equal ones, T = 1: r = (V - 1) e^-D, q = r / (1 + r),
#   log p = -log(1 + r),  H = log(1 + r) + q D,  d log p / d x = 1 - p = q.
# Sums: eight terms at a time by a tree of three levels, where the 1 is rounded
# at most three times, a u each; the rest is summed in fp64.  With the final
# rounding 4 u = 2^-22.  Distances: the product with log2(e) (0.22 u off) is
# rounded once; 2^-21 of the distance covers it at any temperature, and moves
# log p by q D 2^-21 and H by q D^2 2^-21.
# A probability: the sum's 3 u, its rounding and the division's, two
# exponentials near 1 (2 u each), two products and the last sum: 12 u of the
# cotangent.
SUM, DISTANCE = 4 * U, 2.0 ** -21


def _rows(N, V, dtype, gap, at):
    x = torch.zeros(N, V, dtype=dtype, device="cuda")
    x[:, at] = gap
    return x + 1.5  # exact in bf16 too, and no maximum of 0


def _check(N, V, dtype, gap, at):
    x = _rows(N, V, dtype, gap, at)
    D = float(x[0, at].double() - x[0, (at + 1) % V].double())
    r = (V - 1) * math.exp(-D)
    q, lp, H = r / (1 + r), -math.log1p(r), math.log1p(r) + r / (1 + r) * D
    ids = torch.full((N,), at, dtype=torch.int64, device="cuda")
    g = torch.linspace(0.5, 1.5, N, device="cuda")
    new = lambda *s: torch.full(s, math.nan, device="cuda")  # noqa: E731
    bound, bound_H = SUM + q * D * DISTANCE, SUM + q * D * D * DISTANCE
    for K in (0, 5):
        logprob, stats, entropy = new(N), new(N, 2), new(N)
        tops, tids = (new(N, K), torch.zeros(N, K, dtype=torch.int64, device="cuda")) if K else (None, None)
        P.logprob_fwd(x, ids, logprob, stats, entropy, tops, tids)
        alone = new(N)
        P.logprob_fwd(x, ids, alone, new(N, 2), None, tops, tids)
        for got in (logprob, alone) + ((tops[:, 0],) if K else ()):
            assert float((got.double() - lp).abs().max()) <= bound, (K, float((got.double() - lp).abs().max()))
        assert float((entropy.double() - H).abs().max()) <= bound_H, (K, float((entropy.double() - H).abs().max()))
    dx, both = torch.full_like(x, math.nan), torch.full_like(x, math.nan)
    P.logprob_bwd(x, ids, stats, dx, dlogprob=g)
    logprob, entropy = new(N), new(N)
    P.logprob_fwd_bwd(g, x, ids, logprob, new(N, 2), both, None, entropy)
    assert float((logprob.double() - lp).abs().max()) <= bound
    assert float((entropy.double() - H).abs().max()) <= bound_H
    ref = g.double() * q
    off = g.double() * (12 * U + q * D * DISTANCE) + (ref * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    for got in (dx, both):
        assert bool(((got[:, at].double() - ref).abs() <= off).all()), float((got[:, at].double() - ref).abs().max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gap", [16.5, 17.25, 18.0])
@pytest.mark.parametrize("N,V", [(5, 4000), (2100, 500), (2100, 2040), (2100, 4090), (2100, 8190), (2100, 16001), (300, 50021), (7, 50021), (260, 160001), (3, 160001),
                                 (40, 160001)])
def test_a_likely_token(N, V, gap, dtype):
    # streamed, from registers, cut; rows of 32 KiB and more from registers where the gradient is wanted too
    _check(N, V, dtype, gap, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(5, 4000), (2100, 4090), (300, 50021), (3, 160001)])
@pytest.mark.parametrize("place", [0.0, 0.37, 1.0])
def test_wherever_it_stands(N, V, place, dtype):
    # first, within, last: the running maximum rises before or after the rest
    _check(N, V, dtype, 17.25, int(place * (V - 1)))
