"""bf16 linear attention where nothing but a state makes the result: the fp32 state
enters its products with more bits than the type has, so that results are the
definition's but for their own rounding."""
import math

import pytest
import torch

from lm_reference import linattn

pytestmark = pytest.mark.gpu


# The state enters with an error of at most 2^-17 of each element (two parts of 8 bits), and a sum over its rows keeps that of its
# norm: a result moves to the neighbour of the correctly rounded one where it lies that near to the middle of two, 2^-8 apart or
# more for an element of the norm's size: 1 in 256, and more often only for the few elements much smaller than that.  Rounded to
# bf16 first, the state moves about every second element.
MOVED = 0.03


def _moved(got, ref):
    return float((got.cpu() != ref.to(torch.bfloat16)).double().mean())


@pytest.mark.parametrize("T,H,Hk,Dk,Dv", [(64, 2, 2, 64, 64), (200, 2, 1, 128, 128), (130, 2, 2, 32, 48), (90, 1, 1, 256, 64), (70, 2, 2, 33, 30),
                                          (700, 1, 1, 64, 64)])
def test_results_of_a_state(T, H, Hk, Dk, Dv):
    import paper_2211_06934_amd as P
    g = torch.Generator().manual_seed(T)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    bf = lambda *s: r(*s).to(torch.bfloat16)  # noqa: E731
    s0, ds1, lg = r(1, Hk, Dk, Dv), r(1, Hk, Dk, Dv), torch.tensor([-0.01, -0.03])[:Hk]
    scale = 0.25
    # keys of zero leave the state to decay: out and dq are made of it
    q, k, v, do = bf(1, T, H, Dk), torch.zeros(1, T, Hk, Dk).to(torch.bfloat16), torch.zeros(1, T, Hk, Dv).to(torch.bfloat16), bf(1, T, H, Dv)
    qr = q.double().requires_grad_()
    out, _ = linattn(qr, k, v, lg, s0, None, scale)
    (dq_ref,) = torch.autograd.grad(out, qr, do.double())
    o, dq = torch.full(do.shape, math.nan, dtype=q.dtype, device="cuda"), torch.full(q.shape, math.nan, dtype=q.dtype, device="cuda")
    P.linattn_fwd(q.cuda(), k.cuda(), v.cuda(), lg.cuda(), o, state=s0.cuda(), scale=scale)
    P.linattn_bwd(do.cuda(), q.cuda(), k.cuda(), v.cuda(), lg.cuda(), dq, None, None, state=s0.cuda(), scale=scale)
    assert _moved(o, out.detach()) <= MOVED
    assert _moved(dq, dq_ref) <= MOVED
    # queries and cotangents of zero: dk and dv are made of the final state's cotangent
    q, do, k, v = torch.zeros_like(q), torch.zeros_like(do), bf(1, T, Hk, Dk), bf(1, T, Hk, Dv)
    kr, vr = k.double().requires_grad_(), v.double().requires_grad_()
    _, s1 = linattn(q, kr, vr, lg, s0, None, scale)
    dk_ref, dv_ref = torch.autograd.grad(s1, (kr, vr), ds1.double())
    dk, dv = torch.full(k.shape, math.nan, dtype=k.dtype, device="cuda"), torch.full(v.shape, math.nan, dtype=k.dtype, device="cuda")
    P.linattn_bwd(do.cuda(), q.cuda(), k.cuda(), v.cuda(), lg.cuda(), None, dk, dv, state=s0.cuda(), dstate_out=ds1.cuda(), scale=scale)
    assert _moved(dk, dk_ref) <= MOVED
    assert _moved(dv, dv_ref) <= MOVED
