"""bf16 linear attention where the scores make the result: they enter their products
with more bits than the type has, so that results are the definition's but for
their own rounding."""
import math

import pytest
import torch

from lm_reference import linattn
from test_gpu_linattn_state_bits import MOVED, _moved

pytestmark = pytest.mark.gpu


# The scores are exact to 2^-17 of each, as the state is: the same bound on the results that move to a neighbour.
@pytest.mark.parametrize("T,H,Hk,Dk,Dv", [(33, 2, 2, 64, 64), (64, 2, 1, 128, 128), (200, 2, 2, 32, 48), (31, 1, 1, 256, 64), (70, 2, 2, 33, 30)])
def test_results_of_scores(T, H, Hk, Dk, Dv):
    import paper_2211_06934_amd as P
    g = torch.Generator().manual_seed(T)
    q, k, v, do = (torch.randn(1, T, h, w, generator=g).to(torch.bfloat16) for h, w in ((H, Dk), (Hk, Dk), (Hk, Dv), (H, Dv)))
    lg, scale = torch.tensor([-0.01, -0.2])[:Hk], Dk ** -0.5
    ref = [x.double().requires_grad_() for x in (q, k, v)]
    out, _ = linattn(*ref, lg, None, None, scale)
    grads = torch.autograd.grad(out, ref, do.double())
    dev = [x.cuda() for x in (q, k, v, do)]
    o = torch.full(do.shape, math.nan, dtype=q.dtype, device="cuda")
    P.linattn_fwd(*dev[:3], lg.cuda(), o, scale=scale)
    assert _moved(o, out.detach()) <= MOVED
    got = [torch.full_like(x, math.nan) for x in dev[:3]]
    P.linattn_bwd(dev[3], *dev[:3], lg.cuda(), *got, scale=scale)
    for x, want in zip(got, grads):
        assert _moved(x, want) <= MOVED
