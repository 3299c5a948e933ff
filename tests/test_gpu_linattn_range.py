"""Linear attention on values near both ends of fp32's exponents, under decays that
shrink a state by many powers of two on its way: a state that the recurrence holds
in fp32 stays finite and as accurate as ordinary values."""
import math

import pytest
import torch

from lm_reference import F32, assert_close, linattn, tol

pytestmark = pytest.mark.gpu


# what is multiplied by 2^power: results scale by the same power, exactly
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("power", [115, -90])
@pytest.mark.parametrize("which", ["v", "k"])
@pytest.mark.parametrize("T,H,Hk,D", [(700, 3, 3, 32), (520, 2, 1, 64), (2600, 3, 3, 32), (40, 3, 3, 128), (300, 2, 1, 33)])
def test_powers_of_two(T, H, Hk, D, which, power, dtype):
    import paper_2211_06934_amd as P
    g = torch.Generator().manual_seed(T)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q, k, v, do = (r(1, T, h, D).to(dtype) for h in (H, Hk, Hk, H))
    s0, ds1 = r(1, Hk, D, D), r(1, Hk, D, D)
    lg = torch.tensor([-0.05, -0.5, -1e-3])[:Hk]  # 2^-4.6, 2^-46 and 2^-0.1 a chunk of 64
    scale = D ** -0.5
    ref = [x.double().requires_grad_() for x in (q, k, v, s0)]
    out, s1 = linattn(*ref[:3], lg, ref[3], None, scale)
    grads = torch.autograd.grad((out, s1), ref, (do.double(), ds1.double()))

    # out, the states, dq and the gradient of the other factor take the power on; the factor's own gradient does not
    big = lambda x: x * 2.0 ** power  # noqa: E731
    ops = [q, big(k) if which == "k" else k, big(v) if which == "v" else v]
    dev = [x.cuda() for x in (*ops, do)]
    lgd, s0d, ds1d = lg.cuda(), big(s0).cuda(), ds1.cuda()
    nan = lambda x: torch.full(x.shape, math.nan, dtype=x.dtype, device="cuda")  # noqa: E731
    o, so = nan(do), nan(s0)
    P.linattn_fwd(*dev[:3], lgd, o, state=s0d, state_out=so, scale=scale)
    dq, dk, dv, ds0 = nan(q), nan(k), nan(v), nan(s0)
    P.linattn_bwd(dev[3], *dev[:3], lgd, dq, dk, dv, state=s0d, dstate_out=ds1d, dstate=ds0, scale=scale)
    b = tol(dtype, products=True)
    small = lambda x: x.double().cpu() * 2.0 ** -power  # noqa: E731
    assert_close(small(o), out, b, "out")
    assert_close(small(so), s1, F32, "state_out")
    assert_close(small(dq), grads[0], b, "dq")
    assert_close(small(dk) if which == "v" else dk, grads[1], b, "dk")
    assert_close(dv if which == "v" else small(dv), grads[2], b, "dv")
    assert_close(ds0, grads[3], F32, "dstate")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_largest_values(dtype):
    # one value of the type's largest, early, under a decay: the states that follow are finite, and so are the outputs
    import paper_2211_06934_amd as P
    T, D = 700, 32
    q, k, v = (torch.zeros(1, T, 2, D, dtype=dtype) for _ in range(3))
    q[..., 0], k[:, ::64, :, 0], k[:, 5, :, 0] = 0.5, 1e-3, 1.0
    v[:, 5] = torch.finfo(dtype).max
    v[:, 6:] = 1.0
    lg = torch.tensor([-0.05, -1e-3])
    out, so = torch.empty(1, T, 2, D, dtype=dtype, device="cuda"), torch.empty(1, 2, D, D, device="cuda")
    P.linattn_fwd(q.cuda(), k.cuda(), v.cuda(), lg.cuda(), out, state_out=so)
    ref, s1 = linattn(q, k, v, lg)
    # element by element: one head is larger by many powers of two than the other in the end
    for got, want, bound in ((out, ref, tol(dtype, products=True)), (so, s1, F32)):
        got = got.double().cpu()
        assert torch.isfinite(got).all()
        assert bool(((got - want).abs() <= 4 * bound * want.abs()).all())
