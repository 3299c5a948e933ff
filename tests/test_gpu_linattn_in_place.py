"""Linear attention with one tensor as the state before and after: the results of
separate ones, whatever the heads that share a state, the lengths and the cuts."""
import pytest
import torch

from lm_reference import F32, assert_close, linattn, tol

pytestmark = pytest.mark.gpu


def _operands(B, T, H, Hk, D, dtype, ragged, seed):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(B, T, h, D, generator=g).to(dtype) for h in (H, Hk, Hk))
    lg = -torch.rand(Hk, generator=g) * 0.2
    n = None
    if ragged:
        n = torch.randint(0, T + 1, (B,), generator=g).to(torch.int32)
        n[:3] = torch.tensor([0, 1, T])[:B]
    return q, k, v, lg, n, torch.randn(B, Hk, D, D, generator=g)


# far more workgroups than the card holds at once; few; tokens cut into segments (one with shared heads, one without)
CASES = [(600, 96, 8, 2, 64), (400, 65, 4, 4, 64), (300, 70, 16, 2, 128), (3, 70, 4, 2, 32), (3, 70, 4, 1, 33), (1, 3000, 4, 2, 64), (1, 3000, 2, 2, 64),
         (2, 1, 6, 2, 32), (5, 0, 4, 2, 32)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("shape", CASES)
def test_state_in_place(shape, ragged, dtype):
    import paper_2211_06934_amd as P
    B, T, H, Hk, D = shape
    q, k, v, lg, n, s0 = _operands(*shape, dtype, ragged, seed=B + T)
    dev = [x.cuda() for x in (q, k, v, lg)]
    n = None if n is None else n.cuda()
    out, out2 = (torch.full((B, T, H, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    apart, state = torch.full_like(s0, 7.0, device="cuda"), s0.cuda()
    P.linattn_fwd(*dev, out, state=s0.cuda(), state_out=apart, lengths=n, scale=0.25)
    P.linattn_fwd(*dev, out2, state=state, state_out=state, lengths=n, scale=0.25)
    assert torch.equal(out, out2)
    assert_close(state, apart.double().cpu(), F32)  # the same sums, in kernels of their own
    if B * T <= 500 and T:
        ref, s1 = linattn(q, k, v, lg, s0, None if n is None else n.cpu(), 0.25)
        assert_close(out2, ref, tol(dtype, products=True))
        assert_close(state, s1, F32)
    if n is not None and T:
        assert torch.equal(state[0].cpu(), s0[0])  # a length of zero


def test_state_in_place_through_the_python_path(monkeypatch):
    import paper_2211_06934_amd as P
    q, k, v, lg, _, s0 = _operands(40, 80, 4, 2, 32, torch.float32, False, 1)
    dev = [x.cuda() for x in (q, k, v, lg)]
    got = []
    for native in (P.operators._native, P.diffopt._NoNative()):
        monkeypatch.setattr(P.operators, "_native", native)
        out, state = torch.empty(40, 80, 4, 32, device="cuda"), s0.cuda()
        P.linattn_fwd(*dev, out, state=state, state_out=state)
        got.append((out, state))
    assert all(torch.equal(x, y) for x, y in zip(*got))
