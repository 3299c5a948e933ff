"""Single tokens beside a graph that saved their state."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_backward_after_a_step_on_a_saved_state_is_refused():
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(1, 5, 2, 8, generator=gen).cuda() for _ in range(3))
    lg, state = torch.full((2,), -0.1).cuda(), torch.randn(1, 2, 8, 8, generator=gen).cuda()
    q.requires_grad_()
    loss = P.linear_attention(q, k, v, lg, state=state).sum()
    (grad,) = torch.autograd.grad(loss, [q], retain_graph=True)
    P.linear_attention_step(k[:, 0], k[:, 0], v[:, 0], lg, state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    # a copy of the state steps beside the graph
    state = state.clone()
    loss = P.linear_attention(q, k, v, lg, state=state).sum()
    P.linear_attention_step(k[:, 0], k[:, 0], v[:, 0], lg, state.clone())
    loss.backward()
    assert torch.isfinite(grad).all() and torch.isfinite(q.grad).all()
