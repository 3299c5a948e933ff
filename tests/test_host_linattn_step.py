"""What linear_attention_step tells torch.autograd of the state that it updates in
place, and its refusal of operands that ask for a gradient.  No kernel is launched:
the entry point is replaced by one that moves the state behind torch's back."""
import pytest
import torch


@pytest.fixture
def step(monkeypatch):
    import paper_2211_06934_amd as P

    def entry(q, k, v, log_decay, state, out, scale):
        state.numpy()[...] += 1.0  # as a kernel does: through the address
        out.zero_()

    monkeypatch.setattr(P.language._o, "linattn_step", entry)
    return P.linear_attention_step


def _operands():
    q = torch.ones(1, 2, 8)
    return dict(q=q, k=q.clone(), v=q.clone(), log_decay=torch.zeros(2), state=torch.zeros(1, 2, 8, 8))


def test_a_saved_state_that_moved_is_noticed(step):
    a = _operands()
    x = torch.ones(1, 2, 8, 8, requires_grad=True)
    loss = (x * a["state"]).sum()  # saves the state
    before = a["state"]._version
    step(**a)
    assert a["state"]._version > before and float(a["state"].max()) == 1.0
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_a_view_moves_its_base(step):
    a = _operands()
    states = torch.zeros(3, 1, 2, 8, 8)  # one for each layer
    before = states._version
    step(**dict(a, state=states[1]))
    assert states._version > before and float(states[1].min()) == 1.0 and not states[0].any()


@pytest.mark.parametrize("name", ["q", "k", "v", "log_decay", "state"])
def test_operands_that_ask_for_gradients_are_refused(step, name):
    a = _operands()
    a[name] = a[name].requires_grad_()
    with pytest.raises(ValueError, match=name):
        step(**a)
    assert not a["state"].any()  # nothing was run
    with torch.no_grad():
        assert not step(**a).requires_grad
    assert float(a["state"].detach().max()) == 1.0


def test_inference_tensors(step):
    with torch.inference_mode():
        a = _operands()
        step(**a)
        assert float(a["state"].max()) == 1.0
    with torch.no_grad():
        step(**a)
    assert float(a["state"].max()) == 2.0
