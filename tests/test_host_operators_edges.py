"""Edges of the operators' arguments that are refused on the host, before any device call."""
import pytest

from test_host_operators import _distill, _refused


@pytest.mark.parametrize("T", [2.4e-39, 3e-39, 4.2e-39])
def test_temperatures_whose_inverse_overflows_are_refused(T):
    # 1 / T is finite in fp32 from 2.94e-39 on, log2(e) / T, by which the kernels scale, only from 4.24e-39 on
    _refused(_distill(T=T), "temperature")


@pytest.mark.parametrize("call", ["linear_attention", "linear_attention_step"])
@pytest.mark.parametrize("name", ["q", "k", "v"])
@pytest.mark.parametrize("bad", [(8,), (2, 8), ()])
def test_operands_of_other_axes_are_named(call, name, bad):
    import torch

    import paper_2211_06934_amd as P
    shape = (1, 3, 2, 8) if call == "linear_attention" else (1, 2, 8)
    a = {n: torch.zeros(bad if n == name else shape) for n in ("q", "k", "v")}
    extra = {} if call == "linear_attention" else dict(state=torch.zeros(1, 2, 8, 8))
    with pytest.raises(ValueError, match="%s: expected a tensor of %d axes" % (name, len(shape))):
        getattr(P, call)(a["q"], a["k"], a["v"], torch.zeros(2), **extra)
    a[name] = None
    with pytest.raises(ValueError, match="%s: expected a tensor" % name):
        getattr(P, call)(a["q"], a["k"], a["v"], torch.zeros(2), **extra)


def test_workspaces_on_another_device_are_refused():
    import torch

    import paper_2211_06934_amd as P

    class On(torch.Tensor):  # bytes that say which device they are on, without one
        @staticmethod
        def __new__(cls, n, device):
            return torch.Tensor._make_wrapper_subclass(cls, (n,), dtype=torch.uint8, device=device)

        def data_ptr(self):
            return 64

        __torch_dispatch__ = None

    one, two = torch.device("cuda", 0), torch.device("cuda", 1)
    assert P.operators._scratch(On(256, one), 256, one, None)[1:] == (64, 256)
    with pytest.raises(ValueError, match="cuda:1"):
        P.operators._scratch(On(256, two), 256, one, None)
