"""Edges of the operators' arguments that are refused on the host, before any device call."""
import pytest

from test_host_operators import _distill, _refused


@pytest.mark.parametrize("T", [2.4e-39, 3e-39, 4.2e-39])
def test_temperatures_whose_inverse_overflows_are_refused(T):
    # 1 / T is finite in fp32 from 2.94e-39 on, log2(e) / T, by which the kernels scale, only from 4.24e-39 on
    _refused(_distill(T=T), "temperature")
