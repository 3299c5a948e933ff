"""The gated recurrence where a gate of -inf meets a state that is not finite."""
import math

import pytest
import torch

from lm_reference import F32, assert_close
from test_gpu_gscan import _inputs, _reference, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [60, 300, 900, 1500])
def test_a_reset_multiplies_by_zero(T):
    # a gate of -inf forgets any finite state; an infinite one or a NaN stays a NaN, as 0 times it is
    I = _inputs(2, T, 70, torch.float32, resets=False, lengths=False)
    I["x"][0, T // 3, 4], I["x"][1, T // 3, 9], I["s0"][0, 7] = math.nan, math.inf, math.inf
    I["lg"][:, T // 2] = -math.inf
    got, ref = _run(I), _reference(I)
    for k in ("h", "s1"):
        assert torch.equal(torch.isfinite(got[k]).cpu(), torch.isfinite(ref[k])), k
        assert torch.equal(torch.isnan(got[k]).cpu(), torch.isnan(ref[k])), k
    fine = torch.isfinite(ref["h"].detach())
    assert_close(torch.where(fine, got["h"].cpu(), 0.0), torch.where(fine, ref["h"].detach(), 0.0), F32)
    assert bool(torch.isnan(got["h"][0, T // 2:, 4]).all()) and bool(torch.isnan(got["h"][1, T // 2:, 9]).all())
