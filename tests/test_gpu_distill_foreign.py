"""A token that the vocabulary does not have makes its row's results NaN in every
direction, whatever cotangents are given, and no other row's."""
import math

import pytest
import torch

from test_gpu_distill import _inputs

pytestmark = pytest.mark.gpu


# rows in registers, rows read twice, rows cut into slices
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 4099, 140001])
@pytest.mark.parametrize("with_a", [False, True])
@pytest.mark.parametrize("with_c", [False, True])
def test_second_derivative_of_a_foreign_token(with_a, with_c, V, dtype):
    import paper_2211_06934_amd as P
    ops = _inputs(4, V, 6, dtype, holes=False)
    ops[1][2, 3] = V  # not a token
    x, ids, t, g, a, c = (o.cuda() for o in ops)
    loss, stats = torch.empty(4, device="cuda"), torch.empty(4, 2, device="cuda")
    P.distill_fwd(x, ids, t, loss, stats)
    assert torch.isnan(loss[2]) and int(torch.isnan(loss).sum()) == 1
    o = [torch.full_like(y, math.inf) for y in (g, x, t)]
    P.distill_bwd_bwd(a if with_a else None, c if with_c else None, g, x, ids, t, stats, *o)
    for y in o:
        assert torch.isnan(y[2]).all()
        assert torch.isfinite(torch.cat([y[:2], y[3:]])).all()
    assert with_a or not o[1][3].float().abs().sum() > 0 or with_c  # without cotangents the gradient is zero
