"""The gated recurrence where operands and results are views of one buffer: beside
one another they are taken, over one another refused."""
import math

import pytest
import torch

import paper_2211_06934_amd as P
from test_gpu_gscan import _inputs, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,C", [(3, 70, 37), (2, 1500, 8), (1, 300, 130), (66, 1100, 5)])
@pytest.mark.parametrize("kind", ["side by side", "one after another", "odd places"])
def test_parts_of_one_buffer(B, T, C, kind, dtype):
    # operands and results whose rows lie beside one another's are apart
    I = _inputs(B, T, C, dtype, seed=T, resets=False)
    want = _run(I)
    pad = 3 if kind == "odd places" else 0
    if kind == "one after another":
        buf = torch.full((12, B, T, C), math.nan, dtype=dtype, device="cuda")
        part = list(buf)
    else:
        buf = torch.full((B, T, 12 * (C + pad)), math.nan, dtype=dtype, device="cuda")
        part = [buf[:, :, i * (C + pad) + pad // 2 : i * (C + pad) + pad // 2 + C] for i in range(12)]
    free = iter(part)
    got = _run(I, lambda t: next(free).copy_(t), lambda: next(free).zero_())
    for k in want:
        assert torch.equal(got[k], want[k]), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [40, 700, 1500])
def test_shifted_views_are_refused(T, dtype):
    buf, lg, other = (torch.zeros(3, T + 1, 70, dtype=dtype, device="cuda") for _ in range(3))
    early, late, lg, other = buf[:, :-1], buf[:, 1:], lg[:, :-1], other[:, :-1]
    for x, h in ((early, late), (late, early)):
        with pytest.raises(P.DiffoptError, match="h must lie apart from x"):
            P.gscan_fwd(lg, x, h)
        with pytest.raises(P.DiffoptError, match="dx must lie apart from dh"):
            P.gscan_bwd(x, lg, other, None, h)
        with pytest.raises(P.DiffoptError, match="out_dh must lie apart from ddx"):
            P.gscan_bwd_bwd(other, x, other, lg, other, h, torch.empty_like(lg), torch.empty_like(lg))
    state = torch.zeros(9, 70, device="cuda")
    with pytest.raises(P.DiffoptError, match="state must lie apart"):
        P.gscan_step(lg[:, 0].float(), state[1:4], state[:3], torch.empty(3, 70, device="cuda"))
    with pytest.raises(P.DiffoptError, match="out must lie apart"):
        P.gscan_step(state[:3], state[3:6], state[6:], state[1:4])
