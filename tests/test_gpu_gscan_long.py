"""The gated recurrence over sequences of so many chunks that a wave of the join
takes its share of them in several batches."""
import math

import pytest
import torch

import paper_2211_06934_amd as P
from lm_reference import F32, assert_close, tol
from test_gpu_gscan import _inputs, _recurrence, _reference, _run

pytestmark = pytest.mark.gpu


def _in_steps(I):
    """fp64 results of the three directions, token after token from the formulas (autograd of thousands of tokens takes seconds)."""
    lg, x, dh, r, p = (I[k].double() for k in ("lg", "x", "dh", "r", "p"))
    a, (B, T, C) = torch.exp(lg), x.shape
    n = torch.full((B,), T) if I["lengths"] is None else I["lengths"].long().clamp(0, T)
    live = (torch.arange(T)[None, :] < n[:, None])[:, :, None].expand(B, T, C)
    a, x, dh, r, p = (torch.where(live, t, other) for t, other in ((a, 1.0), (x, 0.0), (dh, 0.0), (r, 0.0), (p, 0.0)))
    a, x, dh, r, p = (t.unbind(1) for t in (a, x, dh, r, p))
    h, y, e, f = I["s0"].double(), I["s"].double(), I["ds1"].double(), torch.zeros(B, C, dtype=torch.float64)
    hp, yp, hs, ys = [], [], [], []
    for t in range(T):
        hp.append(h), yp.append(y)
        y = a[t] * (y + r[t] * h) + p[t]
        h = a[t] * h + x[t]
        hs.append(h), ys.append(y)
    back = {k: [None] * T for k in ("dlg", "dx", "out_lg", "out_x")}
    for t in reversed(range(T)):
        g, v = dh[t] + e, r[t] * (dh[t] + e) + f
        back["dx"][t], back["dlg"][t], back["out_x"][t], back["out_lg"][t] = g, a[t] * g * hp[t], f, a[t] * (g * yp[t] + v * hp[t])
        e, f = a[t] * g, a[t] * v
    rows = {k: torch.where(live, torch.stack(v, 1), 0.0) for k, v in (back | dict(h=hs, out_dh=ys)).items()}
    return rows | dict(s1=h, out_ds1=y, ds0=e, out_s0=f)


def test_the_formulas_are_those_of_the_recurrence():
    I = _inputs(3, 60, 4, torch.float32, resets=False)
    ref, got = _reference(I), _in_steps(I)
    assert set(ref) == set(got)
    for k in ref:
        assert_close(got[k], ref[k], 1e-12, k)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [8193, 9000, 16500])
def test_joins_in_batches_backwards(T, dtype):
    # more than 128 chunks of 64 tokens: a wave has 9 or more, in batches of 8; the last batch of one, of some, of all
    I = _inputs(2, T, 5, dtype, seed=T, resets=False)
    got, ref = _run(I), _in_steps(I)
    assert set(got) == set(ref)
    for k in ref:
        assert_close(got[k], ref[k], F32 if k in ("s1", "ds0", "out_ds1", "out_s0") else tol(dtype), k)


@pytest.mark.parametrize("dtype,T", [(torch.float32, 16385), (torch.float32, 20011), (torch.bfloat16, 32769), (torch.bfloat16, 41003)])
@pytest.mark.parametrize("lengths", [False, True])
def test_joins_in_batches_forwards(T, lengths, dtype):
    # more than 256 chunks, of 64 tokens in fp32 and 128 in bf16: a wave has 17 or more, in batches of 16
    I = _inputs(2, T, 3, dtype, seed=T, lengths=lengths, resets=False)
    cuda = {k: None if v is None else v.cuda() for k, v in I.items()}
    h, s1 = torch.full_like(cuda["x"], math.nan), torch.full((2, 3), math.nan, device="cuda")
    P.gscan_fwd(cuda["lg"], cuda["x"], h, cuda["s0"], s1, cuda["lengths"])
    with torch.no_grad():
        ref, last = _recurrence(I["lg"].double(), I["x"].double(), I["s0"].double(), I["lengths"])
    assert_close(h, ref, tol(dtype))
    assert_close(s1, last, F32)
