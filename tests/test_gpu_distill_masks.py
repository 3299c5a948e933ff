"""Distillation over logits masked with large finite values, with a large common
offset, and at tiny temperatures: the loss, the gradients (apart and at once) and
the gradients' own VJP against autograd of the definition in fp64."""
import pytest
import torch

from lm_reference import F32, PEAK, assert_close, tol
from test_gpu_distill import _inputs, _reference, _run

pytestmark = pytest.mark.gpu

MASKS = [-1e9, -1e10, -1e12, -1e15, -1e20, -1e25, -1e30, -3e38, 0.0]


def _compare(ops, T):
    loss, first, second = _reference(*ops, T)
    got, both, got2 = _run(*ops, T)
    t = tol(ops[0].dtype)
    for res, how in ((got, "apart"), (both, "at once")):
        assert_close(res[0], loss, F32, "loss " + how)
        assert_close(res[1], first[0], t, "dlogits " + how)
        assert_close(res[2], first[1], F32, "dteacher " + how)
    assert_close(got2[0], second[0], F32, "out_dloss")
    assert_close(got2[2], second[2], F32, "out_teacher")
    # out_logits is g p (a - [p a]) - g sum_j q_j (c_j - [q c]) e_j: where one token (or entry) has nearly all the weight, a (or c)
    # cancels against its mean, so that an element is held to the rounding of its terms and not of what is left of them
    x, ids, teacher, g, a, c = (o.double() if o.is_floating_point() else o for o in ops)
    p, q, g = torch.softmax(x / T, 1), torch.softmax(teacher / T, 1), g[:, None]
    terms = g * p * (a.abs() + (p * a.abs()).sum(1, keepdim=True))
    terms.scatter_add_(1, ids, g * q * (c.abs() + (q * c.abs()).sum(1, keepdim=True)))
    err = (got2[1].double().cpu() - second[1]).abs()
    assert float(err.norm()) <= t * float(second[1].norm()) + 1e-30
    assert bool((err <= PEAK * t * (terms + second[1].abs() + second[1].square().mean().sqrt()) + 1e-30).all())


# rows that stay in the registers of each size of workgroup, and (512 KiB of fp32) one cut into slices
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1003, 8192, 20011, 50021, 131072])
@pytest.mark.parametrize("T", [0.5, 1.0, 2.0])
def test_finite_masks(T, V, dtype):
    # all but 150 tokens ruled out: most lanes see nothing but the mask
    x, ids, t, g, a, c = _inputs(len(MASKS), V, 8, dtype, seed=V, holes=False)
    ids = torch.stack([torch.randperm(150, generator=torch.Generator().manual_seed(r))[:8] for r in range(len(MASKS))])
    for r, mask in enumerate(MASKS):
        x[r, 150:] = mask
    _compare((x, ids, t, g, a, c), T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [0.5, 1.0])
def test_rows_of_one_value(T, dtype):
    # the row's own maximum is the mask: every token alike
    x, ids, t, g, a, c = _inputs(len(MASKS), 5003, 8, dtype, seed=1, holes=False)
    for r, mask in enumerate(MASKS):
        x[r] = mask
    _compare((x, ids, t, g, a, c), T)


@pytest.mark.parametrize("offset,step", [(1e10, 1024.0), (-1e10, 1024.0), (-1e15, 2.0 ** 27), (2.0 ** 60, 2.0 ** 38)])
def test_common_offset(offset, step):
    # logits a few last places of the offset apart, at a temperature of such a step
    x, ids, t, g, a, c = _inputs(6, 9001, 8, torch.float32, seed=3, holes=False)
    x = offset + step * (4 * x).round()
    assert torch.equal(x, x.double().float())
    _compare((x, ids, t * step, g, a, c), 4 * step)


def test_lanes_of_different_size_side_by_side():
    # lanes at the type's lowest value in one wave with lanes whose own shift is rounded: 1e6 keeps 16 steps a unit
    x, ids, t, g, a, c = _inputs(5, 4099, 8, torch.float32, seed=4, holes=False)
    x = 1e6 + x
    x[:, 200:] = torch.finfo(torch.float32).min
    _compare((x, ids % 200, t, g, a, c), 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_small_temperatures(dtype):
    # the logits' differences over T are enormous: all weight on one token
    _compare(_inputs(6, 3001, 8, dtype, seed=5, holes=False), 2.0 ** -30)
