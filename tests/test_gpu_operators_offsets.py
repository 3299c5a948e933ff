"""Operators on operands whose offsets pass 32 bits (heads, tokens or sequences
gigabytes apart) and on rows aligned to 4 bytes but not to 16.  The results are
those of the same values in compact tensors, element for element where the same
kernels run, else within the type's tolerance of each other."""
import pytest
import torch

from lm_reference import assert_close, tol

pytestmark = pytest.mark.gpu

GIB = 1 << 30


@pytest.fixture(scope="module")
def far():
    """14 GiB of device memory, of which little is touched."""
    buf = torch.empty(14 * GIB, dtype=torch.uint8, device="cuda")
    yield buf
    del buf


def _place(far, x, axis, step_bytes, at=0):
    """x's values with `axis` step_bytes apart (the other axes compact), from byte `at` of the buffer on."""
    flat = far[at:at + (far.numel() - at) // 16 * 16].view(x.dtype)
    strides, run = [0] * x.dim(), 1
    for a in reversed(range(x.dim())):
        if a != axis:
            strides[a] = run
            run *= x.shape[a]
    strides[axis] = step_bytes // x.element_size()
    assert strides[axis] >= run
    return flat.as_strided(x.shape, strides).copy_(x)


# axis, bytes from one to the next, sizes: sequences, heads and tokens far apart
# (tokens 64 MiB apart are past what a chunk's 32-bit offsets hold)
PLACES = [(0, 3 * GIB, (2, 70, 2, 64)), (2, 3 * GIB, (1, 70, 2, 64)), (1, 32 << 20, (1, 70, 2, 64)), (1, 64 << 20, (1, 40, 2, 64))]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("axis,step,shape", PLACES)
def test_linear_attention(far, axis, step, shape, dtype):
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(3)
    q, k, v, do = (torch.randn(*shape, generator=gen).to(dtype).cuda() for _ in range(4))
    lg = torch.tensor([-0.2, -0.01]).cuda()

    def run(put):
        ops = [put(x, i * (GIB // 16)) for i, x in enumerate((q, k, v, do))]
        outs = [put(torch.empty_like(q), (4 + i) * (GIB // 16)) for i in range(4)]
        P.linattn_fwd(*ops[:3], lg, outs[0])
        P.linattn_bwd(ops[3], *ops[:3], lg, *outs[1:])
        return [o.double().cpu() for o in outs]

    # the operands interleave: each starts elsewhere within the step
    sub = step // 8 // 16 * 16
    near = run(lambda x, at: x.clone())
    away = run(lambda x, at: _place(far, x, axis, step, at // (GIB // 16) * sub))
    for x, y in zip(away, near):
        assert_close(x, y, tol(dtype, True))


@pytest.mark.parametrize("axis,step,shape", PLACES[:3])
def test_qknorm_rope(far, axis, step, shape):
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(3)
    q, k, dq, dk = (torch.randn(*shape, generator=gen).cuda() for _ in range(4))
    angle = torch.rand(shape[1], 16, generator=gen)
    cos, sin = torch.cos(angle).cuda(), torch.sin(angle).cuda()
    sub = step // 8 // 16 * 16

    def run(put):
        ops = [put(x, i) for i, x in enumerate((q, k, dq, dk))]
        outs = [put(torch.empty_like(q), 4 + i) for i in range(4)]
        P.qknorm_rope_fwd(*ops[:2], None, None, cos, sin, *outs[:2])
        P.qknorm_rope_bwd(*ops[2:], *ops[:2], None, None, cos, sin, *outs[2:])
        return [o.cpu() for o in outs]

    for x, y in zip(run(lambda x, i: _place(far, x, axis, step, i * sub)), run(lambda x, i: x.clone())):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1001, 40000])
def test_distillation(far, V, dtype):
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(4, V, generator=gen).to(dtype).cuda()
    ids = torch.randint(V, (4, 9), generator=gen).cuda()
    t, g = torch.randn(4, 9, generator=gen).cuda(), torch.randn(4, generator=gen).cuda()

    def run(put):
        loss, stats, a = torch.empty(4, device="cuda"), torch.empty(4, 2, device="cuda"), put(x, 0)
        d = put(torch.empty_like(x), GIB)
        P.distill_fwd(a, ids, t, loss, stats)
        P.distill_bwd(g, a, ids, t, stats, d)
        return loss.cpu(), d.double().cpu()

    # rows of 16-byte alignment in both: sums in pieces run in the same order
    near = run(lambda x, at: torch.zeros(4, 40960, dtype=dtype, device="cuda")[:, :V].copy_(x))
    away = run(lambda x, at: _place(far, x, 0, 3 * GIB, at))
    assert torch.equal(near[0], away[0])
    assert_close(away[1], near[1], tol(dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("skip", [1, 2, 4])
def test_rows_aligned_to_less_than_16_bytes(skip, dtype):
    """Rows a few elements longer than the heads, from an odd place on: 2, 4 or 8 bytes are all the alignment there is."""
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(8)
    B, T, H, D = 2, 131, 2, 64
    q, k, v, do = (torch.randn(B, T, H, D, generator=gen).to(dtype).cuda() for _ in range(4))
    lg = torch.tensor([-0.2, -0.01]).cuda()

    def shifted(x):
        buf = torch.zeros(B * T * H * (D + skip) + skip, dtype=dtype, device="cuda")
        return buf.as_strided(x.shape, (T * H * (D + skip), H * (D + skip), D + skip, 1), skip).copy_(x)

    def run(put):
        ops, outs = [put(x) for x in (q, k, v, do)], [put(torch.empty_like(q)) for _ in range(4)]
        P.linattn_fwd(*ops[:3], lg, outs[0])
        P.linattn_bwd(ops[3], *ops[:3], lg, *outs[1:])
        return [o.double().cpu() for o in outs]

    for x, y in zip(run(shifted), run(lambda x: x.clone())):
        assert_close(x, y, tol(dtype, True))
