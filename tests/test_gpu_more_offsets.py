"""The gated recurrence, log probabilities and clipping on operands whose
offsets pass 32 bits: the results are those of the same values in compact
tensors, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu

GIB = 1 << 30


@pytest.fixture(scope="module")
def far():
    """16 GiB of device memory, of which little is touched."""
    buf = torch.empty(16 * GIB, dtype=torch.uint8, device="cuda")
    yield buf
    del buf


def _place(far, x, axis, step_bytes, at):
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("axis,step,shape", [(0, 3 * GIB, (3, 150, 130)), (1, 64 << 20, (1, 150, 130)), (1, 16 << 20, (1, 700, 70))])
def test_gated_scan(far, axis, step, shape, dtype):
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(3)
    lg, x, dh, r, p = (torch.randn(*shape, generator=gen).to(dtype).cuda() for _ in range(5))
    lg = -lg.abs() * 0.1

    def run(put):
        ops = [put(t, i) for i, t in enumerate((lg, x, dh, r, p))]
        o = [put(torch.empty_like(x), 5 + i) for i in range(6)]
        P.gscan_fwd(ops[0], ops[1], o[0])
        P.gscan_bwd(ops[2], ops[0], ops[1], o[1], o[2])
        P.gscan_bwd_bwd(ops[3], ops[4], ops[2], ops[0], ops[1], *o[3:])
        return [t.cpu() for t in o]

    sub = step // 16 // 16 * 16  # the operands interleave
    for a, b in zip(run(lambda t, i: _place(far, t, axis, step, i * sub)), run(lambda t, i: t.clone())):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1000, 40000])
def test_log_probabilities(far, V, dtype):
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(3)
    x, a = ((2 * torch.randn(4, V, generator=gen)).to(dtype).cuda() for _ in range(2))
    ids = torch.tensor([1, 5, -1, V - 1]).cuda()
    g, h, c = (torch.randn(*s, generator=gen).cuda() for s in ((4,), (4,), (4, 6)))

    def run(put):
        X, A = put(x, 0), put(a, 1)
        dx, ox, both = (put(torch.empty_like(x), 2 + i) for i in range(3))
        lp, ent, st, t, ti = (torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty(4, 2, device="cuda"), torch.empty(4, 6, device="cuda"),
                              torch.empty(4, 6, dtype=torch.int64, device="cuda"))
        P.logprob_fwd(X, ids, lp, st, ent, t, ti)
        how = dict(dlogprob=g, dentropy=h, entropy=ent, dtop_logprob=c, top_ids=ti)
        P.logprob_bwd(X, ids, st, dx, **how)
        P.logprob_bwd_bwd(A, X, ids, st, ox, **how)
        first = [v.cpu() for v in (lp, ent, t, ti)]
        P.logprob_fwd_bwd(g, X, ids, lp, st, both, h, ent)
        return [*first, *(v.cpu() for v in (dx, ox, both, lp, ent))]

    for u, v in zip(run(lambda t, i: _place(far, t, 0, 3 * GIB, i * (GIB // 2))), run(lambda t, i: t.clone())):
        assert torch.equal(u, v)


def test_a_row_of_more_than_2_to_the_31_bytes():
    import paper_2211_06934_amd as P
    V = (1 << 30) + 3
    x = torch.zeros(2, V, dtype=torch.bfloat16, device="cuda")
    x[0, V - 1], x[0, 7], x[1, V - 2] = 40.0, 39.0, 3.0
    ids = torch.tensor([7, V - 1]).cuda()
    lp, st, ent = torch.empty(2, device="cuda"), torch.empty(2, 2, device="cuda"), torch.empty(2, device="cuda")
    t, ti = torch.empty(2, 3, device="cuda"), torch.empty(2, 3, dtype=torch.int64, device="cuda")
    P.logprob_fwd(x, ids, lp, st, ent, t, ti)
    assert ti.tolist() == [[V - 1, 7, 0], [V - 2, 0, 1]]
    # softmax of one, or two, values above 2^30 zeros: a sum of that many equal terms is right to sqrt(2^30 / lanes) 2^-24
    lse = torch.logsumexp(torch.tensor([[40.0, 39.0, 30 * 0.6931471805599453], [3.0, 0.0, 30 * 0.6931471805599453]], dtype=torch.float64), 1)
    want = torch.stack((39.0 - lse[0], -lse[1]))
    assert float((lp.double().cpu() - want).abs().max()) <= 1e-4


def test_more_than_2_to_the_31_elements():
    import paper_2211_06934_amd as P
    n = (1 << 31) + 77
    g = torch.zeros(n, device="cuda")
    g[5], g[1 << 30], g[n - 1] = 3.0, 4.0, 12.0
    stats = torch.empty(2, device="cuda")
    P.clip_norm_fwd(g, 6.5, g, stats, 0.0)
    assert stats.tolist() == [13.0, 0.5]
    assert g[5] == 1.5 and g[1 << 30] == 2.0 and g[n - 1] == 6.0 and int(torch.count_nonzero(g)) == 3
    # and among the leaves of a tree
    small = torch.tensor([5.0], device="cuda")
    table = P.segtable_create([1, n])
    at = P.tree.leaf_pointer_tensor([small, g], "cuda")
    g.zero_()
    g[n - 1] = 12.0
    P.clip_norm_fwd_tree(table, at, 6.5, at, stats, 0.0)
    assert stats.tolist() == [13.0, 0.5] and float(small) == 2.5 and g[n - 1] == 6.0
