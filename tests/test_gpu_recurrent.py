"""The gated recurrence and the log probabilities through torch.autograd: first
and second derivatives against fp64 ones of plain formulas, inside the
meta-optimizers with clipping, the example that runs them together, and
refusals."""
import math
import os
import sys

import pytest
import torch

from lm_reference import F32, assert_close, tol

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def _derivatives(fn, args, cots=None, cc=None, seed=0):
    """(values, first, second derivatives, cotangents, their own) of fn(*args), which gives a list."""
    args = [a.detach().clone().requires_grad_(True) for a in args]
    out = fn(*args)
    gen = torch.Generator().manual_seed(seed)
    if cots is None:
        cots = [torch.randn(o.shape, generator=gen).to(o.dtype) for o in out]
    cots = [c.to(o.device, torch.float64 if o.dtype == torch.float64 else c.dtype).requires_grad_(True) for c, o in zip(cots, out)]
    first = torch.autograd.grad(out, args, cots, create_graph=True)
    if cc is None:
        cc = [torch.randn(g.shape, generator=gen).to(g.dtype) for g in first]
    second = torch.autograd.grad(first, [*cots, *args], [c.to(g.device, g.dtype) for c, g in zip(cc, first)], allow_unused=True)
    second = [torch.zeros_like(x) if s is None else s for s, x in zip(second, [*cots, *args])]
    return out, first, second, [c.detach().cpu() for c in cots], cc


def _compare(ours, ref, bounds):
    for group, r, bound, order in zip(ours[:3], ref[:3], bounds, ("value", "gradient", "second")):
        for i, (x, y) in enumerate(zip(group, r)):
            assert_close(x, y, bound, "%s %d" % (order, i))


def _scan(lg, x, state, lengths):
    h, outs = state, []
    for t in range(x.shape[1]):
        live = (t < lengths)[:, None]
        h = torch.where(live, torch.exp(torch.where(live, lg[:, t], 0.0)) * h + x[:, t], h)
        outs.append(torch.where(live, h, 0.0))
    return torch.stack(outs, 1), h


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(2, 1, 3), (2, 70, 33), (3, 150, 130), (1, 700, 65)])
def test_gated_scan_twice(shape, dtype):
    import paper_2211_06934_amd as P
    B, T, C = shape
    gen = torch.Generator().manual_seed(T)
    lg = (-0.5 * torch.rand(B, T, C, generator=gen)).to(dtype)
    x, s0 = torch.randn(B, T, C, generator=gen).to(dtype), torch.randn(B, C, generator=gen)
    lengths = torch.tensor([T, max(T - 2, 0), 0][:B], dtype=torch.int32)
    ours = _derivatives(lambda *a: P.gated_scan(*a, lengths.cuda(), return_state=True), [v.cuda() for v in (lg, x, s0)])
    ref = _derivatives(lambda *a: _scan(*a, lengths), [v.double() for v in (lg, x, s0)], *ours[3:])
    one = tol(dtype)
    _compare(ours, ref, (one, one, one))


def _scores(logits, ids, T, K):
    """fp64 (logprob, entropy, tops)."""
    lp = torch.log_softmax(logits / T, 1)
    there = (ids >= 0).double()
    by = torch.sort(logits.detach(), dim=1, descending=True, stable=True).indices[:, :K]
    return [lp.gather(1, ids.clamp(min=0)[:, None])[:, 0] * there, -(lp.exp() * lp).sum(1) * there, lp.gather(1, by) * there[:, None]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,K,T", [(5, 97, 7, 1.0), (3, 1030, 16, 2.0), (2, 40000, 1, 0.5), (2, 140001, 20, 1.0)])
def test_token_logprobs_twice(N, V, K, T, dtype):
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(V)
    logits = (2 * torch.randn(N, V, generator=gen)).to(dtype)
    ids = torch.randint(0, V, (N,), generator=gen)
    ids[-1] = -1

    def fn(x):
        got = P.token_logprobs(x, ids.cuda(), T, entropy=True, top=K)
        return [got.logprob, got.entropy, torch.where(got.top_ids >= 0, got.top_logprob, 0.0)]

    ours = _derivatives(fn, [logits.cuda()])
    ref = _derivatives(lambda x: _scores(x, ids, T, K), [logits.double()], *ours[3:])
    one = tol(dtype)
    _compare(ours, ref, (F32, one, one))
    # the cotangents' own gradients are fp32
    for x, y in zip(ours[2][:3], ref[2][:3]):
        assert_close(x, y, F32)


def test_parts_of_token_logprobs():
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(4, 50, generator=gen).cuda().requires_grad_(True)
    ids = torch.tensor([1, 2, -1, 49], dtype=torch.int32).cuda()
    whole = P.token_logprobs(x, ids, entropy=True, top=3)
    alone = P.token_logprobs(x, ids)
    assert alone.entropy is None and alone.top_ids is None and torch.equal(alone.logprob, whole.logprob)
    free = P.token_logprobs(x, top=3)
    assert free.logprob is None and torch.equal(free.top_ids[:2], whole.top_ids[:2]) and (whole.top_ids[2] == -1).all() and (free.top_ids[2] >= 0).all()
    nll = torch.nn.functional.cross_entropy(x.double().cpu(), ids.long().cpu(), ignore_index=-1, reduction="none")
    assert_close(-alone.logprob, nll, F32)
    for got in (alone.logprob.sum(), P.token_logprobs(x, entropy=True).entropy.sum(), free.top_logprob[:, 1].sum()):
        (g,) = torch.autograd.grad(got, [x], create_graph=True)
        (h,) = torch.autograd.grad(g.square().sum(), [x], create_graph=True)
        assert torch.isfinite(h).all() and h.any()
        with pytest.raises(RuntimeError):  # a third order is refused, not taken as zero
            torch.autograd.grad(h.sum(), [x])


# Through two inner steps and back: a chain of about thirty operations, each within one rounding (or F32) of its norm, adding
# like a random walk; sums may cancel to a tenth of their terms: 10 sqrt(30) of the unit.
@pytest.mark.parametrize("dtype,bound", [(torch.float32, 55 * F32), (torch.bfloat16, 55 * 2.0 ** -8)])
@pytest.mark.parametrize("max_norm", [0.2, 50.0])
def test_meta_gradient_through_the_inner_loop(dtype, bound, max_norm):
    """The gradient of the outer loss to the tokens' weights through two clipped inner steps of MetaSGD with momentum, against
    the same loop in fp64 from plain formulas."""
    import recurrent_inner_loop as E
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(0)
    vocab, B, T = 31, 2, 9
    torch.manual_seed(0)
    student = E.Student(vocab, 24, 40, dtype)
    start = {n: t.clone() for n, t in student.state_dict().items()}
    x, target = (torch.randint(vocab, (B, T), generator=gen) for _ in range(2))
    clean = torch.randint(vocab, (B, T), generator=gen)
    target[1, 6:] = -1
    w0 = torch.randn(B, T, generator=gen)

    student = student.cuda()
    weights = w0.cuda().requires_grad_(True)
    opt = P.MetaSGD(student, lr=0.3, momentum=0.9, max_norm=max_norm)
    for _ in range(2):
        opt.step(E.inner_loss(student, x.cuda(), target.cuda(), weights))
    (grad,) = torch.autograd.grad(E.outer_loss(student, x.cuda(), clean.cuda()), [weights])

    names = [n for n, _ in student.named_parameters()]

    def logits(p):
        e = p["embed"][x]
        lg = -torch.nn.functional.softplus(p["rate"]) * torch.sigmoid(e @ p["gate"].T)
        h, _ = _scan(lg, e @ p["into"].T, torch.zeros(B, 40, dtype=torch.float64), torch.full((B,), T))
        return ((e + h @ p["mix"].T) @ p["top"].T).flatten(0, 1)

    p = {n: start[n].double().requires_grad_(True) for n in names}
    w = w0.double().requires_grad_(True)
    trace = [torch.zeros_like(p[n]) for n in names]
    for _ in range(2):
        lp, entropy, _ = _scores(logits(p), target.flatten(), 1.0, 1)
        loss = -(torch.sigmoid(w).flatten() * lp + 0.02 * entropy).sum() / target.numel()
        g = torch.autograd.grad(loss, [p[n] for n in names], create_graph=True)
        norm = torch.sqrt(sum((v * v).sum() for v in g))
        g = [v * torch.clamp(max_norm / (norm + 1e-6), max=1.0) for v in g]
        trace = [a + 0.9 * b for a, b in zip(g, trace)]
        p = {n: p[n] - 0.3 * v for n, v in zip(names, trace)}
    (ref,) = torch.autograd.grad(torch.nn.functional.cross_entropy(logits(p), clean.flatten()), [w])
    assert float((grad.double().cpu() - ref).norm()) <= bound * float(ref.norm())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_example(dtype, capsys):
    import recurrent_inner_loop as E
    outer, inner, got, distilled, back = E.main(["--outer", "3", "--inner", "2", "--dtype", dtype])
    assert all(math.isfinite(v) for v in (*outer, *inner, distilled))
    assert got.shape == (8, 8) and torch.isfinite(back).all() and back.any()


def test_generation_agrees_with_the_prompt():
    """A token at a time from the prompt's state gives the logits that one call over all tokens gives."""
    import recurrent_inner_loop as E
    torch.manual_seed(3)
    student = E.Student().cuda()
    tokens = torch.randint(257, (3, 30), generator=torch.Generator().manual_seed(1)).cuda()
    with torch.no_grad():
        whole = student(tokens)
        _, state = student(tokens[:, :20], return_state=True)
        for t in range(20, 30):
            assert_close(student.step(tokens[:, t], state), whole[:, t].double().cpu(), 4 * F32)  # and four matrix products


def test_expanded_operands_and_cotangents():
    import paper_2211_06934_amd as P
    gen = torch.Generator().manual_seed(4)
    lg = (-0.3 * torch.rand(1, 1, 20, generator=gen)).cuda().requires_grad_(True)
    x = torch.randn(3, 12, 20, generator=gen).cuda().requires_grad_(True)
    s0 = torch.randn(1, 20, generator=gen).cuda().requires_grad_(True)
    h, s1 = P.gated_scan(lg.expand(3, 12, -1), x.transpose(1, 2).contiguous().transpose(1, 2), s0.expand(3, -1), return_state=True)
    grads = torch.autograd.grad(h.sum() + s1.sum(), [lg, x, s0], create_graph=True)
    second = torch.autograd.grad(sum((g * g).sum() for g in grads), [lg, x, s0])
    a, b, c = (t.detach().double().cpu().requires_grad_(True) for t in (lg, x, s0))
    r, r1 = _scan(a.expand(3, 12, -1), b, c.expand(3, -1), torch.full((3,), 12))
    ref = torch.autograd.grad(r.sum() + r1.sum(), [a, b, c], create_graph=True)
    for got, want in zip(grads, ref):
        assert_close(got, want, F32)
    for got, want in zip(second, torch.autograd.grad(sum((g * g).sum() for g in ref), [a, b, c])):
        assert_close(got, want, 3 * F32)
    # one operand alone
    for i, (args, want) in enumerate((((a, b.detach()), a), ((a.detach(), b), b))):
        ours = [t.detach().float().cuda() for t in (a, b)]
        ours[i].requires_grad_(True)
        (got,) = torch.autograd.grad(P.gated_scan(ours[0].expand(3, 12, -1), ours[1]).square().sum(), [ours[i]], create_graph=True)
        (twice,) = torch.autograd.grad(got.square().sum(), [ours[i]])
        r0 = _scan(args[0].expand(3, 12, -1), args[1], torch.zeros(3, 20, dtype=torch.float64), torch.full((3,), 12))[0]
        (ref0,) = torch.autograd.grad(r0.square().sum(), [want], create_graph=True)
        assert_close(got, ref0, 3 * F32)
        assert_close(twice, torch.autograd.grad(ref0.square().sum(), [want])[0], 9 * F32)
    # the state alone, and nothing but h
    (only,) = torch.autograd.grad(P.gated_scan(lg.expand(3, 12, -1), x, s0.expand(3, -1), return_state=True)[1].sum(), [s0])
    assert_close(only, torch.autograd.grad(_scan(a.expand(3, 12, -1), b, c.expand(3, -1), torch.full((3,), 12))[1].sum(), [c])[0], F32)


def test_refusals():
    import paper_2211_06934_amd as P
    x, s = torch.randn(2, 5, 8).cuda().requires_grad_(True), torch.randn(2, 8).cuda()
    (g,) = torch.autograd.grad(P.gated_scan(x, x).sum(), [x], create_graph=True)
    (h,) = torch.autograd.grad(g.square().sum(), [x], create_graph=True)
    with pytest.raises(RuntimeError):  # a third order is refused
        torch.autograd.grad(h.sum(), [x])
    with pytest.raises(ValueError, match="state"):
        P.gated_scan(x, x, s[:1])
    with pytest.raises(ValueError, match="float16"):
        P.gated_scan(x.half(), x.half())
    with pytest.raises(ValueError, match="asks for a gradient"):
        P.gated_scan_step(x[:, 0], x[:, 0].detach(), s)
    state = torch.randn(2, 8).cuda().requires_grad_(True)
    out = P.gated_scan(x, x, state)
    with torch.no_grad():
        P.gated_scan_step(x[:, 0], x[:, 0], state)  # moves the state's version
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(out.sum(), [state])
    with pytest.raises(ValueError, match="top must be"):
        P.token_logprobs(x[0], top=-1)
    with pytest.raises(ValueError, match="ids"):
        P.token_logprobs(x[0], torch.zeros(5).cuda())
    with pytest.raises(ValueError, match="device memory"):
        P.token_logprobs(torch.zeros(2, 9), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="device memory"):
        P.gated_scan(torch.zeros(2, 3, 4), torch.zeros(2, 3, 4))
