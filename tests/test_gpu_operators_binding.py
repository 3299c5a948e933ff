"""The native half of the operators' binding takes and refuses what the Python
path does, with the same results, and calls on a given stream own their scratch."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _calls():
    """name -> (function, results, arguments) of every operator on small operands."""
    import paper_2211_06934_amd as P
    g = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    B, T, H, Hk, D = 2, 600, 4, 2, 64
    q, k, v, do, s0 = r(B, T, H, D), r(B, T, Hk, D), r(B, T, Hk, D), r(B, T, H, D), r(B, Hk, D, D)
    lg, n = -torch.rand(Hk, device="cuda", generator=g), torch.tensor([T, 77], dtype=torch.int32, device="cuda")
    w, c, s = r(D), r(T, 16), r(T, 16)
    pos = torch.randint(0, T, (B, T), device="cuda", generator=g)
    x, a, ids = r(9, 3001), r(9, 3001), torch.randint(0, 3001, (9, 7), device="cuda", generator=g)
    t, ct, gl = r(9, 7), r(9, 7), r(9)
    e = torch.empty_like
    loss, stats = torch.empty(9, device="cuda"), torch.empty(9, 2, device="cuda")
    P.distill_fwd(x, ids, t, loss, stats)
    kw = dict(positions=pos, interleaved=True)

    def case(fn, out, *args, **kws):
        return fn, out, args, kws

    out = {}
    o = [e(do), e(s0)]
    out["linattn_fwd"] = case(P.linattn_fwd, o, q, k, v, lg, o[0], state=s0, state_out=o[1], lengths=n, scale=0.5)
    o = [e(q), e(k), e(v), e(s0)]
    out["linattn_bwd"] = case(P.linattn_bwd, o, do, q, k, v, lg, *o[:3], state=s0, dstate=o[3], lengths=n, scale=0.5)
    o = [e(q[:, 0]), s0.clone()]
    out["linattn_step"] = case(P.linattn_step, o, q[:, 0], k[:, 0], v[:, 0], lg, o[1], o[0])
    o = [e(q), e(k)]
    out["qknorm_rope_fwd"] = case(P.qknorm_rope_fwd, o, q, k, w, None, c, s, *o, **kw)
    o = [e(q), e(k), e(w)]
    out["qknorm_rope_bwd"] = case(P.qknorm_rope_bwd, o, do, v, q, k, w, None, c, s, *o, **kw)
    o = [e(q), e(k), e(q), e(k), e(w), e(w)]
    out["qknorm_rope_bwd_bwd"] = case(P.qknorm_rope_bwd_bwd, o, do, v, w, None, q, k, do, v, w, None, c, s, *o, **kw)
    o = [e(loss), e(stats)]
    out["distill_fwd"] = case(P.distill_fwd, o, x, ids, t, *o, temperature=2.0)
    o = [e(x), e(t)]
    out["distill_bwd"] = case(P.distill_bwd, o, gl, x, ids, t, stats, *o)
    o = [e(loss), e(stats), e(x), e(t)]
    out["distill_fwd_bwd"] = case(P.distill_fwd_bwd, o, gl, x, ids, t, *o)
    o = [e(gl), e(x), e(t)]
    out["distill_bwd_bwd"] = case(P.distill_bwd_bwd, o, a, ct, gl, x, ids, t, stats, *o)
    return out


NAMES = ["linattn_fwd", "linattn_bwd", "linattn_step", "qknorm_rope_fwd", "qknorm_rope_bwd", "qknorm_rope_bwd_bwd", "distill_fwd",
         "distill_bwd", "distill_fwd_bwd", "distill_bwd_bwd"]


@pytest.mark.parametrize("name", NAMES)
def test_native_and_python_paths_agree(name, monkeypatch):
    import paper_2211_06934_amd as P
    taken = []

    class Seen:
        def __getattr__(self, n):
            def call(*args):
                got = getattr(native, n)(*args)
                taken.append(got)
                return got
            return call

    native = P.operators._native
    fn, out, args, kw = _calls()[name]
    monkeypatch.setattr(P.operators, "_native", Seen())
    fn(*args, **kw)
    assert taken == [0]  # the native module ran the call
    fn, out2, args, kw = _calls()[name]
    monkeypatch.setattr(P.operators, "_native", P.diffopt._NoNative())
    fn(*args, **kw)
    assert all(torch.equal(x, y) for x, y in zip(out, out2))


@pytest.mark.parametrize("name", NAMES)
def test_a_given_stream(name):
    fn, ref, args, kw = _calls()[name]
    fn(*args, **kw)
    torch.cuda.synchronize()
    for _ in range(2):
        fn, out, args, kw = _calls()[name]
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        fn(*args, stream=s, **kw)
        junk = [torch.full((1 << 16,), 7.0, device="cuda") for _ in range(8)]  # the current stream allocates and writes meanwhile
        s.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(ref, out))
        del junk


@pytest.mark.parametrize("name", ["linattn_fwd", "linattn_bwd", "qknorm_rope_fwd", "qknorm_rope_bwd", "distill_fwd_bwd", "distill_bwd_bwd"])
def test_graph_replays(name):
    # a captured call gives the eager result on every replay, with eager work between
    fn, ref, args, kw = _calls()[name]
    fn(*args, **kw)
    fn, out, args, kw = _calls()[name]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fn(*args, **kw)
    for _ in range(3):
        for x in out:
            x.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(ref, out))
        fn2, _, args2, kw2 = _calls()[name]
        fn2(*args2, **kw2)
