"""More of the framework's language-model operators as cases that can be timed and checked.

Three operators of one inner step: a layer, the loss, and what the optimizer does to the gradient first.

  gscan    a gated linear recurrence over sequences (whole sequences and single tokens)
  logprob  log probabilities of given tokens, entropy and top alternatives
  clip     the global norm of a tree of gradients, and clipping to it

``run`` makes one pass through one of them: in its plain form (torch products,
sums and exponentials in fp32, rounded once at the end) where ``own`` is false,
through the framework's entry points where it is true.  Both take the same
state.  ``exact`` gives the result from the definitions in fp64.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a long prompt read once, its final state kept for the tokens that follow
        dict(name="scan prompt", op="gscan", mode="prompt", dtype="bf16", B=1, T=16384, C=2048, ragged=False, warm=False, resets=False),
        # a training step's recurrence, both directions
        dict(name="scan train", op="gscan", mode="train", dtype="bf16", B=4, T=4096, C=2048, ragged=False, warm=False, resets=False),
        # an inner step in fp32 whose gradient is differentiated again: padded rows, carried states, documents packed into a row
        dict(name="scan meta f32", op="gscan", mode="meta", dtype="f32", B=8, T=509, C=517, ragged=True, warm=True, resets=True),
        # one token of one user: latency
        dict(name="scan token", op="gscan", mode="step", dtype="bf16", B=1, T=1, C=2048, ragged=False, warm=True, resets=False),
        # one token of many users: the states' traffic
        dict(name="scan tokens", op="gscan", mode="step", dtype="bf16", B=512, T=1, C=4096, ragged=False, warm=True, resets=False),
        # a training step's loss with an entropy bonus and its gradient in one call, odd vocabulary, padding among the rows
        dict(name="logprob train", op="logprob", mode="train", dtype="bf16", N=4096, V=50021, K=0, padded=True, masked=False),
        # a prompt scored: every token's log probability, entropy and top alternatives
        dict(name="logprob prompt", op="logprob", mode="score", dtype="bf16", N=2048, V=50021, K=5, padded=False, masked=False),
        # the next token of a few users under a grammar that rules most of the vocabulary out
        dict(name="logprob answer f32", op="logprob", mode="score", dtype="f32", N=8, V=131072, K=20, padded=False, masked=True),
        # an inner loss whose gradient is differentiated again, through the entropy and the alternatives too
        dict(name="logprob meta f32", op="logprob", mode="meta", dtype="f32", N=1024, V=32000, K=8, padded=True, masked=False),
        # an inner loop's small network, clipped and differentiated: latency
        dict(name="clip tiny", op="clip", mode="train", layout="tiny", n=1761, norm=3.0),
        # many small tensors, clipped and differentiated
        dict(name="clip many", op="clip", mode="train", layout="many", n=20_000_000, norm=3.0),
        # a language model's tensors, clipped before the update
        dict(name="clip model", op="clip", mode="clip", layout="model", n=354_000_000, norm=3.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Sizes over the logarithm of their ranges, odd ones among them."""
    op = rng.choice(["gscan", "gscan", "logprob", "logprob", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "gscan":
        mode = rng.choice(["prompt", "train", "train", "meta", "step"])
        C = rng.choice([_log_int(rng, 16, 4096), 64 * _log_int(rng, 1, 64)])
        if mode == "step":
            return dict(op=op, mode=mode, dtype=dtype, B=_log_int(rng, 1, 512), T=1, C=C, ragged=False, warm=True, resets=rng.random() < 0.2)
        T = _log_int(rng, 1, 2048 if mode == "meta" else 16384)
        most = (4 * 4096 * 2048) // (T * C * (2 if dtype == "f32" else 1) * (4 if mode == "meta" else 1))
        return dict(op=op, mode=mode, dtype=dtype, B=_log_int(rng, 1, max(1, min(32, most))), T=T, C=C if most else 512, ragged=rng.random() < 0.4,
                    warm=rng.random() < 0.4, resets=rng.random() < 0.3)
    if op == "logprob":
        V = _log_int(rng, 100, 160000)
        mode = rng.choice(["train", "score", "split", "meta"])
        most = (4096 * 50021) // (V * (2 if dtype == "f32" else 1) * (2 if mode in ("split", "meta") else 1))
        return dict(op=op, mode=mode, dtype=dtype, N=_log_int(rng, 1, max(1, min(8192, most))), V=V, K=0 if mode == "train" else rng.choice([0, 1, 5, 20, 64, 128]),
                    padded=rng.random() < 0.5, masked=rng.random() < 0.3)
    layout = rng.choice(["flat", "tiny", "many", "model"])
    n = {"flat": (1, 100_000_000), "tiny": (100, 60_000), "many": (10_000, 20_000_000), "model": (1_000_000, 200_000_000)}[layout]
    return dict(op=op, mode=rng.choice(["clip", "train"]), layout=layout, n=_log_int(rng, *n), norm=rng.choice([0.4, 3.0, 3.0, 40.0]))


# ---- inputs -----------------------------------------------------------------


class _Draw:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed) * 6007 + 31)

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=self.gen).to(dtype)

    def uniform(self, *shape):
        return torch.rand(shape, device="cuda", generator=self.gen)


def _inputs_gscan(c, seed):
    r, dt = _Draw(seed), DTYPES[c["dtype"]]
    B, T, C = c["B"], c["T"], c["C"]
    # channels that remember from a few tokens to a few thousand, each token's gate about its channel's
    rate = torch.exp2(-1.0 - 10.0 * (torch.arange(C, device="cuda") + 0.5) / C)
    gate = -2.0 * rate * torch.sigmoid(r.normal(B, T, C))
    S = dict(x=(torch.sqrt(-torch.expm1(2.0 * gate)) * r.normal(B, T, C)).to(dt))
    if c["resets"]:  # documents of a few hundred tokens side by side in a row: nothing passes from one to the next
        gate = torch.where(r.uniform(B, T, 1) < 1.0 / 200.0, -math.inf, gate)
    S["log_gate"] = gate.to(dt)
    S["lengths"] = (T * r.uniform(B) ** 0.5).ceil().to(torch.int32) if c["ragged"] else None
    S["state"] = r.normal(B, C) if c["warm"] else None
    if c["mode"] in ("train", "meta"):
        S["dh"] = r.normal(B, T, C, dtype=dt)
        S["dstate_out"] = r.normal(B, C) if c["warm"] else None
    if c["mode"] == "meta":
        S["ddlog_gate"], S["ddx"] = r.normal(B, T, C, dtype=dt), r.normal(B, T, C, dtype=dt)
        S["ddstate"] = r.normal(B, C) if c["warm"] else None
    return S


def _inputs_logprob(c, seed):
    r, dt = _Draw(seed), DTYPES[c["dtype"]]
    N, V, K = c["N"], c["V"], c["K"]
    S = dict(temperature=0.8 if c["mode"] == "score" else 1.0, K=K)
    S["logits"] = r.normal(N, V, std=2.5, dtype=dt)
    S["ids"] = (V * r.uniform(N)).long().clamp_(max=V - 1)
    if c["masked"]:  # half of the rows allow a share of the vocabulary, from a few tokens on, and the given one
        out = r.uniform(N, V) > torch.where(r.uniform(N, 1) < 0.5, 0.3 * r.uniform(N, 1) ** 8, 1.0)
        S["logits"].masked_fill_(out.scatter_(1, S["ids"][:, None], False), -math.inf)
    if c["padded"]:
        S["ids"] = torch.where(r.uniform(N) < 0.1, -1, S["ids"])
    if c["mode"] != "score":
        S["dlogprob"], S["dentropy"] = -(0.5 + r.uniform(N)) / N, -0.1 * (0.5 + r.uniform(N)) / N
        S["dtop_logprob"] = r.normal(N, K, std=0.3 / N) if K else None
    if c["mode"] == "meta":
        S["ddlogits"] = r.normal(N, V, std=0.1, dtype=dt)
    return S


def _shapes(c):
    """The leaves of a tree of about n elements."""
    n = c["n"]
    if c["layout"] == "flat":
        return [(n,)]
    if c["layout"] == "tiny":  # two hidden layers
        w = max(1, int(math.sqrt(n + 4.0)) - 2)
        return [(w, 1), (w,), (w, w), (w,), (1, w), (1,)]
    if c["layout"] == "many":  # sizes spread over the logarithm, from one element on; the same tree for every seed
        hi = max(8, min(65536, n // 4))
        count = max(2, int(n * math.log(hi) / hi))
        gen = torch.Generator().manual_seed(n)
        return [(int(s),) for s in torch.exp(torch.rand(count, generator=gen, dtype=torch.float64) * math.log(hi)).round()]
    layers = 24 if n > 50_000_000 else 6
    w = max(16, int(math.sqrt(n / (14.0 * layers))) // 2 * 2)
    block = [(w, w)] * 4 + [(4 * w, w), (w, 4 * w)] + [(w,), (w,)]
    rest = n - layers * sum(math.prod(s) for s in block)
    return block * layers + [(max(1, rest // w), w)]


def _inputs_clip(c, seed):
    r = _Draw(seed)
    shapes = _shapes(c)
    n = sum(math.prod(s) for s in shapes)
    S = dict(max_norm=1.0, eps=1e-6)
    S["grad"] = [r.normal(*s, std=c["norm"] / math.sqrt(n)) for s in shapes]
    if c["mode"] == "train":
        S["dout"] = [r.normal(*s) for s in shapes]
        S["dnorm"] = r.normal(1)
    return S


_INPUTS = {"gscan": _inputs_gscan, "logprob": _inputs_logprob, "clip": _inputs_clip}


def _place(shapes):
    """First elements of a tree's leaves in one buffer, each on a 128-byte line of its own, and the buffer's length."""
    at, places = 0, []
    for s in shapes:
        places.append(at)
        at += -(-math.prod(s) // 32) * 32
    return places, at


def _leaves(buffer, shapes):
    return [buffer[i:i + math.prod(s)].view(s) for i, s in zip(_place(shapes)[0], shapes)]


def _new(x):
    return None if x is None else torch.zeros_like(x, memory_format=torch.contiguous_format)


def prepare(case, seed):
    """The inputs and the result buffers that a program keeps, for a tree (whose results lie in one buffer) also its table and its leaves' addresses."""
    op, mode = case["op"], case["mode"]
    S = _INPUTS[op](case, seed)
    S["op"], S["mode"] = op, mode
    if op == "gscan":
        B, T, C = (case[k] for k in ("B", "T", "C"))
        if mode == "step":
            S["log_gate"], S["x"] = S["log_gate"][:, 0].contiguous(), S["x"][:, 0].contiguous()
            S["out"] = _new(S["x"])
        else:
            S["h"] = _new(S["x"])
            S["state_out"] = torch.zeros(B, C, device="cuda") if mode == "prompt" or case["warm"] else None
        if mode in ("train", "meta"):
            S["dx"], S["dlog_gate"], S["dstate"] = _new(S["x"]), _new(S["x"]), _new(S["state"])
        if mode == "meta":
            S["out_dh"], S["out_x"], S["out_log_gate"] = _new(S["x"]), _new(S["x"]), _new(S["x"])
            S["out_state"], S["out_dstate_out"] = _new(S["state"]), _new(S["state"])
    elif op == "logprob":
        N, K = case["N"], case["K"]
        S["logprob"], S["entropy"], S["stats"] = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda"), torch.zeros(N, 2, device="cuda")
        S["top_logprob"] = torch.zeros(N, K, device="cuda") if K else None
        S["top_ids"] = torch.zeros(N, K, dtype=torch.int64, device="cuda") if K else None
        if mode != "score":
            S["dlogits"] = _new(S["logits"])
        if mode == "meta":
            S["out_logits"], S["out_dlogprob"], S["out_dentropy"], S["out_dtop_logprob"] = (_new(S[k]) for k in ("logits", "dlogprob", "dentropy", "dtop_logprob"))
    else:
        S["stats"] = torch.zeros(2, device="cuda")
        shapes = [x.shape for x in S["grad"]]
        for k in ("out", "dgrad") if mode == "train" else ("out",):
            S[k] = torch.zeros(_place(shapes)[1], device="cuda")
            S[k + "_leaves"] = _leaves(S[k], shapes)
        S["flat"] = case["layout"] == "flat"
        if own and not S["flat"]:
            import paper_2211_06934_amd as P
            S["table"] = P.segtable_create([x.numel() for x in S["grad"]])
            S["at"] = {k: P.tree.leaf_pointer_tensor(S[k], "cuda") for k in ("grad", "out_leaves", "dout", "dgrad_leaves") if k in S}
    return S


# ---- one pass ---------------------------------------------------------------

_SCAN = ("h", "state_out", "dlog_gate", "dx", "dstate")
_LOGPROB = ("logprob", "entropy", "top_logprob", "top_ids", "dlogits")
_RESULTS = {
    "gscan": {"prompt": ("h", "state_out"), "train": _SCAN, "meta": _SCAN + ("out_dh", "out_dstate_out", "out_log_gate", "out_x", "out_state"), "step": ("out", "state")},
    "logprob": {"train": _LOGPROB, "split": _LOGPROB, "score": _LOGPROB[:-1], "meta": _LOGPROB + ("out_dlogprob", "out_dentropy", "out_dtop_logprob", "out_logits")},
    "clip": {"clip": ("stats", "out"), "train": ("stats", "out", "dgrad")},
}


def run(state):
    if own:
        _OWN[state["op"]](state)
        got = state
    else:
        got = _PLAIN[state["op"]](state)
    return {k: got[k] for k in _RESULTS[state["op"]][state["mode"]] if got.get(k) is not None}


def _own_gscan(S):
    import paper_2211_06934_amd as P
    if S["mode"] == "step":
        P.gscan_step(S["log_gate"], S["x"], S["state"], S["out"])
        return
    P.gscan_fwd(S["log_gate"], S["x"], S["h"], state=S["state"], state_out=S["state_out"], lengths=S["lengths"])
    if S["mode"] != "prompt":
        P.gscan_bwd(S["dh"], S["log_gate"], S["x"], S["dlog_gate"], S["dx"], state=S["state"], dstate_out=S["dstate_out"], dstate=S["dstate"],
                    lengths=S["lengths"])
    if S["mode"] == "meta":
        P.gscan_bwd_bwd(S["ddlog_gate"], S["ddx"], S["dh"], S["log_gate"], S["x"], S["out_dh"], S["out_log_gate"], S["out_x"], state=S["state"],
                        dstate_out=S["dstate_out"], ddstate=S["ddstate"], out_dstate_out=S["out_dstate_out"], out_state=S["out_state"], lengths=S["lengths"])


def _own_logprob(S):
    import paper_2211_06934_amd as P
    T = S["temperature"]
    if S["mode"] == "train":
        P.logprob_fwd_bwd(S["dlogprob"], S["logits"], S["ids"], S["logprob"], S["stats"], S["dlogits"], dentropy=S["dentropy"], entropy=S["entropy"],
                          temperature=T)
        return
    P.logprob_fwd(S["logits"], S["ids"], S["logprob"], S["stats"], entropy=S["entropy"], top_logprob=S["top_logprob"], top_ids=S["top_ids"], temperature=T)
    given = dict(dlogprob=S.get("dlogprob"), dentropy=S.get("dentropy"), entropy=S["entropy"], dtop_logprob=S.get("dtop_logprob"), top_ids=S["top_ids"], temperature=T)
    if S["mode"] != "score":
        P.logprob_bwd(S["logits"], S["ids"], S["stats"], S["dlogits"], **given)
    if S["mode"] == "meta":
        P.logprob_bwd_bwd(S["ddlogits"], S["logits"], S["ids"], S["stats"], S["out_logits"], out_dlogprob=S["out_dlogprob"], out_dentropy=S["out_dentropy"],
                          out_dtop_logprob=S["out_dtop_logprob"], **given)


def _own_clip(S):
    import paper_2211_06934_amd as P
    if S["flat"]:
        P.clip_norm_fwd(S["grad"][0], S["max_norm"], S["out_leaves"][0], S["stats"], eps=S["eps"])
        if S["mode"] == "train":
            P.clip_norm_bwd(S["dout"][0], S["dnorm"], S["grad"][0], S["stats"], S["dgrad_leaves"][0], eps=S["eps"])
        return
    at = S["at"]
    P.clip_norm_fwd_tree(S["table"], at["grad"], S["max_norm"], at["out_leaves"], S["stats"], eps=S["eps"])
    if S["mode"] == "train":
        P.clip_norm_bwd_tree(S["table"], at["dout"], S["dnorm"], at["grad"], S["stats"], at["dgrad_leaves"], eps=S["eps"])


_OWN = {"gscan": _own_gscan, "logprob": _own_logprob, "clip": _own_clip}


# ---- plain forms ------------------------------------------------------------


def _scan(a, x, first):
    """h_t = a_t h_{t-1} + x_t along the second axis, h_{-1} = first (or None: 0), by doubling."""
    x = x.clone()
    if first is not None and x.shape[1]:
        x[:, 0] += a[:, 0] * first
    step = 1
    while step < x.shape[1]:
        x = torch.cat((x[:, :step], x[:, step:] + a[:, step:] * x[:, :-step]), 1)
        a = torch.cat((a[:, :step], a[:, step:] * a[:, :-step]), 1)
        step *= 2
    return x


def _before(h, first):
    """h_{t-1}, beginning with `first`."""
    return torch.cat((torch.zeros_like(h[:, :1]) if first is None else first[:, None], h[:, :-1]), 1)


def _adjoint(a, u, last):
    """v_t = u_t + a_{t+1} v_{t+1}, with `last` (or None: 0) as the term after the last token."""
    one = torch.ones_like(a[:, :1])
    return _scan(torch.cat((a[:, 1:], one), 1).flip(1), u.flip(1), last).flip(1)


def _plain_gscan(S):
    dt, s0 = S["x"].dtype, S["state"]
    lg, x = S["log_gate"].float(), S["x"].float()
    if S["mode"] == "step":
        state = s0.mul_(torch.exp(lg)).add_(x)
        return dict(out=state.to(dt), state=state)
    live = None
    if S["lengths"] is not None:
        live = (torch.arange(x.shape[1], device=x.device)[None, :] < S["lengths"].long()[:, None])[:, :, None]
    masked = lambda v, other=0.0: v if live is None else torch.where(live, v, torch.full((), other, device=v.device))
    a, x = masked(torch.exp(lg), 1.0), masked(x)  # tokens past the end leave the state as it is
    h = _scan(a, x, s0)
    got = dict(h=masked(h).to(dt))
    if S["state_out"] is not None:
        got["state_out"] = h[:, -1].contiguous()
    if S["mode"] == "prompt":
        return got
    dh, hp = masked(S["dh"].float()), _before(h, s0)
    g = _adjoint(a, dh, S["dstate_out"])
    got["dx"], got["dlog_gate"] = masked(g).to(dt), masked(a * hp * g).to(dt)
    if s0 is not None:
        got["dstate"] = a[:, 0] * g[:, 0]
    if S["mode"] == "meta":
        r, p, first = masked(S["ddlog_gate"].float()), masked(S["ddx"].float()), S["ddstate"]
        y = _scan(a, p + r * a * hp, first)
        v = _adjoint(a, r * g, None)
        got["out_dh"], got["out_x"] = masked(y).to(dt), masked(v - r * g).to(dt)
        got["out_log_gate"] = masked(a * (g * _before(y, first) + hp * v)).to(dt)
        if s0 is not None:
            got["out_dstate_out"], got["out_state"] = y[:, -1].contiguous(), a[:, 0] * v[:, 0]
    return got


def _top(x, K):
    """The K largest of each row of fp32 values: [N, K] values and ids, the lowest id first among equals; -1 from the last finite one on."""
    N, V = x.shape
    bits = (x + 0.0).view(torch.int32).long()  # -0 as +0
    order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF))  # as the values order
    key = order * (1 << 31) + ((1 << 31) - 1 - torch.arange(V, device=x.device))  # all different
    key = torch.topk(key, min(K, V), dim=1).values
    ids = (1 << 31) - 1 - (key & 0x7FFFFFFF)
    values = x.gather(1, ids)
    if K > V:
        ids, values = (torch.nn.functional.pad(t, (0, K - V), value=v) for t, v in ((ids, -1), (values, -math.inf)))
    return values, torch.where(values == -math.inf, -1, ids)


def _plain_logprob(S):
    T, K, ids = S["temperature"], S["K"], S["ids"][:, None]
    raw = S["logits"].float()
    x, dt = raw / T, S["logits"].dtype
    there, at = ids >= 0, ids.clamp(min=0)
    nought = torch.zeros((), device=x.device)
    m = x.max(1, keepdim=True).values
    e = torch.exp(x - m)
    s = e.sum(1, keepdim=True)
    p, l = e / s, (x - m) - torch.log(s)
    l = torch.where(p > 0, l, nought)  # 0 log 0 = 0
    H = -(p * l).sum(1, keepdim=True)
    got = dict(logprob=torch.where(there, x.gather(1, at) - m - torch.log(s), nought)[:, 0], entropy=torch.where(there, H, nought)[:, 0])
    if K:
        values, got["top_ids"] = _top(raw, K)
        got["top_logprob"] = torch.where(there, values / T - m - torch.log(s), -math.inf)
        got["top_ids"] = torch.where(there, got["top_ids"], -1)
    if S["mode"] == "score":
        return got
    g, h = S["dlogprob"][:, None], S["dentropy"][:, None]
    G = g
    if K:
        c, top = torch.where(got["top_ids"] >= 0, S["dtop_logprob"], nought), got["top_ids"].clamp(min=0)
        G = g + c.sum(1, keepdim=True)
    d = (-p * (G + h * (l + H))).scatter_add(1, at, g)
    if K:
        d = d.scatter_add(1, top, c)
    got["dlogits"] = torch.where(there, d / T, nought).to(dt)
    if S["mode"] == "meta":
        b = S["ddlogits"].float()
        mean = (p * b).sum(1, keepdim=True)
        k = (p * (b - mean) * (l + H)).sum(1, keepdim=True)
        got["out_dlogprob"] = torch.where(there, (b.gather(1, at) - mean) / T, nought)[:, 0]
        got["out_dentropy"] = torch.where(there, -k / T, nought)[:, 0]
        got["out_logits"] = torch.where(there, -p * (G * (b - mean) + h * ((b - mean) * (l + H + 1) - k)) / (T * T), nought).to(dt)
        if K:
            got["out_dtop_logprob"] = torch.where(there & (got["top_ids"] >= 0), (b.gather(1, top) - mean) / T, nought)
    return got


def _plain_clip(S):
    total = sum((x * x).sum(dtype=torch.float64) for x in S["grad"])
    norm = torch.sqrt(total)
    scale = torch.clamp(S["max_norm"] / (norm + S["eps"]), max=1.0).float()
    for x, out in zip(S["grad"], S["out_leaves"]):
        torch.mul(x, scale, out=out)
    got = dict(stats=torch.stack((norm.float(), scale)), out=S["out"])
    if S["mode"] == "train":
        dot = sum((x * d).sum(dtype=torch.float64) for x, d in zip(S["grad"], S["dout"]))
        slope = (S["dnorm"].double() - torch.where(scale < 1.0, scale.double() * dot / (norm + S["eps"]), 0.0)) / norm
        slope = torch.where(norm > 0, slope, 0.0).float()
        for x, d, to in zip(S["grad"], S["dout"], S["dgrad_leaves"]):
            torch.add(scale * d, slope * x, out=to)
        got["dgrad"] = S["dgrad"]
    return got


_PLAIN = {"gscan": _plain_gscan, "logprob": _plain_logprob, "clip": _plain_clip}


# ---- what a pass cannot do without ------------------------------------------


def work(case):
    op, mode = case["op"], case["mode"]
    if op == "gscan":
        n, state = case["B"] * case["T"] * case["C"], 4 * case["B"] * case["C"]
        e = {"bf16": 2, "f32": 4}[case["dtype"]]
        # gate and input, then h; dh, then the two gradients; two cotangents, then three results
        arrays, states, flops = {"step": (3, 2, 3), "prompt": (3, 1 + case["warm"], 3), "train": (6, 4 * case["warm"], 9), "meta": (11, 7 * case["warm"], 24)}[mode]
        return {"bytes": arrays * n * e + states * state, "flops": flops * n}
    if op == "logprob":
        n, N, K = case["N"] * case["V"], case["N"], case["K"]
        arrays, flops = {"score": (1, 6), "train": (2, 12), "split": (2, 12), "meta": (4, 30)}[mode]
        small = {"score": 8 + 8 + 12 * K, "train": 8 + 16, "split": 8 + 16 + 16 * K, "meta": 8 + 24 + 20 * K}[mode]
        return {"bytes": arrays * n * {"bf16": 2, "f32": 4}[case["dtype"]] + N * small, "flops": flops * n}
    n = sum(math.prod(s) for s in _shapes(case))
    return {"bytes": 4 * n * (4 if mode == "train" else 2), "flops": n * (8 if mode == "train" else 3)}


# ---- in 64 bits, from the definitions ---------------------------------------


def exact(case, seed):
    S = _INPUTS[case["op"]](case, seed)
    got = {"gscan": _exact_gscan, "logprob": _exact_logprob, "clip": _exact_clip}[case["op"]](case, S)
    return {k: got[k] for k in _RESULTS[case["op"]][case["mode"]] if k in got}


def _exact_gscan(c, S):
    """A token after another; the derivatives by autograd."""
    B, T, mode = c["B"], c["T"], c["mode"]
    train, meta = mode in ("train", "meta"), mode == "meta"
    lg, x = (S[k].double().requires_grad_(train) for k in ("log_gate", "x"))
    s0 = S["state"].double().requires_grad_(train) if c["warm"] else torch.zeros(B, c["C"], dtype=torch.float64, device="cuda")
    ends = torch.full((B,), T, device="cuda") if S["lengths"] is None else S["lengths"].long()
    h, hs = s0, []
    for t, (gate, new) in enumerate(zip(torch.exp(lg).unbind(1), x.unbind(1))):
        live = (t < ends)[:, None]
        step = gate * h + new
        h = step if S["lengths"] is None else torch.where(live, step, h)
        hs.append(h if S["lengths"] is None else torch.where(live, h, 0.0))
    out = torch.stack(hs, 1)
    if mode == "step":
        return dict(out=out[:, 0], state=h)
    got = dict(h=out.detach())
    if mode == "prompt" or c["warm"]:
        got["state_out"] = h.detach()
    if not train:
        return got
    leaves, cots, outs = [lg, x], [S["dh"].double().requires_grad_(meta)], [out]
    if c["warm"]:
        leaves.append(s0)
        cots.append(S["dstate_out"].double().requires_grad_(meta))
        outs.append(h)
    grads = torch.autograd.grad(outs, leaves, cots, create_graph=meta)
    got |= dict(zip(("dlog_gate", "dx", "dstate"), (g.detach() for g in grads)))
    if meta:
        second = [S[k].double() for k in ("ddlog_gate", "ddx", "ddstate")[:len(grads)]]
        back = torch.autograd.grad(grads, cots + leaves, second, allow_unused=True)
        names = ("out_dh", "out_dstate_out", "out_log_gate", "out_x", "out_state") if c["warm"] else ("out_dh", "out_log_gate", "out_x")
        got |= {k: torch.zeros_like(of) if b is None else b for k, b, of in zip(names, back, cots + leaves)}
    return got


def _exact_logprob(c, S):
    """log_softmax in fp64, some rows at a time; alternatives by a stable sort, the derivatives by autograd."""
    N, V, K, T, mode = c["N"], c["V"], c["K"], S["temperature"], c["mode"]
    step = max(1, 40_000_000 // V)
    parts = []
    for i in range(0, N, step):
        rows = slice(i, min(N, i + step))
        x = S["logits"][rows].double().requires_grad_(mode != "score")
        ids = S["ids"][rows]
        there = ids >= 0
        lp = torch.log_softmax(x / T, 1)
        masked = torch.isinf(S["logits"][rows])
        finite = lp.masked_fill(masked, 0.0)
        p = torch.softmax(x / T, 1)
        outs = [torch.where(there, lp.gather(1, ids.clamp(min=0)[:, None])[:, 0], 0.0), torch.where(there, -(p * finite).sum(1), 0.0)]
        part = dict(logprob=outs[0], entropy=outs[1])
        if K:
            by = torch.sort(S["logits"][rows], dim=1, descending=True, stable=True).indices[:, :K]
            by = torch.nn.functional.pad(by, (0, K - by.shape[1]), value=V)
            gone = ~there[:, None] | (by == V)
            by = by.clamp(max=V - 1)
            gone = gone | masked.gather(1, by)
            outs.append(finite.gather(1, by).masked_fill(gone, 0.0))
            part["top_ids"], part["top_logprob"] = by.masked_fill(gone, -1), outs[2].masked_fill(gone, -math.inf)
        if mode != "score":
            cots = [S[k][rows].double().requires_grad_(mode == "meta") for k in ("dlogprob", "dentropy", "dtop_logprob")[:len(outs)]]
            (part["dlogits"],) = torch.autograd.grad(outs, x, cots, create_graph=mode == "meta")
            if mode == "meta":
                back = torch.autograd.grad(part["dlogits"], [*cots, x], S["ddlogits"][rows].double())
                part |= dict(zip(("out_dlogprob", "out_dentropy", "out_dtop_logprob")[:len(cots)], back))
                part["out_logits"] = back[-1]
        parts.append({k: v.detach() for k, v in part.items()})
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_clip(c, S):
    """The norm of all elements as one vector, the derivative by autograd."""
    train = c["mode"] == "train"
    flat = torch.cat([x.reshape(-1) for x in S["grad"]]).double().requires_grad_(train)
    norm = torch.linalg.vector_norm(flat)
    scale = torch.clamp(S["max_norm"] / (norm + S["eps"]), max=1.0)
    out = flat * scale
    shapes = [x.shape for x in S["grad"]]

    def back(v):
        buffer = torch.zeros(_place(shapes)[1], dtype=torch.float64, device="cuda")
        for t, to in zip(v.split([x.numel() for x in S["grad"]]), _leaves(buffer, shapes)):
            to.copy_(t.view(to.shape))
        return buffer

    got = dict(stats=torch.stack((norm, scale)).detach(), out=back(out.detach()))
    if train:
        dout = torch.cat([x.reshape(-1) for x in S["dout"]]).double()
        (d,) = torch.autograd.grad((out, norm), flat, (dout, S["dnorm"].double()[0]))
        got["dgrad"] = back(d)
    return got
