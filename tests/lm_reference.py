"""fp64 references of the language-model operators, from their definitions, and
the tolerances their tests use.  Token after token, row after row, on the CPU;
derivatives by autograd of the fp64 forward."""
import math

import torch

# Tolerances, derived from the arithmetic before any run.
# fp32 results: every sum has at most a few thousand fp32 terms whose rounding
# errors (2^-24 each) add like a random walk, at most sqrt(4096) 2^-24 = 4e-6 of
# the norm of the terms; the exponentials add an error of 2^-22 of each term.
# Inputs are drawn so that sums do not cancel below a tenth of their terms'
# norm, in the 2-norm of a whole result: 1e-5 (the framework's forward bar).
F32 = 1e-5
# bf16 results: 8 significant bits, so that one rounding is at most 2^-8 of each
# element (3.9e-3; torch's own conversion of 1 + 2^-8 is that far off).  Linear
# attention also rounds the scores and the state to bf16 once each where they
# enter a matrix product: three independent roundings, sqrt(3) 2^-8 = 6.8e-3.
BF16 = 2.0 ** -8
BF16_PRODUCTS = 3.0 ** 0.5 * 2.0 ** -8
# one element's error is held to this many times the bound on the norm, against
# the result's root mean square (or the element itself, where larger): 4e5
# elements' worst rounding lies below 8 times their root mean square
PEAK = 16.0


def tol(dtype, products=False):
    if dtype == torch.float32:
        return F32
    return BF16_PRODUCTS if products else BF16


def assert_close(got, ref, bound, what=""):
    """got (any type) against ref (fp64, CPU): finite where ref is, within
    `bound` in the 2-norm, each element within PEAK * bound."""
    got = got.detach().double().cpu()
    ref = ref.detach().double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    if ref.numel() == 0:
        return
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got)), (what, "finite elsewhere")
    g, r = got[fine], ref[fine]
    if r.numel() == 0:
        return
    norm = float(r.norm())
    err = float((g - r).norm())
    assert err <= bound * norm + 1e-30, (what, "norm", err / max(norm, 1e-300))
    rms = norm / math.sqrt(r.numel())
    worst = float(((g - r).abs() / torch.clamp(r.abs(), min=rms + 1e-30)).max())
    assert worst <= PEAK * bound, (what, "element", worst)


# ---- linear attention -------------------------------------------------------


def linattn(q, k, v, log_decay, state=None, lengths=None, scale=1.0):
    """fp64 (out, final state), one token after another."""
    B, T, H, Dk = q.shape
    Hk, Dv = k.shape[2], v.shape[3]
    q, k, v, lg = q.double(), k.double(), v.double(), log_decay.double()
    S = torch.zeros(B, Hk, Dk, Dv, dtype=torch.float64) if state is None else state.double()
    n = torch.full((B,), T) if lengths is None else lengths.clamp(0, T)
    g = torch.exp(lg)[None, :, None, None]
    outs = []
    for t in range(T):
        live = (t < n)[:, None, None, None]
        nought = torch.zeros((), dtype=torch.float64)
        kt, vt, qt = (torch.where(live[..., 0], x[:, t], nought) for x in (k, v, q))
        S = torch.where(live, g * S + kt[..., :, None] * vt[..., None, :], S)
        o = scale * torch.einsum("bhgd,bhde->bhge", qt.reshape(B, Hk, H // Hk, Dk), S).reshape(B, H, Dv)
        outs.append(torch.where(live[..., 0], o, nought))
    out = torch.stack(outs, 1) if T else torch.zeros(B, 0, H, Dv, dtype=torch.float64)
    return out, S


# ---- norms and rotation -----------------------------------------------------


def qknorm_rope(x, w, cos, sin, where, eps, interleaved):
    """fp64 x [B,T,h,D] normed, scaled and rotated by rows where [B,T] of cos, sin [rows, rot/2] (None: not rotated)."""
    z = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
    if w is not None:
        z = z * w
    if cos is None:
        return z
    half = cos.shape[1]
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = (t.double()[where][:, :, None] for t in (cos, sin))
    out = z.clone()
    out[..., a] = z[..., a] * c - z[..., b] * s
    out[..., b] = z[..., b] * c + z[..., a] * s
    return out


# ---- distillation -----------------------------------------------------------


def distill(logits, ids, teacher, temperature):
    """fp64 loss [N], a row at a time."""
    losses = []
    for x, id_, t in zip(logits, ids, teacher):
        keep = (id_ >= 0) & (t.detach() != -math.inf)
        if not bool(keep.any()):
            losses.append(torch.zeros((), dtype=torch.float64))
            continue
        if bool((id_[keep] >= x.numel()).any()):
            losses.append(torch.full((), math.nan, dtype=torch.float64))
            continue
        lq = torch.log_softmax(t[keep] / temperature, 0)
        lp = torch.log_softmax(x / temperature, 0)[id_[keep]]
        q = lq.exp()
        on = q.detach() > 0
        losses.append(temperature ** 2 * (q[on] * (lq[on] - lp[on])).sum())
    return torch.stack(losses)
