"""A recurrent student fine-tuned by an inner loop whose per-token weights an
outer loop learns, then sampling: the gated recurrence, the log probabilities
and the clipped step together, on synthetic data.

The student is one block of a gated linear recurrence.  Listing 1's inner loop
takes a few MetaAdam steps, their gradients clipped to a global norm, on the
weighted negative log likelihood of the tokens with an entropy bonus; the outer
loss (the likelihood of clean text after those steps) is differentiated through
them to the weights of the noisy corpus's tokens.  At the end the adapted
student reads a prompt in one call, keeps its state, and continues it a token
at a time from its likeliest alternatives; these also serve a second student as
its teacher's top logits.

  python examples/recurrent_inner_loop.py [--outer 5 --inner 3 --dtype bf16]
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2211_06934_amd as P  # noqa: E402


class Student(torch.nn.Module):
    """Embedding, one residual block of the gated recurrence, output head."""

    def __init__(self, vocab=257, width=96, inner=160, dtype=torch.float32):
        super().__init__()
        self.dtype = dtype
        new = lambda *s: torch.nn.Parameter(torch.randn(*s) * s[-1] ** -0.5)
        self.embed = torch.nn.Parameter(torch.randn(vocab, width) * 0.5)
        self.gate = new(inner, width)
        self.rate = torch.nn.Parameter(torch.linspace(-4.0, 1.0, inner))  # channels remember from a token to a few hundred
        self.into = new(inner, width)
        self.mix = new(width, inner)
        self.top = new(vocab, width)

    def _operands(self, x):
        """Log gates and inputs of the recurrence, [..., inner]."""
        p = self._parameters
        log_gate = -F.softplus(p["rate"]) * torch.sigmoid(F.linear(x, p["gate"]))
        return log_gate.to(self.dtype), F.linear(x, p["into"]).to(self.dtype)

    def _logits(self, x, h):
        p = self._parameters
        return F.linear(x + F.linear(h.float(), p["mix"]), p["top"]).to(self.dtype)

    def forward(self, tokens, lengths=None, return_state=False):
        x = self._parameters["embed"][tokens]
        got = P.gated_scan(*self._operands(x), lengths=lengths, return_state=return_state)
        h, state = got if return_state else (got, None)
        return (self._logits(x, h), state) if return_state else self._logits(x, h)

    @torch.no_grad()
    def step(self, tokens, state):
        """The next token's logits [B, vocab] for tokens [B]; the state moves on."""
        x = self._parameters["embed"][tokens]
        return self._logits(x, P.gated_scan_step(*self._operands(x), state))


def inner_loss(student, tokens, target, weights, bonus=0.02):
    """Weighted negative log likelihood of target [B, T] (-1: padding) after tokens, less an entropy bonus."""
    got = P.token_logprobs(student(tokens).flatten(0, 1), target.flatten(), entropy=True)
    return -(torch.sigmoid(weights).flatten() * got.logprob + bonus * got.entropy).sum() / target.numel()


def adapt(student, tokens, target, weights, steps, lr=3e-3, max_norm=1.0):
    opt = P.MetaAdam(student, lr=lr, max_norm=max_norm)
    losses, norms = [], []
    for _ in range(steps):
        loss = inner_loss(student, tokens, target, weights)
        losses.append(loss.detach())
        opt.step(loss)
        norms.append(opt.grad_norm)
    return opt, losses, norms


def outer_loss(student, tokens, target):
    return -P.token_logprobs(student(tokens).flatten(0, 1), target.flatten()).logprob.mean()


def generate(student, prompt, count, top=5):
    """Continuation [B, count] of prompt [B, T] by the likeliest token, with the alternatives' ids and log probabilities."""
    with torch.no_grad():
        logits, state = student(prompt, return_state=True)
        logits, got = logits[:, -1], []
        for _ in range(count):
            choice = P.token_logprobs(logits, top=top)
            got.append(choice)
            logits = student.step(choice.top_ids[:, 0], state)
    return torch.stack([c.top_ids[:, 0] for c in got], 1), torch.stack([c.top_ids for c in got], 1), torch.stack([c.top_logprob for c in got], 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--outer", type=int, default=5)
    ap.add_argument("--inner", type=int, default=3)
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="bf16")
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args(argv)
    gen = torch.Generator().manual_seed(args.seed)
    torch.manual_seed(args.seed)
    vocab, B, T = 257, 8, 61
    dtype = torch.bfloat16 if args.dtype == "bf16" else torch.float32
    # a language to learn: the next token is an affine map of this one; the corpus has every third token wrong
    tokens = torch.randint(vocab, (B, 1), generator=gen)
    for _ in range(T):
        tokens = torch.cat([tokens, (tokens[:, -1:] * 5 + 3) % vocab], 1)
    x, clean = tokens[:, :-1].cuda(), tokens[:, 1:].cuda()
    wrong = torch.rand(B, T, generator=gen) < 1 / 3
    noisy = torch.where(wrong, torch.randint(vocab, (B, T), generator=gen), tokens[:, 1:]).cuda()
    noisy[-1, T // 2:] = -1  # a shorter text
    weights = torch.zeros(B, T, device="cuda", requires_grad=True)
    start = Student(vocab, dtype=dtype).state_dict()
    outer = []
    for it in range(args.outer):
        student = Student(vocab, dtype=dtype).cuda()
        student.load_state_dict(start)
        _, _, norms = adapt(student, x, noisy, weights, args.inner)
        loss = outer_loss(student, x, clean)
        (grad,) = torch.autograd.grad(loss, [weights])
        with torch.no_grad():
            weights -= grad / grad.square().mean().sqrt()
        outer.append(float(loss.detach()))
        print("outer step %d: loss after %d inner steps %.4f, last gradient's norm %.3f" % (it, args.inner, outer[-1], float(norms[-1])), flush=True)
    student = Student(vocab, dtype=dtype).cuda()
    student.load_state_dict(start)
    opt, inner, _ = adapt(student, x, noisy, weights.detach(), 60)
    opt.detach_()
    print("weighted loss %.4f -> %.4f over %d steps" % (float(inner[0]), float(inner[-1]), len(inner)))
    got, ids, logprob = generate(student, x[:, :40], 8)
    print("continued tokens that follow the language: %d of %d" % (int((got == clean[:, 39:47]).sum()), got.numel()))
    # the alternatives as a teacher's top logits
    other = Student(vocab, dtype=dtype).cuda()
    seen = other(x[:, :47])[:, 39:].flatten(0, 1)
    distilled = P.distillation_loss(seen, ids.flatten(0, 1), logprob.flatten(0, 1)).mean()
    (back,) = torch.autograd.grad(distilled, [other.embed])
    return outer, [float(v) for v in inner], got, float(distilled.detach()), back


if __name__ == "__main__":
    main()
