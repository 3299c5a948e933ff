"""A student that an inner loop distils, its teacher tuned through that loop,
then generation: the operators of a language model together, on synthetic data.

The student is one block of linear attention over normed, rotated queries and
keys.  Listing 1's inner loop takes a few MetaAdam steps on the distillation
loss against the teacher's top logits; the outer loss (next-token cross
entropy of the adapted student) is differentiated through those steps to the
teacher's logits, which move against it.  At the end the adapted student reads
a prompt in one call, keeps its state, and generates a token at a time.

  python examples/distill_inner_loop.py [--outer 5 --inner 3 --dtype bf16]
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2211_06934_amd as P  # noqa: E402


class Student(torch.nn.Module):
    """Embedding, one residual block of linear attention (query heads share k/v heads), output head."""

    def __init__(self, vocab=257, width=96, heads=4, kv_heads=2, head=32, rows=512, dtype=torch.float32):
        super().__init__()
        self.heads, self.kv, self.head, self.dtype = heads, kv_heads, head, dtype
        new = lambda *s: torch.nn.Parameter(torch.randn(*s) * s[-1] ** -0.5)
        self.embed = torch.nn.Parameter(torch.randn(vocab, width) * 0.5)
        self.qkv = new((heads + 2 * kv_heads) * head, width)
        self.q_weight, self.k_weight = (torch.nn.Parameter(torch.ones(head)) for _ in range(2))
        self.mix = new(width, heads * head)
        self.top = new(vocab, width)
        angle = torch.arange(rows)[:, None] * 10000.0 ** (-torch.arange(head // 2) / (head // 2))
        self.register_buffer("cos", torch.cos(angle))
        self.register_buffer("sin", torch.sin(angle))
        self.register_buffer("log_decay", torch.log(1 - 2.0 ** -(3.0 + torch.arange(kv_heads))))

    def _qkv(self, x, positions=None, first=0):
        """x [B, T, width] -> normed and rotated q, k, and v: views of one projection's output."""
        p = self._parameters
        y = F.linear(x, p["qkv"]).to(self.dtype).unflatten(-1, (-1, self.head))
        q, k, v = y.split([self.heads, self.kv, self.kv], 2)
        q, k = P.qknorm_rope(q, k, p["q_weight"], p["k_weight"], self.cos, self.sin, positions, first)
        return q, k, v

    def _logits(self, x, out):
        p = self._parameters
        x = x + F.linear(out.flatten(2).float(), p["mix"])
        return F.linear(x, p["top"])

    def forward(self, tokens, lengths=None, return_state=False):
        x = self._parameters["embed"][tokens]
        q, k, v = self._qkv(x)
        got = P.linear_attention(q, k, v, self.log_decay, lengths=lengths, scale=self.head ** -0.5, return_state=return_state)
        out, state = got if return_state else (got, None)
        return (self._logits(x, out), state) if return_state else self._logits(x, out)

    @torch.no_grad()
    def step(self, tokens, place: int, state):
        """The next token's logits [B, vocab] for tokens [B] at this place; the state moves on."""
        x = self._parameters["embed"][tokens][:, None]
        q, k, v = self._qkv(x, first=place)
        out = P.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], self.log_decay, state, self.head ** -0.5)
        return self._logits(x, out[:, None])[:, 0]


def inner_loss(student, tokens, ids, teacher, temperature=2.0):
    """Mean distillation loss over the tokens: logits [B, T, vocab] as rows against the teacher's [B, T, K]."""
    logits = student(tokens).flatten(0, 1).to(student.dtype)
    return P.distillation_loss(logits, ids.flatten(0, 1), teacher.flatten(0, 1), temperature).mean()


def adapt(student, tokens, ids, teacher, steps, lr=3e-3):
    opt = P.MetaAdam(student, lr=lr)
    losses = []
    for _ in range(steps):
        loss = inner_loss(student, tokens, ids, teacher)
        losses.append(loss.detach())
        opt.step(loss)
    return opt, losses


def outer_loss(student, tokens, target):
    return F.cross_entropy(student(tokens).flatten(0, 1), target.flatten())


def generate(student, prompt, count):
    """Greedy continuation of prompt [B, T]: the prompt in one call, then a token at a time."""
    with torch.no_grad():
        logits, state = student(prompt, return_state=True)
        token, got = logits[:, -1].argmax(-1), []
        for i in range(count):
            got.append(token)
            token = student.step(token, prompt.shape[1] + i, state).argmax(-1)
    return torch.stack(got, 1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--outer", type=int, default=5)
    ap.add_argument("--inner", type=int, default=3)
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="bf16")
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args(argv)
    gen = torch.Generator().manual_seed(args.seed)
    torch.manual_seed(args.seed)
    vocab, B, T, K = 257, 8, 61, 16
    dtype = torch.bfloat16 if args.dtype == "bf16" else torch.float32
    # a language to learn: the next token is an affine map of this one
    tokens = torch.randint(vocab, (B, 1), generator=gen)
    for _ in range(T):
        tokens = torch.cat([tokens, (tokens[:, -1:] * 5 + 3) % vocab], 1)
    x, target = tokens[:, :-1].cuda(), tokens[:, 1:].cuda()
    # the teacher names the right token among others, but does not tell it apart yet
    ids = torch.randint(vocab, (B, T, K), generator=gen)
    ids[..., 0] = tokens[:, 1:]
    ids = ids.cuda()
    teacher = torch.zeros(B, T, K, device="cuda", requires_grad=True)
    start = Student(vocab, dtype=dtype).state_dict()
    outer = []
    for it in range(args.outer):
        student = Student(vocab, dtype=dtype).cuda()
        student.load_state_dict(start)
        adapt(student, x, ids, teacher, args.inner)
        loss = outer_loss(student, x, target)
        (grad,) = torch.autograd.grad(loss, [teacher])
        with torch.no_grad():
            teacher -= 0.5 * grad / grad.square().mean().sqrt()
        outer.append(float(loss.detach()))
        print("outer step %d: loss after %d inner steps %.4f" % (it, args.inner, outer[-1]), flush=True)
    student = Student(vocab, dtype=dtype).cuda()
    student.load_state_dict(start)
    opt, inner = adapt(student, x, ids, teacher.detach(), 60)
    opt.detach_()
    print("distillation loss %.4f -> %.4f over %d steps" % (float(inner[0]), float(inner[-1]), len(inner)))
    got = generate(student, x[:, :40], 8)
    print("generated tokens that follow the language: %d of %d" % (int((got == target[:, 39:47]).sum()), got.numel()))
    return outer, [float(x) for x in inner], got


if __name__ == "__main__":
    main()
