"""Data-parallel distillation of a small language model, every worker on one GPU.

    python examples/distill.py [--workers 4] [--steps 20] [--vocab 4096] [--dim 256] [--layers 2]

Each worker holds a student and a shard of the batch.  A step, on every worker: the teacher's log
probabilities of its likeliest next tokens (TokenLogprobs), the student's forward pass with the residual
connections and norms between its blocks (ResidualNorm), the loss against the teacher's alternatives with
the logits' gradient in the same pass (DistillLoss), and the backward pass; then every worker's
gradients are averaged (FusedAllreduce) and applied.  The first parameters are worker 0's (TensorBroadcast).
Matrix products are torch's; nothing here uses automatic differentiation.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1802_05799_amd as hv  # noqa: E402


class Model:
    """Embedding, `layers` blocks (a two-layer network, then norm, gate and residual), a head.  The language it
    learns is a table: the next token depends on the present one."""

    def __init__(self, rows, vocab, dim, layers, seed, grad):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape, std: std * torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
        hidden = 2 * dim
        self.parameters = {"embedding": new(vocab, dim, std=0.5), "weight": torch.ones(dim, device="cuda"),
                           "head": new(dim, vocab, std=2.0 / dim ** 0.5)}
        for i in range(layers):
            self.parameters.update({f"up{i}": new(dim, hidden, std=dim ** -0.5), f"down{i}": new(hidden, dim, std=hidden ** -0.5),
                                    f"post{i}": torch.ones(dim, device="cuda"), f"gate{i}": torch.full((1, dim), 0.5, device="cuda"),
                                    f"weight{i}": torch.ones(dim, device="cuda")})
        self.layers = layers
        f32 = torch.float32
        self.norms = [hv.ResidualNorm(rows, dim, f32, block=False, grad=grad)]
        self.norms += [hv.ResidualNorm(rows, dim, f32, gate_rows=rows, grad=grad) for _ in range(layers)]
        if grad:
            self.gradients = {k: torch.zeros_like(v) for k, v in self.parameters.items()}

    def forward(self, tokens):
        p, self.tokens, self.kept = self.parameters, tokens, []
        x = p["embedding"][tokens]
        self.norms[0](x, None, p["weight"])
        for i, norm in enumerate(self.norms[1:]):
            h = self.norms[i].h
            a = h @ p[f"up{i}"]
            y = torch.relu(a) @ p[f"down{i}"]
            norm(self.norms[i].x, y, p[f"weight{i}"], p[f"post{i}"], p[f"gate{i}"])
            self.kept.append((h, a, y))
        return self.norms[-1].h @ p["head"]

    def backward(self, grad_logits):
        p, g = self.parameters, self.gradients
        torch.mm(self.norms[-1].h.t(), grad_logits, out=g["head"])
        grad_x, grad_h = None, grad_logits @ p["head"].t()
        for i in reversed(range(self.layers)):
            h, a, y = self.kept[i]
            norm = self.norms[i + 1]
            norm.grad(y, grad_x, grad_h, p[f"weight{i}"], p[f"post{i}"], p[f"gate{i}"])
            g[f"weight{i}"].copy_(norm.grad_weight)
            g[f"post{i}"].copy_(norm.grad_post)
            g[f"gate{i}"].copy_(norm.grad_gate)
            torch.mm(torch.relu(a).t(), norm.grad_y, out=g[f"down{i}"])
            grad_a = (norm.grad_y @ p[f"down{i}"].t()) * (a > 0)
            torch.mm(h.t(), grad_a, out=g[f"up{i}"])
            grad_x, grad_h = norm.grad_x, grad_a @ p[f"up{i}"].t()
        self.norms[0].grad(None, grad_x, grad_h, p["weight"])
        g["weight"].copy_(self.norms[0].grad_weight)
        g["embedding"].zero_().index_add_(0, self.tokens, self.norms[0].grad_x)


def train(workers=4, steps=20, rows=512, vocab=4096, dim=256, layers=2, alternatives=16, rate=2.0, say=print):
    """Mean loss of each step; raises if the workers' parameters ever differ."""
    teacher = Model(rows, vocab, dim, layers, seed=1, grad=False)
    students = [Model(rows, vocab, dim, layers, seed=100 + r, grad=True) for r in range(workers)]
    hv.TensorBroadcast([list(s.parameters.values()) for s in students])(root=0)
    average = hv.FusedAllreduce([list(s.gradients.values()) for s in students], op="average")
    answer = hv.TokenLogprobs(rows, vocab, top=alternatives)
    loss = hv.DistillLoss(rows, vocab, alternatives)
    grad_loss = torch.full((rows,), 1.0 / rows, device="cuda")
    data = torch.Generator(device="cuda").manual_seed(7)
    seen = torch.randint(0, vocab, (256,), generator=data, device="cuda")  # the tokens that occur
    means = []
    for step in range(steps):
        total = torch.zeros((), device="cuda")
        for s in students:
            tokens = seen[torch.randint(0, len(seen), (rows,), generator=data, device="cuda")]
            answer(teacher.forward(tokens))
            logits = s.forward(tokens)
            loss(logits, answer.top_ids, answer.top_logprobs, grad_loss=grad_loss, out=logits)  # the gradient over the logits
            total += loss.loss.mean()
            s.backward(logits)
        average()
        for s in students:
            for k, v in s.parameters.items():
                v.sub_(s.gradients[k], alpha=rate)
        means.append((total / workers).item())
        say(f"step {step}: loss {means[-1]:.4f}")
        first = students[0].parameters
        if not all(torch.equal(v, first[k]) for s in students[1:] for k, v in s.parameters.items()):
            raise AssertionError("the workers' parameters differ")
    return means


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("workers", 4), ("steps", 20), ("rows", 512), ("vocab", 4096), ("dim", 256), ("layers", 2), ("alternatives", 16)):
        ap.add_argument(f"--{name}", type=int, default=value)
    ap.add_argument("--rate", type=float, default=2.0)
    train(**vars(ap.parse_args()))
