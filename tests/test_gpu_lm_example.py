"""The distillation example: its hand-written backward pass against automatic differentiation of the same
model in 64 bits, and a few data-parallel steps, whose loss falls and whose workers stay alike."""
import os
import sys

import pytest
import torch

import paper_1802_05799_amd as hv
from _gpu import say

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def reference_loss(p, tokens, layers, ids, lp):
    def normed(v, w):
        return v * (v.square().mean(1, keepdim=True) + 1e-6).rsqrt() * w
    x = p["embedding"][tokens]
    h = normed(x, p["weight"])
    for i in range(layers):
        y = torch.relu(h @ p[f"up{i}"]) @ p[f"down{i}"]
        x = x + normed(y, p[f"post{i}"]) * p[f"gate{i}"]
        h = normed(x, p[f"weight{i}"])
    logp = torch.log_softmax(h @ p["head"], 1)
    q = lp.exp()
    left = 1 - q.sum(1)
    rest = 1 - logp.gather(1, ids).exp().sum(1)
    return ((q * (lp - logp.gather(1, ids))).sum(1) + left * (left.log() - rest.log())).mean()


def test_gradients_of_the_whole_model():
    import distill

    rows, vocab, dim, layers, top = 96, 501, 40, 2, 7
    say("example: gradients")
    model = distill.Model(rows, vocab, dim, layers, seed=3, grad=True)
    teacher = distill.Model(rows, vocab, dim, layers, seed=4, grad=False)
    tokens = torch.randint(0, vocab, (rows,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    answer, loss = hv.TokenLogprobs(rows, vocab, top=top), hv.DistillLoss(rows, vocab, top)
    answer(teacher.forward(tokens))
    logits = model.forward(tokens)
    loss(logits, answer.top_ids, answer.top_logprobs, grad_loss=torch.full((rows,), 1 / rows, device="cuda"), out=logits)
    model.backward(logits)
    p = {k: v.double().requires_grad_(True) for k, v in model.parameters.items()}
    want = reference_loss(p, tokens, layers, answer.top_ids, answer.top_logprobs.double())
    want.backward()
    assert loss.loss.mean().item() == pytest.approx(want.item(), rel=1e-5)
    # the products are torch's in 32 bits: sums of up to `vocab` terms, a few of them in a row
    for k, v in p.items():
        assert (model.gradients[k].double() - v.grad).norm().item() <= 2e-5 * v.grad.norm().item(), k


def test_data_parallel_steps():
    import distill

    means = distill.train(workers=3, steps=6, rows=256, vocab=2000, dim=128, layers=2, alternatives=8, say=say)
    assert means[-1] < 0.9 * means[0]
