"""Plain references in 64 bits for the language-model operators, written from their definitions, and the
error bounds of the tests (test helper).

Bounds, with u = 2^-24 (binary32's half unit): a sum of n positive terms, taken as at most n/64 serial
steps in a lane and some 20 joins, is off by at most (n/64 + 20) u of itself; a term 2^d is off by the
hardware exponential's 2 u and by the 3 u |d| of its argument; a logarithm adds u of itself.
The tests double what these give.  A result rounded to a type with unit e is off by e/2 of itself
besides, or by half the smallest subnormal.
"""
import math

import torch

U = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -23, torch.float16: 2.0 ** -10, torch.bfloat16: 2.0 ** -7}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
INF, NAN = float("inf"), float("nan")


def sum_error(n):
    """Relative error allowed a sum over a row of n terms."""
    return 2 * U * (n / 64 + 20)


def log_error(n, depth):
    """Absolute error allowed a log probability whose logits lie `depth` (scaled) below the maximum."""
    return sum_error(n) + 2 * U * (8 * depth + 2 * math.log(n + 1) + 8)


def softmax_parts(z, scale):
    """(log p, p) in 64 bits; rows of minus infinity throughout: minus infinity and 0; broken rows: NaN."""
    x = z.double()
    broken = (x.isnan() | (x == INF)).any(1, keepdim=True)
    m = x.amax(1, keepdim=True)
    none = m == -INF
    d = (x - torch.where(none | broken, 0.0, m)) * scale
    lse = torch.where(none, 0.0, torch.logsumexp(d, 1, keepdim=True))
    logp = torch.where(none, -INF, d - lse)
    logp = torch.where(broken, NAN, logp)
    return logp, torch.where(broken, NAN, logp.exp())


def logprobs(z, tokens, scale, top):
    vocab = z.shape[1]
    logp, p = softmax_parts(z, scale)
    at = tokens.clamp(0, vocab - 1)[:, None]
    mine = torch.where(tokens < 0, 0.0, logp.gather(1, at)[:, 0])
    mine = torch.where(tokens >= vocab, NAN, mine)
    entropy = -torch.where(p == 0, 0.0, p * logp).sum(1)
    out = {"logprob": mine, "entropy": entropy}
    if top:
        broken = p.isnan().any(1, keepdim=True)
        order = torch.where(broken, 0.0, z.double() + 0.0).sort(dim=1, descending=True, stable=True).indices[:, :top]
        out["top_ids"] = torch.where(broken, -1, order)
        out["top_logprobs"] = torch.where(broken, NAN, logp.gather(1, order))
    return out


def logprobs_grad(z, tokens, scale, a, b):
    """a, b: [rows] in 64 bits (zeros for none)."""
    vocab = z.shape[1]
    logp, p = softmax_parts(z, scale)
    none = (z.double() == -INF).all(1, keepdim=True)
    entropy = -torch.where(p == 0, 0.0, p * logp).sum(1, keepdim=True)
    a = torch.where(tokens >= 0, a, 0.0)[:, None]
    a = torch.where(tokens[:, None] >= vocab, NAN, a)
    hit = torch.arange(vocab, device=z.device) == tokens[:, None]
    g = torch.where(hit, a, 0.0) - a * p - b[:, None] * torch.where(p == 0, 0.0, p * (logp + entropy))
    return torch.where(none, 0.0, g * scale)


def teacher(ids, t, rest):
    """(probability of each entry, what they leave) in 64 bits."""
    there = ids >= 0
    t = torch.where(there, t.double(), -INF)
    if rest:
        q = t.exp()
        return q, (1.0 - q.sum(1)).clamp(min=0.0)
    high = t.amax(1, keepdim=True)
    e = (t - torch.where(high == -INF, 0.0, high)).exp()
    total = e.sum(1, keepdim=True)
    return torch.where(total > 0, e / total.clamp(min=1e-300), 0.0), torch.zeros(ids.shape[0], dtype=torch.float64, device=ids.device)


def distill(z, ids, t, scale, rest):
    """(loss, gradient for grad_loss 1, log of the unlisted mass)"""
    rows, vocab = z.shape
    bad = (ids >= vocab).any(1)
    ids = torch.where(ids >= vocab, -1, ids)
    there, at = ids >= 0, ids.clamp(min=0)
    logp, p = softmax_parts(z, scale)
    q, left = teacher(ids, t, rest)
    log_q = torch.where(q > 0, q, 1.0).log()
    loss = torch.where(there & (q != 0), q * (log_q - logp.gather(1, at)), 0.0).sum(1)
    listed = torch.zeros_like(p).scatter_add_(1, at, there.double()) > 0
    log_rest = torch.logsumexp(torch.where(listed, -INF, logp), 1)
    gone = (log_rest == -INF)
    if rest:
        loss = loss + torch.where(gone, torch.where(left > 1e-6, INF, 0.0),
                                  torch.where(left > 0, left * (torch.where(left > 0, left, 1.0).log() - log_rest), 0.0))
    total = q.sum(1) + left
    grad = total[:, None] * p - torch.zeros_like(p).scatter_add_(1, at, q)
    if rest:
        share = torch.where(gone[:, None], 0.0, (logp - torch.where(gone, 0.0, log_rest)[:, None]).exp())
        grad = grad - torch.where(listed, 0.0, left[:, None] * share)
    none = (z.double() == -INF).all(1)
    grad = torch.where(none[:, None], 0.0, grad * scale)
    return torch.where(bad, NAN, loss), torch.where(bad[:, None], NAN, grad), log_rest


def residual_norm(x, y, weight, post, gate, scale, eps):
    """(x_out, h_out) of 64-bit operands; gate: [groups, dim] or None."""
    def factor(v):
        return ((v * v).mean(1, keepdim=True) + eps).rsqrt()
    if y is not None:
        if post is not None:
            y = y * factor(y) * post
        if gate is not None:
            y = y * gate.repeat_interleave(x.shape[0] // gate.shape[0], 0)
        x = x + scale * y
    h = x * factor(x)
    return x, h if weight is None else h * weight


def assert_close(got, want, bound, dtype, what):
    """|got - want| <= bound + rounding to `dtype`; the same NaNs and infinities."""
    got, want = got.double(), want.double()
    bound = torch.as_tensor(bound, dtype=torch.float64, device=want.device).expand_as(want)
    fine = want.isfinite()
    limit = torch.finfo(dtype).max
    over = fine & (want.abs() > limit)  # rounds to infinity, or to the largest value
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaNs differ"
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities differ"
    fine &= ~over
    off = (got - want).abs()[fine]
    may = (bound + want.abs() * (UNIT[dtype] / 2) * 1.01 + TINY[dtype] / 2)[fine]
    assert not bool(off.isnan().any()), f"{what}: not finite where it should be"
    if off.numel():
        worst = (off / may).max().item()
        assert worst <= 1.0, f"{what}: {worst:.3g} times the bound (off by {off.max().item():.3g})"
