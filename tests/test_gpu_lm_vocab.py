"""TokenLogprobs and DistillLoss on the GPU against plain references in 64 bits (tests/_lm.py): every
type, lengths from one token up, unaligned and padded rows, masks, ties, broken rows; the gradients against
the formula and against differences."""
import math

import pytest
import torch

import _lm as R
import paper_1802_05799_amd as hv
from _gpu import say

pytestmark = pytest.mark.gpu
INF, NAN = R.INF, R.NAN
TYPES = [torch.float32, torch.float16, torch.bfloat16]
SENTINEL = 7.25


def matrix(rows, length, dtype, pad=0, offset=0, fill=SENTINEL):
    """(a [rows, length] view whose rows are `pad` elements apart and which starts `offset` elements into its
    storage, that storage)"""
    base = torch.full((offset + rows * (length + pad) + 64,), fill, dtype=dtype, device="cuda")
    return base[offset:offset + rows * (length + pad)].view(rows, length + pad)[:, :length], base


def untouched(base, view):
    """The storage outside the view still holds its fill."""
    seen = torch.zeros_like(base, dtype=torch.bool)
    torch.as_strided(seen, view.shape, view.stride(), view.storage_offset()).fill_(True)
    rest = base[~seen]
    return bool((rest == SENTINEL).all())


def logits(rows, vocab, dtype, seed, pad=0, offset=0, std=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z, _ = matrix(rows, vocab, dtype, pad, offset)
    z.copy_(torch.randn(rows, vocab, generator=g, device="cuda") * std)
    return z


def special_rows(z):
    """Overwrites the first rows with the cases where it can go wrong; returns their names by row."""
    vocab, low = z.shape[1], torch.finfo(z.dtype).min
    half = torch.arange(vocab, device="cuda") % 2 == 0
    rows = {
        "all masked": lambda r: r.fill_(-INF),
        "all lowest": lambda r: r.fill_(low),
        "half masked": lambda r: r.masked_fill_(half, -INF),
        "half lowest": lambda r: r.masked_fill_(half, low),
        "one left": lambda r: r.fill_(-INF)[-1:].fill_(2.0),
        "lowest and masked": lambda r: r.fill_(-INF)[vocab // 2:].fill_(low),
        "constant": lambda r: r.fill_(1.5),
        "zeros of both signs": lambda r: r.zero_()[::2].neg_(),
        "ties": lambda r: r.copy_((torch.arange(vocab, device="cuda") % 3).to(r.dtype)),
        "ascending": lambda r: r.copy_(torch.linspace(-8, 8, vocab, device="cuda").to(r.dtype)),
        "descending": lambda r: r.copy_(torch.linspace(8, -8, vocab, device="cuda").to(r.dtype)),
        "largest": lambda r: r[:1].fill_(-low),
        "plus infinity": lambda r: r[vocab // 3:vocab // 3 + 1].fill_(INF),
        "NaN": lambda r: r[vocab - 1:].fill_(NAN),
        "all NaN": lambda r: r.fill_(NAN),
        "one far above": lambda r: r[vocab // 2:vocab // 2 + 1].fill_(250.0),
    }
    assert len(rows) <= z.shape[0]
    for i, make in enumerate(rows.values()):
        make(z[i])
    return list(rows)


def depth_of(z, scale):
    """The largest scaled distance below the maximum whose log probability a test looks at."""
    x = z.double()
    x = torch.where(x.isfinite(), x, NAN)
    d = (x.nan_to_num(-1e308).amax(1) - x.nan_to_num(1e308).amin(1)) * scale
    return d.clamp(min=0.0)


def check_logprobs(z, tokens, scale, top, what, call=None, rows=None):
    say(f"{what}: {tuple(z.shape)} {z.dtype} stride {z.stride()} scale {scale} top {top}")
    call = call or hv.TokenLogprobs(z.shape[0], z.shape[1], top=top)
    call(z, tokens, scale=scale)
    torch.cuda.synchronize()
    n, v = z.shape
    want = R.logprobs(z, tokens, scale, top)
    bound = R.log_error(v, depth_of(z, scale))
    entropy = (R.sum_error(v) + 16 * R.U) * (2 + math.log(v + 1)) * 3
    R.assert_close(call.logprob[:n], want["logprob"], bound, torch.float32, f"{what} logprob")
    R.assert_close(call.entropy[:n], want["entropy"], entropy, torch.float32, f"{what} entropy")
    if top:
        assert torch.equal(call.top_ids[:n], want["top_ids"]), f"{what} top_ids"
        R.assert_close(call.top_logprobs[:n], want["top_logprobs"], bound[:, None], torch.float32, f"{what} top_logprobs")
    return call, want


SIZES = [(1, 0, 0), (2, 0, 1), (7, 1, 0), (8, 0, 3), (9, 3, 1), (64, 0, 0), (65, 5, 0), (257, 0, 1), (1000, 0, 0), (4097, 7, 2),
         (20011, 0, 0), (32768, 0, 0), (70001, 1, 1)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab,pad,offset", SIZES, ids=lambda v: str(v))
def test_logprobs_and_top(vocab, pad, offset, dtype):
    rows = 24
    z = logits(rows, vocab, dtype, vocab, pad, offset)
    special_rows(z)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    tokens[3], tokens[20], tokens[21] = -1, -5, vocab  # none, none, outside
    for top, scale in ((0, 1.0), (min(vocab, 5), 0.5), (min(vocab, 64), 1.7)):
        check_logprobs(z, tokens, scale, top, f"vocab {vocab}")


@pytest.mark.parametrize("rows,vocab,top", [(1, 32768, 8), (1, 50001, 64), (2, 131072, 20), (5, 200003, 64), (40, 131072, 1), (300, 9001, 33),
                                            (700, 40001, 16)])
def test_few_and_many_rows(rows, vocab, top):
    """Long rows split over blocks, and rows enough for a block each."""
    for dtype in (torch.float32, torch.bfloat16):
        z = logits(rows, vocab, dtype, rows, offset=rows % 3)
        if rows >= 16:
            special_rows(z)
        tokens = torch.arange(rows, device="cuda") * 7919 % vocab
        check_logprobs(z, tokens, 1.0, top, f"rows {rows}")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("rows", [1, 3, 600])
def test_top_where_the_largest_lie_together(rows, dtype):
    """Rows whose largest values recur with every period that a block's threads might read by, or fill one stretch."""
    vocab = 100003
    for period in (256, 512, 1024, 2048, 4096, 8192, 16384):
        z = torch.zeros(rows, vocab, dtype=dtype, device="cuda")
        near = torch.arange(vocab, device="cuda") % period < 9
        z += near.to(dtype) * (1 + torch.arange(vocab, device="cuda") % 7).to(dtype)
        check_logprobs(z, torch.zeros(rows, dtype=torch.int64, device="cuda"), 1.0, 64, f"period {period}")
    z = torch.zeros(rows, vocab, dtype=dtype, device="cuda")
    z[:, 40000:44000] = 3.0
    check_logprobs(z, torch.zeros(rows, dtype=torch.int64, device="cuda"), 1.0, 64, "one stretch")


def grad_bound(z, want, scale, a, b, vocab):
    logp, p = R.softmax_parts(z, scale)
    p, logp = p.nan_to_num(0.0), logp.nan_to_num(0.0, neginf=0.0)
    rel = R.log_error(vocab, logp.abs() + math.log(vocab + 1))
    size = a.abs()[:, None] + b.abs()[:, None] * (logp.abs() + math.log(vocab + 1) + 1)
    return scale * (rel * p * size + 4 * R.U * a.abs()[:, None]) + 1e-37


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab,pad,offset", [s for s in SIZES if s[0] < 60000], ids=lambda v: str(v))
def test_logprobs_grad(vocab, pad, offset, dtype):
    rows, scale = 24, 0.8
    z = logits(rows, vocab, dtype, vocab + 1, pad, offset)
    special_rows(z)
    g = torch.Generator(device="cuda").manual_seed(vocab)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    tokens[3], tokens[20], tokens[21] = -1, -5, vocab
    a, b = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    call = hv.TokenLogprobs(rows, vocab)
    call(z, tokens, scale=scale)
    zero = torch.zeros_like(a)
    for ga, gb in ((a, b), (a, None), (None, b)):
        say(f"grad vocab {vocab} {dtype} {ga is not None} {gb is not None}")
        out, base = matrix(rows, vocab, dtype, pad + 2, offset + 1)
        call.grad(z, tokens, ga, gb, out=out)
        torch.cuda.synchronize()
        pa, pb = (zero if ga is None else ga).double(), (zero if gb is None else gb).double()
        want = R.logprobs_grad(z, tokens if ga is not None else tokens.clamp(max=vocab - 1), scale, pa, pb)
        R.assert_close(out, want, grad_bound(z, want, scale, pa, pb, vocab), dtype, f"grad vocab {vocab}")
        assert untouched(base, out)
    copy = z.clone() if pad == 0 and offset == 0 else z
    out = call.grad(copy, tokens, a, b)
    assert torch.equal(call.grad(copy, tokens, a, b, out=copy).nan_to_num(9.0), out.nan_to_num(9.0))  # in place


def test_logprobs_grad_against_differences():
    """A direction's derivative by central differences of the 64-bit definition: off by h^2 / 6 times the third derivative,
    which for a sum of log probabilities and entropies of bounded logits is below 40 |v|^3."""
    rows, vocab, scale, h = 6, 501, 0.7, 2.0 ** -10
    g = torch.Generator(device="cuda").manual_seed(5)
    z = torch.randn(rows, vocab, generator=g, device="cuda")
    v = torch.randn(rows, vocab, generator=g, device="cuda").clamp(-2, 2)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    a, b = torch.rand(rows, generator=g, device="cuda"), torch.rand(rows, generator=g, device="cuda")
    call = hv.TokenLogprobs(rows, vocab)
    call(z, tokens, scale=scale)
    grad = call.grad(z, tokens, a, b)

    def at(x):
        w = R.logprobs(x, tokens, scale, 0)
        return (a.double() * w["logprob"] + b.double() * w["entropy"]).sum()
    numeric = (at(z.double() + h * v.double()) - at(z.double() - h * v.double())) / (2 * h)
    assert abs((grad.double() * v.double()).sum().item() - numeric.item()) <= h * h / 6 * 40 * 8 * rows + rows * vocab * 4 * R.U


# --- distillation -----------------------------------------------------------------------------

def alternatives(rows, vocab, top, seed):
    """Distinct tokens (as far as there are any) with log probabilities that leave part of the mass."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:top] if vocab >= top else
                       torch.cat([torch.randperm(vocab, generator=g, device="cuda"), torch.full((top - vocab,), -1, device="cuda")])
                       for _ in range(rows)])
    t = torch.log_softmax(2 * torch.randn(rows, top + 1, generator=g, device="cuda"), 1)[:, :top].contiguous()
    return ids, t


def check_distill(z, ids, t, scale, rest, what, in_place=False):
    rows, vocab = z.shape
    top = ids.shape[1]
    dtype = z.dtype
    say(f"{what}: {tuple(z.shape)} {dtype} stride {z.stride()} entries {top} scale {scale} rest {rest}")
    g = torch.linspace(0.5, 2.0, rows, device="cuda")
    loss, grad, log_rest = R.distill(z, ids, t, scale, rest)
    q, left = R.teacher(torch.where(ids >= vocab, -1, ids), t, rest)
    logp, p = R.softmax_parts(z, scale)
    clean = logp.nan_to_num(0.0, neginf=0.0)
    at = ids.clamp(0, vocab - 1)
    rel = R.log_error(vocab, clean.gather(1, at).abs() + math.log(vocab + 1))
    off_left = 4 * R.U * (top + 4) * rest  # 1 - sum q, and q itself
    span = log_rest.nan_to_num(0.0, neginf=0.0).abs() + left.clamp(min=1e-12).log().abs()
    loss_bound = (q * (rel + 8 * R.U * (clean.gather(1, at).abs() + q.clamp(min=1e-30).log().abs() + 4))).sum(1) \
        + left * (R.log_error(vocab, span) + 8 * R.U * span) + off_left * (span + 2) + 1e-30
    rel_v = R.log_error(vocab, clean.abs() + log_rest.nan_to_num(0.0, neginf=0.0).abs()[:, None] + math.log(vocab + 1))
    share = torch.where((log_rest == -INF)[:, None], 0.0, (clean - log_rest.nan_to_num(0.0, neginf=0.0)[:, None]).exp().clamp(max=1.0))
    dense = torch.zeros_like(clean).scatter_add_(1, at, q)
    total = (q.sum(1) + left)[:, None]
    grad_bound = scale * g.double()[:, None] * (rel_v * (p.nan_to_num(0.0) * total + left[:, None] * share) + off_left * (share + p.nan_to_num(0.0))
                                                + 8 * R.U * (top + 4) * dense) + 1e-37
    want = grad * g.double()[:, None]
    call = hv.DistillLoss(rows, vocab, top, rest=rest)
    out, base = matrix(rows, vocab, dtype, 3, 1)
    call(z, ids, t, scale=scale, grad_loss=g, out=out)
    torch.cuda.synchronize()
    R.assert_close(call.loss, loss, loss_bound, torch.float32, f"{what} loss")
    R.assert_close(out, want, grad_bound, dtype, f"{what} grad")
    assert untouched(base, out)
    call.loss.fill_(SENTINEL)
    call(z, ids, t, scale=scale)  # the loss alone, then the gradient alone
    R.assert_close(call.loss, loss, loss_bound, torch.float32, f"{what} loss alone")
    alone, base = matrix(rows, vocab, dtype, 0, 0)
    call.grad(z, ids, t, g, out=alone)
    torch.cuda.synchronize()
    R.assert_close(alone, want, grad_bound, dtype, f"{what} grad alone")
    assert untouched(base, alone)
    if in_place:
        twice = z.clone()
        call.grad(twice, ids, t, g, out=twice)
        assert torch.equal(twice.nan_to_num(9.0), alone.nan_to_num(9.0))
        twice, apart = z.clone(), torch.empty_like(z.clone())
        call(twice, ids, t, scale=scale, grad_loss=g, out=apart)  # the same rows at the same alignment
        both = call.loss.clone()
        call(twice, ids, t, scale=scale, grad_loss=g, out=twice)
        assert torch.equal(twice.nan_to_num(9.0), apart.nan_to_num(9.0)) and torch.equal(call.loss.nan_to_num(9.0), both.nan_to_num(9.0))


@pytest.mark.parametrize("rest", [True, False], ids=["rest", "renormalised"])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("vocab,pad,offset", SIZES, ids=lambda v: str(v))
def test_distill(vocab, pad, offset, dtype, rest):
    rows = 24
    z = logits(rows, vocab, dtype, vocab + 2, pad, offset)
    special_rows(z)
    for top, scale in ((1, 1.0), (5, 0.5), (64, 1.3)):
        ids, t = alternatives(rows, vocab, top, vocab + top)
        ids[17, top // 2:] = -1
        ids[18] = -1
        ids[19, 0] = vocab
        ids[20, 0] = ids[20, top - 1]  # a token twice
        t[21, 0] = -INF
        check_distill(z, ids, t, scale, rest, f"vocab {vocab}", in_place=True)


@pytest.mark.parametrize("rows,vocab,dtype", [(1, 32768, torch.bfloat16), (3, 200003, torch.float32), (33, 131072, torch.float16),
                                              (300, 66001, torch.bfloat16), (520, 131072, torch.bfloat16), (300, 131073, torch.bfloat16),
                                              (260, 65537, torch.float32), (1000, 1000, torch.float32)])
def test_distill_sizes(rows, vocab, dtype):
    z = logits(rows, vocab, dtype, rows)
    if rows >= 16:
        special_rows(z)
    for rest in (True, False):
        ids, t = alternatives(rows, vocab, 40, rows)
        ids[:, 0], ids[:, 1] = vocab - 1, 0  # both ends of a row
        check_distill(z, ids, t, 0.9, rest, f"rows {rows}")


@pytest.mark.parametrize("rows,vocab,dtype", [(60, 140001, torch.float32), (50, 300007, torch.bfloat16), (7, 300007, torch.float16),
                                              (2, 10, torch.bfloat16), (70, 17, torch.float32)])
def test_distill_rows_read_twice(rows, vocab, dtype):
    """Rows too long for registers (whose bitmap has fewer bytes than they have vectors), and of less than a vector or two."""
    z = logits(rows, vocab, dtype, rows, offset=1)
    if rows >= 16:
        special_rows(z)
    for rest in (True, False):
        ids, t = alternatives(rows, vocab, 33, rows)
        ids[:, 2] = vocab // 2
        ids[:, 3] = min(vocab - 1, vocab // 2 + 16384 * 8)  # the same byte of a smaller bitmap
        check_distill(z, ids, t, 1.1, rest, f"twice {vocab}", in_place=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_long_vocabulary(dtype):
    """Positions that binary32 does not hold exactly."""
    rows, vocab = 2, 40_000_003
    z = logits(rows, vocab, dtype, 6)
    tokens = torch.tensor([vocab - 1, 33_554_433], device="cuda")
    z[0, vocab - 1] = 30.0
    z[1, 33_554_433] = 30.0
    call, _ = check_logprobs(z, tokens, 1.0, 16, "long")
    a, b = torch.ones(rows, device="cuda"), torch.full((rows,), 0.1, device="cuda")
    out = call.grad(z, tokens, a, b)
    want = R.logprobs_grad(z, tokens, 1.0, a.double(), b.double())
    R.assert_close(out, want, grad_bound(z, want, 1.0, a.double(), b.double(), vocab), dtype, "long grad")
    del want, out
    ids, t = torch.tensor([[vocab - 1, 5], [33_554_433, 33_554_432]], device="cuda"), torch.tensor([[-0.5, -2.0]] * rows, device="cuda")
    check_distill(z, ids, t, 1.0, True, "long")


def test_distill_peaked_student():
    """The listed tokens hold all but 1e-3 .. 1e-60 of the student's probability: the unlisted mass must not come from a
    difference."""
    rows, vocab, top = 16, 5003, 8
    z = logits(rows, vocab, torch.float32, 11, std=1.0)
    ids, t = alternatives(rows, vocab, top, 3)
    z.scatter_(1, ids[:, :2], torch.linspace(15.0, 145.0, rows, device="cuda")[:, None].expand(rows, 2).contiguous())
    check_distill(z, ids, t, 1.0, True, "peaked")
    t = torch.log_softmax(t, 1) - 1e-5  # a teacher that is as sure
    check_distill(z, ids, t, 1.0, True, "peaked, sure teacher")


def test_distill_every_token_listed():
    for vocab in (1, 5, 8, 64):
        z = logits(4, vocab, torch.float32, vocab)
        ids = torch.stack([torch.randperm(vocab, device="cuda") for _ in range(4)])
        t = torch.log_softmax(torch.randn(4, vocab, device="cuda"), 1)
        for rest in (True, False):
            check_distill(z, ids, t, 1.0, rest, f"all of {vocab}")
        if vocab > 1:
            check_distill(z, ids, t - 1.0, 1.0, True, f"all of {vocab}, mass left")  # nowhere for it: infinite


def test_distill_against_differences():
    rows, vocab, top, scale, h = 5, 401, 7, 0.9, 2.0 ** -10
    g = torch.Generator(device="cuda").manual_seed(9)
    z = torch.randn(rows, vocab, generator=g, device="cuda")
    v = torch.randn(rows, vocab, generator=g, device="cuda").clamp(-2, 2)
    ids, t = alternatives(rows, vocab, top, 2)
    w = torch.rand(rows, generator=g, device="cuda")
    for rest in (True, False):
        call = hv.DistillLoss(rows, vocab, top, rest=rest)
        out = torch.empty_like(z)
        call(z, ids, t, scale=scale, grad_loss=w, out=out)
        at = lambda x: (w.double() * R.distill(x, ids, t, scale, rest)[0]).sum()  # noqa: E731
        numeric = (at(z.double() + h * v.double()) - at(z.double() - h * v.double())) / (2 * h)
        got = (out.double() * v.double()).sum()
        assert abs(got.item() - numeric.item()) <= h * h / 6 * 40 * 8 * rows + rows * vocab * 4 * R.U


def test_cross_entropy_is_one_certain_alternative():
    rows, vocab = 9, 777
    z = logits(rows, vocab, torch.float32, 4)
    tokens = torch.arange(rows, device="cuda") * 31
    lp, ds = hv.TokenLogprobs(rows, vocab), hv.DistillLoss(rows, vocab, 1, rest=False)
    out, g = torch.empty_like(z), torch.ones(rows, device="cuda")
    lp(z, tokens)
    ds(z, tokens[:, None], torch.zeros(rows, 1, device="cuda"), grad_loss=g, out=out)
    assert (ds.loss + lp.logprob).abs().max().item() <= 2 * R.log_error(vocab, 30.0)
    assert (out + lp.grad(z, tokens, g)).abs().max().item() <= 2 * R.log_error(vocab, 30.0)


# --- both -------------------------------------------------------------------------------------

def test_offsets_past_32_bits():
    """Rows so far apart that elements lie past 2^31, and bytes past 2^32."""
    rows, vocab, stride = 3, 1001, (1 << 30) + 5
    base = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    z = torch.as_strided(base, (rows, vocab), (stride, 1))
    z.copy_(logits(rows, vocab, torch.bfloat16, 1))
    tokens = torch.tensor([5, 1000, 77], device="cuda")
    call, _ = check_logprobs(z, tokens, 1.0, 5, "far rows")
    near = z.contiguous()
    a = torch.ones(rows, device="cuda")
    want = call.grad(near, tokens, a)
    ids, t = alternatives(rows, vocab, 6, 1)
    ds = hv.DistillLoss(rows, vocab, 6)
    ref = torch.empty_like(near)
    ds(near, ids, t, grad_loss=a, out=ref)
    out = torch.as_strided(torch.empty_like(base), (rows, vocab), (stride, 1))
    ds(z, ids, t, grad_loss=a, out=out)
    assert torch.equal(out, ref)
    assert torch.equal(call.grad(z, tokens, a, out=z), want)


def test_fewer_rows_than_built_for():
    call = hv.TokenLogprobs(40, 1000, top=3)
    for name in ("logprob", "entropy", "top_logprobs"):
        getattr(call, name).fill_(SENTINEL)
    call.top_ids.fill_(77)
    z = logits(11, 1000, torch.float16, 3)
    tokens = torch.arange(11, device="cuda")
    check_logprobs(z, tokens, 1.0, 3, "fewer rows", call=call)
    for name in ("logprob", "entropy", "top_logprobs"):
        assert bool((getattr(call, name)[11:] == SENTINEL).all())
    assert bool((call.top_ids[11:] == 77).all())
    call(z[:0], tokens[:0])  # no rows: nothing happens
    call(z[5:6], tokens[5:6])
    assert torch.allclose(call.logprob[0], R.logprobs(z[5:6], tokens[5:6], 1.0, 0)["logprob"][0].float(), atol=1e-5)


def test_objects_refuse():
    call, ds = hv.TokenLogprobs(4, 100, top=2), hv.DistillLoss(4, 100, 3)
    z, tokens = torch.zeros(4, 100, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    ids, t = torch.zeros(4, 3, dtype=torch.int64, device="cuda"), torch.zeros(4, 3, device="cuda")
    g = torch.ones(4, device="cuda")
    for bad in (z.double(), z.cpu(), z[:, :99], torch.zeros(5, 100, device="cuda"), z.t().contiguous().t(), z[:1].expand(4, 100), z[0]):
        with pytest.raises(ValueError):
            call(bad, tokens)
        with pytest.raises(ValueError):
            ds(bad, ids, t)
    for bad in (tokens[:3], tokens.int(), tokens.cpu(), torch.zeros(8, dtype=torch.int64, device="cuda")[::2]):
        with pytest.raises(ValueError):
            call(z, bad)
    with pytest.raises(hv.HvdxError, match="scale"):
        call(z, tokens, scale=0.0)
    with pytest.raises(hv.HvdxError, match="scale"):
        call(z, tokens, scale=2e30)
    with pytest.raises(ValueError, match="rows after"):
        call.grad(z, tokens, g)  # before any call
    call(z, tokens)
    with pytest.raises(ValueError, match="rows after"):
        call.grad(z[:2], tokens[:2], g[:2])
    with pytest.raises(ValueError, match="out"):
        call.grad(z, tokens, g, out=z.half())
    with pytest.raises(hv.HvdxError, match="overlaps"):
        wide = torch.zeros(4, 101, device="cuda")
        call(wide[:, :100], tokens)
        call.grad(wide[:, :100], tokens, g, out=wide[:, 1:])
    with pytest.raises(ValueError, match="go together"):
        ds(z, ids, t, grad_loss=g)
    with pytest.raises(ValueError, match="ids"):
        ds(z, ids[:, :2], t)
    with pytest.raises(ValueError, match="logprobs"):
        ds(z, ids, t.half())


def test_another_stream():
    rows, vocab = 64, 50001
    z = logits(rows, vocab, torch.bfloat16, 8)
    tokens = torch.arange(rows, device="cuda")
    ids, t = alternatives(rows, vocab, 9, 5)
    g = torch.ones(rows, device="cuda")
    lp, ds = hv.TokenLogprobs(rows, vocab, top=9), hv.DistillLoss(rows, vocab, 9)
    grad, grad2 = torch.empty_like(z), torch.empty_like(z)
    lp(z, tokens)
    ds(z, ids, t, grad_loss=g, out=grad)
    want = [x.clone() for x in (lp.logprob, lp.entropy, lp.top_ids, lp.top_logprobs, ds.loss, grad)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    lp(z, tokens, stream=s.cuda_stream)
    with torch.cuda.stream(s):
        ds(z, ids, t, grad_loss=g, out=grad2)
    s.synchronize()
    for x, y in zip((lp.logprob, lp.entropy, lp.top_ids, lp.top_logprobs, ds.loss, grad2), want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("rows", [2, 400])
def test_replayed_from_a_graph(rows):
    vocab = 40001
    z = logits(rows, vocab, torch.bfloat16, 8)
    tokens = torch.arange(rows, device="cuda")
    ids, t = alternatives(rows, vocab, 9, 5)
    g = torch.ones(rows, device="cuda")
    lp, ds = hv.TokenLogprobs(rows, vocab, top=9), hv.DistillLoss(rows, vocab, 9)
    grad, glp = torch.empty_like(z), torch.empty_like(z)

    def step():
        lp(z, tokens)
        lp.grad(z, tokens, g, g, out=glp)
        ds(z, ids, t, grad_loss=g, out=grad)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        z.copy_(logits(rows, vocab, torch.bfloat16, 100 + seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (lp.logprob, lp.entropy, lp.top_ids, lp.top_logprobs, ds.loss, grad, glp)]
        step()
        torch.cuda.synchronize()
        for x, y in zip(got, (lp.logprob, lp.entropy, lp.top_ids, lp.top_logprobs, ds.loss, grad, glp)):
            assert torch.equal(x, y)


def test_timeline_names_the_operators():
    z = logits(32, 2000, torch.float32, 1)
    tokens = torch.arange(32, device="cuda")
    lp = hv.TokenLogprobs(32, 2000, top=2)
    with hv.Timeline() as tl:
        lp(z, tokens)
        lp.grad(z, tokens, torch.ones(32, device="cuda"))
    kinds = [r["kind"] for r in tl.records]
    assert kinds[-1] == hv._lib.KERNEL_LOGPROBS_GRAD and set(kinds[:-1]) == {hv._lib.KERNEL_LOGPROBS}
    assert all(r["duration_us"] > 0 and r["count"] == 64000 for r in tl.records)
    names = {e["name"] for e in tl.chrome_trace()["traceEvents"]}
    assert "token log probabilities" in names


@pytest.mark.parametrize("rows,vocab,top,dtype", [(1100, 2087, 20, torch.bfloat16), (1300, 1081, 32, torch.float32), (4100, 8001, 7, torch.float16),
                                                  (700, 3500, 0, torch.bfloat16), (300, 2000, 64, torch.bfloat16), (20, 2000, 64, torch.float16),
                                                  (20, 1000, 64, torch.float32), (700, 8000, 64, torch.bfloat16), (30, 8003, 33, torch.bfloat16),
                                                  (300, 70, 64, torch.float32)])
def test_short_rows(rows, vocab, top, dtype):
    """A wavefront a row over several batches of its vectors, and many alternatives of short rows."""
    z = logits(rows, vocab, dtype, rows, offset=1)
    special_rows(z)
    tokens = torch.arange(rows, device="cuda") * 7919 % vocab
    check_logprobs(z, tokens, 0.8, top, f"short {rows}")


@pytest.mark.parametrize("rows,vocab,dtype", [(600, 3500, torch.bfloat16), (1100, 1081, torch.float32), (2100, 8003, torch.bfloat16), (600, 20000, torch.float16),
                                              (600, 32767, torch.bfloat16), (20, 3500, torch.bfloat16), (20, 8001, torch.float16)])
def test_distill_short_rows(rows, vocab, dtype):
    z = logits(rows, vocab, dtype, rows, offset=1)
    special_rows(z)
    for rest in (True, False):
        ids, t = alternatives(rows, vocab, 9, rows)
        ids[:, 0], ids[:, 1] = vocab - 1, 0
        check_distill(z, ids, t, 1.2, rest, f"short {rows}", in_place=True)
