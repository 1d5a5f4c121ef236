"""The language-model operators' argument checks through the C-ABI, without a GPU (they return before any
HIP call), the backward pass's division of rows, and the Python objects' own checks that need no device."""
import pytest
import torch

import paper_1802_05799_amd as hv

FAKE = 0x7F0000000000  # a plausible device address; never dereferenced by these calls
MIB = 1 << 20


def at(k, offset=0):
    return FAKE + k * 64 * MIB + offset


def refused(call, args, status, **change):
    a = dict(args, **change)
    try:
        call(*a.values(), 0)
    except hv.HvdxError as e:
        assert e.status == status, (change, e)
        return
    assert status == hv.OK, change


LOGPROBS = dict(logits=at(1), stride=1000, dtype=hv.BFLOAT16, rows=4, vocab=1000, scale=1.0, tokens=at(2), logprob=at(3), entropy=at(4),
                top=5, top_ids=at(5), top_logprobs=at(6), stats=at(7), workspace=at(8), workspace_bytes=64 * MIB)


def test_logprobs_refusals():
    def no(status, **change):
        refused(hv.hvdx_token_logprobs, LOGPROBS, status, **change)
    no(hv.ERR_INVALID, dtype=3)
    no(hv.ERR_INVALID, rows=-1)
    no(hv.ERR_INVALID, rows=(1 << 31) + 1)
    no(hv.ERR_INVALID, vocab=0, top=0)
    no(hv.ERR_UNSUPPORTED, vocab=1 << 31, stride=1 << 31)
    no(hv.ERR_INVALID, stride=999)
    no(hv.ERR_INVALID, stride=1 << 61)
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        no(hv.ERR_INVALID, scale=scale)
    no(hv.ERR_INVALID, top=-1)
    no(hv.ERR_INVALID, top=65)
    no(hv.ERR_INVALID, vocab=4, stride=4)  # top 5 of 4
    no(hv.ERR_INVALID, logits=0)
    no(hv.ERR_INVALID, tokens=0)
    no(hv.ERR_INVALID, top_ids=0)
    no(hv.ERR_INVALID, top_logprobs=0)
    no(hv.ERR_INVALID, logits=at(1, 1))
    no(hv.ERR_INVALID, tokens=at(2, 4))
    no(hv.ERR_INVALID, stats=at(7, 8))
    no(hv.ERR_INVALID, entropy=at(4, 2))
    no(hv.ERR_ALIAS, entropy=at(1, 7992))
    no(hv.ERR_ALIAS, entropy=at(3, 12))
    no(hv.ERR_ALIAS, top_ids=at(2, 24))
    no(hv.OK, rows=0, logits=0, tokens=0, workspace=0, workspace_bytes=0)
    assert "logits" in hv.hvdx_last_error() or hv.hvdx_last_error()


def test_logprobs_workspace():
    for rows, vocab, top in ((0, 1, 0), (1, 131072, 64), (24, 200000, 20), (4096, 131072, 32), (1, 8, 8)):
        need = hv.hvdx_token_logprobs_workspace_bytes(rows, vocab, top)
        assert 0 <= need <= 64 * MIB
        if need:
            args = dict(LOGPROBS, rows=rows, vocab=vocab, stride=vocab, top=top, logits=at(20))
            refused(hv.hvdx_token_logprobs, args, hv.ERR_WORKSPACE, workspace=0)
            refused(hv.hvdx_token_logprobs, args, hv.ERR_WORKSPACE, workspace_bytes=need - 1)
            refused(hv.hvdx_token_logprobs, args, hv.ERR_WORKSPACE, workspace=at(8, 8))
            refused(hv.hvdx_token_logprobs, args, hv.ERR_ALIAS, workspace=at(3))
    for rows, vocab in ((0, 1), (1, 131072), (24, 200000), (4096, 131072)):
        assert 0 <= hv.hvdx_distill_workspace_bytes(rows, vocab) <= 64 * MIB
    assert hv.hvdx_token_logprobs_workspace_bytes(-1, 5, 0) == 0 and hv.hvdx_distill_workspace_bytes(1, -5) == 0


def test_logprobs_grad_refusals():
    args = dict(logits=at(1), stride=1000, dtype=hv.FLOAT16, rows=4, vocab=1000, scale=1.0, tokens=at(2), stats=at(3), a=at(4), b=at(5),
                grad=at(6), grad_stride=1000)

    def no(status, **change):
        refused(hv.hvdx_token_logprobs_grad, args, status, **change)
    no(hv.ERR_INVALID, stats=0)
    no(hv.ERR_INVALID, grad=0)
    no(hv.ERR_INVALID, tokens=0)  # grad_logprob needs them
    no(hv.ERR_INVALID, grad_stride=10)
    no(hv.ERR_INVALID, scale=0.0)
    no(hv.ERR_INVALID, stats=at(3, 4))
    no(hv.ERR_ALIAS, grad=at(1, 2))  # over the logits, but not the very matrix
    no(hv.ERR_ALIAS, grad=at(1), grad_stride=1001)
    no(hv.ERR_ALIAS, grad=at(3))
    no(hv.OK, rows=0, logits=0)


def test_distill_refusals():
    args = dict(logits=at(1), stride=1000, dtype=hv.FLOAT32, rows=4, vocab=1000, scale=1.0, ids=at(2), teacher=at(3), entries=8, rest=1,
                grad_loss=at(4), loss=at(5), stats=at(6), grad=at(7), grad_stride=1000, workspace=at(8), workspace_bytes=64 * MIB)

    def no(status, **change):
        refused(hv.hvdx_distill, args, status, **change)
    no(hv.ERR_INVALID, entries=0)
    no(hv.ERR_INVALID, entries=65)
    no(hv.ERR_INVALID, rest=2)
    no(hv.ERR_INVALID, ids=0)
    no(hv.ERR_INVALID, teacher=0)
    no(hv.ERR_INVALID, grad_loss=0)
    no(hv.ERR_INVALID, grad_stride=999)
    no(hv.ERR_INVALID, dtype=-1)
    no(hv.ERR_INVALID, vocab=-3)
    no(hv.ERR_INVALID, scale=float("nan"))
    no(hv.ERR_INVALID, stats=at(6, 4))
    no(hv.ERR_ALIAS, grad=at(1, 4000))
    no(hv.ERR_ALIAS, loss=at(3))
    no(hv.ERR_ALIAS, stats=at(7, 16))
    no(hv.OK, rows=0, logits=0, ids=0)
    grad = {k: args[k] for k in ("logits", "stride", "dtype", "rows", "vocab", "scale", "ids", "teacher", "entries", "rest", "stats",
                                 "grad_loss", "grad", "grad_stride")}

    def no_grad(status, **change):
        refused(hv.hvdx_distill_grad, grad, status, **change)
    no_grad(hv.ERR_INVALID, stats=0)
    no_grad(hv.ERR_INVALID, grad_loss=0)
    no_grad(hv.ERR_INVALID, grad=0)
    no_grad(hv.ERR_INVALID, entries=100)
    no_grad(hv.ERR_ALIAS, grad=at(6))
    no_grad(hv.OK, rows=0)


NORM = dict(x=at(1), x_stride=512, y=at(2), y_stride=512, dtype=hv.BFLOAT16, rows=6, dim=512, post=at(3), gate=at(4),
            gate_dtype=hv.BFLOAT16, gate_rows=3, scale=1.0, weight=at(5), eps=1e-6, x_out=at(6), h_out=at(7), stats=at(8))


def test_norm_refusals():
    def no(status, **change):
        refused(hv.hvdx_residual_norm, NORM, status, **change)
    no(hv.ERR_UNSUPPORTED, dim=32769, x_stride=32769, y_stride=32769)
    no(hv.ERR_INVALID, dim=0)
    no(hv.ERR_INVALID, dtype=9)
    no(hv.ERR_INVALID, x_stride=511)
    no(hv.ERR_INVALID, y_stride=1)
    no(hv.ERR_INVALID, gate_rows=4)
    no(hv.ERR_INVALID, gate_rows=0)
    no(hv.ERR_INVALID, gate_dtype=hv.FLOAT16)
    no(hv.ERR_INVALID, scale=float("inf"))
    no(hv.ERR_INVALID, eps=-1.0)
    no(hv.ERR_INVALID, eps=float("nan"))
    no(hv.ERR_INVALID, x=0)
    no(hv.ERR_INVALID, y=0)  # post and gate need it
    no(hv.ERR_INVALID, y=0, post=0, gate=0)  # x_out without it
    no(hv.ERR_INVALID, x_out=0, h_out=0, stats=0)
    no(hv.ERR_INVALID, weight=at(5, 2))
    no(hv.ERR_INVALID, stats=at(8, 4))
    no(hv.ERR_ALIAS, h_out=at(1))  # x is not h_out's to overwrite
    no(hv.ERR_ALIAS, x_out=at(1), x_stride=600)
    no(hv.ERR_ALIAS, x_out=at(1, 2))
    no(hv.ERR_ALIAS, h_out=at(6))
    no(hv.ERR_ALIAS, x_out=at(5))
    no(hv.OK, rows=0, x=0)


def test_norm_grad_refusals():
    args = dict(x=at(1), x_stride=512, y=at(2), y_stride=512, dx=at(3), dx_stride=512, dh=at(4), dh_stride=512, dtype=hv.FLOAT16, rows=6,
                dim=512, post=at(5), gate=at(6), gate_dtype=hv.FLOAT32, gate_rows=6, scale=1.0, weight=at(7), stats=at(8), grad_x=at(9),
                grad_y=at(10), grad_weight=at(11), grad_post=at(12), grad_gate=at(13), workspace=at(14), workspace_bytes=64 * MIB)

    def no(status, **change):
        refused(hv.hvdx_residual_norm_grad, args, status, **change)
    no(hv.ERR_INVALID, stats=0)
    no(hv.ERR_INVALID, x=0)
    no(hv.ERR_INVALID, dx=0, dh=0)
    no(hv.ERR_INVALID, y=0, post=0, gate=0)  # grad_y without y
    no(hv.ERR_INVALID, post=0)
    no(hv.ERR_INVALID, gate=0)
    no(hv.ERR_INVALID, gate_rows=5)
    no(hv.ERR_INVALID, dh_stride=4)
    no(hv.ERR_INVALID, grad_x=0, grad_y=0, grad_weight=0, grad_post=0, grad_gate=0)
    need = hv.hvdx_residual_norm_grad_workspace_bytes(6, 512, 6)
    assert need > 0
    no(hv.ERR_WORKSPACE, workspace=0)
    no(hv.ERR_WORKSPACE, workspace_bytes=need - 1)
    no(hv.ERR_WORKSPACE, workspace=at(14, 4))
    no(hv.ERR_ALIAS, grad_x=at(1))
    no(hv.ERR_ALIAS, grad_y=at(9))
    no(hv.ERR_ALIAS, workspace=at(13))
    no(hv.OK, rows=0)
    for bad in ((0, 8, 0), (-1, 8, 0), (6, 0, 0), (6, 40000, 0), (6, 8, 4), (6, 8, -1)):
        assert hv.hvdx_residual_norm_grad_workspace_bytes(*bad) == 0


def test_objects_refuse_before_they_allocate():
    with pytest.raises(ValueError, match="GPU"):
        hv.TokenLogprobs(4, 100, device="cpu")
    with pytest.raises(ValueError, match="top"):
        hv.TokenLogprobs(4, 100, top=65)
    with pytest.raises(ValueError, match="top"):
        hv.TokenLogprobs(4, 10, top=11)
    with pytest.raises(ValueError):
        hv.TokenLogprobs(-1, 10)
    with pytest.raises(ValueError, match="alternatives"):
        hv.DistillLoss(4, 100, 0)
    with pytest.raises(ValueError, match="alternatives"):
        hv.DistillLoss(4, 100, 65)
    with pytest.raises(ValueError, match="GPU"):
        hv.DistillLoss(4, 100, 4, device="cpu")
    with pytest.raises(ValueError, match="rows of"):
        hv.ResidualNorm(4, 40000, torch.float32)
    with pytest.raises(ValueError, match="divide"):
        hv.ResidualNorm(4, 64, torch.float32, gate_rows=3)
