"""ResidualNorm on the GPU against plain references in 64 bits (tests/_lm.py): every type, widths from one
element up, each kind of gate, with and without the norm after the block and the block itself; the gradients
against automatic differentiation of the 64-bit definition and against differences."""
import pytest
import torch

import _lm as R
import paper_1802_05799_amd as hv
from _gpu import say

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
SENTINEL = 7.25
DIMS = [1, 3, 8, 9, 64, 100, 511, 1001, 1024, 2047, 4096, 5001, 8192, 16385, 32768]


def strided(rows, dim, dtype, g, pad=0, std=1.0):
    base = torch.empty(rows, dim + pad, dtype=dtype, device="cuda")
    base.copy_(torch.randn(rows, dim + pad, generator=g, device="cuda") * std)
    return base[:, :dim]


def operands(rows, dim, dtype, seed, post, gate_rows, gate_dtype, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, y = strided(rows, dim, dtype, g, pad, 1.5), strided(rows, dim, dtype, g, 2 * pad, 0.7)
    f = lambda: 1 + 0.2 * torch.randn(dim, generator=g, device="cuda")  # noqa: E731
    gate = (0.5 + 0.3 * torch.randn(rows // gate_rows, dim, generator=g, device="cuda")).to(gate_dtype) if gate_rows else None
    return x, y, f(), f() if post else None, gate


def doubles(*xs):
    return [None if x is None else x.double() for x in xs]


def bounds(dim):
    """Relative error of a norm's factor (half its sum's, and the root and division), of a result of it."""
    return R.sum_error(dim) / 2 + 8 * R.U


VARIANTS = [(True, 0, None), (False, 0, None), (True, "all", torch.float32), (False, "all", None), (True, 3, None), (True, 1, None),
            (False, 1, torch.float32), (True, 4, torch.float32)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim", DIMS)
def test_forward(dim, dtype):
    rows = 12
    for post, gate_rows, gate_dtype in VARIANTS:
        gate_rows = rows if gate_rows == "all" else gate_rows
        gate_dtype = gate_dtype or dtype
        say(f"forward {rows}x{dim} {dtype} post {post} gate_rows {gate_rows} {gate_dtype}")
        x, y, w, p, gate = operands(rows, dim, dtype, dim, post, gate_rows, gate_dtype, pad=dim % 5)
        call = hv.ResidualNorm(rows, dim, dtype, post=post, gate_rows=gate_rows, gate_dtype=gate_dtype, eps=1e-5)
        call(x, y, w, p, gate, scale=0.6)
        torch.cuda.synchronize()
        new, h = R.residual_norm(*doubles(x, y, w, p, gate), 0.6, 1e-5)
        part = (new - x.double()).abs()
        rel = bounds(dim)
        R.assert_close(call.x, new, part * (rel + 8 * R.U) + 4 * R.U * (x.double().abs() + part), dtype, "x")
        spread = (part * (rel + 8 * R.U) + 4 * R.U * (x.double().abs() + part)) / new.square().mean(1, keepdim=True).add(1e-5).sqrt()
        R.assert_close(call.h, h, h.abs() * (rel + 8 * R.U) + spread * w.double().abs() + h.abs() * spread.square().mean(1, keepdim=True).sqrt(),
                       dtype, "h")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_norm_alone_and_unweighted(dtype):
    rows, dim = 7, 777
    x, *_ = operands(rows, dim, dtype, 3, False, 0, None, pad=3)
    call = hv.ResidualNorm(rows, dim, dtype, block=False, grad=True)
    for weight in (None, torch.linspace(0.5, 1.5, dim, device="cuda")):
        call(x, None, weight)
        _, h = R.residual_norm(x.double(), None, None if weight is None else weight.double(), None, None, 1.0, 1e-6)
        R.assert_close(call.h, h, h.abs() * (bounds(dim) + 8 * R.U), dtype, "h")
        assert call.x is x
        check_grads(call, x, None, weight, None, None, 1.0, dtype, seed=2)


def reference_grads(x_out, y, w, p, gate, scale, eps, dx, dh):
    """Automatic differentiation of the definition in 64 bits, at the stream that leads to x_out."""
    args = [None if v is None else v.double().requires_grad_(True) for v in (y, w, p, gate)]
    zero = torch.zeros_like(x_out, dtype=torch.float64)
    with torch.no_grad():
        part = R.residual_norm(zero, *args, scale, eps)[0] if y is not None else 0.0
    x = (x_out.double() - part).requires_grad_(True)
    new, h = R.residual_norm(x, *args, scale, eps)
    keep = [x] + [a for a in args if a is not None]
    outs, grads = ([new, h], [dx, dh]) if dx is not None and dh is not None else ([new], [dx]) if dh is None else ([h], [dh])
    got = torch.autograd.grad(outs, keep, [v.double() for v in grads], allow_unused=True)
    it = iter(got)
    out = {"x": next(it)}
    for name, a in zip(("y", "weight", "post", "gate"), args):
        v = next(it) if a is not None else None
        out[name] = torch.zeros_like(a) if a is not None and v is None else v
    return out


def check_grads(call, x_out, y, w, p, gate, scale, dtype, seed, parts="both", eps=1e-6):
    rows, dim = x_out.shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    dx = strided(rows, dim, dtype, g, 1, 0.3) if parts != "h" else None
    dh = strided(rows, dim, dtype, g, 2, 0.3) if parts != "x" else None
    say(f"grad {rows}x{dim} {dtype} post {p is not None} gate {None if gate is None else tuple(gate.shape)} of {parts}")
    # the factors of the stored stream, so that the reference differentiates at the same point
    r = lambda v: (v.double().square().mean(1) + eps).rsqrt().float()  # noqa: E731
    call.stats.copy_(torch.stack([r(y) if p is not None else torch.ones(rows, device="cuda"), r(x_out)], 1))
    call.grad(y, dx, dh, w, p, gate, scale=scale)
    torch.cuda.synchronize()
    want = reference_grads(x_out, y, w, p, gate, scale, eps, dx, dh)
    # the size of the terms that each result is a sum of, and how far each may be off
    rx = call.stats[:, 1:].double()
    xh = x_out.double() * rx
    gw = (dh.double() if dh is not None else torch.zeros_like(xh)) * (1.0 if w is None else w.double())
    size = (dx.double().abs() if dx is not None else 0.0) + rx * (gw.abs() + xh.abs() * (gw * xh).abs().mean(1, keepdim=True))
    rel = R.sum_error(dim) + 24 * R.U
    R.assert_close(call.grad_x, want["x"], rel * size, dtype, "grad_x")
    if dh is not None and w is not None:
        terms = (dh.double() * xh).abs().sum(0)
        R.assert_close(call.grad_weight, want["weight"], (R.sum_error(rows) + 16 * R.U) * terms, torch.float32, "grad_weight")
    elif dh is None:
        assert not bool(call.grad_weight.any())
    if y is None:
        return
    ry = call.stats[:, :1].double()
    yh = y.double() * ry
    post = p.double() if p is not None else torch.ones(dim, dtype=torch.float64, device="cuda")
    over = gate.double().repeat_interleave(rows // gate.shape[0], 0).abs() if gate is not None else 1.0
    du = scale * size * over
    if gate is not None:
        span = rows // gate.shape[0]
        terms = (scale * size * (yh * post).abs()).view(-1, span, dim).sum(1)
        R.assert_close(call.grad_gate, want["gate"], (R.sum_error(span) + rel + 16 * R.U) * terms, gate.dtype, "grad_gate")
    if p is not None:
        R.assert_close(call.grad_post, want["post"], (R.sum_error(rows) + rel + 16 * R.U) * (du * yh.abs()).sum(0), torch.float32, "grad_post")
        t = du * post.abs()
        du = ry * (t + yh.abs() * (t * yh.abs()).mean(1, keepdim=True))
    R.assert_close(call.grad_y, want["y"], 2 * rel * du, dtype, "grad_y")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("dim", DIMS)
def test_backward(dim, dtype):
    rows = 12
    for i, (post, gate_rows, gate_dtype) in enumerate(VARIANTS):
        gate_rows = rows if gate_rows == "all" else gate_rows
        gate_dtype = gate_dtype or dtype
        x, y, w, p, gate = operands(rows, dim, dtype, dim, post, gate_rows, gate_dtype, pad=dim % 5)
        call = hv.ResidualNorm(rows, dim, dtype, post=post, gate_rows=gate_rows, gate_dtype=gate_dtype, grad=True)
        call.x.copy_(x)
        check_grads(call, call.x, y, w, p, gate, 0.6, dtype, seed=dim + i, parts=("both", "h", "x")[i % 3])


@pytest.mark.parametrize("rows,dim,gate_rows", [(1, 4096, 1), (2, 100, 2), (777, 513, 777), (2000, 1024, 100), (4096, 640, 16), (3000, 257, 1),
                                                (5000, 72, 2500), (1030, 5001, 103)])
def test_many_rows(rows, dim, gate_rows):
    """Sums over rows dealt out to many blocks, in segments of a group or whole groups."""
    for dtype in (torch.float32, torch.bfloat16):
        x, y, w, p, gate = operands(rows, dim, dtype, rows, True, gate_rows, dtype)
        call = hv.ResidualNorm(rows, dim, dtype, gate_rows=gate_rows, gate_dtype=dtype, grad=True)
        call.x.copy_(x)
        check_grads(call, call.x, y, w, p, gate, 1.1, dtype, seed=rows)
        first = [v.clone() for v in (call.grad_x, call.grad_y, call.grad_weight, call.grad_post, call.grad_gate)]
        g = torch.Generator(device="cuda").manual_seed(rows)
        dx, dh = strided(rows, dim, dtype, g, 1, 0.3), strided(rows, dim, dtype, g, 2, 0.3)
        call.grad(y, dx, dh, w, p, gate, scale=1.1)
        for a, b in zip(first, (call.grad_x, call.grad_y, call.grad_weight, call.grad_post, call.grad_gate)):
            assert torch.equal(a, b)  # the same bits again


def test_backward_against_differences():
    rows, dim, scale, h = 4, 96, 0.8, 2.0 ** -10
    x, y, w, p, gate = operands(rows, dim, torch.float32, 5, True, 2, torch.float32)
    call = hv.ResidualNorm(rows, dim, torch.float32, gate_rows=2, grad=True)
    call(x, y, w, p, gate, scale=scale)
    g = torch.Generator(device="cuda").manual_seed(6)
    dx, dh = strided(rows, dim, torch.float32, g), strided(rows, dim, torch.float32, g)
    call.grad(y, dx, dh, w, p, gate, scale=scale)
    ops = doubles(x, y, w, p, gate)
    grads = [call.grad_x, call.grad_y, call.grad_weight, call.grad_post, call.grad_gate]

    def at(args):
        new, out = R.residual_norm(*args, scale, 1e-6)
        return ((new * dx.double()).sum() + (out * dh.double()).sum()).item()
    for i, grad in enumerate(grads):
        v = torch.randn(ops[i].shape, generator=g, device="cuda", dtype=torch.float64).clamp(-2, 2)
        plus, minus = [list(ops), list(ops)]
        plus[i], minus[i] = ops[i] + h * v, ops[i] - h * v
        numeric = (at(plus) - at(minus)) / (2 * h)
        # truncation: h^2 / 6 times a third derivative below 200 a unit of the rows' sums
        assert abs((grad.double() * v).sum().item() - numeric) <= h * h / 6 * 200 * rows * dim + 1e-4 * rows


def test_rows_of_zeros_and_extremes():
    """A row of zeros has the factor eps^-1/2; NaN and infinity stay in their row."""
    rows, dim = 6, 300
    x, y, w, p, gate = operands(rows, dim, torch.float32, 1, True, 0, None)
    x[0], y[0] = 0.0, 0.0
    x[1, 5], y[2, 7], x[3, 9] = float("nan"), float("inf"), 1e19
    call = hv.ResidualNorm(rows, dim, torch.float32, grad=True)
    call(x, y, w, p)
    assert not bool(call.x[0].any()) and not bool(call.h[0].any())
    assert call.stats[0].tolist() == pytest.approx([1e3, 1e3], rel=1e-5)
    assert bool(call.h[1].isnan().all()) and bool(call.h[2].isnan().any())
    assert bool(call.h[4:].isfinite().all()) and bool(call.x[4:].isfinite().all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_in_place_through_the_abi(dtype):
    """x_out over x, h_out over y, grad_x over dx and grad_y over dh; nothing past the rows is written."""
    rows, dim = 9, 1003
    code = {torch.float32: hv.FLOAT32, torch.bfloat16: hv.BFLOAT16}[dtype]
    x, y, w, p, gate = operands(rows, dim, dtype, 4, True, rows, torch.float32)
    ref = hv.ResidualNorm(rows, dim, dtype, gate_rows=rows, grad=True)
    ref(x, y, w, p, gate)
    pad = lambda v: torch.cat([v.contiguous().view(-1), torch.full((64,), SENTINEL, dtype=dtype, device="cuda")])  # noqa: E731
    a, b = pad(x), pad(y)
    stats = torch.empty(rows, 2, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    hv.hvdx_residual_norm(a.data_ptr(), dim, b.data_ptr(), dim, code, rows, dim, p.data_ptr(), gate.data_ptr(), hv.FLOAT32, rows,
                          1.0, w.data_ptr(), 1e-6, a.data_ptr(), b.data_ptr(), stats.data_ptr(), s)
    assert torch.equal(a[:-64].view(rows, dim), ref.x) and torch.equal(b[:-64].view(rows, dim), ref.h)
    assert torch.equal(stats, ref.stats) and bool((a[-64:] == SENTINEL).all()) and bool((b[-64:] == SENTINEL).all())
    g = torch.Generator(device="cuda").manual_seed(3)
    dx, dh = strided(rows, dim, dtype, g), strided(rows, dim, dtype, g)
    ref.grad(y, dx, dh, w, p, gate)
    c, d = pad(dx), pad(dh)
    need = hv.hvdx_residual_norm_grad_workspace_bytes(rows, dim, rows)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    gw, gp, gg = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda"), torch.empty(1, dim, device="cuda")
    y = y.contiguous()
    hv.hvdx_residual_norm_grad(a.data_ptr(), dim, y.data_ptr(), dim, c.data_ptr(), dim, d.data_ptr(), dim, code, rows, dim,
                               p.data_ptr(), gate.data_ptr(), hv.FLOAT32, rows, 1.0, w.data_ptr(), stats.data_ptr(), c.data_ptr(),
                               d.data_ptr(), gw.data_ptr(), gp.data_ptr(), gg.data_ptr(), ws.data_ptr(), need, s)
    torch.cuda.synchronize()
    assert torch.equal(c[:-64].view(rows, dim), ref.grad_x) and torch.equal(d[:-64].view(rows, dim), ref.grad_y)
    assert torch.equal(gw, ref.grad_weight) and torch.equal(gp, ref.grad_post) and torch.equal(gg, ref.grad_gate)
    assert bool((c[-64:] == SENTINEL).all()) and bool((d[-64:] == SENTINEL).all())


def test_objects_refuse():
    x, w = torch.zeros(6, 64, device="cuda"), torch.ones(64, device="cuda")
    gate = torch.ones(2, 64, device="cuda")
    call = hv.ResidualNorm(6, 64, torch.float32, gate_rows=3)
    for bad in (x[:5], x.half(), x.cpu(), x[:, :63], x.t().contiguous().t()):
        with pytest.raises(ValueError):
            call(bad, x, w, w, gate)
        with pytest.raises(ValueError):
            call(x, bad, w, w, gate)
    for bad in ((w, None, gate), (w, w, None), (w[:5], w, gate), (w.half(), w, gate), (w, w, gate[:1]), (w, w, gate.half())):
        with pytest.raises(ValueError):
            call(x, x, *bad)
    with pytest.raises(ValueError, match="y must be given"):
        call(x, None, w, w, gate)
    with pytest.raises(ValueError, match="grad=True"):
        call.grad(x, x, x, w, w, gate)
    call = hv.ResidualNorm(6, 64, torch.float32, block=False, grad=True)
    with pytest.raises(ValueError, match="first call"):
        call.grad(None, None, x, w)
    call(x, None, w)
    with pytest.raises(hv.HvdxError, match="dx and dh"):
        call.grad(None, None, None, w)
    with pytest.raises(ValueError, match="gate_dtype"):
        hv.ResidualNorm(6, 64, torch.bfloat16, gate_rows=3, gate_dtype=torch.float16)


def test_offsets_past_32_bits():
    """More than 2^31 elements: the last rows as if they were alone."""
    dim, rows = 16384, (1 << 17) + 40  # 2^31 + 655,360 elements
    x = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(1, dim, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x[-40:] = torch.randn(40, dim, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.ones(dim, device="cuda")
    whole = hv.ResidualNorm(rows, dim, torch.bfloat16, block=False)
    part = hv.ResidualNorm(40, dim, torch.bfloat16, block=False)
    whole(x, None, w)
    part(x[-40:], None, w)
    assert torch.equal(whole.h[-40:], part.h) and torch.equal(whole.stats[-40:], part.stats)
    del y


def test_graph_stream_and_timeline():
    rows, dim = 300, 1024
    x, y, w, p, gate = operands(rows, dim, torch.bfloat16, 5, True, 100, torch.bfloat16)
    call = hv.ResidualNorm(rows, dim, torch.bfloat16, gate_rows=100, gate_dtype=torch.bfloat16, grad=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    dx, dh = strided(rows, dim, torch.bfloat16, g), strided(rows, dim, torch.bfloat16, g)
    names = ("x", "h", "stats", "grad_x", "grad_y", "grad_weight", "grad_post", "grad_gate")

    def step(stream=None):
        call(x, y, w, p, gate, stream=stream)
        call.grad(y, dx, dh, w, p, gate, stream=stream)
        torch.cuda.synchronize()
        return [getattr(call, n).clone() for n in names]
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(x, y, w, p, gate)
        call.grad(y, dx, dh, w, p, gate)
    for seed in range(3):
        x.copy_(strided(rows, dim, torch.bfloat16, torch.Generator(device="cuda").manual_seed(50 + seed)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [getattr(call, n).clone() for n in names]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
    s = torch.cuda.Stream()
    want = step()
    assert all(torch.equal(a, b) for a, b in zip(step(s.cuda_stream), want))
    with hv.Timeline() as tl:
        step()
    kinds = [r["kind"] for r in tl.records]
    assert kinds[0] == hv._lib.KERNEL_RESIDUAL_NORM and set(kinds[1:]) == {hv._lib.KERNEL_RESIDUAL_NORM_GRAD}
