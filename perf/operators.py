"""Performance cases of the language-model operators: log probabilities of given tokens with
entropy and top alternatives (`TokenLogprobs`), distillation from a teacher's top alternatives
(`DistillLoss`) and the residual connection between two blocks with the norms on either side
(`ResidualNorm`), each forward and backward.

A case's values: `op` names the pass; `rows` are token positions; `vocab` or `dim` the row's
length; `dtype` the rows' type; `pad` the elements between one row's end and the next one's start
(logits that are a slice of a padded vocabulary's); `masked` the share of the vocabulary
that constrained decoding has set to minus infinity; `top` the alternatives asked for, or the
teacher's; `rest` whether what the teacher's alternatives leave of its probability counts as one
more outcome; `gate` "none", "channel" (one vector), "group" (a vector for each sequence of
`span` rows) or "full" (a vector for each row).

`own` selects the framework's kernels; otherwise `run` computes the same from elementary torch
operations in 32 bits.
"""
import torch

own = False

_TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_LOWEST = torch.finfo(torch.float32).min


def _lp(name, op, rows, vocab, dtype, top, **kw):
    case = {"name": name, "op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "top": top, "scale": 1.0, "pad": 0,
            "masked": 0.0}
    case.update(kw)
    return case


def _ds(name, op, rows, vocab, dtype, top, **kw):
    case = {"name": name, "op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "top": top, "scale": 1.0, "pad": 0,
            "rest": True}
    case.update(kw)
    return case


def _rn(name, op, rows, dim, dtype, **kw):
    case = {"name": name, "op": op, "rows": rows, "dim": dim, "dtype": dtype, "post": True, "gate": "channel", "span": 1,
            "scale": 1.0}
    case.update(kw)
    return case


def listed():
    return [
        # one sequence's next token with its alternatives: a call that is all latency
        _lp("logprobs_token", "logprobs", 1, 32768, "bf16", 8),
        # a decoding batch over a large vocabulary, some of it masked: few long rows
        _lp("logprobs_batch", "logprobs", 24, 131072, "bf16", 20, masked=0.25, scale=1.25),
        # scoring a text in full precision, an odd vocabulary cut from a padded one
        _lp("logprobs_score", "logprobs", 2048, 50021, "f32", 0, pad=155),
        # the teacher's pass over a training batch: every position's top alternatives
        _lp("logprobs_teacher", "logprobs", 4096, 131072, "bf16", 32, scale=0.5),
        # a policy-gradient step: log probabilities and entropy, then the logits' gradient
        _lp("logprobs_train", "logprobs_train", 4096, 65536, "bf16", 0),
        # an image classifier's 1000 classes, a worker's batch of 64: a small call
        _ds("distill_classes", "distill", 64, 1000, "f32", 5, rest=False),
        # an ordinary step's loss and gradient at once, an odd vocabulary in half precision
        _ds("distill_mid", "distill", 1024, 32003, "f16", 16, scale=0.5),
        # loss first, gradient in a second call, in full precision
        _ds("distill_apart", "distill_apart", 2048, 65537, "f32", 32),
        # the largest step: 4096 positions of a large vocabulary, 64 alternatives
        _ds("distill_large", "distill", 4096, 131072, "bf16", 64),
        # one token through a block's end, when serving
        _rn("norm_token", "norm", 1, 4096, "bf16"),
        # a training batch forward, gated by one vector
        _rn("norm_forward", "norm", 8192, 4096, "bf16", scale=0.7),
        # a backward pass: an odd width in full precision, a gate for each of 16 sequences
        _rn("norm_grad_odd", "norm_grad", 4096, 5001, "f32", gate="group", span=256),
    ]


_MOST_LOGITS = 4096 * 131072
_MOST_NORM = 16384 * 4096


def _log_uniform(rng, low, high):
    return int(round(low * (high / low) ** rng.random()))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "logprobs_train", "distill", "distill", "distill_apart", "norm", "norm_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    rows = _log_uniform(rng, 1, 8192)
    if op in ("norm", "norm_grad"):
        dim = _log_uniform(rng, 64, 16384)
        if rng.random() < 0.6:
            dim = max(64, dim // 64 * 64)
        while rows * dim > _MOST_NORM:
            rows = -(-rows // 2)
        gate = rng.choice(["none", "channel", "channel", "group", "full"])
        span = 1
        if gate == "group":
            span = rng.choice([16, 64, 100, 256])
            rows = max(1, rows // span) * span
            if rows * dim > _MOST_NORM:
                rows -= span
        return {"op": op, "rows": rows, "dim": dim, "dtype": dtype, "post": rng.random() < 0.75, "gate": gate, "span": span,
                "scale": round(rng.uniform(0.1, 1.5), 3)}
    vocab = _log_uniform(rng, 1000, 200000)
    if rng.random() < 0.5:
        vocab = vocab // 64 * 64
    while rows * vocab * (1 if dtype != "f32" else 2) > _MOST_LOGITS:
        rows = -(-rows // 2)
    case = {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "scale": rng.choice([1.0, 0.5, round(rng.uniform(0.3, 2.0), 3)]),
            "pad": rng.choice([0, 0, 7, 64])}
    if op in ("logprobs", "logprobs_train"):
        case["top"] = 0 if op == "logprobs_train" else rng.choice([0, 1, 5, 20, 64])
        case["masked"] = rng.choice([0.0, 0.0, 0.5])
    else:
        case["top"] = rng.choice([1, 4, 10, 32, 64])
        case["rest"] = rng.random() < 0.6
    return case


# --- inputs ---------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)


def _logits(case, g):
    """Logits as a language model's head gives them: a broad bulk, a few high ones in each row."""
    rows, vocab = case["rows"], case["vocab"]
    wide = torch.empty(rows, vocab + case["pad"], dtype=_TORCH[case["dtype"]], device="cuda").normal_(0.0, 2.0, generator=g)
    z = wide[:, :vocab]
    ids = torch.randint(0, vocab, (rows, 16), generator=g, device="cuda")
    high = 6.0 + 4.0 * torch.randn(rows, 16, generator=g, device="cuda")
    z.scatter_(1, ids, high.to(z.dtype))
    return z


def _alternatives(case, g):
    """A teacher's top alternatives: distinct tokens in descending order of log probability, which
    leave part of its mass; some rows have fewer, some (padding positions) none: token -1."""
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    step = torch.randint(1, max(2, vocab // top), (rows, 1), generator=g, device="cuda")
    start = torch.randint(0, vocab, (rows, 1), generator=g, device="cuda")
    slot = torch.arange(top, device="cuda")
    ids = (start + slot * step) % vocab
    score = 2.5 * torch.randn(rows, top + 1, generator=g, device="cuda")
    lp = torch.log_softmax(score, 1)[:, :top].sort(1, descending=True).values.contiguous()
    kept = torch.randint(0, 8 * top, (rows, 1), generator=g, device="cuda")
    return torch.where(slot <= kept, ids, -1).contiguous(), lp


def _loss_scale(case):
    """Half-precision training scales its loss, so that small gradients are not lost."""
    return 2.0 ** 14 if case["dtype"] == "f16" else 1.0


def _gate_rows(case):
    """Rows that share one vector of the gate."""
    return {"channel": case["rows"], "group": case["span"], "full": 1}.get(case["gate"], 0)


def _inputs(case, seed):
    g = _generator(seed)
    op, rows = case["op"], case["rows"]
    state = {"case": case, "op": op}
    if op in ("logprobs", "logprobs_train"):
        z = _logits(case, g)
        if case["masked"]:
            off = torch.rand(1, case["vocab"], generator=g, device="cuda") < case["masked"]
            z.masked_fill_(off, float("-inf"))
        tokens = torch.randint(0, case["vocab"], (rows,), generator=g, device="cuda")
        if case["masked"]:  # the tokens that were taken are among those allowed
            tokens = (tokens + (~off[0]).int().argmax()) % case["vocab"]
            tokens = torch.where(off[0][tokens], (~off[0]).int().argmax(), tokens)
        if rows > 1:
            tokens = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.03, -1, tokens)  # padding positions
        state.update(z=z, tokens=tokens)
        if op == "logprobs_train":
            state["a"] = torch.randn(rows, generator=g, device="cuda") * (_loss_scale(case) / rows)
            state["b"] = torch.full((rows,), 0.01 * _loss_scale(case) / rows, device="cuda")
            state["grad"] = torch.empty(rows, case["vocab"], dtype=z.dtype, device="cuda")
    elif op in ("distill", "distill_apart"):
        state["z"] = z = _logits(case, g)
        ids, lp = _alternatives(case, g)
        # a student that has learnt some of it: its logits at those tokens stand out
        known = (lp / max(case["scale"], 0.25) + 9.0 + 0.5 * torch.randn(lp.shape, generator=g, device="cuda")).to(z.dtype)
        at = ids.clamp(min=0)
        z.scatter_(1, at, torch.where(ids >= 0, known, z.gather(1, at)))
        state.update(ids=ids, lp=lp, g=torch.full((rows,), _loss_scale(case) / rows, device="cuda"))
        state["grad"] = torch.empty(rows, case["vocab"], dtype=z.dtype, device="cuda")
    else:
        dim, dtype = case["dim"], _TORCH[case["dtype"]]
        def new(*shape, mean=0.0, std=1.0, of=dtype):
            return torch.empty(*shape, dtype=of, device="cuda").normal_(mean, std, generator=g)
        state["x"], state["y"] = new(rows, dim, std=1.5), new(rows, dim, std=0.8)
        state["weight"] = new(dim, mean=1.0, std=0.2, of=torch.float32)
        state["post"] = new(dim, mean=1.0, std=0.2, of=torch.float32) if case["post"] else None
        per = _gate_rows(case)  # one vector of the gate is a parameter, in 32 bits; more are activations
        state["gate"] = new(rows // per, dim, mean=0.5, std=0.3, of=torch.float32 if per == rows else dtype) if per else None
        if op == "norm_grad":
            # x is then the stream after the block, as the forward pass stored it, and stats its norms' factors
            state["dx"], state["dh"] = new(rows, dim, std=0.02), new(rows, dim, std=0.02)
            state["stats"] = torch.stack([(t.double().square().mean(1) + 1e-6).rsqrt().float() if t is not None else torch.ones(rows, device="cuda")
                                          for t in (state["y"] if case["post"] else None, state["x"])], 1)
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    if not own:
        return state
    import paper_1802_05799_amd as hv

    op, rows = case["op"], case["rows"]
    if op in ("logprobs", "logprobs_train"):
        state["call"] = hv.TokenLogprobs(rows, case["vocab"], top=case["top"], device="cuda")
    elif op in ("distill", "distill_apart"):
        state["call"] = hv.DistillLoss(rows, case["vocab"], case["top"], rest=case["rest"], device="cuda")
    else:
        gate, back = state["gate"], op == "norm_grad"
        state["call"] = rn = hv.ResidualNorm(rows, case["dim"], _TORCH[case["dtype"]], post=case["post"], gate_rows=_gate_rows(case),
                                             gate_dtype=None if gate is None else gate.dtype, eps=1e-6, grad=back, device="cuda")
        if back:
            rn.x.copy_(state["x"])
            rn.stats.copy_(state["stats"])
    return state


# --- the plain forms ------------------------------------------------------------------------

def _softmax_parts(z, scale):
    """(scaled distance from the row's maximum, its exponential, the sum's logarithm)"""
    z = z.float()
    d = (z - z.amax(1, keepdim=True)) * scale
    e = d.exp()
    return d, e, e.sum(1, keepdim=True).log()


def _plain_logprobs(state, case):
    z, tokens = state["z"], state["tokens"]
    d, e, lse = _softmax_parts(z, case["scale"])
    at = tokens.clamp(min=0)[:, None]
    logprob = torch.where(tokens < 0, 0.0, (d.gather(1, at) - lse)[:, 0])
    inner = (e * d.clamp(min=_LOWEST)).sum(1, keepdim=True) / lse.exp()
    entropy = lse - inner
    out = {"logprob": logprob, "entropy": entropy[:, 0]}
    if case["op"] == "logprobs_train":
        p = (d - lse).exp()
        grad = -state["a"][:, None] * p * (tokens >= 0)[:, None] - state["b"][:, None] * p * ((d - lse).clamp(min=_LOWEST) + entropy)
        grad.scatter_add_(1, at, (state["a"] * (tokens >= 0))[:, None])
        out["grad"] = (grad * case["scale"]).to(z.dtype)
    if case["top"]:
        left, index = z.float().clone(), torch.arange(z.shape[1], device=z.device)
        found = []
        for _ in range(case["top"]):
            high = left.amax(1, keepdim=True)
            found.append(torch.where(left == high, index, z.shape[1]).amin(1))
            left.scatter_(1, found[-1][:, None], float("-inf"))
        out["top_ids"] = torch.stack(found, 1)
        out["top_logprobs"] = d.gather(1, out["top_ids"]) - lse
    return out


def _plain_distill(state, case):
    z, ids, lp, g = state["z"], state["ids"], state["lp"], state["g"]
    d, e, lse = _softmax_parts(z, case["scale"])
    there, at = ids >= 0, ids.clamp(min=0)
    q = torch.where(there, lp.exp(), 0.0)
    if not case["rest"]:
        q = q / q.sum(1, keepdim=True).clamp(min=1e-30)
    total = q.sum(1, keepdim=True)
    log_q = torch.where(q > 0, q, 1.0).log()
    loss = (q * (log_q - torch.where(q > 0, d.gather(1, at) - lse, 0.0))).sum(1)
    dense = torch.zeros_like(d).scatter_add_(1, at, q)
    factor = total
    if case["rest"]:
        left = (1.0 - total).clamp(min=0.0)
        total = total + left
        listed = torch.zeros_like(d).scatter_add_(1, at, there.float()) > 0
        p_left = torch.where(listed, 0.0, e).sum(1, keepdim=True) / lse.exp()
        loss = loss + torch.where(left > 0, left * ((left / p_left).log()), 0.0)[:, 0]
        factor = torch.where(listed, total, total - left / p_left)
    grad = ((d - lse).exp() * factor - dense) * g[:, None] * case["scale"]
    return {"loss": loss, "grad": grad.to(z.dtype)}


def _over_rows(gate, rows):
    return gate.float().repeat_interleave(rows // gate.shape[0], 0)


def _plain_norm(state, case):
    x, y, gate = state["x"].float(), state["y"].float(), state["gate"]
    if case["post"]:
        y = y * (y.square().mean(1, keepdim=True) + 1e-6).rsqrt() * state["post"]
    if gate is not None:
        y = y * _over_rows(gate, x.shape[0])
    x = x + case["scale"] * y
    h = x * (x.square().mean(1, keepdim=True) + 1e-6).rsqrt() * state["weight"]
    return {"x": x.to(state["x"].dtype), "h": h.to(state["x"].dtype)}


def _plain_norm_grad(state, case):
    x, y, dx, dh, gate = state["x"].float(), state["y"].float(), state["dx"].float(), state["dh"].float(), state["gate"]
    dtype, rows = state["x"].dtype, x.shape[0]
    r_y, r_x = state["stats"][:, :1], state["stats"][:, 1:]
    out = {}
    xh, gw = x * r_x, dh * state["weight"]
    out["weight"] = (dh * xh).sum(0)
    dx = dx + r_x * (gw - xh * (gw * xh).mean(1, keepdim=True))
    out["x"] = dx.to(dtype)
    yh = y * r_y if case["post"] else y
    u = yh * state["post"] if case["post"] else yh
    du = case["scale"] * dx
    if gate is not None:
        out["gate"] = (du * u).view(gate.shape[0], rows // gate.shape[0], -1).sum(1).to(gate.dtype)
        du = du * _over_rows(gate, rows)
    if case["post"]:
        out["post"] = (du * yh).sum(0)
        du = du * state["post"]
        du = r_y * (du - yh * (du * yh).mean(1, keepdim=True))
    out["y"] = du.to(dtype)
    return out


_PLAIN = {"logprobs": _plain_logprobs, "logprobs_train": _plain_logprobs, "distill": _plain_distill,
          "distill_apart": _plain_distill, "norm": _plain_norm, "norm_grad": _plain_norm_grad}


# --- one pass -------------------------------------------------------------------------------

def run(state):
    case, op = state["case"], state["op"]
    if not own:
        return _PLAIN[op](state, case)
    call = state["call"]
    if op in ("logprobs", "logprobs_train"):
        call(state["z"], state["tokens"], scale=case["scale"])
        out = {"logprob": call.logprob, "entropy": call.entropy}
        if op == "logprobs_train":
            out["grad"] = call.grad(state["z"], state["tokens"], state["a"], state["b"], out=state["grad"])
        if case["top"]:
            out["top_ids"], out["top_logprobs"] = call.top_ids, call.top_logprobs
        return out
    if op == "distill":
        call(state["z"], state["ids"], state["lp"], scale=case["scale"], grad_loss=state["g"], out=state["grad"])
        return {"loss": call.loss, "grad": state["grad"]}
    if op == "distill_apart":
        call(state["z"], state["ids"], state["lp"], scale=case["scale"])
        return {"loss": call.loss, "grad": call.grad(state["z"], state["ids"], state["lp"], state["g"], out=state["grad"])}
    if op == "norm":
        call(state["x"], state["y"], state["weight"], state["post"], state["gate"], scale=case["scale"])
        return {"x": call.x, "h": call.h}
    call.grad(state["y"], state["dx"], state["dh"], state["weight"], state["post"], state["gate"], scale=case["scale"])
    out = {"weight": call.grad_weight, "x": call.grad_x}
    if state["gate"] is not None:
        out["gate"] = call.grad_gate
    if state["post"] is not None:
        out["post"] = call.grad_post
    out["y"] = call.grad_y
    return out


def work(case):
    """Every input read once, every output written once."""
    size = _TORCH[case["dtype"]].itemsize
    op, rows = case["op"], case["rows"]
    if op in ("logprobs", "logprobs_train"):
        row = case["vocab"] * size * (1 if op == "logprobs" else 2) + 8 + 8 + 12 * case["top"]
        return {"bytes": rows * row, "flops": rows * case["vocab"] * (6 if op == "logprobs" else 12)}
    if op in ("distill", "distill_apart"):
        row = case["vocab"] * size * 2 + 12 * case["top"] + 8
        return {"bytes": rows * row, "flops": rows * case["vocab"] * 8}
    dim = case["dim"]
    per = _gate_rows(case)
    gate = (rows // per * dim * (4 if per == rows else size)) if per else 0
    vectors = 4 * dim * (2 if case["post"] else 1)
    if op == "norm":
        return {"bytes": 4 * rows * dim * size + vectors + gate, "flops": 12 * rows * dim}
    return {"bytes": 6 * rows * dim * size + 8 * rows + 2 * (vectors + gate), "flops": 30 * rows * dim}


# --- the definitions in 64 bits -------------------------------------------------------------

def _exact_logprobs(state, case):
    keep = {k: [] for k in ("logprob", "entropy", "grad", "top_ids", "top_logprobs")}
    rows, vocab = state["z"].shape
    step = max(1, (1 << 25) // vocab)
    for i in range(0, rows, step):
        x = (state["z"][i:i + step].double() * case["scale"]).requires_grad_(case["op"] == "logprobs_train")
        tokens = state["tokens"][i:i + step]
        logp = torch.log_softmax(x, 1)
        mine = logp.gather(1, tokens.clamp(min=0)[:, None])[:, 0] * (tokens >= 0)
        entropy = -(logp.exp() * logp.clamp(min=-1e300)).sum(1)
        if x.requires_grad:
            sl = slice(i, i + step)
            total = (state["a"][sl].double() * mine + state["b"][sl].double() * entropy).sum()
            keep["grad"].append(torch.autograd.grad(total, x)[0] * case["scale"])
        keep["logprob"].append(mine.detach())
        keep["entropy"].append(entropy.detach())
        if case["top"]:
            order = state["z"][i:i + step].float().sort(dim=1, descending=True, stable=True).indices[:, :case["top"]]
            keep["top_ids"].append(order)
            keep["top_logprobs"].append(logp.detach().gather(1, order))
    return {k: torch.cat(v) for k, v in keep.items() if v}


def _exact_distill(state, case):
    losses, grads = [], []
    rows, vocab = state["z"].shape
    step = max(1, (1 << 25) // vocab)
    for i in range(0, rows, step):
        x = (state["z"][i:i + step].double() * case["scale"]).requires_grad_(True)
        ids, t = state["ids"][i:i + step], state["lp"][i:i + step].double()
        there = ids >= 0
        logp = torch.log_softmax(x, 1)
        mine = logp.gather(1, ids.clamp(min=0))
        t = t.masked_fill(~there, float("-inf"))
        if not case["rest"]:
            t = t - torch.logsumexp(t, 1, keepdim=True)
        q = torch.where(there, t.exp(), 0.0)
        loss = torch.where(there, q * (torch.where(there, t, 0.0) - mine), 0.0).sum(1)
        if case["rest"]:
            left = (1.0 - q.sum(1)).clamp(min=0.0)
            hit = torch.zeros(x.shape, dtype=torch.bool, device=x.device)
            r, c = there.nonzero(as_tuple=True)
            hit[r, ids[r, c]] = True
            loss = loss + left * (left.clamp(min=1e-300).log() - torch.logsumexp(logp.masked_fill(hit, float("-inf")), 1))
        grads.append(torch.autograd.grad((loss * state["g"][i:i + step].double()).sum(), x)[0] * case["scale"])
        losses.append(loss.detach())
    return {"loss": torch.cat(losses), "grad": torch.cat(grads)}


def _exact_norm_of(x, y, weight, post, gate, scale):
    def normed(v, w):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w
    if post is not None:
        y = normed(y, post)
    if gate is not None:
        y = (y.view(gate.shape[0], -1, y.shape[1]) * gate[:, None]).view_as(y)
    x = x + scale * y
    return x, normed(x, weight)


def _exact_norm(state, case):
    args = [None if state[k] is None else state[k].double() for k in ("x", "y", "weight", "post", "gate")]
    x, h = _exact_norm_of(*args, case["scale"])
    return {"x": x, "h": h}


def _exact_norm_grad(state, case):
    """The pass that led to the stored stream, backwards: its input is the stream less the block's part."""
    names = ("y", "weight", "post", "gate")
    args = {k: None if state[k] is None else state[k].double() for k in names}
    part, _ = _exact_norm_of(torch.zeros_like(args["y"]), *args.values(), case["scale"])
    x = (state["x"].double() - part).requires_grad_(True)
    for v in args.values():
        if v is not None:
            v.requires_grad_(True)
    new, h = _exact_norm_of(x, *args.values(), case["scale"])
    wanted = {"weight": args["weight"], "x": x}
    if args["gate"] is not None:
        wanted["gate"] = args["gate"]
    if args["post"] is not None:
        wanted["post"] = args["post"]
    wanted["y"] = args["y"]
    got = torch.autograd.grad([new, h], list(wanted.values()), [state["dx"].double(), state["dh"].double()])
    return dict(zip(wanted, got))


def exact(case, seed):
    state = _inputs(case, seed)
    op = case["op"]
    if op in ("logprobs", "logprobs_train"):
        return _exact_logprobs(state, case)
    if op in ("distill", "distill_apart"):
        return _exact_distill(state, case)
    return _exact_norm(state, case) if op == "norm" else _exact_norm_grad(state, case)
