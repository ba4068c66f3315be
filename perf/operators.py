"""Cases of the token-model operators around the block-circulant layers: the embedding lookup and its gradient, the RMS
norm with the residual's addition, the softmax cross entropy, and the clipping of gradients by their global norm.

``run`` computes an operator either in plain float32 torch operations (``own`` false) or through the library (``own``
true), on the same inputs.  ``exact`` gives the results in 64 bits from the definitions.
"""
import math

import torch

own = False

F32, BF16 = torch.float32, torch.bfloat16
DTYPES = {"f32": F32, "bf16": BF16}
SIZES = {"f32": 4, "bf16": 2, "e4m3": 1, "i32": 4, "i64": 8}
E4M3_MAX = 448.0
EPS = 1e-5
CLIP_EPS = 1e-6
PADDING = 0          # the id that fills short sequences up
NO_TARGET = -100     # the target of positions that are not predicted


def listed():
    return [
        # one token of a decoding step: nothing but latency
        dict(name="embed_one_token", op="embed", tokens=1, vocab=32768, dim=4096, table="bf16", out="bf16", ids="i32"),
        # the tokens of a training batch from float32 master weights, into bfloat16 activations
        dict(name="embed_batch", op="embed", tokens=8192, vocab=65536, dim=4096, table="f32", out="bf16", ids="i64"),
        # a small model with odd sizes
        dict(name="embed_grad_odd", op="embed_grad", tokens=513, vocab=10007, dim=1000, out="f32", table="f32", ids="i32"),
        # a training batch: most rows of the table get no token, a few get thousands
        dict(name="embed_grad_batch", op="embed_grad", tokens=32768, vocab=65536, dim=2048, out="bf16", table="f32", ids="i64"),
        # one token of a decoding step
        dict(name="norm_one_token", op="norm", rows=1, dim=4096, x="bf16", y="bf16", group=0, residual=True),
        # a long prompt, activations handed on in 8 bits, one scale for 128 values
        dict(name="norm_e4m3_prompt", op="norm", rows=8192, dim=9216, x="bf16", y="e4m3", group=128, residual=True),
        # training in float32 at an odd width
        dict(name="norm_grad_odd", op="norm_grad", rows=1003, dim=1001, x="f32", y="f32", carry=False),
        # a training batch in bfloat16, with the gradient that flows past the layer
        dict(name="norm_grad_batch", op="norm_grad", rows=16384, dim=4096, x="bf16", y="bf16", carry=True),
        # scoring a few positions over many classes: few long rows
        dict(name="loss_few_rows", op="loss", rows=24, classes=131072, logits="f32", ids="i32", masked=64, grad=False),
        # a training batch; rows of an odd length start at every alignment
        dict(name="loss_grad_batch", op="loss", rows=8192, classes=50001, logits="bf16", ids="i64", masked=0, grad=True),
        # the gradients of circulant layers of several block sizes with their biases: many small tensors, float32, in one buffer
        dict(name="clip_circulant_layers", op="clip", tensors=192, largest=262144, grads="f32", outs="f32", over=3.0),
        # a large model's gradients in bfloat16, clipped into the float32 buffers that the optimizer reads
        dict(name="clip_large_model", op="clip", tensors=24, largest=67108864, grads="bf16", outs="f32", over=20.0),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "loss", "loss", "clip"])
    ids = rng.choice(["i32", "i64"])
    if op in ("embed", "embed_grad"):
        tokens, vocab = _log_uniform(rng, 1, 65536), _log_uniform(rng, 64, 131072)
        most = 1 << 28 if op == "embed" else 1 << 27
        dim = min(_log_uniform(rng, 16, 8192), max(16, most // max(tokens, vocab)))
        dim = dim if rng.random() < 0.3 else -(-dim // 8) * 8
        return dict(op=op, tokens=tokens, vocab=vocab, dim=dim, table=rng.choice(["f32", "bf16"]), out=rng.choice(["f32", "bf16"]), ids=ids)
    if op in ("norm", "norm_grad"):
        rows = _log_uniform(rng, 1, 32768)
        dim = min(_log_uniform(rng, 32, 16384), (1 << 26) // rows)
        x = rng.choice(["f32", "bf16"])
        if op == "norm_grad":
            return dict(op=op, rows=rows, dim=dim, x=x, y=rng.choice(["f32", "bf16"]), carry=rng.random() < 0.5)
        y = rng.choice(["f32", "bf16", "e4m3", "e4m3"])
        group = rng.choice([0, 32, 64, 128]) if y == "e4m3" else 0
        if group:
            dim = max(1, dim // group) * group
        return dict(op=op, rows=rows, dim=dim, x=x, y=y, group=group, residual=rng.random() < 0.7)
    if op == "loss":
        rows = _log_uniform(rng, 1, 16384)
        classes = min(_log_uniform(rng, 16, 200000), (1 << 28) // rows)
        return dict(op=op, rows=rows, classes=classes, logits=rng.choice(["f32", "bf16"]), ids=ids, masked=rng.choice([0, classes // 50]),
                    grad=rng.random() < 0.6)
    return dict(op=op, tensors=_log_uniform(rng, 1, 500), largest=_log_uniform(rng, 100, 1 << 20), grads=rng.choice(["f32", "bf16"]),
                outs=rng.choice(["f32", "bf16"]), over=rng.choice([0.5, 3.0, 100.0]))


def _clip_sizes(case):
    """Elements of each tensor: matrices of the largest size and of fractions of it, biases between them, odd sizes among them."""
    n = case["largest"]
    return ([n, n // 4, n // 64 + 1, n // 4, n, n // 1024 + 3] * -(-case["tensors"] // 6))[:case["tensors"]]


def _chance(case):
    """Probability of every id: log-uniform over ids 1 .. vocab - 1 (few frequent, many rare), the padding id for one token in 16."""
    v = torch.arange(1, case["vocab"], dtype=torch.float64)
    return torch.log1p(1 / v) / math.log(case["vocab"]) * (15 / 16)


def work(case):
    op = case["op"]
    if op in ("embed", "embed_grad"):
        t, d = case["tokens"], case["dim"]
        table, out = SIZES[case["table"]] * d, SIZES[case["out"]] * d
        if op == "embed":
            rows = float((-torch.expm1(t * torch.log1p(-_chance(case)))).sum())   # distinct rows that are read
            return {"bytes": t * SIZES[case["ids"]] + rows * table + t * out, "flops": t * d}
        return {"bytes": t * SIZES[case["ids"]] + t * 15 / 16 * out + case["vocab"] * table, "flops": 2 * t * d}
    if op == "norm":
        n, x = case["rows"] * case["dim"], SIZES[case["x"]]
        groups = 0 if case["y"] != "e4m3" else n // case["group"] if case["group"] else case["rows"]
        return {"bytes": n * ((3 if case["residual"] else 1) * x + SIZES[case["y"]]) + 4 * (groups + case["rows"] + case["dim"]), "flops": 5 * n}
    if op == "norm_grad":
        n, x = case["rows"] * case["dim"], SIZES[case["x"]]
        return {"bytes": n * ((3 if case["carry"] else 2) * x + SIZES[case["y"]]) + 4 * (case["rows"] + 2 * case["dim"]), "flops": 10 * n}
    if op == "loss":
        n, z = case["rows"] * case["classes"], SIZES[case["logits"]]
        return {"bytes": n * z * (2 if case["grad"] else 1) + case["rows"] * (SIZES[case["ids"]] + 8), "flops": (6 if case["grad"] else 3) * n}
    n = sum(_clip_sizes(case))
    return {"bytes": n * (SIZES[case["grads"]] + SIZES[case["outs"]]), "flops": 3 * n}


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, dtype=F32, std=1.0):
        return torch.randn(*shape, device="cuda", dtype=dtype, generator=g).mul_(std)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=g)

    op = case["op"]
    it = torch.int32 if case.get("ids") == "i32" else torch.int64
    if op in ("embed", "embed_grad"):
        t, v, d = case["tokens"], case["vocab"], case["dim"]
        ids = torch.exp(uniform(t).double() * math.log(v)).long().clamp_(1, v - 1)
        ids = torch.where(uniform(t) < 1 / 16, PADDING, ids).to(it)
        s = {"ids": ids, "scale": math.sqrt(d)}
        if op == "embed":
            s["table"] = normal(v, d, dtype=DTYPES[case["table"]], std=0.02)
        else:
            s["grad"] = normal(t, d, dtype=DTYPES[case["out"]], std=1e-2)
        return s
    if op in ("norm", "norm_grad"):
        r, d, x = case["rows"], case["dim"], DTYPES[case["x"]]
        s = {"gain": 1 + normal(d, std=0.1)}
        if op == "norm":
            s["x"] = normal(r, d, dtype=x)
            s["residual"] = normal(r, d, dtype=x, std=2.0) if case["residual"] else None
        else:
            s["sum"] = normal(r, d, dtype=x, std=2.0)
            s["rstd"] = torch.rsqrt(s["sum"].float().square().mean(1) + EPS)
            s["grad"] = normal(r, d, dtype=DTYPES[case["y"]], std=1e-2)
            s["carry"] = normal(r, d, dtype=x, std=1e-2) if case["carry"] else None
        return s
    if op == "loss":
        r, c = case["rows"], case["classes"]
        logits = normal(r, c, dtype=DTYPES[case["logits"]], std=2.5)
        targets = (uniform(r) * (c - case["masked"])).long().clamp_(max=c - case["masked"] - 1)
        logits[torch.arange(r, device="cuda"), targets] += 6 * uniform(r).to(logits.dtype)    # a model that has learnt something
        if case["masked"]:
            logits[:, c - case["masked"]:] = -math.inf                                         # classes that fill the matrix up
        targets = torch.where(uniform(r) < 1 / 10, NO_TARGET, targets)
        return {"logits": logits, "targets": targets.to(it)}
    sizes = _clip_sizes(case)
    n = sum(sizes)
    return {"flat": normal(n, dtype=DTYPES[case["grads"]], std=1e-3), "sizes": sizes, "max_norm": math.sqrt(n) * 1e-3 / case["over"]}


class _Handle:
    """A library handle that is destroyed with the state that holds it."""

    def __init__(self, value, destroy):
        self.value, self.destroy = value, destroy

    def __del__(self):
        self.destroy(self.value)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "clip":      # the gradients and their clipped copies are views of two buffers that such a program keeps
        s["out"] = torch.empty(s["flat"].numel(), device="cuda", dtype=DTYPES[case["outs"]])
    if own:                       # the handle and the output buffers that a user of the library keeps
        _prepare_own(s, case)
    return s


def _prepare_own(s, case):
    import paper_1708_08917_b200 as circ
    op = case["op"]
    code = {"f32": circ.CIRC_F32, "bf16": circ.CIRC_BF16, "e4m3": circ.CIRC_E4M3, "i32": circ.CIRC_I32, "i64": circ.CIRC_I64}
    s["circ"], s["stream"] = circ, torch.cuda.current_stream()
    if op in ("embed", "embed_grad"):
        h = circ.circ_embed_create(case["vocab"], case["dim"])
        s["handle"] = _Handle(h, circ.circ_embed_destroy)
        circ.circ_embed_set_dtypes(h, code[case["table"]], code[case["out"]], code[case["ids"]])
        circ.circ_embed_set_scale(h, s["scale"])
        circ.circ_embed_set_padding(h, PADDING)
        if op == "embed":
            s["y"] = torch.empty(case["tokens"], case["dim"], device="cuda", dtype=DTYPES[case["out"]])
        else:
            circ.circ_embed_reserve(h, case["tokens"])
            s["grad_table"] = torch.empty(case["vocab"], case["dim"], device="cuda", dtype=DTYPES[case["table"]])
    elif op in ("norm", "norm_grad"):
        h = circ.circ_norm_create(case["dim"], EPS)
        s["handle"] = _Handle(h, circ.circ_norm_destroy)
        circ.circ_norm_set_dtypes(h, code[case["x"]], code[case["y"]])
        if op == "norm":
            n, d = case["rows"], case["dim"]
            group = case["group"] or d
            s["y"] = torch.empty(n, d, device="cuda", dtype=torch.float8_e4m3fn if case["y"] == "e4m3" else DTYPES[case["y"]])
            s["y_scale"] = None
            if case["y"] == "e4m3":
                circ.circ_norm_set_group(h, case["group"])
                s["y_scale"] = torch.empty(n, d // group, device="cuda")
            s["sum"] = torch.empty_like(s["x"]) if case["residual"] else None
            s["rstd"] = torch.empty(n, device="cuda")
        else:
            circ.circ_norm_reserve(h)
            s["grad_x"], s["grad_gain"] = torch.empty_like(s["sum"]), torch.empty_like(s["gain"])
    elif op == "loss":
        h = circ.circ_loss_create(case["classes"])
        s["handle"] = _Handle(h, circ.circ_loss_destroy)
        circ.circ_loss_set_dtypes(h, code[case["logits"]], code[case["ids"]])
        circ.circ_loss_set_ignore(h, NO_TARGET)
        s["row_loss"], s["lse"] = torch.empty(case["rows"], device="cuda"), torch.empty(case["rows"], device="cuda")
        s["mean"] = torch.empty(1, device="cuda")
        if case["grad"]:
            s["grad"] = torch.empty_like(s["logits"])
    else:
        h = circ.circ_clip_create(s["sizes"], code[case["grads"]], code[case["outs"]])
        s["handle"] = _Handle(h, circ.circ_clip_destroy)
        circ.circ_clip_set_tensors(h, s["flat"].split(s["sizes"]), s["out"].split(s["sizes"]), s["stream"])
        s["norm"] = torch.empty(1, device="cuda")


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    circ, case, h, stream = s["circ"], s["case"], s["handle"].value, s["stream"]
    op = case["op"]
    if op == "embed":
        circ.circ_embed_forward(h, s["table"], s["ids"], s["y"], case["tokens"], stream)
        return s["y"]
    if op == "embed_grad":
        circ.circ_embed_backward(h, s["ids"], s["grad"], s["grad_table"], case["tokens"], stream)
        return s["grad_table"]
    if op == "norm":
        circ.circ_norm_forward(h, s["x"], s["residual"], s["gain"], s["sum"], s["y"], s["y_scale"], s["rstd"], case["rows"], stream)
        return {k: s[k] for k in ("sum", "y", "y_scale", "rstd") if s[k] is not None}
    if op == "norm_grad":
        circ.circ_norm_backward(h, s["sum"], s["gain"], s["rstd"], s["grad"], s["carry"], s["grad_x"], s["grad_gain"], case["rows"], stream)
        return {"grad_x": s["grad_x"], "grad_gain": s["grad_gain"]}
    if op == "loss":
        c = case["classes"]
        if case["grad"]:
            circ.circ_loss_backward(h, s["logits"], c, s["targets"], s["row_loss"], s["lse"], s["mean"], s["grad"], c, 1.0, case["rows"], stream)
            return {k: s[k] for k in ("row_loss", "lse", "mean", "grad")}
        circ.circ_loss_forward(h, s["logits"], c, s["targets"], s["row_loss"], s["lse"], s["mean"], case["rows"], stream)
        return {k: s[k] for k in ("row_loss", "lse", "mean")}
    circ.circ_clip_forward(h, s["max_norm"], s["norm"], stream)
    return {"norm": s["norm"], "out": s["out"]}


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "embed":
        y = s["table"][s["ids"].long()].float() * s["scale"]
        return torch.where((s["ids"] != PADDING)[:, None], y, 0.0).to(DTYPES[case["out"]])
    if op == "embed_grad":
        grad = torch.where((s["ids"] != PADDING)[:, None], s["grad"].float() * s["scale"], 0.0)
        table = torch.zeros(case["vocab"], case["dim"], device="cuda")
        return table.index_add_(0, s["ids"].long(), grad).to(DTYPES[case["table"]])
    if op == "norm":
        total = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
        rstd = torch.rsqrt((total * total).mean(1) + EPS)
        y = total * rstd[:, None] * s["gain"]
        out = {"rstd": rstd}
        if s["residual"] is not None:
            out["sum"] = total.to(DTYPES[case["x"]])
        if case["y"] == "e4m3":
            y = y.view(case["rows"], -1, case["group"] or case["dim"])
            top = y.abs().amax(2)
            scale = torch.where(top > 0, top / E4M3_MAX, 1.0)
            out["y"] = (y / scale[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(case["rows"], case["dim"])
            out["y_scale"] = scale
        else:
            out["y"] = y.to(DTYPES[case["y"]])
        return out
    if op == "norm_grad":
        total, grad, rstd = s["sum"].float(), s["grad"].float(), s["rstd"][:, None]
        u = grad * s["gain"]
        dx = rstd * u - total * (rstd * rstd * rstd * (u * total).mean(1, keepdim=True))
        if s["carry"] is not None:
            dx = dx + s["carry"].float()
        return {"grad_x": dx.to(DTYPES[case["x"]]), "grad_gain": (grad * total * rstd).sum(0)}
    if op == "loss":
        z, rows = s["logits"].float(), torch.arange(case["rows"], device="cuda")
        valid = s["targets"] != NO_TARGET
        target = torch.where(valid, s["targets"], 0).long()
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(1, keepdim=True)
        lse = (torch.log(total) + top).squeeze(1)
        row = torch.where(valid, lse - z[rows, target], 0.0)
        count = valid.sum().clamp(min=1)
        out = {"row_loss": row, "lse": lse, "mean": (row.sum() / count).view(1)}
        if case["grad"]:
            grad = e / total
            grad[rows, target] -= 1.0
            out["grad"] = (grad * (valid / count)[:, None]).to(DTYPES[case["logits"]])
        return out
    norm = torch.sqrt(s["flat"].float().square().sum())
    factor = torch.clamp(s["max_norm"] / (norm + CLIP_EPS), max=1.0)
    s["out"].copy_(s["flat"].float() * factor)
    return {"norm": norm.view(1), "out": s["out"]}


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("embed", "embed_grad"):
        keep = s["ids"].long().ne(PADDING).nonzero().squeeze(1)
        if op == "embed":
            y = torch.zeros(case["tokens"], case["dim"], device="cuda", dtype=torch.float64)
            y[keep] = s["scale"] * s["table"].index_select(0, s["ids"].long()[keep]).double()
            return y
        ids, order = torch.sort(s["ids"].long()[keep], stable=True)         # sums of runs as differences of a running sum, in slices
        ends = torch.searchsorted(ids, torch.arange(case["vocab"], device="cuda"), right=True)
        out = torch.empty(case["vocab"], case["dim"], device="cuda", dtype=torch.float64)
        for c in range(0, case["dim"], 512):
            run_sum = torch.nn.functional.pad(s["grad"][:, c:c + 512].double()[keep][order].cumsum(0), (0, 0, 1, 0))[ends]
            out[:, c:c + 512] = s["scale"] * torch.diff(run_sum, dim=0, prepend=torch.zeros_like(run_sum[:1]))
        return out
    if op == "norm":
        total = s["x"].double()
        if s["residual"] is not None:
            total += s["residual"].double()
        rstd = 1 / torch.sqrt(torch.linalg.vector_norm(total, dim=1) ** 2 / case["dim"] + EPS)
        out = {"rstd": rstd}
        if s["residual"] is not None:
            out["sum"] = total
        y = torch.einsum("rd,r,d->rd", total, rstd, s["gain"].double())
        if case["y"] == "e4m3":
            blocks = y.reshape(case["rows"], -1, case["group"] or case["dim"])
            scale = torch.linalg.vector_norm(blocks, ord=math.inf, dim=2) / E4M3_MAX
            scale[scale == 0] = 1
            out["y_scale"] = scale
            y = (blocks / scale.unsqueeze(2)).reshape(case["rows"], case["dim"])
        out["y"] = y
        return out
    if op == "norm_grad":
        total, grad = s["sum"].double(), s["grad"].double()
        rstd = s["rstd"].double()
        unit = total * rstd[:, None]                                       # y = unit g, d unit = (1 - unit unit^T / n) rstd
        w = grad * s["gain"].double()
        dx = (w - unit * ((w * unit).sum(1) / case["dim"])[:, None]) * rstd[:, None]
        if s["carry"] is not None:
            dx += s["carry"].double()
        return {"grad_x": dx, "grad_gain": torch.einsum("rd,rd->d", grad, unit)}
    if op == "loss":
        valid = s["targets"].long() >= 0
        count = max(1, int(valid.sum()))
        lse = torch.empty(case["rows"], device="cuda", dtype=torch.float64)
        row = torch.zeros_like(lse)
        grad = torch.empty(case["rows"], case["classes"], device="cuda", dtype=torch.float64) if case["grad"] else None
        for r in range(0, case["rows"], 512):
            z, t, ok = s["logits"][r:r + 512].double(), s["targets"][r:r + 512].long(), valid[r:r + 512]
            lse[r:r + 512] = torch.logsumexp(z, 1)
            hot = torch.zeros_like(z)
            hot[ok.nonzero().squeeze(1), t[ok]] = 1
            row[r:r + 512][ok] = lse[r:r + 512][ok] - z[ok].gather(1, t[ok][:, None]).squeeze(1)
            if grad is not None:
                grad[r:r + 512] = (torch.softmax(z, 1) - hot) * (ok.double() / count)[:, None]
        out = {"row_loss": row, "lse": lse, "mean": row.sum().view(1) / count}
        if grad is not None:
            out["grad"] = grad
        return out
    total = torch.zeros((), device="cuda", dtype=torch.float64)
    for part in s["flat"].split(1 << 26):
        total += torch.dot(part.double(), part.double())
    norm = float(total.sqrt())
    out = s["flat"].double()
    return {"norm": torch.tensor([norm], dtype=torch.float64), "out": out.mul_(min(1.0, s["max_norm"] / (norm + CLIP_EPS)))}
