"""Cases of the operators that train a compressed network in the place of an uncompressed one: the selection of a teacher's top logits,
the distillation loss against them with its gradient, and the group norm with an activation behind channel-last convolutions.

``run`` computes an operator either in plain torch operations (``own`` false) or through the library (``own`` true), on the same
inputs.  ``exact`` gives the results in 64 bits from the definitions.
"""
import math

import torch

own = False

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
DTYPES = {"f32": F32, "bf16": BF16}
SIZES = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
EPS = 1e-5
NO_CLASS = -1        # the id of an entry that a short list does not have
SKIPPED = 1 / 10     # share of the rows that carry no weight (positions that are not predicted)


def listed():
    return [
        # the teacher's answer for one position of a long vocabulary: nothing but latency
        dict(name="top_one_row", op="top", rows=1, classes=131072, count=8, logits="bf16", ids="i32", tau=1.0, masked=0),
        # a teacher's batch, stored as lists of 64; rows of an odd length start at every alignment
        dict(name="top_batch", op="top", rows=8192, classes=50001, count=64, logits="bf16", ids="i32", tau=2.0, masked=0),
        # scoring a few positions against the teacher over many classes: few long rows
        dict(name="distill_few_rows", op="distill", rows=24, classes=131072, count=64, logits="f32", values="f32", ids="i32", tau=1.0,
             rest=True, weights=False, grad=False),
        # the validation loss of a batch
        dict(name="distill_batch", op="distill", rows=4096, classes=50001, count=50, logits="bf16", values="bf16", ids="i64", tau=2.0,
             rest=False, weights=True, grad=False),
        # a stack of circulant layers that ends in 1024 classes, trained against the dense stack's five best
        dict(name="distill_grad_stack", op="distill", rows=128, classes=1024, count=5, logits="f32", values="f32", ids="i64", tau=4.0,
             rest=False, weights=False, grad=True),
        # odd sizes, the classes outside the list counted as one class more
        dict(name="distill_grad_odd", op="distill", rows=513, classes=10007, count=20, logits="f32", values="f32", ids="i32", tau=2.0,
             rest=True, weights=True, grad=True),
        # a training batch
        dict(name="distill_grad_batch", op="distill", rows=8192, classes=50001, count=64, logits="bf16", values="bf16", ids="i32", tau=1.0,
             rest=True, weights=True, grad=True),
        # one image behind a convolution of 256 channels: nothing but latency
        dict(name="gnorm_one_image", op="gnorm", images=1, height=28, width=28, channels=256, groups=32, x="bf16", y="bf16", act="relu"),
        # odd images of few channels, float32
        dict(name="gnorm_odd", op="gnorm", images=5, height=37, width=41, channels=60, groups=12, x="f32", y="f32", act="silu"),
        # a batch of large images at an early layer
        dict(name="gnorm_large", op="gnorm", images=32, height=112, width=112, channels=256, groups=32, x="bf16", y="bf16", act="silu"),
        # the training batch of a 256-channel convolution on 28 x 28 pixels
        dict(name="gnorm_grad_batch", op="gnorm_grad", images=32, height=28, width=28, channels=256, groups=32, x="bf16", y="bf16", act="relu"),
        # a batch of larger images
        dict(name="gnorm_grad_large", op="gnorm_grad", images=64, height=56, width=56, channels=256, groups=32, x="bf16", y="bf16", act="silu"),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["top", "distill", "distill", "gnorm", "gnorm_grad"])
    if op in ("top", "distill"):
        rows = _log_uniform(rng, 1, 16384)
        classes = min(_log_uniform(rng, 16, 200000), (1 << 28) // rows)
        case = dict(op=op, rows=rows, classes=classes, count=_log_uniform(rng, 1, min(256, classes // 2)), logits=rng.choice(["f32", "bf16"]),
                    ids=rng.choice(["i32", "i64"]), tau=rng.choice([1.0, 2.0, 4.0]))
        if op == "top":
            return dict(case, masked=rng.choice([0, classes // 50]))
        return dict(case, values=rng.choice(["f32", "bf16"]), rest=rng.random() < 0.5, weights=rng.random() < 0.5, grad=rng.random() < 0.6)
    groups = rng.choice([1, 2, 4, 8, 16, 32])
    channels = groups * _log_uniform(rng, 1, max(2, 512 // groups))
    height, width = _log_uniform(rng, 1, 160), _log_uniform(rng, 1, 160)
    most = 1 << 26 if op == "gnorm" else 1 << 25
    images = max(1, min(_log_uniform(rng, 1, 128), most // (height * width * channels)))
    return dict(op=op, images=images, height=height, width=width, channels=channels, groups=groups, x=rng.choice(["f32", "bf16"]),
                y=rng.choice(["f32", "bf16"]), act=rng.choice(["none", "relu", "silu"]))


def work(case):
    op = case["op"]
    if op in ("top", "distill"):
        r, n, z = case["rows"], case["rows"] * case["classes"], SIZES[case["logits"]]
        if op == "top":
            return {"bytes": n * z + r * (case["count"] * (z + SIZES[case["ids"]]) + 4), "flops": 3 * n}
        live = 1 - SKIPPED if case["weights"] else 1       # the others are not read
        lists = live * r * case["count"] * (SIZES[case["values"]] + SIZES[case["ids"]])
        single = r * (8 + (4 if case["rest"] else 0) + (4 if case["weights"] else 0))
        return {"bytes": n * z * (live + (1 if case["grad"] else 0)) + lists + single, "flops": (6 if case["grad"] else 3) * live * n}
    n, c, g = case["images"] * case["height"] * case["width"] * case["channels"], case["channels"], case["images"] * case["groups"]
    if op == "gnorm":
        return {"bytes": n * (SIZES[case["x"]] + SIZES[case["y"]]) + 8 * (g + c), "flops": (6 if case["act"] == "none" else 8) * n}
    return {"bytes": n * (2 * SIZES[case["x"]] + SIZES[case["y"]]) + 8 * g + 16 * c, "flops": (12 if case["act"] == "none" else 18) * n}


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, dtype=F32, std=1.0):
        return torch.randn(*shape, device="cuda", dtype=dtype, generator=g).mul_(std)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=g)

    op = case["op"]
    it = torch.int32 if case.get("ids") == "i32" else torch.int64
    if op in ("top", "distill"):
        r, c, k = case["rows"], case["classes"], case["count"]
        z = normal(r, c, dtype=DTYPES[case["logits"]], std=2.5)
        if op == "top":
            if case["masked"]:
                z[:, c - case["masked"]:] = -math.inf            # classes that fill the matrix up
            return {"logits": z}
        # a list's classes: one of each of `count` equal parts of the classes, in random order; the values descend
        part = torch.argsort(uniform(r, k), 1)
        low, high = part * c // k, (part + 1) * c // k
        ids = low + (uniform(r, k).double() * (high - low)).long()
        values = (8 + normal(r, k, std=2.0)).sort(1, descending=True).values.to(DTYPES[case["values"]])
        z.scatter_(1, ids, (values.float() + normal(r, k)).to(z.dtype))                     # a student that has learnt something
        ids = torch.where(uniform(r, k) < 1 / 50, NO_CLASS, ids)
        s = {"logits": z, "values": values, "ids": ids.to(it), "lse": None, "weights": None}
        if case["rest"]:     # between 1 and 30 percent of the teacher's probability lie outside the list
            share = 0.01 + 0.29 * uniform(r)
            listed_values = torch.where(ids >= 0, values.float() / case["tau"], -math.inf)
            s["lse"] = torch.where((ids >= 0).any(1), torch.logsumexp(listed_values, 1) - torch.log1p(-share), 8.0)
        if case["weights"]:
            s["weights"] = torch.where(uniform(r) < SKIPPED, 0.0, 0.5 + uniform(r))
        return s
    n, h, w, c = case["images"], case["height"], case["width"], case["channels"]
    offset = normal(c)
    x = (normal(n, h, w, c, std=1.5) + offset).to(DTYPES[case["x"]])
    s = {"x": x, "gain": 1 + normal(c, std=0.1), "bias": normal(c, std=0.1)}
    if op == "gnorm_grad":
        groups = [p.float().view(p.shape[0], h * w, case["groups"], -1) for p in x.split(max(1, (1 << 26) // (h * w * c)))]
        s["mean"] = torch.cat([p.mean((1, 3)) for p in groups])
        s["rstd"] = torch.cat([torch.rsqrt(p.var((1, 3), unbiased=False) + EPS) for p in groups])
        s["grad"] = normal(n, h, w, c, dtype=DTYPES[case["y"]], std=1e-2)
    return s


class _Handle:
    """A library handle that is destroyed with the state that holds it."""

    def __init__(self, value, destroy):
        self.value, self.destroy = value, destroy

    def __del__(self):
        self.destroy(self.value)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:                       # the handle and the output buffers that a user of the library keeps
        _prepare_own(s, case)
    return s


def _prepare_own(s, case):
    import paper_1708_08917_b200 as circ
    op = case["op"]
    code = {"f32": circ.CIRC_F32, "bf16": circ.CIRC_BF16, "i32": circ.CIRC_I32, "i64": circ.CIRC_I64}
    s["circ"], s["stream"] = circ, torch.cuda.current_stream()
    if op == "top":
        r, k = case["rows"], case["count"]
        h = circ.circ_top_create(case["classes"], k)
        s["handle"] = _Handle(h, circ.circ_top_destroy)
        circ.circ_top_set_dtypes(h, code[case["logits"]], code[case["ids"]])
        circ.circ_top_set_temperature(h, case["tau"])
        s["values"] = torch.empty(r, k, device="cuda", dtype=DTYPES[case["logits"]])
        s["ids"] = torch.empty(r, k, device="cuda", dtype=torch.int32 if case["ids"] == "i32" else torch.int64)
        s["lse"] = torch.empty(r, device="cuda")
    elif op == "distill":
        h = circ.circ_distill_create(case["classes"], case["count"])
        s["handle"] = _Handle(h, circ.circ_distill_destroy)
        circ.circ_distill_set_dtypes(h, code[case["logits"]], code[case["values"]], code[case["ids"]])
        circ.circ_distill_set_temperature(h, case["tau"])
        circ.circ_distill_set_rest(h, case["rest"])
        circ.circ_distill_reserve(h, case["rows"])
        s["row_loss"], s["student_lse"] = torch.empty(case["rows"], device="cuda"), torch.empty(case["rows"], device="cuda")
        s["mean"] = torch.empty(1, device="cuda")
        if case["grad"]:
            s["grad"] = torch.empty_like(s["logits"])
    else:
        h = circ.circ_gnorm_create(case["channels"], case["groups"], EPS)
        s["handle"] = _Handle(h, circ.circ_gnorm_destroy)
        circ.circ_gnorm_set_dtypes(h, code[case["x"]], code[case["y"]])
        circ.circ_gnorm_set_activation(h, {"none": circ.CIRC_ACT_NONE, "relu": circ.CIRC_ACT_RELU, "silu": circ.CIRC_ACT_SILU}[case["act"]])
        circ.circ_gnorm_reserve(h, case["images"], case["height"], case["width"])
        if op == "gnorm":
            s["y"] = torch.empty(s["x"].shape, device="cuda", dtype=DTYPES[case["y"]])
            s["mean"], s["rstd"] = (torch.empty(case["images"], case["groups"], device="cuda") for _ in range(2))
        else:
            s["grad_x"] = torch.empty_like(s["x"])
            s["grad_gain"], s["grad_bias"] = torch.empty_like(s["gain"]), torch.empty_like(s["bias"])


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    circ, case, h, stream = s["circ"], s["case"], s["handle"].value, s["stream"]
    op = case["op"]
    if op == "top":
        circ.circ_top_forward(h, s["logits"], case["classes"], s["values"], s["ids"], s["lse"], case["rows"], stream)
        return {k: s[k] for k in ("values", "ids", "lse")}
    if op == "distill":
        c, lists = case["classes"], (s["values"], s["ids"], s["lse"], s["weights"])
        if case["grad"]:
            circ.circ_distill_backward(h, s["logits"], c, *lists, s["row_loss"], s["student_lse"], s["mean"], s["grad"], c, case["tau"] ** 2,
                                       case["rows"], stream)
            return {k: s[k] for k in ("row_loss", "student_lse", "mean", "grad")}
        circ.circ_distill_forward(h, s["logits"], c, *lists, s["row_loss"], s["student_lse"], s["mean"], case["rows"], stream)
        return {k: s[k] for k in ("row_loss", "student_lse", "mean")}
    sizes = case["images"], case["height"], case["width"]
    if op == "gnorm":
        circ.circ_gnorm_forward(h, s["x"], s["gain"], s["bias"], s["y"], s["mean"], s["rstd"], *sizes, stream)
        return {k: s[k] for k in ("y", "mean", "rstd")}
    circ.circ_gnorm_backward(h, s["x"], s["gain"], s["bias"], s["mean"], s["rstd"], s["grad"], s["grad_x"], s["grad_gain"], s["grad_bias"],
                             *sizes, stream)
    return {k: s[k] for k in ("grad_x", "grad_gain", "grad_bias")}


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "top":
        z, k = s["logits"], case["count"]
        values, ids = torch.empty(len(z), k, device="cuda", dtype=z.dtype), torch.empty(len(z), k, device="cuda", dtype=torch.int64)
        lse = torch.empty(len(z), device="cuda")
        behind = torch.arange(case["classes"] - 1, -1, -1, device="cuda")           # the lower of two equal classes has the larger one
        for r in range(0, len(z), 1024):
            f = z[r:r + 1024].float()
            bits = (f + 0.0).view(torch.int32).long()
            order = torch.where(bits < 0, -1 - (bits & 0x7fffffff), bits)             # whole numbers in the order of the values
            ids[r:r + 1024] = case["classes"] - 1 - torch.topk((order << 32) + behind, k, 1).values.remainder(1 << 32)
            values[r:r + 1024] = z[r:r + 1024].gather(1, ids[r:r + 1024])
            f = f * (1 / case["tau"])
            top = f.amax(1, keepdim=True)
            lse[r:r + 1024] = (torch.log(torch.exp(f - top).sum(1, keepdim=True)) + top).squeeze(1)
        return {"values": values, "ids": ids.to(torch.int32 if case["ids"] == "i32" else torch.int64), "lse": lse}
    if op == "distill":
        z, tau, valid = s["logits"].float() * (1 / case["tau"]), case["tau"], s["ids"] >= 0
        ids = torch.where(valid, s["ids"], 0).long()
        w = torch.ones(len(z), device="cuda", dtype=F64) if s["weights"] is None else s["weights"].double()
        t = torch.where(valid, s["values"].double() / tau, -math.inf)                 # the lists in 64 bits: what they leave over is small
        has = valid.any(1)
        lse_t = torch.logsumexp(t, 1) if s["lse"] is None else s["lse"].double()
        p = torch.where(has[:, None], torch.exp(t - lse_t[:, None]), 0.0)
        p_rest = torch.zeros_like(w) if s["lse"] is None else (1 - p.sum(1)).clamp(min=0)
        student = torch.where(valid, z.gather(1, ids), -math.inf).double()
        rows, entries = valid.nonzero(as_tuple=True)
        rest = z
        rest[rows, ids[rows, entries]] = -math.inf
        top = rest.amax(1, keepdim=True)
        e = torch.exp(rest - top)
        a = torch.log(e.sum(1).double()) + top.squeeze(1).double()
        lse = torch.logaddexp(a, torch.logsumexp(student, 1))
        loss = torch.where(p > 0, p * (torch.log(p) - student + lse[:, None]), 0.0).sum(1)
        loss += torch.where(p_rest > 0, p_rest * (torch.log(p_rest) - a + lse), 0.0)
        total = w.sum().clamp(min=1e-300)
        live = w > 0
        out = {"row_loss": torch.where(live, loss, 0.0).float(), "student_lse": torch.where(live, lse, 0.0).float(),
               "mean": ((torch.where(live, loss, 0.0) * w).sum() / total).float().view(1)}
        if case["grad"]:
            scale = torch.where(has, w * (tau / total), 0.0)                          # tau^2 mean, and 1 / tau from z / tau
            all_p = p.sum(1) + p_rest
            grad = e * (scale * (all_p * torch.exp(a - lse) - p_rest) / e.sum(1)).float()[:, None]
            listed_grad = (scale[:, None] * (all_p[:, None] * torch.exp(student - lse[:, None]) - p)).float()
            grad[rows, ids[rows, entries]] = listed_grad[rows, entries]
            out["grad"] = grad.to(DTYPES[case["logits"]])
        return out
    n, hw, c, g = case["images"], case["height"] * case["width"], case["channels"], case["groups"]
    x = s["x"].float().view(n, hw, g, c // g)
    gain, bias = s["gain"].view(g, -1), s["bias"].view(g, -1)
    if op == "gnorm":
        mean = x.mean((1, 3))
        x = x - mean[:, None, :, None]
        rstd = torch.rsqrt((x * x).mean((1, 3)) + EPS)
        v = x * rstd[:, None, :, None] * gain + bias
        if case["act"] == "relu":
            v = torch.where(v > 0, v, 0.0)
        elif case["act"] == "silu":
            v = v / (1 + torch.exp(-v))
        return {"y": v.to(DTYPES[case["y"]]).view(s["x"].shape), "mean": mean, "rstd": rstd}
    grad = s["grad"].float().view(x.shape)
    rstd = s["rstd"][:, None, :, None]
    if case["act"] == "relu":                   # which side of 0 a value lies on: in 64 bits
        v = (x.double() - s["mean"].double()[:, None, :, None]) * (s["rstd"].double()[:, None, :, None] * gain.double()) + bias.double()
        grad = torch.where(v > 0, grad, 0.0)
        del v
    x = (x - s["mean"][:, None, :, None]) * rstd
    if case["act"] == "silu":
        v = x * gain + bias
        sig = 1 / (1 + torch.exp(-v))
        grad = grad * (sig * (1 + v * (1 - sig)))
        del v, sig
    grad_gain, grad_bias = (grad * x).sum((0, 1)).view(c), grad.sum((0, 1)).view(c)
    grad = grad * gain
    a, b = grad.mean((1, 3), keepdim=True), (grad * x).mean((1, 3), keepdim=True)
    grad = rstd * (grad - a - x * b)
    return {"grad_x": grad.to(DTYPES[case["x"]]).view(s["x"].shape), "grad_gain": grad_gain, "grad_bias": grad_bias}


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "top":
        out = {"values": [], "ids": [], "lse": []}
        for z in s["logits"].split(max(1, (1 << 25) // case["classes"])):
            v, i = torch.sort(z.double(), dim=1, descending=True, stable=True)
            out["values"].append(v[:, :case["count"]].clone())
            out["ids"].append(i[:, :case["count"]].clone())
            out["lse"].append(torch.logsumexp(v / case["tau"], 1))
        return {k: torch.cat(v) for k, v in out.items()}
    if op == "distill":
        return _exact_distill(case, s)
    groups, c, parts = case["groups"], case["channels"], []
    gain, bias = s["gain"].double(), s["bias"].double()
    sums = [torch.zeros(c, device="cuda", dtype=F64) for _ in range(2)]
    for i in range(case["images"]):
        x = s["x"][i].double().reshape(-1, groups, c // groups)
        if op == "gnorm":
            flat = x.permute(1, 0, 2).reshape(groups, -1)
            mean = flat.sum(1) / flat.shape[1]
            deviation = torch.linalg.vector_norm(flat - mean[:, None], dim=1) / math.sqrt(flat.shape[1])
            rstd = 1 / torch.sqrt(deviation ** 2 + EPS)
        else:
            mean, rstd = s["mean"][i].double(), s["rstd"][i].double()
        unit = torch.einsum("pgd,g->pgd", x - mean[None, :, None], rstd).reshape(-1, c)
        v = torch.addcmul(bias, unit, gain)
        if op == "gnorm":
            y = v if case["act"] == "none" else v.clamp(min=0) if case["act"] == "relu" else v * torch.sigmoid(v)
            parts.append((y, mean, rstd))
            continue
        slope = s["grad"][i].double().reshape(-1, c)
        if case["act"] == "relu":
            slope = slope * (v > 0)
        elif case["act"] == "silu":
            sig = torch.sigmoid(v)
            slope = slope * (sig + v * sig * torch.sigmoid(-v))
        sums[0] += torch.einsum("pc,pc->c", slope, unit)
        sums[1] += slope.sum(0)
        w, u = ((t * f).reshape(-1, groups, c // groups) for t, f in ((slope, gain), (unit, 1.0)))
        m = w.shape[0] * w.shape[2]
        parts.append((w - w.sum((0, 2))[:, None] / m - u * (torch.einsum("pgd,pgd->g", w, u)[:, None] / m)) * rstd[:, None])
    if op == "gnorm":
        y, mean, rstd = (torch.stack(t) for t in zip(*parts))
        return {"y": y.view(s["x"].shape), "mean": mean, "rstd": rstd}
    return {"grad_x": torch.stack(parts).view(s["x"].shape), "grad_gain": sums[0], "grad_bias": sums[1]}


def _exact_distill(case, s):
    """Row by row over the classes: the teacher's probabilities as a dense row, the classes outside the list as a mask."""
    tau, parts = case["tau"], []
    w = torch.ones(case["rows"], device="cuda", dtype=F64) if s["weights"] is None else s["weights"].double()
    for r in range(0, case["rows"], 256):
        z, ids, t = s["logits"][r:r + 256].double() / tau, s["ids"][r:r + 256].long(), s["values"][r:r + 256].double() / tau
        listed_classes, dense = torch.zeros_like(z, dtype=torch.bool), torch.full_like(z, -math.inf)
        row, entry = (ids != NO_CLASS).nonzero(as_tuple=True)
        listed_classes[row, ids[row, entry]] = True
        dense[row, ids[row, entry]] = t[row, entry]
        some = listed_classes.sum(1) > 0
        if case["rest"]:
            p = torch.exp(dense - s["lse"][r:r + 256].double()[:, None])
            outside = torch.clamp(1 - p.sum(1), min=0)
        else:
            p = torch.softmax(dense, 1).nan_to_num(0.0)
            outside = torch.zeros_like(p[:, 0])
        log_q = torch.log_softmax(z, 1)
        log_rest = torch.logsumexp(torch.where(listed_classes, -math.inf, log_q), 1)
        loss = (torch.special.xlogy(p, p) - torch.where(p > 0, p * log_q, 0.0)).sum(1)
        loss = loss + torch.special.xlogy(outside, outside) - torch.where(outside > 0, outside * log_rest, 0.0)
        live = w[r:r + 256] > 0
        part = {"row_loss": torch.where(live, loss, 0.0), "student_lse": torch.where(live, torch.logsumexp(z, 1), 0.0)}
        if case["grad"]:
            mass = (p.sum(1) + outside)[:, None]
            beside = torch.where(listed_classes, 0.0, torch.exp(log_q - log_rest[:, None]) * outside[:, None])
            grad = (mass * torch.exp(log_q) - p - beside) * (tau * w[r:r + 256] * some / w.sum().clamp(min=1e-300))[:, None]
            part["grad"] = grad
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    out["mean"] = ((out["row_loss"] * w).sum() / w.sum().clamp(min=1e-300)).view(1)
    return out
