"""Distillation from a teacher's lists against the formulas in 64 bits: one class to many, one entry to 256, odd row lengths and strides, lists
with repeated and missing entries, rows without weight, without a teacher, with nothing left; the gradient in place, added, captured;
refusals.

Bounds (u: unit roundoff of float32).  With (s - max) / tau at most R in magnitude, an exponential has a relative error of at most
(2 + 3 R) u, a sum of v positive terms by at least 32 lanes adds (v / 32 + 16) u (together: `total`).  The teacher's side is float64.
loss: the student's logarithms enter with the weights mass and p_rest.  gradient: P q_k - p_k on the list, outside the softmax of the
outside times P q_rest - p_rest, each q with `total`, a few roundings, and the output's own."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, U, device, guarded, rng, rounding, small, within

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
SHAPES = [(1, 1, 1), (1, 7, 3), (5, 32, 8), (3, 1000, 64), (40, 257, 20), (2, 50001, 256), (1, 131072, 64), (130, 2056, 50), (9, 16384, 100), (200, 8, 2),
          (3, 70003, 64), (1500, 40, 5), (700, 5001, 10), (1, 300000, 33), (333, 1025, 1), (310, 30002, 64)]


def plain(z, values, ids, tau, lse=None, weights=None, grad_mean=1.0):
    """(row_loss, student_lse, mean, gradient, parts for the bounds), everything float64."""
    rows, classes = z.shape
    top = z.double().max(1, keepdim=True).values
    top = torch.where(torch.isfinite(top), top, 0.0)               # differences first: a row of a type's lowest value keeps its digits
    s, t = (z.double() - top) / tau, values.double() / tau
    w = torch.ones(rows, dtype=F64) if weights is None else weights.double()
    live = w > 0
    total_w = float(w[live].sum()) if bool(live.any()) else 1.0
    loss, out, grad = torch.zeros(rows, dtype=F64), torch.zeros(rows, dtype=F64), torch.zeros(rows, classes, dtype=F64)
    weight_sum, scale_bound = torch.zeros(rows, dtype=F64), torch.zeros(rows, classes, dtype=F64)
    for r in range(rows):
        if not live[r]:
            continue
        entries, seen = [], set()
        for k, c in enumerate(ids[r].tolist()):
            if 0 <= c < classes and c not in seen:
                seen.add(c)
                entries.append(k)
        listed = ids[r, entries].long()
        u = t[r, entries]
        outside = torch.ones(classes, dtype=torch.bool)
        outside[listed] = False
        out[r] = torch.logsumexp(s[r], 0)
        given = float(lse[r]) if lse is not None else (float(torch.logsumexp(u, 0)) if entries else -torch.inf)
        if given == -torch.inf:
            continue
        p = torch.exp(u - given)
        a = torch.logsumexp(s[r, outside], 0) if bool(outside.any()) else torch.tensor(-torch.inf, dtype=F64)
        p_rest = max(0.0, 1.0 - float(p.sum())) if lse is not None and a != -torch.inf else 0.0
        mass = float(p.sum()) + p_rest
        weight_sum[r] = mass + p_rest
        if mass == 0:
            continue
        if out[r] == -torch.inf:
            loss[r] = torch.inf
            continue
        on = p > 0
        loss[r] = (p[on] * (u[on] - given - s[r, listed][on] + out[r])).sum()
        if p_rest > 0:
            loss[r] += p_rest * (torch.log(torch.tensor(p_rest, dtype=F64)) - a + out[r])
        q = torch.exp(s[r] - out[r])
        soft = torch.where(outside, torch.exp(s[r] - (a if a != -torch.inf else 0.0)), 0.0)
        q_rest = float(torch.exp(a - out[r]))
        scale = grad_mean * float(w[r]) / total_w / tau
        g = soft * (mass * q_rest - p_rest)
        g[listed] = mass * q[listed] - p
        grad[r] = scale * g
        b = soft * (mass * q_rest + p_rest)
        b[listed] = mass * q[listed] + p
        scale_bound[r] = abs(scale) * b
    out = torch.where(live, out + top[:, 0] / tau, 0.0)
    mean = (loss * torch.where(live, w, 0.0)).sum() / total_w if bool(live.any()) else torch.zeros((), dtype=F64)
    return loss, out, mean.view(1), grad, weight_sum, scale_bound


def strided(t, stride, offset=0):
    buf = torch.full((t.shape[0] * stride + offset,), float("nan"), dtype=t.dtype, device="cuda")
    out = buf[offset:].as_strided(t.shape, (stride, 1), offset)
    out.copy_(t)
    return out


def draw(rows, classes, count, dtype, values_dtype, seed, rest, weighted, tau, missing=True):
    g = rng(seed)
    z = 3 * torch.randn(rows, classes, generator=g)
    ids = torch.stack([torch.randperm(classes, generator=g)[:count] for _ in range(rows)]) if classes >= count else torch.randint(classes, (rows, count), generator=g)
    values = (3 * torch.randn(rows, count, generator=g) + 6).to(values_dtype)
    z.scatter_(1, ids, values.float() + torch.randn(rows, count, generator=g))
    if missing and count > 3:
        ids[:, 2] = -1
        ids[0, 3] = classes + 5
        ids[rows // 2, -1] = ids[rows // 2, 0]            # an entry that the list has already had
    lse = weights = None
    if rest:
        v = torch.where((ids >= 0) & (ids < classes), values.float() / tau, -torch.inf)
        lse = torch.where(v.max(1).values > -torch.inf, torch.logsumexp(v, 1) + 0.3 * torch.rand(rows, generator=g), 3.0)
    if weighted:
        weights = torch.rand(rows, generator=g) + 0.1
        weights[::5] = 0.0
        weights[rows // 2] = -1.0
    return z.to(dtype), values, ids, lse, weights


def handle(z, values, count, ids, tau, rest, add=False):
    h = circ.circ_distill_create(z.shape[1], count)
    circ.circ_distill_set_dtypes(h, CODE[z.dtype], CODE[values.dtype], CODE[ids])
    circ.circ_distill_set_temperature(h, tau)
    circ.circ_distill_set_rest(h, rest)
    circ.circ_distill_set_add(h, add)
    return h


def up(t):
    return None if t is None else device(t)


def run(z, values, ids, lse, weights, tau=1.0, it=torch.int64, extra=0, offset=0, grad_extra=None, grad_offset=None, grad_mean=1.0, in_place=False, add=None):
    rows, classes = z.shape
    count = ids.shape[1]
    stream = torch.cuda.current_stream()
    h = handle(z, values, count, it, tau, lse is not None, add is not None)
    stride = classes + extra
    zd, vd, idd, ld, wd = strided(z, stride, offset), device(values), device(ids.to(it)), up(lse), up(weights)
    row, row_ok = guarded((rows,), F32)
    out, out_ok = guarded((rows,), F32)
    mean, mean_ok = guarded((1,), F32)
    circ.circ_distill_forward(h, zd, stride, vd, idd, ld, wd, row, out, mean, rows, stream)
    only = torch.empty(1, device="cuda")
    circ.circ_distill_forward(h, zd, stride, vd, idd, ld, wd, None, None, only, rows, stream)
    row2, out2, mean2 = torch.empty_like(row), torch.empty_like(out), torch.empty_like(mean)
    grad_stride = classes + (extra if grad_extra is None else grad_extra)
    grad = zd if in_place else strided(torch.zeros_like(z) if add is None else add, grad_stride, offset if grad_offset is None else grad_offset)
    circ.circ_distill_backward(h, zd, stride, vd, idd, ld, wd, row2, out2, mean2, grad, grad_stride, grad_mean, rows, stream)
    torch.cuda.synchronize()
    circ.circ_distill_destroy(h)
    for ok in (row_ok, out_ok, mean_ok):
        ok()
    assert torch.equal(only.view(torch.int32), mean.view(torch.int32))        # the same call, with nothing else asked for
    between = grad.as_strided((rows, grad_stride - classes), (grad_stride, 1), grad.storage_offset() + classes)
    if rows > 1:
        assert bool(between[:-1].isnan().all())          # what lies between the rows is left alone
    return (row.cpu(), out.cpu(), mean.cpu()), (row2.cpu(), out2.cpu(), mean2.cpu()), grad.cpu()


def check(z, values, ids, lse, weights, got, tau=1.0, grad_mean=1.0, add=None):
    loss_ref, out_ref, mean_ref, grad_ref, mass, scale = plain(z, values, ids, tau, lse, weights, grad_mean)
    zz = z.double() / tau
    top = zz.max(1, keepdim=True).values
    spread = (top - torch.where(zz == -torch.inf, top, zz)).max(1).values.nan_to_num(0.0)
    total = (2 + 3 * spread + z.shape[1] / 32 + 16) * U
    loss_bound = 1.1 * total * mass + 4 * U * loss_ref.abs()
    out_bound = 1.1 * total + 2 * U * out_ref.abs()
    finite = torch.where(torch.isfinite(loss_bound), loss_bound, 0.0)
    mean_bound = (finite.max() + 4 * U * mean_ref.abs())
    for three in got[:2]:
        for g, ref, b in zip(three, (loss_ref, out_ref, mean_ref), (loss_bound, out_bound, mean_bound)):
            g, fine = g.double(), torch.isfinite(ref)
            assert torch.equal(g[~fine], ref[~fine])                          # infinities in their places
            within(g[fine], ref[fine], b[fine])
    old = torch.zeros_like(grad_ref) if add is None else add.double()
    want = grad_ref + old
    within(got[2], want, 2 * (total + 6 * U)[:, None] * scale + (rounding(z.dtype)) * want.abs() + small(z.dtype) + (2 * U * old.abs()))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,count", SHAPES)
@pytest.mark.parametrize("dtype,values_dtype,it,extra,offset,tau,rest,weighted", [
    (F32, F32, torch.int64, 0, 0, 1.0, False, False), (BF16, BF16, torch.int32, 0, 0, 2.0, True, True), (BF16, F32, torch.int64, 5, 3, 1.0, True, False),
    (F32, BF16, torch.int32, 3, 1, 0.7, False, True), (BF16, F32, torch.int32, 8, 0, 4.0, False, False), (F32, F32, torch.int64, 3, 0, 3.0, True, True)])
def test_loss_and_gradient(rows, classes, count, dtype, values_dtype, it, extra, offset, tau, rest, weighted):
    case = draw(rows, classes, count, dtype, values_dtype, rows + classes, rest, weighted, tau)
    check(*case, run(*case, tau=tau, it=it, extra=extra, offset=offset), tau=tau)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,dtype", [(4, 1000, F32), (300, 513, BF16), (2, 60001, BF16), (5, 40000, F32), (330, 9001, BF16), (400, 200, F32)])
@pytest.mark.parametrize("rest", [False, True])
def test_gradient_in_place_scaled_and_added(rows, classes, dtype, rest):
    case = draw(rows, classes, 30, dtype, F32, 77, rest, True, 2.0)
    check(*case, run(*case, tau=2.0, in_place=True, grad_mean=-2.5), tau=2.0, grad_mean=-2.5)
    other = run(*case, tau=2.0, extra=1, grad_extra=4, grad_offset=1, grad_mean=-2.5)       # another alignment
    check(*case, other, tau=2.0, grad_mean=-2.5)
    old = (1e-3 * torch.randn(rows, classes, generator=rng(3))).to(dtype)
    check(*case, run(*case, tau=2.0, add=old, grad_mean=4.0), tau=2.0, grad_mean=4.0, add=old)
    check(*case, run(*case, tau=2.0, add=old, extra=3, grad_extra=6, grad_offset=1, grad_mean=4.0), tau=2.0, grad_mean=4.0, add=old)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,count", [(2047, 40, 5), (2048, 40, 5), (2300, 517, 64), (2050, 2300, 9), (310, 70003, 20), (15, 140001, 256), (16, 140001, 256),
                                                (2, 500001, 50)])
@pytest.mark.parametrize("dtype,offset,rest,weighted", [(F32, 0, False, True), (BF16, 0, True, False), (BF16, 1, False, True), (F32, 3, True, True)])
def test_many_rows_and_the_longest(rows, classes, count, dtype, offset, rest, weighted):
    case = draw(rows, classes, count, dtype, F32, rows + classes, rest, weighted, 2.0)
    check(*case, run(*case, tau=2.0, offset=offset), tau=2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [60, 700, 3001, 40000, 130001])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", [False, True])
def test_masked_classes_empty_lists_and_rows_with_nothing_left(classes, dtype, rest):
    rows, count = 12, 40
    z, values, ids, lse, weights = draw(rows, classes, count, dtype, F32, 5, rest, False, 1.0)
    z[0, classes // 2:] = -torch.inf                       # the teacher's classes among them
    z[1, classes // 2:] = torch.finfo(dtype).min
    ids[1] = torch.arange(count) % (classes // 2)          # repeats where there are few
    z[2] = -torch.inf
    ids[3] = -1                                            # no entry
    values[4] = -torch.inf
    values[5, 1:] = -torch.inf
    outside = torch.ones(classes, dtype=torch.bool)
    outside[ids[6][(ids[6] >= 0) & (ids[6] < classes)]] = False
    z[6, outside] = -torch.inf                             # the student gives the outside nothing
    ids[7] = 4                                             # the same class all over
    z[8] = 1.5                                             # every logit the same
    values[9] = 2.0
    z[10] = torch.finfo(dtype).min
    if rest:
        lse[0] = 40.0                                      # the list holds next to nothing
        lse[4] = -torch.inf                                # no teacher
        lse[11] = float(torch.logsumexp(values[11].double(), 0)) - 0.5      # more than all of it
    got = run(z, values, ids, lse, weights)
    check(z, values, ids, lse, weights, got)
    grad = got[2]
    assert bool((grad[2:5] == 0).all()) if not rest else bool((grad[2:4] == 0).all())
    assert got[0][0][2] == torch.inf and got[0][1][2] == -torch.inf and got[0][0][3] == 0
    assert bool(torch.isfinite(grad).all())


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [50, 2048, 40000])
@pytest.mark.parametrize("rest", [False, True])
def test_values_that_are_not_finite_stay_in_their_rows(classes, rest):
    case = draw(6, classes, 20, F32, F32, 6, rest, False, 1.0)
    z, values, ids, lse, _ = case
    clean = run(*case)
    z[1, classes - 1] = float("nan")
    z[2, ids[2, 0]] = float("inf")
    values[3, 1] = float("nan")
    if rest:
        lse[4] = float("nan")
    (row, out, mean), _, grad = run(*case)
    assert bool(row[1:4].isnan().all()) and bool(mean.isnan()) and bool(out[1:3].isnan().all())
    assert bool(grad[1:4].isnan().any(1).all()) and (not rest or (bool(row[4].isnan()) and bool(grad[4].isnan().all())))
    for r in (0, 5):
        assert torch.equal(grad[r], clean[2][r]) and row[r] == clean[0][0][r]


@pytest.mark.gpu
@pytest.mark.parametrize("classes,count", [(256, 256), (100, 100), (2000, 256), (3, 3)])
def test_lists_that_hold_every_class(classes, count):
    case = draw(20, classes, count, F32, F32, 8, True, False, 1.0, missing=False)
    check(*case, run(*case))
    if classes == count:       # then it is the divergence of two softmaxes, whatever the teacher's lse leaves over
        z, values, ids, _, _ = case
        got = run(z, values, ids, None, None)
        teacher = torch.zeros(20, classes, dtype=F64).scatter_(1, ids, values.double())
        want = torch.nn.functional.kl_div(torch.log_softmax(z.double(), 1), torch.log_softmax(teacher, 1), reduction="none", log_target=True).sum(1)
        assert float((got[0][0].double() - want).abs().max()) <= 1e-5


@pytest.mark.gpu
def test_no_rows_no_weights_and_one_entry():
    h = circ.circ_distill_create(10, 3)
    mean = torch.full((1,), float("nan"), device="cuda")
    circ.circ_distill_forward(h, None, 10, None, None, None, None, None, None, mean, 0, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_distill_destroy(h)
    assert float(mean) == 0
    z, values, ids, lse, _ = draw(7, 33, 5, F32, F32, 1, False, False, 1.0)
    (row, out, mean), _, grad = run(z, values, ids, lse, torch.zeros(7))
    assert bool((row == 0).all()) and bool((out == 0).all()) and float(mean) == 0 and bool((grad == 0).all())
    # a list of one entry is a label: the loss is the cross entropy
    ids = torch.randint(33, (7, 1), generator=rng(2))
    (row, out, mean), _, grad = run(z, torch.zeros(7, 1), ids, None, None)
    want = torch.nn.functional.cross_entropy(z.double(), ids[:, 0], reduction="none")
    assert float((row.double() - want).abs().max()) <= 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("classes", [37, 1500])
def test_gradient_is_the_derivative_of_the_mean(rest, classes):
    case = draw(8, classes, 12, F32, F32, 21, rest, True, 1.7)
    grad = run(*case, tau=1.7)[2]
    z = case[0].double()
    v = torch.randn(z.shape, generator=rng(4), dtype=F64)
    step = 1e-4                                                      # central differences in 64 bits: error step^2 times third derivatives
    slope = float(plain(z + step * v, *case[1:3], 1.7, *case[3:])[2] - plain(z - step * v, *case[1:3], 1.7, *case[3:])[2]) / (2 * step)
    mine = grad.double() * v
    assert abs(float(mine.sum()) - slope) <= 1e-5 * float(mine.abs().sum())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(50, 1000), (3, 70003), (1200, 300), (300, 12001)])
def test_a_captured_graph_keeps_its_workspace(rows, classes):
    case = draw(rows, classes, 20, F32, F32, 19, True, True, 2.0)
    z, values, ids, lse, weights = case
    h = handle(z, values, 20, torch.int64, 2.0, True)
    tensors = [device(t) for t in (values, ids, lse, weights)]
    zd = device(z)
    circ.circ_distill_reserve(h, rows)
    row, out, mean, grad = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros_like(zd)
    args = (h, zd, classes, *tensors, row, out, mean, grad, classes, 4.0, rows)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_distill_backward(*args, torch.cuda.current_stream())
    for more in (2 * rows, 20000):
        circ.circ_distill_reserve(h, more)               # the graph's workspace stays
        other = torch.full((1 << 20,), float("nan"), device="cuda")
        for _ in range(2):
            for t in (row, out, mean, grad):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            three = (row.cpu(), out.cpu(), mean.cpu())
            check(*case, (three, three, grad.cpu()), tau=2.0, grad_mean=4.0)
        eager = torch.zeros_like(grad)
        circ.circ_distill_backward(h, zd, classes, *tensors, row, out, mean, eager, classes, 4.0, rows, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(eager, grad) and bool(other.isnan().all())
    del graph
    circ.circ_distill_destroy(h)


@pytest.mark.gpu
def test_a_workspace_that_cannot_be_allocated():
    h = circ.circ_distill_create(64, 4)
    try:
        circ.circ_debug_fail_alloc_after(1)
        refused(circ.CIRC_ERR_ALLOC, circ.circ_distill_reserve, h, 10)
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_distill_reserve(h, 10)
    finally:
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_distill_destroy(h)


def refused(code, call, *args):
    with pytest.raises(circ.CircError) as e:
        call(*args)
    assert e.value.code == code


def test_refusals_before_any_device_call():
    for args in ((0, 1), (10, 0), (1000, 257), ((1 << 28) + 1, 1)):
        refused(circ.CIRC_ERR_SHAPE, circ.circ_distill_create, *args)
    for call, args in ((circ.circ_distill_forward, (None, 64, 8, 64, 64, None, None, 64, None, None, 1)),
                       (circ.circ_distill_backward, (None, 64, 8, 64, 64, None, None, 64, None, None, 256, 8, 1.0, 1)),
                       (circ.circ_distill_set_dtypes, (None, 0, 0, 0)), (circ.circ_distill_set_temperature, (None, 1.0)),
                       (circ.circ_distill_set_rest, (None, 1)), (circ.circ_distill_set_add, (None, 1)), (circ.circ_distill_reserve, (None, 1))):
        refused(circ.CIRC_ERR_ARG, call, *args)
    circ.circ_distill_destroy(None)


@pytest.mark.gpu
def test_refusals_of_bad_arguments():
    h = circ.circ_distill_create(16, 4)
    z, v = torch.empty(4, 16, device="cuda"), torch.empty(4, 4, device="cuda")
    i, out = torch.zeros(4, 4, dtype=torch.int64, device="cuda"), torch.empty(4, device="cuda")
    try:
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_set_dtypes, h, circ.CIRC_E4M3, 0, 0)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_set_dtypes, h, 0, circ.CIRC_E4M3, 0)
        for tau in (0.0, -1.0, float("nan"), float("inf")):
            refused(circ.CIRC_ERR_ARG, circ.circ_distill_set_temperature, h, tau)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_distill_forward, h, z, 15, v, i, None, None, out, None, None, 4)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_distill_forward, h, z, 16, v, i, None, None, out, None, None, -1)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_forward, h, z, 16, v, i, None, None, None, None, None, 4)          # nothing to compute
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_forward, h, None, 16, v, i, None, None, out, None, None, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_forward, h, z, 16, None, i, None, None, out, None, None, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_forward, h, z, 16, v, None, None, None, out, None, None, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_forward, h, z, 16, v, i, out, None, out, None, None, 4)            # an lse without the rest
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_forward, h, z.data_ptr() + 2, 16, v, i, None, None, out, None, None, 1)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_backward, h, z, 16, v, i, None, None, out, None, None, None, 16, 1.0, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_backward, h, z, 16, v, i, None, None, out, None, None, z, 17, 1.0, 3)
        circ.circ_distill_set_rest(h, 1)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_forward, h, z, 16, v, i, None, None, out, None, None, 4)           # the rest without an lse
        circ.circ_distill_set_rest(h, 0)
        circ.circ_distill_set_add(h, 1)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_backward, h, z, 16, v, i, None, None, out, None, None, z, 16, 1.0, 4)   # added in place
        with pytest.raises(AssertionError):
            circ.circ_distill_forward(h, z.t(), 16, v, i, None, None, out, None, None, 4)
    finally:
        circ.circ_distill_destroy(h)
