"""Softmax cross entropy and its gradient against the formulas in 64 bits: one class to many, odd row lengths and strides,
ignored and impossible targets, masked classes, rows with nothing left, values that are not finite; refusals.

Bounds (u: unit roundoff of float32).  With z - max at most R in magnitude, exp has a relative error of at most (2 + 2 R) u
(rounding of the argument and the function's own), a sum of v positive terms by at least 32 lanes adds (v / 32 + 16) u;
lse = max + log(sum) adds two roundings.  Probabilities are quotients of the two."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, U, device, guarded, rng, rounding, small, within

F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(1, 1), (1, 7), (5, 32), (3, 1000), (40, 257), (2, 50001), (1, 131072), (130, 2056), (9, 16384), (200, 8), (3, 70003), (1500, 40), (1100, 3001), (1, 500000)]


def handle(classes, dtype, ids, ignore=-100):
    h = circ.circ_loss_create(classes)
    circ.circ_loss_set_dtypes(h, CODE[dtype], CODE[ids])
    circ.circ_loss_set_ignore(h, ignore)
    return h


def plain(z, targets, ignore=-100, grad_mean=1.0):
    z = z.double()
    rows, classes = z.shape
    valid = (targets >= 0) & (targets < classes) & (targets != ignore)
    count = int(valid.sum())
    top = z.max(1).values
    base = torch.where(top == -torch.inf, 0.0, top)
    e = torch.exp(z - base[:, None])
    total = e.sum(1)
    lse = base + torch.log(total)
    loss, grad = torch.zeros(rows, dtype=torch.float64), torch.zeros_like(z)
    for r in range(rows):
        if valid[r]:
            loss[r] = torch.inf if z[r, targets[r]] == -torch.inf else lse[r] - z[r, targets[r]]
            if total[r] > 0:
                grad[r] = e[r] / total[r]
                grad[r, targets[r]] -= 1
    mean = loss.sum() / count if count else torch.zeros((), dtype=torch.float64)
    return loss, lse, mean, grad * (grad_mean / max(1, count))


def strided(t, stride, offset=0):
    """A copy on the GPU with `stride` elements between rows (NaN between), starting `offset` elements behind an aligned address."""
    buf = torch.full((t.shape[0] * stride + offset,), float("nan"), dtype=t.dtype, device="cuda")
    out = buf[offset:].as_strided(t.shape, (stride, 1), offset)
    out.copy_(t)
    return out


def draw(rows, classes, dtype, seed, masked=0):
    g = rng(seed)
    z = 3 * torch.randn(rows, classes, generator=g)
    targets = torch.randint(classes - masked, (rows,), generator=g)
    z[torch.arange(rows), targets] += 4
    if masked:
        z[:, classes - masked:] = -torch.inf
    targets = torch.where(torch.rand(rows, generator=g) < 0.2, -100, targets)
    return z.to(dtype), targets


def run(z, targets, dtype, ids, stride, offset=0, grad_stride=None, grad_offset=0, grad_mean=1.0, in_place=False, ignore=-100):
    rows, classes = z.shape
    h = handle(classes, dtype, ids, ignore)
    zd, td = strided(z, stride, offset), device(targets.to(ids))
    row, row_ok = guarded((rows,), F32)
    lse, lse_ok = guarded((rows,), F32)
    mean, mean_ok = guarded((1,), F32)
    circ.circ_loss_forward(h, zd, stride, td, row, lse, mean, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    only = torch.empty(1, device="cuda")
    circ.circ_loss_forward(h, zd, stride, td, None, None, only, rows, torch.cuda.current_stream())
    row2, lse2, mean2 = torch.empty_like(row), torch.empty_like(lse), torch.empty_like(mean)
    grad_stride = stride if grad_stride is None else grad_stride
    grad = zd if in_place else strided(torch.zeros(rows, classes, dtype=dtype), grad_stride, grad_offset)
    circ.circ_loss_backward(h, zd, stride, td, row2, lse2, mean2, grad, grad_stride, grad_mean, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_loss_destroy(h)
    for ok in (row_ok, lse_ok, mean_ok):
        ok()
    check_values(z, targets, ignore, row, lse, mean)
    check_values(z, targets, ignore, row2, lse2, mean2)
    assert torch.equal(only.view(torch.int32), mean.view(torch.int32))        # the same call, with nothing else asked for
    between = grad.as_strided((rows, grad_stride - classes), (grad_stride, 1), grad.storage_offset() + classes)
    if rows > 1:
        assert bool(between[:-1].isnan().all())          # what lies between the rows is left alone
    return row2.cpu(), lse2.cpu(), mean2.cpu(), grad.cpu()


def row_bounds(z, lse_ref):
    """(error of an exponential, of the sum of them, of its logarithm) for every row."""
    zz = z.double()
    top = zz.max(1, keepdim=True).values
    spread = (top - torch.where(zz == -torch.inf, top, zz)).max(1).values
    term = (2 + 2 * spread) * U
    total = term + (z.shape[1] / 32 + 16) * U
    return term, total, 1.1 * total + 3 * U * (lse_ref.abs() + zz.max(1).values.abs())


def check_values(z, targets, ignore, row, lse, mean):
    loss_ref, lse_ref, mean_ref, _ = plain(z, targets, ignore)
    _, _, bound = row_bounds(z, lse_ref)
    for got, ref, b in ((lse, lse_ref, bound), (row, loss_ref, bound + 2 * U * loss_ref.abs()), (mean, mean_ref.view(1), (bound.max() + 4 * U * mean_ref.abs()).view(1))):
        got, fine = got.double().cpu(), torch.isfinite(ref)
        assert torch.equal(got[~fine].nan_to_num(5.0), ref[~fine].nan_to_num(5.0))        # NaN and the infinities in their places
        within(got[fine], ref[fine], b[fine])


def check(z, targets, dtype, got, ignore=-100, grad_mean=1.0):
    grad = got[3]
    _, lse_ref, _, grad_ref = plain(z, targets, ignore, grad_mean)
    term, total, _ = row_bounds(z, lse_ref)
    count = max(1, int(((targets >= 0) & (targets < z.shape[1]) & (targets != ignore)).sum()))
    p = grad_ref.abs() + (grad_ref < 0) * abs(grad_mean) / count          # the larger of the two that are subtracted
    within(grad, grad_ref, ((term + total)[:, None] + 10 * U) * p + rounding(dtype) * grad_ref.abs() + small(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", SHAPES)
@pytest.mark.parametrize("dtype,ids,extra,offset", [(F32, torch.int64, 0, 0), (BF16, torch.int32, 0, 0), (BF16, torch.int64, 5, 3), (F32, torch.int32, 3, 1),
                                                    (BF16, torch.int32, 8, 0)])
def test_loss_and_gradient(rows, classes, dtype, ids, extra, offset):
    z, targets = draw(rows, classes, dtype, rows + classes)
    check(z, targets, dtype, run(z, targets, dtype, ids, classes + extra, offset))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,dtype", [(4, 1000, F32), (300, 513, BF16), (2, 60001, BF16), (5, 40000, F32)])
def test_gradient_in_place_and_scaled(rows, classes, dtype):
    z, targets = draw(rows, classes, dtype, 77, masked=classes // 10)
    got = run(z, targets, dtype, torch.int64, classes, in_place=True, grad_mean=-2.5)
    check(z, targets, dtype, got, grad_mean=-2.5)
    other = run(z, targets, dtype, torch.int64, classes + 1, grad_stride=classes + 4, grad_offset=1, grad_mean=-2.5)   # another alignment
    check(z, targets, dtype, other, grad_mean=-2.5)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,dtype,extra", [(400, 30000, F32, 0), (400, 30001, F32, 2), (310, 60003, BF16, 0), (170, 60001, F32, 0), (90, 131073, F32, 3)])
@pytest.mark.parametrize("in_place", [False, True])
def test_clusters_that_walk_over_several_rows(rows, classes, dtype, extra, in_place):
    """Rows of 2, 4 and 8 blocks, two or more for each cluster that the machine holds at once: the copies of a row run behind the
    gradient of the one before, and the places for the peers' sums are used again."""
    z, targets = draw(rows, classes, dtype, rows)
    check(z, targets, dtype, run(z, targets, dtype, torch.int64, classes + extra, in_place=in_place))


@pytest.mark.gpu
@pytest.mark.parametrize("masked", [-torch.inf, "lowest"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_masked_classes_and_impossible_targets(masked, dtype):
    rows, classes = 6, 300
    z, targets = draw(rows, classes, F32, 5)
    low = torch.finfo(dtype).min if masked == "lowest" else masked
    z[:, 100:] = low
    z = z.to(dtype)
    targets[:] = torch.tensor([3, 99, 0, -100, 300, -1])            # the last two lie outside the classes
    row, lse, mean, grad = run(z, targets, dtype, torch.int64, classes)
    loss_ref, lse_ref, mean_ref, grad_ref = plain(z, targets)
    assert torch.allclose(row.double(), loss_ref, rtol=1e-5) and torch.allclose(lse.double(), lse_ref, rtol=1e-5)
    assert torch.allclose(mean.double(), mean_ref.view(1), rtol=1e-5)
    assert bool((grad[:, 100:] == 0).all()) and bool((grad[3:] == 0).all()) and bool((row[3:] == 0).all())
    assert torch.allclose(grad.double(), grad_ref, rtol=4 * rounding(dtype) + 1e-5, atol=1e-6)
    targets[0] = 200                                                # a masked class as the target
    row, _, _, grad = run(z, targets, dtype, torch.int64, classes)
    assert (row[0] == torch.inf) if masked != "lowest" else (row[0] > 1e38)
    assert bool(torch.isfinite(grad).all()) and float(grad[0, 200]) < 0


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [50, 2048, 40000])
def test_rows_with_nothing_left_and_values_that_are_not_finite(classes):
    z = torch.randn(5, classes, generator=rng(2))
    z[1] = -torch.inf
    z[2, 3] = float("nan")
    z[3, classes - 1] = float("inf")
    targets = torch.tensor([1, 2, 3, 4, -100])
    row, lse, mean, grad = run(z, targets, F32, torch.int64, classes)
    assert bool(torch.isfinite(row[0])) and bool(torch.isfinite(grad[0]).all())
    assert row[1] == torch.inf and lse[1] == -torch.inf and bool((grad[1] == 0).all())
    assert bool(row[2].isnan()) and bool(lse[2].isnan()) and bool(grad[2].isnan().all())
    assert bool(row[3].isnan()) and bool(grad[3].isnan().all())
    assert row[4] == 0 and bool((grad[4] == 0).all()) and bool(mean.isnan().all())


@pytest.mark.gpu
def test_no_rows_no_targets_and_an_ignored_class():
    h = handle(10, F32, torch.int64)
    mean = torch.full((1,), float("nan"), device="cuda")
    circ.circ_loss_forward(h, None, 10, None, None, None, mean, 0, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_loss_destroy(h)
    assert float(mean) == 0
    z, _ = draw(7, 33, F32, 1)
    row, lse, mean, grad = run(z, torch.full((7,), -100), F32, torch.int32, 33)
    assert bool((row == 0).all()) and float(mean) == 0 and bool((grad == 0).all()) and bool(torch.isfinite(lse).all())
    targets = torch.tensor([0, 1, 2, 0, 5, 0, 32])
    got = run(z, targets, F32, torch.int32, 33, ignore=0)
    check(z, targets, F32, got, ignore=0)
    assert bool((got[0][targets == 0] == 0).all())


@pytest.mark.gpu
def test_gradient_is_the_derivative_of_the_mean():
    rows, classes = 8, 37
    z, targets = draw(rows, classes, F32, 21)
    *_, grad = run(z, targets, F32, torch.int64, classes)
    v = torch.randn(rows, classes, generator=rng(4), dtype=torch.float64)
    step = 1e-4                                                      # central differences in 64 bits: error step^2 times third derivatives
    slope = float(plain(z.double() + step * v, targets)[2] - plain(z.double() - step * v, targets)[2]) / (2 * step)
    mine = grad.double() * v
    assert abs(float(mine.sum()) - slope) <= 1e-5 * float(mine.abs().sum())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(50, 1000), (3, 70003), (1200, 300), (1030, 3000)])
def test_captured_graph(rows, classes):
    z, targets = draw(rows, classes, F32, 9)
    zd, td = device(z), device(targets)
    h = handle(classes, F32, torch.int64)
    circ.circ_loss_reserve(h, rows)
    mean, grad = torch.zeros(1, device="cuda"), torch.zeros_like(zd)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_loss_backward(h, zd, classes, td, None, None, mean, grad, classes, 1.0, rows, torch.cuda.current_stream())
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    ref = plain(z, targets)
    assert abs(float(mean) - float(ref[2])) <= 1e-5 * float(ref[2]) and torch.allclose(grad.double().cpu(), ref[3], atol=1e-7)
    del graph
    circ.circ_loss_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(50, 1000), (1200, 300), (30, 70003)])
def test_a_captured_graph_keeps_its_workspace(rows, classes):
    """Calls behind the capture need more, and other memory takes what they leave."""
    z, targets = draw(rows, classes, F32, 19)
    zd, td = device(z), device(targets)
    h = handle(classes, F32, torch.int64)
    circ.circ_loss_reserve(h, rows)
    mean, grad = torch.zeros(1, device="cuda"), torch.zeros_like(zd)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_loss_backward(h, zd, classes, td, None, None, mean, grad, classes, 1.0, rows, torch.cuda.current_stream())
    ref = plain(z, targets)
    for more in (20000, 400000, 1600000):                # blocks of 8 rows: 2500, 50000, 200000 sums
        circ.circ_loss_reserve(h, more)
        other = torch.full((more,), float("nan"), device="cuda")
        for _ in range(2):
            mean.zero_()
            grad.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert abs(float(mean) - float(ref[2])) <= 1e-5 * float(ref[2]) and torch.allclose(grad.double().cpu(), ref[3], atol=1e-7)
        eager = torch.zeros(1, device="cuda")
        circ.circ_loss_backward(h, zd, classes, td, None, None, eager, grad, classes, 1.0, rows, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(eager, mean) and bool(other.isnan().all())
    del graph
    circ.circ_loss_destroy(h)


@pytest.mark.gpu
def test_a_workspace_that_cannot_be_allocated():
    h = handle(64, F32, torch.int64)
    try:
        circ.circ_debug_fail_alloc_after(1)
        refused(circ.CIRC_ERR_ALLOC, circ.circ_loss_reserve, h, 10)
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_loss_reserve(h, 10)
    finally:
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_loss_destroy(h)


def refused(code, call, *args):
    with pytest.raises(circ.CircError) as e:
        call(*args)
    assert e.value.code == code


def test_refusals_before_any_device_call():
    refused(circ.CIRC_ERR_SHAPE, circ.circ_loss_create, 0)
    for call, args in ((circ.circ_loss_forward, (None, 64, 8, 64, 128, None, None, 1)),
                       (circ.circ_loss_backward, (None, 64, 8, 64, 128, None, None, 256, 8, 1.0, 1)), (circ.circ_loss_set_dtypes, (None, 0, 0)),
                       (circ.circ_loss_set_ignore, (None, 0)), (circ.circ_loss_reserve, (None, 1))):
        refused(circ.CIRC_ERR_ARG, call, *args)
    circ.circ_loss_destroy(None)


@pytest.mark.gpu
def test_refusals_of_bad_arguments():
    h = handle(16, F32, torch.int64)
    z, t, out = torch.empty(4, 16, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.empty(4, device="cuda")
    try:
        refused(circ.CIRC_ERR_ARG, circ.circ_loss_set_dtypes, h, circ.CIRC_E4M3, 0)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_loss_forward, h, z, 15, t, out, None, None, 4)              # rows overlap
        refused(circ.CIRC_ERR_SHAPE, circ.circ_loss_forward, h, z, 16, t, out, None, None, -1)
        refused(circ.CIRC_ERR_ARG, circ.circ_loss_forward, h, z, 16, t, None, None, None, 4)               # nothing to compute
        refused(circ.CIRC_ERR_ARG, circ.circ_loss_forward, h, None, 16, t, out, None, None, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_loss_forward, h, z.data_ptr() + 2, 16, t, out, None, None, 1)
        refused(circ.CIRC_ERR_ARG, circ.circ_loss_backward, h, z, 16, t, out, None, None, None, 16, 1.0, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_loss_backward, h, z, 16, t, out, None, None, z, 17, 1.0, 3)   # in place, another stride
        with pytest.raises(AssertionError):
            circ.circ_loss_forward(h, z.t(), 16, t, out, None, None, 4)
    finally:
        circ.circ_loss_destroy(h)
