"""What the header says of the ends of the ranges of top logits, distillation and group norm: sizes and temperatures that are refused, the smallest and largest
that are served, logits that are not finite, deviations from tiny to huge."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import U, device, rng

F64 = torch.float64
NAN, INF = float("nan"), float("inf")


def refused(code, call, *args):
    with pytest.raises(circ.CircError) as e:
        call(*args)
    assert e.value.code == code


@pytest.mark.gpu
def test_sizes_and_temperatures_beyond_the_limits_are_refused():
    t, d, g = circ.circ_top_create(8, 2), circ.circ_distill_create(8, 2), circ.circ_gnorm_create(8, 2, 1e-5)
    z = torch.empty(64, device="cuda")
    try:
        for tau in (9e-7, 1.1e6):
            refused(circ.CIRC_ERR_ARG, circ.circ_top_set_temperature, t, tau)
            refused(circ.CIRC_ERR_ARG, circ.circ_distill_set_temperature, d, tau)
        many = (1 << 24) + 1
        refused(circ.CIRC_ERR_SHAPE, circ.circ_top_forward, t, z, 8, z, None, None, many)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_distill_forward, d, z, 8, z, z, None, None, z, None, None, many)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_distill_backward, d, z, 8, z, z, None, None, z, None, None, z, 8, 1.0, many)
        refused(circ.CIRC_ERR_ARG, circ.circ_top_reserve, t, many)
        refused(circ.CIRC_ERR_ARG, circ.circ_distill_reserve, d, many)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_gnorm_forward, g, z, None, None, z, None, None, (1 << 20) + 1, 1, 1)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_gnorm_forward, g, z, None, None, z, None, None, 1, 1 << 14, (1 << 14) + 1)
    finally:
        circ.circ_top_destroy(t)
        circ.circ_distill_destroy(d)
        circ.circ_gnorm_destroy(g)


@pytest.mark.gpu
@pytest.mark.parametrize("tau", [1e-6, 1e6])
@pytest.mark.parametrize("classes", [40, 3001])
def test_the_smallest_and_largest_temperature(tau, classes):
    rows, count = 6, 5
    z = torch.randn(rows, classes, generator=rng(classes))
    top, di = circ.circ_top_create(classes, count), circ.circ_distill_create(classes, count)
    circ.circ_top_set_temperature(top, tau)
    circ.circ_distill_set_temperature(di, tau)
    zd = device(z)
    values, ids, lse = torch.empty(rows, count, device="cuda"), torch.empty(rows, count, dtype=torch.int64, device="cuda"), torch.empty(rows, device="cuda")
    row, out, mean = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(1, device="cuda")
    s = torch.cuda.current_stream()
    circ.circ_top_forward(top, zd, classes, values, ids, lse, rows, s)
    student = device(z.flip(1).contiguous())
    circ.circ_distill_forward(di, student, classes, values, ids, None, None, row, out, mean, rows, s)
    torch.cuda.synchronize()
    circ.circ_top_destroy(top)
    circ.circ_distill_destroy(di)
    tau = float(torch.tensor(tau))
    want = torch.logsumexp(z.double() / tau, 1)
    # sums of up to 3001 exponentials by 32 lanes: (94 + 16 + 2) u, the value itself u; at 1e-6 the largest takes all
    for got in (lse, out):
        assert bool(((got.double().cpu() - want).abs() <= 120 * U + 2 * U * want.abs()).all())
    p = torch.softmax(values.double().cpu() / tau, 1)
    log_q = torch.log_softmax(z.flip(1).double() / tau, 1).gather(1, ids.cpu())
    loss = (torch.special.xlogy(p, p) - torch.where(p > 0, p * log_q, 0.0)).sum(1)
    assert bool(((row.double().cpu() - loss).abs() <= 120 * U + 4 * U * loss.abs()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(6, 50), (6, 3001), (400, 5000), (6, 140001)])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_logits_that_leave_no_probabilities(rows, classes, rest, bad):
    count = 9
    g = rng(classes)
    z, values = torch.randn(rows, classes, generator=g), torch.randn(rows, count, generator=g)
    ids = torch.arange(count).expand(rows, count).contiguous()
    z[1, 4] = bad                  # of the list
    z[2, classes - 1] = bad        # outside
    z[3, 4] = bad                  # of a row without a teacher
    ids[3] = -1
    lse = torch.logsumexp(values, 1) + 0.1 if rest else None
    if rest:
        lse[3] = -INF
    h = circ.circ_distill_create(classes, count)
    circ.circ_distill_set_rest(h, rest)
    row, out, mean, grad = (torch.zeros(n, device="cuda") for n in (rows, rows, 1, rows * classes))
    circ.circ_distill_backward(h, device(z), classes, device(values), device(ids), None if lse is None else device(lse), None, row, out, mean, grad, classes, 1.0,
                               rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_distill_destroy(h)
    row, out, grad = row.cpu(), out.cpu(), grad.view(rows, classes).cpu()
    assert bool(row[1:3].isnan().all()) and bool(out[1:4].isnan().all()) and bool(mean.isnan())
    assert bool(grad[1:3].isnan().all()) and row[3] == 0 and bool((grad[3] == 0).all())
    for r in (0, 4, rows - 1):
        assert bool(torch.isfinite(grad[r]).all()) and bool(torch.isfinite(row[r])) and bool(torch.isfinite(out[r]))


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 9, 11, 60, 12), (1, 90, 75, 24, 3), (3, 28, 28, 256, 32), (2, 20, 20, 515, 5)])
@pytest.mark.parametrize("size", [1e-15, 1e15, 1e30])
def test_deviations_from_tiny_to_huge(n, h, w, c, groups, size):
    x = (torch.randn(n, h, w, c, generator=rng(c), dtype=F64) * size).float()
    hd = circ.circ_gnorm_create(c, groups, 0.0)
    y, mean, rstd = torch.empty(n, h, w, c, device="cuda"), torch.empty(n, groups, device="cuda"), torch.empty(n, groups, device="cuda")
    circ.circ_gnorm_forward(hd, device(x), None, None, y, mean, rstd, n, h, w, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_gnorm_destroy(hd)
    if size > 1e20:
        assert bool((rstd == 0).all())
        return
    g = x.double().view(n, h * w, groups, -1)
    want = 1 / g.var((1, 3), unbiased=False).sqrt()
    # at most 264 + 256 + 103 additions a sum, twice that where the sums' difference is taken, halved by the root
    assert bool(((rstd.double().cpu() - want).abs() <= 1300 * U * want).all())
    v = (g - g.mean((1, 3), keepdim=True)) * want[:, None, :, None]
    assert bool(((y.double().cpu().view(v.shape) - v).abs() <= 1300 * U * (v.abs() + 5)).all())
