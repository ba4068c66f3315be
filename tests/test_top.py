"""The largest logits of rows against a stable sort in 64 bits: one class to many, odd row lengths and strides, ties, rows in every order,
masked classes, rows with nothing left, NaN and infinities; log sum exp at a temperature; refusals.

Values and ids are exact.  Bounds of lse (u: unit roundoff of float32): with (z - max) / tau at most R in magnitude, an exponential has a
relative error of at most (2 + 3 R) u (rounding of the factor, of the argument, and the function's own), a sum of v positive terms by at
least 32 lanes adds (v / 32 + 16) u, and the result is rounded once."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, U, device, guarded, rng, within

F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(1, 1, 1), (1, 7, 7), (5, 32, 3), (3, 1000, 64), (40, 257, 20), (2, 50001, 256), (1, 131072, 8), (130, 2056, 50), (9, 16384, 100), (200, 8, 4),
          (3, 70003, 64), (1500, 40, 5), (400, 20001, 64), (1, 500000, 200), (700, 300, 256), (333, 1025, 1)]


def strided(t, stride, offset=0):
    buf = torch.full((t.shape[0] * stride + offset,), float("nan"), dtype=t.dtype, device="cuda")
    out = buf[offset:].as_strided(t.shape, (stride, 1), offset)
    out.copy_(t)
    return out


def plain(z, count):
    # NaN is above everything: a stable sort by (is NaN, value)
    d = z.double()
    nan = torch.isnan(d)
    order = torch.argsort(torch.where(nan, -torch.inf, d), dim=1, descending=True, stable=True)
    order = order.gather(1, torch.argsort(nan.gather(1, order).int(), dim=1, descending=True, stable=True))
    return order[:, :count]


def run(z, count, ids=torch.int64, extra=0, offset=0, tau=1.0):
    rows, classes = z.shape
    h = circ.circ_top_create(classes, count)
    circ.circ_top_set_dtypes(h, CODE[z.dtype], CODE[ids])
    circ.circ_top_set_temperature(h, tau)
    zd = strided(z, classes + extra, offset)
    values, values_ok = guarded((rows, count), z.dtype)
    which, which_ok = guarded((rows, count), ids)
    lse, lse_ok = guarded((rows,), F32)
    circ.circ_top_forward(h, zd, classes + extra, values, which, lse, rows, torch.cuda.current_stream())
    again = [torch.empty_like(t) for t in (values, which, lse)]
    for i, t in enumerate(again):                # each alone
        circ.circ_top_forward(h, zd, classes + extra, *(t if j == i else None for j in range(3)), rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_top_destroy(h)
    for ok in (values_ok, which_ok, lse_ok):
        ok()
    as_bits = torch.int16 if z.dtype == BF16 else torch.int32
    assert torch.equal(again[0].view(as_bits), values.view(as_bits)) and torch.equal(again[1], which)
    assert torch.equal(again[2].view(torch.int32), lse.view(torch.int32))
    return values.cpu(), which.cpu().long(), lse.cpu()


def check(z, count, got, tau=1.0):
    values, which, lse = got
    want = plain(z, count)
    assert torch.equal(which, want)
    picked = z.gather(1, want)
    assert torch.equal(values.float().nan_to_num(7.5, 1e38, -1e38), picked.float().nan_to_num(7.5, 1e38, -1e38))
    zz = z.double() / tau
    ref = torch.logsumexp(zz, 1)
    top = zz.max(1, keepdim=True).values
    spread = (top - torch.where(zz == -torch.inf, top, zz)).max(1).values
    fine = torch.isfinite(zz).any(1) & torch.isfinite(top[:, 0])
    bound = 1.1 * ((2 + 3 * spread) + z.shape[1] / 32 + 16) * U + 2 * U * ref.abs()
    within(lse[fine], ref[fine], bound[fine])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,count", SHAPES)
@pytest.mark.parametrize("dtype,ids,extra,offset,tau", [(F32, torch.int64, 0, 0, 1.0), (BF16, torch.int32, 0, 0, 2.0), (BF16, torch.int64, 5, 3, 1.0),
                                                        (F32, torch.int32, 3, 1, 0.7), (BF16, torch.int32, 8, 0, 4.0)])
def test_random_rows(rows, classes, count, dtype, ids, extra, offset, tau):
    z = (3 * torch.randn(rows, classes, generator=rng(rows + classes))).to(dtype)
    check(z, count, run(z, count, ids, extra, offset, tau), tau)


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [100, 1000, 3001, 20000, 50001, 120000])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("count", [1, 40, 256])
def test_rows_in_every_order(classes, dtype, count):
    count = min(count, classes)
    g = rng(classes)
    n = torch.arange(classes, dtype=torch.float64)
    rows = [n / 7, -n / 7, torch.zeros(classes), torch.full((classes,), -2.5), (n % 3), (n % 17) * (n > classes // 2), -(n % 2) * 0.0,
            torch.where(n < count // 2, n, -torch.inf),                         # fewer left than are asked for
            torch.where((n >= classes // 3) & (n < classes // 3 + 2 * count), 50 + n % 5, torch.randn(classes, generator=g)),     # all of them side by side
            torch.where(n % 64 == 5, 9.0, torch.randn(classes, generator=g)),     # all of them the same, far apart
            torch.full((classes,), -torch.inf), torch.full((classes,), torch.finfo(dtype).min),
            torch.where(n == classes - 1, torch.finfo(dtype).max, torch.finfo(dtype).min),
            torch.where(n % 2 == 0, -0.0, 0.0), torch.where(n < 3, 1e-40, -1e-40)]
    z = torch.stack([r.double() for r in rows]).to(dtype)
    check(z, count, run(z, count, torch.int32, extra=1), 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,count", [(1480, 1000, 1), (1500, 2870, 20), (1501, 5001, 64), (1600, 520, 33), (400, 30000, 8), (300, 30000, 200),
                                                (1, 700000, 40), (47, 600000, 3), (48, 600000, 3)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["random", "few_values", "rising", "mostly_masked"])
def test_many_rows_and_the_longest(rows, classes, count, dtype, kind):
    n = torch.arange(classes)
    if kind == "rising":
        z = (n / 7 + torch.arange(rows)[:, None]).float()
    else:
        z = 3 * torch.randn(rows, classes, generator=rng(classes))
    if kind == "few_values":
        z = torch.round(z)
    if kind == "mostly_masked":
        z[::2, n % 97 != 5] = -torch.inf
        z[1::2, n % 89 != 7] = torch.finfo(dtype).min
        z[::7] = -torch.inf
        z[3:4, 11] = float("nan")
    z = z.to(dtype)
    got = run(z, count, tau=2.0)
    check(z, count, got, 2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [30, 2048, 40001, 150000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_with_nothing_left_and_values_that_are_not_finite(classes, dtype):
    z = torch.randn(6, classes, generator=rng(2)).to(dtype)
    z[1] = -torch.inf
    z[2, [3, 20]] = float("nan")
    z[3, classes - 1] = float("inf")
    z[4] = float("nan")
    z[5, ::2] = float("inf")
    got = run(z, 20)
    check(z, 20, got)
    lse = got[2]
    assert bool(torch.isfinite(lse[0])) and lse[1] == -torch.inf and bool(lse[2].isnan()) and bool(lse[4].isnan())
    assert not bool(torch.isfinite(lse[3])) and not bool(torch.isfinite(lse[5]))


@pytest.mark.gpu
def test_no_rows_other_streams_and_the_same_bits_again():
    h = circ.circ_top_create(10, 3)
    circ.circ_top_forward(h, None, 10, None, None, None, 0, torch.cuda.current_stream())
    circ.circ_top_destroy(h)
    z = torch.randn(37, 30011, generator=rng(5))
    first = run(z, 33)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = run(z, 33)
    for a, b in zip(first, second):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(1, 131072), (50, 1000), (300, 30000), (3, 400)])
def test_captured_graph(rows, classes):
    z = torch.randn(rows, classes, generator=rng(9))
    h = circ.circ_top_create(classes, 17)
    circ.circ_top_reserve(h, rows)
    zd = device(z)
    values, ids, lse = torch.zeros(rows, 17, device="cuda"), torch.zeros(rows, 17, dtype=torch.int64, device="cuda"), torch.zeros(rows, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_top_forward(h, zd, classes, values, ids, lse, rows, torch.cuda.current_stream())
    for seed in (9, 10):
        z = torch.randn(rows, classes, generator=rng(seed))
        zd.copy_(z)
        circ.circ_top_reserve(h, 4 * rows)             # what the graph holds stays
        graph.replay()
        torch.cuda.synchronize()
        check(z, 17, (values.cpu(), ids.cpu(), lse.cpu()))
    del graph
    circ.circ_top_destroy(h)


def refused(code, call, *args):
    with pytest.raises(circ.CircError) as e:
        call(*args)
    assert e.value.code == code


def test_refusals_before_any_device_call():
    for args in ((0, 1), (10, 0), (10, 11), (1000, 257), ((1 << 28) + 1, 1)):
        refused(circ.CIRC_ERR_SHAPE, circ.circ_top_create, *args)
    for call, args in ((circ.circ_top_forward, (None, 64, 8, 64, 64, 64, 1)), (circ.circ_top_set_dtypes, (None, 0, 0)),
                       (circ.circ_top_set_temperature, (None, 1.0)), (circ.circ_top_reserve, (None, 1))):
        refused(circ.CIRC_ERR_ARG, call, *args)
    circ.circ_top_destroy(None)


@pytest.mark.gpu
def test_refusals_of_bad_arguments():
    h = circ.circ_top_create(16, 4)
    z, v, i = torch.empty(4, 16, device="cuda"), torch.empty(4, 4, device="cuda"), torch.empty(4, 4, dtype=torch.int64, device="cuda")
    try:
        refused(circ.CIRC_ERR_ARG, circ.circ_top_set_dtypes, h, circ.CIRC_E4M3, 0)
        refused(circ.CIRC_ERR_ARG, circ.circ_top_set_dtypes, h, 0, 2)
        for tau in (0.0, -1.0, float("nan"), float("inf")):
            refused(circ.CIRC_ERR_ARG, circ.circ_top_set_temperature, h, tau)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_top_forward, h, z, 15, v, i, None, 4)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_top_forward, h, z, 16, v, i, None, -1)
        refused(circ.CIRC_ERR_ARG, circ.circ_top_forward, h, z, 16, None, None, None, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_top_forward, h, None, 16, v, i, None, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_top_forward, h, z.data_ptr() + 2, 16, v, i, None, 1)
        refused(circ.CIRC_ERR_ARG, circ.circ_top_forward, h, z, 16, v, i.data_ptr() + 4, None, 1)
    finally:
        circ.circ_top_destroy(h)
