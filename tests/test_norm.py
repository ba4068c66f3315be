"""RMS norm with the residual's addition, its 8-bit output and its gradients against the formulas in 64 bits: one element to
long rows, odd widths, unaligned buffers, rows of zeros, in-place sums, values that are not finite; refusals.

Bounds (u: unit roundoff of float32).  A float32 sum over a row of d terms by at least 32 lanes has chains of at most
d / 32 + 16 additions, so sums of squares (all positive) have a relative error of at most c = (d / 32 + 16) u and rstd of
c / 2 + 4 u.  The other bounds follow through the formulas; each result is rounded once to its type."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, U, device, guarded, rng, rounding, small, within

F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
EPS = 1e-5
SHAPES = [(1, 1), (1, 4096), (3, 31), (5, 64), (2, 250), (17, 1001), (9, 1024), (4, 2056), (3, 8200), (2, 20000), (300, 96), (3, 40000), (700, 2048)]


def handle(dim, x, y, group=0, eps=EPS):
    h = circ.circ_norm_create(dim, eps)
    circ.circ_norm_set_dtypes(h, CODE[x], CODE[y])
    circ.circ_norm_set_group(h, group)
    return h


def chain(dim):
    return (dim / 32 + 16) * U


def plain_forward(x, residual, gain, eps=EPS):
    s = x.double() + (residual.double() if residual is not None else 0.0)
    rstd = 1 / torch.sqrt((s * s).mean(1) + float(torch.tensor(eps, dtype=F32)))
    return s, rstd, s * rstd[:, None] * (gain.double() if gain is not None else 1.0)


def inputs(rows, dim, x_dtype, residual, gain, seed):
    g = rng(seed)
    x = torch.randn(rows, dim, generator=g).to(x_dtype)
    r = (2 * torch.randn(rows, dim, generator=g)).to(x_dtype) if residual else None
    w = 1 + 0.2 * torch.randn(dim, generator=g) if gain else None
    return x, r, w


def on_device(t, offset=0):
    return None if t is None else device(t, offset)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype,residual,gain,offset", [(F32, F32, True, True, 0), (BF16, BF16, True, True, 0), (BF16, F32, False, True, 0),
                                                                  (F32, BF16, False, False, 1), (BF16, BF16, True, False, 3)])
def test_forward(rows, dim, x_dtype, y_dtype, residual, gain, offset):
    x, r, w = inputs(rows, dim, x_dtype, residual, gain, rows + dim)
    h = handle(dim, x_dtype, y_dtype)
    y, y_ok = guarded((rows, dim), y_dtype, offset)
    s, s_ok = guarded((rows, dim), x_dtype, offset)
    rstd, rstd_ok = guarded((rows,), F32)
    circ.circ_norm_forward(h, device(x, offset), on_device(r, offset), on_device(w, offset), s, y, None, rstd, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    for ok in (y_ok, s_ok, rstd_ok):
        ok()
    s_ref, rstd_ref, y_ref = plain_forward(x, r, w)
    # one rounding of the sum to float32 (relative to the sum), then one to its type
    within(s, s_ref, (U + rounding(x_dtype)) * s_ref.abs() + small(x_dtype))
    c = chain(dim) / 2 + 6 * U
    within(rstd, rstd_ref, c * rstd_ref)
    within(y, y_ref, (c + 4 * U + rounding(y_dtype)) * y_ref.abs() + small(y_dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim,group", [(1, 32, 32), (3, 4096, 128), (7, 192, 64), (5, 1001, 0), (2, 9216, 128), (3, 9216, 0), (2, 20000, 32),
                                            (40, 96, 32), (1, 1, 0), (2, 24576, 64)])
@pytest.mark.parametrize("x_dtype,residual,offset", [(BF16, True, 0), (F32, False, 0), (F32, True, 1)])
def test_eight_bits(rows, dim, group, x_dtype, residual, offset):
    x, r, w = inputs(rows, dim, x_dtype, residual, True, rows * 7 + dim)
    x[0, : dim // 2] = 0                          # groups of nothing but zeros
    if residual:
        r[0, : dim // 2] = 0
    h = handle(dim, x_dtype, E4M3, group)
    width = group or dim
    q, q_ok = guarded((rows, dim), E4M3, offset)
    scale, scale_ok = guarded((rows, dim // width), F32)
    circ.circ_norm_forward(h, device(x, offset), on_device(r, offset), device(w), None, q, scale, None, rows, torch.cuda.current_stream())
    out = torch.full((rows, dim), float("nan"), device="cuda")
    circ.circ_norm_unpack(h, q, scale, out, circ.CIRC_F32, rows, torch.cuda.current_stream())
    out16 = torch.full((rows, dim), float("nan"), device="cuda", dtype=BF16)
    circ.circ_norm_unpack(h, q, scale, out16, circ.CIRC_BF16, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    q_ok()
    scale_ok()
    _, _, y = plain_forward(x, r, w)
    blocks = y.view(rows, -1, width)
    top = blocks.abs().amax(2)
    want = torch.where(top > 0, top / 448, 1.0)
    c = chain(dim) / 2 + 12 * U
    within(scale, want, c * want)
    # the stored value is the nearest e4m3 number (3 bits behind the point: 1/16 relative, 2^-10 below 2^-6) of a quotient
    # that is itself off by twice c
    ratio = blocks / want[:, :, None]
    within(q.float().view_as(blocks), ratio, (1 / 16 + 4 * c) * ratio.abs() + 2.0 ** -10)
    got = (q.double().cpu().view_as(blocks) * scale.double().cpu()[:, :, None]).view(rows, dim)
    within(out, got, U * got.abs())
    within(out16, got, (rounding(BF16) + U) * got.abs())
    assert float(q.float().abs().max()) <= 448


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim,group", [(64, 4096, 128), (100, 1001, 0), (200, 64, 32), (2, 20000, 32)])
@pytest.mark.parametrize("x_dtype,offset", [(BF16, 0), (F32, 1)])
def test_eight_bits_are_the_nearest(rows, dim, group, x_dtype, offset):
    """Codes lie at half their spacing from the quotient at most, but for what the norm (c) and the inverse of the scale are off by."""
    x, r, w = inputs(rows, dim, x_dtype, True, True, dim)
    h = handle(dim, x_dtype, E4M3, group)
    width = group or dim
    q, scale = torch.empty(rows, dim, device="cuda", dtype=E4M3), torch.empty(rows, dim // width, device="cuda")
    circ.circ_norm_forward(h, device(x, offset), device(r, offset), device(w), None, q, scale, None, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    _, _, y = plain_forward(x, r, w)
    ratio = y.view(rows, -1, width) / scale.double().cpu()[:, :, None]
    half = torch.exp2(torch.floor(torch.log2(ratio.abs().clamp(min=2.0 ** -6))) - 4)        # 3 bits behind the point; 2^-10 below 2^-6
    within(q.float().view_as(ratio), ratio, half + (chain(dim) / 2 + 12 * U) * ratio.abs())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype,carry,gain,offset", [(F32, F32, True, True, 0), (BF16, BF16, True, True, 0), (BF16, F32, False, True, 0),
                                                               (F32, BF16, False, False, 1), (F32, E4M3, True, True, 0)])
def test_backward(rows, dim, x_dtype, y_dtype, carry, gain, offset):
    g = rng(rows * 3 + dim)
    s = (2 * torch.randn(rows, dim, generator=g)).to(x_dtype)
    grad_dtype = x_dtype if y_dtype == E4M3 else y_dtype
    dy = torch.randn(rows, dim, generator=g).to(grad_dtype)
    ds = torch.randn(rows, dim, generator=g).to(x_dtype) if carry else None
    w = 1 + 0.2 * torch.randn(dim, generator=g) if gain else None
    rstd = torch.rsqrt((s.float() ** 2).mean(1) + EPS)
    h = handle(dim, x_dtype, y_dtype)
    dx, dx_ok = guarded((rows, dim), x_dtype, offset)
    dg, dg_ok = guarded((dim,), F32, offset)
    args = (device(s, offset), on_device(w, offset), device(rstd), device(dy, offset), on_device(ds, offset))
    circ.circ_norm_backward(h, *args, dx, dg, rows, torch.cuda.current_stream())
    dx_alone, dg_alone = torch.empty_like(dx), torch.empty_like(dg)
    circ.circ_norm_backward(h, *args, dx_alone, None, rows, torch.cuda.current_stream())
    circ.circ_norm_backward(h, *args, None, dg_alone, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    dx_ok()
    dg_ok()
    assert torch.equal(dx, dx_alone) and torch.equal(dg, dg_alone)
    k = rstd.double()[:, None]
    unit = s.double() * k
    u = dy.double() * (w.double() if gain else 1.0)
    mean = (u * unit).mean(1, keepdim=True)
    ref = k * (u - unit * mean) + (ds.double() if carry else 0.0)
    # three roundings in u, four in unit * mean, whose mean is off by c times the mean of magnitudes; two in the difference and
    # the product, one in the addition
    size = k * (6 * U * u.abs() + unit.abs() * (8 * U * mean.abs() + (chain(dim) + 4 * U) * (u * unit).abs().mean(1, keepdim=True)))
    within(dx, ref, size + 2 * U * ref.abs() + (3 * U * ds.double().abs() if carry else 0.0) + rounding(x_dtype) * ref.abs() + small(x_dtype))
    terms = dy.double() * unit
    within(dg, terms.sum(0), (rows + 4) * U * terms.abs().sum(0) + 1e-40)


# Rows enough that a launch has four of them in a block (at least 592), that a thread has 2, 4 or 8 vectors of a row (more than 148 rows, or
# long ones), and that a block of the backward pass walks over more rows than its ring holds (4 rows, at most 592 blocks).
MANY = [(700, 96), (700, 97), (700, 31), (200, 300), (200, 301), (200, 1001), (200, 2047), (150, 9001), (150, 16001), (150, 20001)]
WALKS = [(5000, 96), (5000, 97), (3000, 1001), (2600, 2056), (1500, 2047), (150, 5001), (200, 8201), (150, 9001), (150, 20001)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim", MANY)
@pytest.mark.parametrize("x_dtype,y_dtype,residual,gain", [(F32, F32, True, True), (BF16, BF16, True, True), (BF16, F32, False, False)])
def test_forward_of_many_rows(rows, dim, x_dtype, y_dtype, residual, gain):
    test_forward(rows, dim, x_dtype, y_dtype, residual, gain, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim,group", [(700, 96, 32), (700, 97, 0), (700, 64, 64), (200, 1001, 0), (200, 2048, 128), (150, 9001, 0), (150, 20001, 0)])
@pytest.mark.parametrize("x_dtype", [BF16, F32])
def test_eight_bits_of_many_rows(rows, dim, group, x_dtype):
    test_eight_bits(rows, dim, group, x_dtype, True, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim", WALKS)
@pytest.mark.parametrize("x_dtype,y_dtype,carry,gain", [(F32, F32, True, True), (BF16, BF16, True, True), (BF16, F32, False, True)])
def test_backward_of_many_rows(rows, dim, x_dtype, y_dtype, carry, gain):
    test_backward(rows, dim, x_dtype, y_dtype, carry, gain, 0)


@pytest.mark.gpu
def test_gradients_are_the_derivatives_of_the_forward_pass():
    rows, dim = 6, 50
    x, r, w = inputs(rows, dim, F32, True, True, 11)
    g = rng(12)
    dy, ds = torch.randn(rows, dim, generator=g), torch.randn(rows, dim, generator=g)
    h = handle(dim, F32, F32)
    s, y, rstd = torch.empty(rows, dim, device="cuda"), torch.empty(rows, dim, device="cuda"), torch.empty(rows, device="cuda")
    dx, dg = torch.empty_like(s), torch.empty(dim, device="cuda")
    wd = device(w)
    circ.circ_norm_forward(h, device(x), device(r), wd, s, y, None, rstd, rows, torch.cuda.current_stream())
    circ.circ_norm_backward(h, s, wd, rstd, device(dy), device(ds), dx, dg, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)

    def value(x, w):
        s, _, y = plain_forward(x, r, w)
        return float((y * dy.double()).sum() + (s * ds.double()).sum())

    step = 1e-4                                       # central differences in 64 bits: error step^2 times third derivatives
    for got, slope in ((dx, lambda v: (value(x.double() + step * v, w) - value(x.double() - step * v, w)) / (2 * step)),
                       (dg, lambda v: (value(x, w.double() + step * v) - value(x, w.double() - step * v)) / (2 * step))):
        v = torch.randn(got.shape, generator=g, dtype=torch.float64)
        mine = got.double().cpu() * v
        assert abs(float(mine.sum()) - slope(v)) <= 1e-5 * float(mine.abs().sum())


@pytest.mark.gpu
@pytest.mark.parametrize("y_dtype,dim", [(BF16, 1024), (E4M3, 1024), (F32, 1001), (E4M3, 20000), (BF16, 20000)])
@pytest.mark.parametrize("into", ["x", "residual"])
def test_sum_in_place(y_dtype, dim, into):
    rows = 5
    x, r, w = inputs(rows, dim, BF16, True, True, dim)
    h = handle(dim, BF16, y_dtype)
    results = []
    for place in (None, into):
        xd, rd = device(x), device(r)
        s = torch.empty_like(xd) if place is None else xd if place == "x" else rd
        y = torch.empty(rows, dim, device="cuda", dtype=y_dtype)
        scale = torch.empty(rows, 1, device="cuda") if y_dtype == E4M3 else None
        circ.circ_norm_forward(h, xd, rd, device(w), s, y, scale, None, rows, torch.cuda.current_stream())
        torch.cuda.synchronize()
        results.append((s.float(), y.float()))
    circ.circ_norm_destroy(h)
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])


@pytest.mark.gpu
def test_gradient_in_the_place_of_the_one_that_flows_past():
    rows, dim = 9, 1032
    g = rng(3)
    s, dy, ds = (torch.randn(rows, dim, generator=g).to(BF16) for _ in range(3))
    rstd = torch.rsqrt((s.float() ** 2).mean(1) + EPS)
    h = handle(dim, BF16, BF16)
    dx, carry = torch.empty(rows, dim, device="cuda", dtype=BF16), device(ds)
    circ.circ_norm_backward(h, device(s), None, device(rstd), device(dy), carry, dx, None, rows, torch.cuda.current_stream())
    circ.circ_norm_backward(h, device(s), None, device(rstd), device(dy), carry, carry, None, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    assert torch.equal(dx, carry)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim,dtype", [(5000, 97, BF16), (3000, 1001, F32), (200, 8201, BF16)])
def test_gradient_of_shared_vectors_in_the_place_of_the_one_that_flows_past(rows, dim, dtype):
    """Neighbouring rows share a vector, and other blocks have them."""
    g = rng(4)
    s, dy, ds = (torch.randn(rows, dim, generator=g).to(dtype) for _ in range(3))
    rstd = torch.rsqrt((s.float() ** 2).mean(1) + EPS)
    w = 1 + 0.2 * torch.randn(dim, generator=g)
    h = handle(dim, dtype, dtype)
    dx, carry = torch.empty(rows, dim, device="cuda", dtype=dtype), device(ds)
    dg, dg2 = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    args = (device(s), device(w), device(rstd), device(dy))
    circ.circ_norm_backward(h, *args, carry, dx, dg, rows, torch.cuda.current_stream())
    circ.circ_norm_backward(h, *args, carry, carry, dg2, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    assert torch.equal(dx, carry) and torch.equal(dg, dg2)


@pytest.mark.gpu
def test_rows_of_zeros_and_values_that_are_not_finite():
    dim = 256
    x = torch.randn(4, dim, generator=rng(1))
    x[1] = 0
    x[2, 5] = float("inf")
    x[3, 200] = float("nan")
    h = handle(dim, F32, F32)
    y, rstd = torch.empty(4, dim, device="cuda"), torch.empty(4, device="cuda")
    circ.circ_norm_forward(h, device(x), None, None, None, y, None, rstd, 4, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    y = y.cpu()
    assert bool(torch.isfinite(y[0]).all()) and bool((y[1] == 0).all())
    assert bool((y[2, :5] == 0).all()) and bool(y[2, 5].isnan())            # rstd of an infinite row is 0, and 0 * inf is NaN
    assert bool(y[3].isnan().all())
    h = handle(dim, F32, E4M3, 128)
    q, scale = torch.empty(4, dim, device="cuda", dtype=E4M3), torch.empty(4, 2, device="cuda")
    circ.circ_norm_forward(h, device(x), None, None, None, q, scale, None, 4, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    scale, q = scale.cpu(), q.float().cpu()
    assert scale[1].tolist() == [1.0, 1.0] and bool((q[1] == 0).all())
    assert bool(scale[2, 0].isnan()) and bool((q[2, 128:] == 0).all()) and scale[2, 1] == 1.0
    assert bool(scale[3].isnan().all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim,offset", [(6, 31, 0), (6, 1024, 0), (700, 64, 0), (200, 1001, 0), (5, 4096, 1), (2, 40000, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size,eps", [(1e15, 1e-5), (1e-15, 0.0), (1e-24, 1e-30)])
def test_large_and_small_rows(rows, dim, offset, dtype, size, eps):
    """Every second row of this size, the others of size 1."""
    x, r, w = inputs(rows, dim, F32, True, True, dim)
    x[::2] *= size
    r[::2] *= size
    x, r = x.to(dtype), r.to(dtype)
    h = handle(dim, dtype, F32, eps=eps)
    y, s, rstd = torch.empty(rows, dim, device="cuda"), guarded((rows, dim), dtype, offset)[0], torch.empty(rows, device="cuda")
    circ.circ_norm_forward(h, device(x, offset), device(r, offset), device(w), s, y, None, rstd, rows, torch.cuda.current_stream())
    h8 = handle(dim, dtype, E4M3, eps=eps)
    q, scale, out = torch.empty(rows, dim, device="cuda", dtype=E4M3), torch.empty(rows, 1, device="cuda"), torch.empty(rows, dim, device="cuda")
    circ.circ_norm_forward(h8, device(x, offset), device(r, offset), device(w), None, q, scale, None, rows, torch.cuda.current_stream())
    circ.circ_norm_unpack(h8, q, scale, out, circ.CIRC_F32, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    circ.circ_norm_destroy(h8)
    _, rstd_ref, y_ref = plain_forward(x, r, w, eps)
    c = chain(dim) / 2 + 6 * U
    within(rstd, rstd_ref, c * rstd_ref)
    within(y, y_ref, (c + 4 * U + rounding(F32)) * y_ref.abs() + small(F32))
    within(out, y_ref, 1 / 16 * (1 + 2.0 ** -10) * y_ref.abs() + y_ref.abs().amax(1, keepdim=True) / 448 * 2.0 ** -9)


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [31, 1024, 40000])
def test_rows_beyond_the_range_of_their_squares(dim):
    """A sum of squares that float32 does not hold is infinite: rstd and the row are 0."""
    x = torch.randn(3, dim, generator=rng(9))
    x[1] *= 1e25
    h = handle(dim, F32, F32)
    y, rstd = torch.empty(3, dim, device="cuda"), torch.empty(3, device="cuda")
    circ.circ_norm_forward(h, device(x), None, None, None, y, None, rstd, 3, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    assert float(rstd[1]) == 0 and bool((y[1] == 0).all()) and bool((rstd[::2] > 0.3).all())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,dim,offset", [(6, 31, 0), (6, 1024, 0), (5, 4096, 1), (700, 1001, 0), (3, 9001, 0)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e12, 1e15, 1e-12, 1e-15])
def test_gradients_of_large_and_small_rows(rows, dim, offset, dtype, size):
    g = rng(dim + 5)
    s = torch.randn(rows, dim, generator=g)
    s[::2] *= size
    s = s.to(dtype)
    dy, w = torch.randn(rows, dim, generator=g).to(dtype), 1 + 0.2 * torch.randn(dim, generator=g)
    rstd = (1 / torch.sqrt((s.double() ** 2).mean(1))).float()
    h = handle(dim, dtype, dtype, eps=0.0)
    dx, dg = torch.empty(rows, dim, device="cuda", dtype=dtype), torch.empty(dim, device="cuda")
    circ.circ_norm_backward(h, device(s, offset), device(w), device(rstd), device(dy, offset), None, dx, dg, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    k = rstd.double()[:, None]
    unit = s.double() * k
    u = dy.double() * w.double()
    mean = (u * unit).mean(1, keepdim=True)
    ref = k * (u - unit * mean)
    bound = k * (6 * U * u.abs() + unit.abs() * (8 * U * mean.abs() + (chain(dim) + 4 * U) * (u * unit).abs().mean(1, keepdim=True)))   # as above
    within(dx, ref, bound + 2 * U * ref.abs() + rounding(dtype) * ref.abs() + small(dtype))
    terms = dy.double() * unit
    within(dg, terms.sum(0), (rows + 4) * U * terms.abs().sum(0) + 1e-40)


@pytest.mark.gpu
def test_no_rows():
    h = handle(64, F32, F32)
    circ.circ_norm_forward(h, None, None, None, None, None, None, None, 0)
    dg = torch.full((64,), float("nan"), device="cuda")
    circ.circ_norm_backward(h, None, None, None, None, None, None, dg, 0, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_norm_destroy(h)
    assert bool((dg == 0).all())


@pytest.mark.gpu
def test_captured_graph():
    rows, dim = 600, 512
    g = rng(8)
    s, dy = device(torch.randn(rows, dim, generator=g)), device(torch.randn(rows, dim, generator=g))
    rstd = torch.rsqrt((s ** 2).mean(1) + EPS)
    h = handle(dim, F32, F32)
    dx, dg = torch.zeros_like(s), torch.zeros(dim, device="cuda")
    circ.circ_norm_reserve(h)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_norm_backward(h, s, None, rstd, dy, None, dx, dg, rows, torch.cuda.current_stream())
    graph.replay()
    want_x, want_g = torch.empty_like(dx), torch.empty_like(dg)
    circ.circ_norm_backward(h, s, None, rstd, dy, None, want_x, want_g, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(dx, want_x) and torch.equal(dg, want_g)
    del graph
    circ.circ_norm_destroy(h)


@pytest.mark.gpu
def test_a_workspace_that_cannot_be_allocated():
    h = handle(64, F32, F32)
    try:
        circ.circ_debug_fail_alloc_after(1)
        refused(circ.CIRC_ERR_ALLOC, circ.circ_norm_reserve, h)
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_norm_reserve(h)
    finally:
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_norm_destroy(h)


def refused(code, call, *args):
    with pytest.raises(circ.CircError) as e:
        call(*args)
    assert e.value.code == code


def test_refusals_before_any_device_call():
    refused(circ.CIRC_ERR_SHAPE, circ.circ_norm_create, 0, EPS)
    refused(circ.CIRC_ERR_ARG, circ.circ_norm_create, 8, -1.0)
    refused(circ.CIRC_ERR_ARG, circ.circ_norm_create, 8, float("nan"))
    for call, args in ((circ.circ_norm_forward, (None, 64, None, None, None, 128, None, None, 1)),
                       (circ.circ_norm_backward, (None, 64, None, 64, 64, None, 128, None, 1)), (circ.circ_norm_set_dtypes, (None, 0, 0)),
                       (circ.circ_norm_set_group, (None, 0)), (circ.circ_norm_reserve, (None,)), (circ.circ_norm_unpack, (None, 64, 64, 128, 0, 1))):
        refused(circ.CIRC_ERR_ARG, call, *args)
    circ.circ_norm_destroy(None)


@pytest.mark.gpu
def test_refusals_of_bad_arguments():
    h = handle(96, F32, F32)
    a, b = torch.empty(4, 96, device="cuda"), torch.empty(4, 96, device="cuda")
    try:
        refused(circ.CIRC_ERR_ARG, circ.circ_norm_set_dtypes, h, circ.CIRC_E4M3, 0)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_norm_set_group, h, 64)                      # does not divide 96
        refused(circ.CIRC_ERR_SHAPE, circ.circ_norm_set_group, h, 48)
        refused(circ.CIRC_ERR_ARG, circ.circ_norm_forward, h, a, None, None, None, a, None, None, 4)       # y is x
        refused(circ.CIRC_ERR_ARG, circ.circ_norm_forward, h, a, None, None, None, None, None, None, 4)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_norm_forward, h, a, None, None, None, b, None, None, -1)
        refused(circ.CIRC_ERR_ARG, circ.circ_norm_forward, h, a.data_ptr() + 2, None, None, None, b, None, None, 1)
        refused(circ.CIRC_ERR_ARG, circ.circ_norm_backward, h, a, None, None, b, None, a, None, 4)         # no rstd
        refused(circ.CIRC_ERR_ARG, circ.circ_norm_backward, h, a, None, b, b, None, None, None, 4)         # nothing to compute
        refused(circ.CIRC_ERR_ARG, circ.circ_norm_unpack, h, a, b, None, circ.CIRC_F32, 4)
        circ.circ_norm_set_dtypes(h, circ.CIRC_F32, circ.CIRC_E4M3)
        refused(circ.CIRC_ERR_ARG, circ.circ_norm_forward, h, a, None, None, None, b, None, None, 4)       # no place for the scales
        with pytest.raises(AssertionError):
            circ.circ_norm_forward(h, a.t(), None, None, None, b, None, None, 4)
    finally:
        circ.circ_norm_destroy(h)
