"""Group norm with an activation, channels last, against the formulas in 64 bits: one pixel to many, groups of one channel to all, odd channel
counts, types that differ, large offsets, in place, unaligned; gradients against the formulas and against differences; refusals.

Bounds (u: unit roundoff of float32, P pixels, D channels a group): the terms of a channel's sum are at most P, those of a group are joined in
float64.  mean: (P + 8) u of the largest |x - x'| in the group; variance: relative (2 P + 8) u; a value v = (x - mean) rstd gain + bias takes
both and four roundings; the activations have slopes of at most 1.1, sigmoid(v) a relative error of (4 + 2 |v|) u."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, U, device, guarded, rng, rounding, small, within

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
EPS = 1e-5
NONE, RELU, SILU = circ.CIRC_ACT_NONE, circ.CIRC_ACT_RELU, circ.CIRC_ACT_SILU
SHAPES = [(1, 1, 1, 8, 2), (2, 1, 1, 8, 8), (1, 5, 7, 16, 4), (3, 4, 4, 6, 3), (2, 9, 11, 60, 12), (1, 28, 28, 256, 32), (4, 13, 13, 64, 1), (2, 33, 17, 40, 5),
          (5, 3, 2, 1, 1), (1, 2, 3, 1025, 5), (70, 2, 2, 32, 4), (2, 40, 40, 8, 2), (3, 30, 30, 96, 32), (1, 90, 75, 24, 3), (2, 6, 6, 4096, 16)]


def act(v, kind):
    return v if kind == NONE else v.clamp(min=0) if kind == RELU else v * torch.sigmoid(v)


def slope(v, kind):
    if kind == NONE:
        return torch.ones_like(v)
    if kind == RELU:
        return (v > 0).double()
    s = torch.sigmoid(v)
    return s * (1 + v * (1 - s))


def grouped(x, groups):
    n, h, w, c = x.shape
    return x.double().view(n, h * w, groups, c // groups)


def plain(x, gain, bias, groups, kind, eps=EPS):
    g = grouped(x, groups)
    mean = g.mean((1, 3))
    d = g - mean[:, None, :, None]
    var = (d * d).mean((1, 3))
    rstd = 1 / torch.sqrt(var + eps)
    shape = (1, 1, groups, -1)
    t = d * rstd[:, None, :, None] * gain.double().view(shape)
    v = t + bias.double().view(shape)
    # bounds
    p = g.shape[1]
    reach = (g.amax((1, 3)) - g.amin((1, 3)))
    mean_err = (p + 8) * U * reach + U * mean.abs()
    rstd_err = ((2 * p + 8) * U * var / (var + eps) + 2 * (p + 8) ** 2 * U * U * reach ** 2 / (var + eps)) * rstd + U * rstd
    v_err = gain.double().abs().view(shape) * (rstd * mean_err)[:, None, :, None] + t.abs() * (rstd_err / rstd + 4 * U)[:, None, :, None] + U * v.abs()
    return dict(mean=mean, rstd=rstd, v=v, y=act(v, kind), mean_err=mean_err, rstd_err=rstd_err, v_err=v_err)


def draw(n, h, w, c, dtype, seed, offset=1.0):
    g = rng(seed)
    x = (1.5 * torch.randn(n, h, w, c, generator=g) + offset * torch.randn(c, generator=g)).to(dtype)
    return x, 1 + 0.3 * torch.randn(c, generator=g), 0.3 * torch.randn(c, generator=g)


def handle(c, groups, x_dtype, y_dtype, kind, eps=EPS):
    h = circ.circ_gnorm_create(c, groups, eps)
    circ.circ_gnorm_set_dtypes(h, CODE[x_dtype], CODE[y_dtype])
    circ.circ_gnorm_set_activation(h, kind)
    return h


def forward(x, gain, bias, groups, kind, y_dtype, offset=0, eps=EPS, stats=True):
    n, hh, w, c = x.shape
    h = handle(c, groups, x.dtype, y_dtype, kind, eps)
    xd = device(x, offset)
    y, y_ok = guarded(x.shape, y_dtype, offset)
    mean, mean_ok = guarded((n, groups), F32)
    rstd, rstd_ok = guarded((n, groups), F32)
    gd, bd = (None if t is None else device(t, offset) for t in (gain, bias))
    circ.circ_gnorm_forward(h, xd, gd, bd, y, mean if stats else None, rstd if stats else None, n, hh, w, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_gnorm_destroy(h)
    for ok in (y_ok, mean_ok, rstd_ok):
        ok()
    assert torch.equal(xd.cpu().view(torch.int16 if x.dtype == BF16 else torch.int32), x.view(torch.int16 if x.dtype == BF16 else torch.int32))
    return y.cpu(), mean.cpu(), rstd.cpu()


def check(x, gain, bias, groups, kind, got, eps=EPS):
    ref = plain(x, gain, bias, groups, kind, eps)
    y, mean, rstd = got
    within(mean, ref["mean"], ref["mean_err"])
    within(rstd, ref["rstd"], ref["rstd_err"])
    want = ref["y"].reshape(x.shape)
    err = 1.1 * ref["v_err"] + (ref["y"].abs() * (4 + 2 * ref["v"].abs()) * U if kind == SILU else 0.0)
    within(y, want, err.reshape(x.shape) + rounding(y.dtype) * want.abs() * (1 + 2 ** -7) + small(y.dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype,kind,offset", [(F32, F32, NONE, 0), (BF16, BF16, RELU, 0), (BF16, F32, SILU, 0), (F32, BF16, RELU, 0), (F32, F32, SILU, 1),
                                                         (BF16, BF16, SILU, 3), (BF16, BF16, NONE, 0)])
def test_forward(n, h, w, c, groups, x_dtype, y_dtype, kind, offset):
    x, gain, bias = draw(n, h, w, c, x_dtype, n + h + w + c)
    check(x, gain, bias, groups, kind, forward(x, gain, bias, groups, kind, y_dtype, offset))


def backward(x, gain, bias, mean, rstd, grad_y, groups, kind, offset=0, only=None, place=None):
    n, hh, w, c = x.shape
    h = handle(c, groups, x.dtype, grad_y.dtype, kind)
    xd, gyd = device(x, offset), device(grad_y, offset)
    gx, gx_ok = guarded(x.shape, x.dtype, offset)
    gg, gg_ok = guarded((c,), F32)
    gb, gb_ok = guarded((c,), F32)
    gd, bd, md, rd = (None if t is None else device(t, offset) for t in (gain, bias, mean, rstd))
    outs = [gx, gg, gb]
    if place == "grad_y":
        outs[0] = gyd
    if place == "x":
        outs[0] = xd
    if only is not None:
        outs = [t if i == only else None for i, t in enumerate(outs)]
    circ.circ_gnorm_backward(h, xd, gd, bd, md, rd, gyd, *outs, n, hh, w, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_gnorm_destroy(h)
    for ok in (gx_ok, gg_ok, gb_ok):
        ok()
    return [None if t is None else t.cpu() for t in outs]


def plain_backward(x, gain, bias, mean, rstd, grad_y, groups, kind):
    """The gradients from a given mean and rstd, with their bounds."""
    n, hh, w, c = x.shape
    shape = (1, 1, groups, -1)
    ga, be = gain.double().view(shape), bias.double().view(shape)
    r = rstd.double()[:, None, :, None]
    u = (grouped(x, groups) - mean.double()[:, None, :, None]) * r
    v = u * ga + be
    gy = grouped(grad_y, groups)
    g = gy * slope(v, kind)
    g_err = torch.zeros_like(g)
    if kind == SILU:
        v_err = U * (4 * (u * ga).abs() + 2 * v.abs())
        g_err = gy.abs() * (0.5 * v_err + (8 + 3 * v.abs()) * U * 1.1)
    p, d = u.shape[1], u.shape[3]
    m = p * d
    a, b = (ga * g).sum((1, 3), keepdim=True) / m, (ga * g * u).sum((1, 3), keepdim=True) / m
    u_err = 3 * U * u.abs()
    term_a, term_b = (p + 4) * U * g.abs() + g_err, ((p + 6) * U * (g * u).abs() + g_err * u.abs())
    a_err, b_err = (ga.abs() * term_a).sum((1, 3), keepdim=True) / m + U * a.abs(), (ga.abs() * term_b).sum((1, 3), keepdim=True) / m + U * b.abs()
    gx = r * (ga * g - a - u * b)
    gx_err = r * (ga.abs() * g_err + a_err + u.abs() * b_err + u_err * b.abs() + 4 * U * ((ga * g).abs() + a.abs() + (u * b).abs()))
    sums = (g * u).sum((0, 1)).view(c), g.sum((0, 1)).view(c)
    errs = term_b.sum((0, 1)).view(c) + U * sums[0].abs(), term_a.sum((0, 1)).view(c) + U * sums[1].abs()
    return (gx.reshape(x.shape), *sums), (gx_err.reshape(x.shape), *errs)


def check_backward(args, got):
    refs, errs = plain_backward(*args)
    x = args[0]
    for i, (g, ref, err) in enumerate(zip(got, refs, errs)):
        if g is not None:
            within(g, ref, err + (rounding(x.dtype) * ref.abs() * (1 + 2 ** -7) + small(x.dtype) if i == 0 else U * ref.abs() + small(F32)))


def draw_backward(n, h, w, c, groups, x_dtype, y_dtype, kind, seed):
    x, gain, bias = draw(n, h, w, c, x_dtype, seed)
    ref = plain(x, gain, bias, groups, kind)
    grad_y = (0.1 * torch.randn(n, h, w, c, generator=rng(seed + 1))).to(y_dtype)
    return x, gain, bias, ref["mean"].float(), ref["rstd"].float(), grad_y, groups, kind


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype,kind,offset", [(F32, F32, NONE, 0), (BF16, BF16, RELU, 0), (BF16, F32, SILU, 0), (F32, BF16, RELU, 0), (F32, F32, SILU, 1),
                                                         (BF16, BF16, SILU, 3), (BF16, BF16, NONE, 0)])
def test_backward(n, h, w, c, groups, x_dtype, y_dtype, kind, offset):
    args = draw_backward(n, h, w, c, groups, x_dtype, y_dtype, kind, n + h + w + c)
    got = backward(*args, offset=offset)
    check_backward(args, got)
    bits = torch.int16 if x_dtype == BF16 else torch.int32
    for i in range(3):                           # each alone: the same bits
        alone = backward(*args, offset=offset, only=i)[i]
        assert torch.equal(alone.view(bits if i == 0 else torch.int32), got[i].view(bits if i == 0 else torch.int32))


MANY = [(1800, 3, 3, 8, 2), (1776, 11, 12, 64, 8), (1775, 11, 12, 64, 8), (400, 12, 12, 64, 8), (2, 64, 64, 2048, 32), (2, 17, 19, 1028, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", MANY)
@pytest.mark.parametrize("dtype,kind", [(F32, SILU), (BF16, RELU), (BF16, SILU)])
def test_many_images_and_wide_pixels(n, h, w, c, groups, dtype, kind):
    x, gain, bias = draw(n, h, w, c, dtype, n + c)
    check(x, gain, bias, groups, kind, forward(x, gain, bias, groups, kind, dtype))
    args = draw_backward(n, h, w, c, groups, dtype, dtype, kind, n + c)
    check_backward(args, backward(*args))


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 9, 11, 60, 12), (1, 28, 28, 256, 32), (1, 90, 75, 24, 3), (3, 5, 5, 6, 2)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place(n, h, w, c, groups, dtype):
    x, gain, bias = draw(n, h, w, c, dtype, 31)
    y = forward(x, gain, bias, groups, SILU, dtype)[0]
    handle_ = handle(c, groups, dtype, dtype, SILU)
    xd, gd, bd = device(x), device(gain), device(bias)
    circ.circ_gnorm_forward(handle_, xd, gd, bd, xd, None, None, n, h, w, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(xd.cpu(), y)
    circ.circ_gnorm_destroy(handle_)
    args = draw_backward(n, h, w, c, groups, dtype, dtype, RELU, 32)
    want = backward(*args)
    for place in ("grad_y", "x"):
        for a, b in zip(backward(*args, place=place), want):
            assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,groups", [((2, 20, 20, 32), 4), ((1, 60, 60, 16), 2), ((1, 1, 3, 8), 8)])
def test_large_offsets_constant_groups_and_missing_parameters(shape, groups):
    """A mean a thousand times the deviation; groups whose values are all the same (variance 0: rstd is 1 / sqrt(eps)); no gain, no bias."""
    c = shape[-1]
    x, gain, bias = draw(*shape, F32, 3, offset=0.0)
    x += 1500.0
    x[..., :c // groups] = 3.25
    ones, zeros = torch.ones(c), torch.zeros(c)
    check(x, gain, bias, groups, NONE, forward(x, gain, bias, groups, NONE, F32))
    check(x, ones, zeros, groups, RELU, forward(x, None, None, groups, RELU, F32))
    got = forward(x, gain, bias, groups, NONE, F32)
    y, mean, rstd = got
    assert bool((mean[:, 0] == 3.25).all()) and torch.equal(y[..., :c // groups], bias[:c // groups].expand(*shape[:3], -1))
    alone = forward(x, gain, bias, groups, NONE, F32, stats=False)[0]
    assert torch.equal(alone, y)
    args = draw_backward(*shape, groups, F32, F32, SILU, 5)
    none = (args[0], None, None, *args[3:])
    plain_args = (args[0], ones, zeros, *args[3:])
    check_backward(plain_args, backward(*none))


@pytest.mark.gpu
def test_the_sides_of_a_relu_do_not_depend_on_rounding():
    """Values whose v is 0, or a few float32 roundings beside it: v = (x - mean) rstd gain + bias with a bias that cancels it."""
    n, h, w, c = 1, 64, 64, 32
    g = rng(8)
    x = torch.randn(n, h, w, c, generator=g)
    gain, mean, rstd = 1 + 0.3 * torch.randn(c, generator=g), torch.tensor([[0.3, -0.1]]), torch.tensor([[1.7, 0.9]])
    m, r = mean[0].repeat_interleave(16), rstd[0].repeat_interleave(16)
    base = x[0, 0, 0].clone()
    bias = -((base.double() - m.double()) * r.double() * gain.double()).float()
    steps = torch.randint(-3, 4, (n, h, w, c), generator=g)
    x = (base.view(torch.int32) + steps.int()).view(F32).clone()                     # neighbours of the value where v is 0
    grad_y = torch.ones(n, h, w, c)
    args = (x, gain, bias, mean, rstd, grad_y, 2, RELU)
    gx, gg, gb = backward(*args)
    v = (x.double() - m.double()) * (r.double() * gain.double()) + bias.double()
    assert torch.equal(gb.double(), (v > 0).double().sum((0, 1, 2)))                 # whole numbers: the sum is exact
    check_backward(args, (gx, gg, gb))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite_stay_in_their_groups(bad):
    n, h, w, c, groups = 2, 6, 7, 32, 4
    x, gain, bias = draw(n, h, w, c, F32, 11)
    clean = forward(x, gain, bias, groups, SILU, F32)
    x[1, 3, 2, 9] = bad
    y, mean, rstd = forward(x, gain, bias, groups, SILU, F32)
    assert bool(y[1, :, :, 8:16].isnan().any()) and not bool(torch.isfinite(mean[1, 1]))
    y[1, :, :, 8:16] = clean[0][1, :, :, 8:16]
    assert torch.equal(y, clean[0])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [NONE, RELU, SILU])
def test_gradients_are_the_derivatives(kind):
    n, h, w, c, groups = 2, 3, 5, 12, 3
    x, gain, bias = draw(n, h, w, c, F32, 13)
    ref = plain(x, gain, bias, groups, kind)
    if kind == RELU:            # away from the kink
        x = torch.where((ref["v"].abs() < 1e-2).view(x.shape), x + 0.1, x)
        ref = plain(x, gain, bias, groups, kind)
        assert float(ref["v"].abs().min()) > 1e-3
    grad_y = torch.randn(n, h, w, c, generator=rng(14))
    got = backward(x, gain, bias, ref["mean"].float(), ref["rstd"].float(), grad_y, groups, kind)

    def value(x, gain, bias):
        return float((plain(x, gain, bias, groups, kind)["y"].reshape(n, h, w, c) * grad_y.double()).sum())

    step = 1e-5
    for i, t in enumerate((x, gain, bias)):
        d = torch.randn(t.shape, generator=rng(15 + i), dtype=F64)
        three = [x.double(), gain.double(), bias.double()]
        lo, hi = list(three), list(three)
        lo[i], hi[i] = three[i] - step * d, three[i] + step * d
        numeric = (value(*hi) - value(*lo)) / (2 * step)
        mine = got[i].double() * d
        assert abs(float(mine.sum()) - numeric) <= 2e-5 * float(mine.abs().sum()), i


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", [(2, 9, 11, 60, 12), (3, 28, 28, 64, 8), (1, 90, 75, 24, 3)])
def test_captured_graph_and_another_stream(n, h, w, c, groups):
    x, gain, bias = draw(n, h, w, c, F32, 41)
    grad_y = 0.1 * torch.randn(n, h, w, c, generator=rng(42))
    want = forward(x, gain, bias, groups, SILU, F32)
    want_back = backward(x, gain, bias, want[1], want[2], grad_y, groups, SILU)
    hd = handle(c, groups, F32, F32, SILU)
    circ.circ_gnorm_reserve(hd, n, h, w)
    xd, gd, bd, gyd = (device(t) for t in (x, gain, bias, grad_y))
    y, gx = torch.zeros_like(xd), torch.zeros_like(xd)
    mean, rstd, gg, gb = torch.zeros(n, groups, device="cuda"), torch.zeros(n, groups, device="cuda"), torch.zeros(c, device="cuda"), torch.zeros(c, device="cuda")

    def calls():
        s = torch.cuda.current_stream()
        circ.circ_gnorm_forward(hd, xd, gd, bd, y, mean, rstd, n, h, w, s)
        circ.circ_gnorm_backward(hd, xd, gd, bd, mean, rstd, gyd, gx, gg, gb, n, h, w, s)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    circ.circ_gnorm_reserve(hd, 50 * n, h, w)              # what the graph holds stays
    other = torch.full((1 << 20,), float("nan"), device="cuda")

    def on_another_stream():
        with torch.cuda.stream(torch.cuda.Stream()):
            calls()

    for go in (graph.replay, graph.replay, calls, on_another_stream):
        for t in (y, gx, mean, rstd, gg, gb):
            t.zero_()
        torch.cuda.synchronize()
        go()
        torch.cuda.synchronize()
        for a, b in zip((y, mean, rstd, gx, gg, gb), (*want, *want_back)):
            assert torch.equal(a.cpu(), b)
    assert bool(other.isnan().all())
    del graph
    circ.circ_gnorm_destroy(hd)


@pytest.mark.gpu
def test_no_images_and_a_workspace_that_cannot_be_allocated():
    h = circ.circ_gnorm_create(8, 2, EPS)
    gg, gb = torch.full((8,), float("nan"), device="cuda"), torch.full((8,), float("nan"), device="cuda")
    circ.circ_gnorm_forward(h, None, None, None, None, None, None, 0, 4, 4, torch.cuda.current_stream())
    circ.circ_gnorm_backward(h, None, None, None, None, None, None, None, gg, gb, 0, 4, 4, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert bool((gg == 0).all()) and bool((gb == 0).all())
    try:
        circ.circ_debug_fail_alloc_after(1)
        refused(circ.CIRC_ERR_ALLOC, circ.circ_gnorm_reserve, h, 3, 8, 8)
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_gnorm_reserve(h, 3, 8, 8)
    finally:
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_gnorm_destroy(h)


def refused(code, call, *args):
    with pytest.raises(circ.CircError) as e:
        call(*args)
    assert e.value.code == code


def test_refusals_before_any_device_call():
    for args in ((0, 1, EPS), (8, 0, EPS), (8, 3, EPS), (8, 16, EPS), (8, 2, -1.0), (8, 2, float("nan")), (1 << 17, 1, EPS)):
        refused(circ.CIRC_ERR_SHAPE, circ.circ_gnorm_create, *args)
    for call, args in ((circ.circ_gnorm_forward, (None, 64, None, None, 64, None, None, 1, 1, 1)),
                       (circ.circ_gnorm_backward, (None, 64, None, None, 64, 64, 64, 64, None, None, 1, 1, 1)),
                       (circ.circ_gnorm_set_dtypes, (None, 0, 0)), (circ.circ_gnorm_set_activation, (None, 0)), (circ.circ_gnorm_reserve, (None, 1, 1, 1))):
        refused(circ.CIRC_ERR_ARG, call, *args)
    circ.circ_gnorm_destroy(None)


@pytest.mark.gpu
def test_refusals_of_bad_arguments():
    h = circ.circ_gnorm_create(8, 2, EPS)
    x, y, m = torch.empty(2, 3, 3, 8, device="cuda"), torch.empty(2, 3, 3, 8, device="cuda"), torch.empty(2, 2, device="cuda")
    try:
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_set_dtypes, h, circ.CIRC_E4M3, 0)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_set_activation, h, 3)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_set_activation, h, -1)
        for sizes in ((-1, 3, 3), (2, 0, 3), (2, 3, 0), (2, 1 << 15, 1 << 14)):
            refused(circ.CIRC_ERR_SHAPE, circ.circ_gnorm_forward, h, x, None, None, y, None, None, *sizes)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_forward, h, None, None, None, y, None, None, 2, 3, 3)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_forward, h, x, None, None, None, None, None, 2, 3, 3)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_forward, h, x.data_ptr() + 2, None, None, y, None, None, 1, 3, 3)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_forward, h, x, m.data_ptr() + 1, None, y, None, None, 1, 3, 3)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_backward, h, x, None, None, None, m, y, x, None, None, 2, 3, 3)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_backward, h, x, None, None, m, m, y, None, None, None, 2, 3, 3)
        circ.circ_gnorm_set_dtypes(h, circ.CIRC_F32, circ.CIRC_BF16)
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_forward, h, x, None, None, x, None, None, 2, 3, 3)          # in place, another type
        refused(circ.CIRC_ERR_ARG, circ.circ_gnorm_backward, h, x, None, None, m, m, y, y, None, None, 2, 3, 3)
        with pytest.raises(AssertionError):
            circ.circ_gnorm_forward(h, x.transpose(1, 3), None, None, y, None, None, 2, 3, 3)
    finally:
        circ.circ_gnorm_destroy(h)
