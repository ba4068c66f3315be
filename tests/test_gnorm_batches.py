"""Group norm of batches whose images are walked in several pieces of several rounds, the last of them partial: the kernels of training batches.

The values are whole numbers (or quarters) whose float32 sums are exact, so that a pixel lost or counted twice shows: the gradients of gain and bias are compared for
equality, mean and rstd within 40 u (u: unit roundoff of float32) of the largest difference, or relative: a thread's quotients, the joining of at most 17
threads a channel and of a group's channels in float32, float64 behind it."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import U, rng, rounding, small, within
from test_gnorm import EPS, NONE, RELU, SILU, backward, check, check_backward, draw, draw_backward, forward, grouped

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
SHAPES = [(32, 29, 29, 256, 32), (16, 57, 55, 256, 8), (24, 61, 47, 60, 5), (12, 67, 67, 255, 15), (64, 33, 31, 63, 9), (6, 45, 43, 515, 5)]
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype", TYPES)
@pytest.mark.parametrize("kind", [NONE, RELU])
def test_statistics_of_whole_numbers(n, h, w, c, groups, x_dtype, y_dtype, kind):
    x = torch.randint(-3, 4, (n, h, w, c), generator=rng(n + c)).to(x_dtype)
    y, mean, rstd = forward(x, None, None, groups, kind, y_dtype)
    g = grouped(x, groups)
    m = g.mean((1, 3))
    d = g - m[:, None, :, None]
    var = (d * d).mean((1, 3))
    r = 1 / torch.sqrt(var + EPS)
    mean_err, rstd_err = 40 * U * 6 + 0 * m, 40 * U * r
    within(mean, m, mean_err)
    within(rstd, r, rstd_err)
    v = d * r[:, None, :, None]
    want = (v if kind == NONE else v.clamp(min=0)).reshape(x.shape)
    err = ((r * mean_err)[:, None, :, None] + v.abs() * 44 * U).reshape(x.shape)
    within(y, want, err + rounding(y_dtype) * want.abs() * (1 + 2 ** -7) + small(y_dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype", TYPES)
@pytest.mark.parametrize("kind", [NONE, RELU])
def test_gradients_of_whole_numbers(n, h, w, c, groups, x_dtype, y_dtype, kind):
    """mean 1/2, rstd 1/2: u are quarters; a bias of quarters, so that some v are 0."""
    g = rng(n + c + 1)
    x, grad_y = torch.randint(-3, 4, (n, h, w, c), generator=g).to(x_dtype), torch.randint(-2, 3, (n, h, w, c), generator=g).to(y_dtype)
    gain, bias = torch.ones(c), torch.randint(-3, 4, (c,), generator=g) / 4
    mean, rstd = torch.full((n, groups), 0.5), torch.full((n, groups), 0.5)
    gx, gg, gb = backward(x, gain, bias, mean, rstd, grad_y, groups, kind)
    u = (x.double() - 0.5) * 0.5
    slope = grad_y.double() * (1.0 if kind == NONE else (u + bias.double() > 0).double())
    assert torch.equal(gb.double(), slope.sum((0, 1, 2)))
    assert torch.equal(gg.double(), (slope * u).sum((0, 1, 2)))
    s, t = grouped(slope, groups), grouped(u, groups)
    a, b = s.mean((1, 3), keepdim=True), (s * t).mean((1, 3), keepdim=True)
    want = 0.5 * (s - a - t * b)
    err = 0.5 * 5 * U * (s.abs() + a.abs() + (t * b).abs())
    within(gx, want.reshape(x.shape), err.reshape(x.shape) + rounding(x_dtype) * want.reshape(x.shape).abs() * (1 + 2 ** -7) + small(x_dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups", SHAPES)
@pytest.mark.parametrize("x_dtype,y_dtype", TYPES)
def test_silu(n, h, w, c, groups, x_dtype, y_dtype):
    x, gain, bias = draw(n, h, w, c, x_dtype, n + c)
    check(x, gain, bias, groups, SILU, forward(x, gain, bias, groups, SILU, y_dtype))
    args = draw_backward(n, h, w, c, groups, x_dtype, y_dtype, SILU, n + c)
    check_backward(args, backward(*args))


@pytest.mark.parametrize("n,h,w,c,groups", SHAPES)
def test_a_pixel_left_out_of_the_sums_would_show(n, h, w, c, groups):
    """One pixel of one image missing from the oracle's sums is beyond the bounds of mean or rstd in some of its groups."""
    x = torch.randint(-3, 4, (n, h, w, c), generator=rng(n + c))
    g = grouped(x[:1], groups)
    kept = g.clone()
    kept[:, g.shape[1] // 2] = 0
    mean, less = g.mean((1, 3)), kept.sum((1, 3)) / (g[0, :, 0].numel())
    rstd, other = (1 / torch.sqrt((v * v).mean((1, 3)) + EPS) for v in (g, kept))
    assert bool((((mean - less).abs() > 40 * U * 6) | ((rstd - other).abs() > 40 * U * rstd)).any())


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,groups,x_dtype", [(1, 68, 80, 3, 1, F32), (2, 68, 80, 24, 1, BF16), (3, 64, 68, 60, 2, F32), (5, 32, 32, 256, 1, BF16), (70, 16, 16, 64, 4, F32),
                                                    (1800, 16, 16, 64, 1, BF16)])
def test_means_that_are_small_beside_the_first_pixel(n, h, w, c, groups, x_dtype):
    """Threads of 8 to 32 whole numbers: their means are exact, and what they are joined to, in float64, is rounded once (and once more where the first pixel is
    added)."""
    x = torch.randint(-3, 4, (n, h, w, c), generator=rng(n + c)).to(x_dtype)
    x[:, 0, 0] = 200.0
    x[:, -1, -1] = -200.0
    mean = forward(x, None, None, groups, NONE, x_dtype)[1]
    want = grouped(x, groups).mean((1, 3))
    assert float(want.abs().max()) < 0.2                     # a thousandth of the first pixel
    within(mean, want, 2 * U * want.abs() + 2.0 ** -45)
