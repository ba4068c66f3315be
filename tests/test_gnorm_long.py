"""Group norm of images whose channels have many pixels a thread: what rounding costs does not grow with the pixels, and a pixel far from the others
in the place that the sums start from costs no digits.

Bounds (u: unit roundoff of float32).  A thread adds up at most 264 values in float32, around the mean of its first 4 or 8 or, behind a run, around the mean
so far.  The values here are whole numbers, at most 3 and OUT: a first run's sums are exact (multiples of 1/8, their squares' sum below 2^18; of 1/4, below
2^20), and what its two sums' difference loses is at most 3 u of the sum of squares, 75 u of those around the mean.  Further runs: a difference u, the sum of
squares s 266 u, the sum 265 u of the magnitudes', so that a run's squares around its mean are off by at most (267 + 2 * 265) u s, and all runs' s are at most
twice the squares around the mean of all (a run has no more values than those whose mean it starts from).  Joined in float64, rounded once and joined over at
most 256 threads: relative 1700 u of the variance.  The mean: 265 u sqrt(2) of the deviation, and (256 + 8) u of the distance from the first pixel."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, U, rounding

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
OUT = 100
EPS = 1e-5


def whole_numbers(n, h, w, c, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.empty(n, h * w, c, dtype=dtype, device="cuda")
    for part in x.split(max(1, (1 << 28) // (h * w * c))):
        part.copy_(torch.randint(-3, 4, part.shape, dtype=torch.int8, device="cuda", generator=g))
    return x


def handle(c, groups, x_dtype, y_dtype, kind=circ.CIRC_ACT_NONE):
    h = circ.circ_gnorm_create(c, groups, EPS)
    circ.circ_gnorm_set_dtypes(h, CODE[x_dtype], CODE[y_dtype])
    circ.circ_gnorm_set_activation(h, kind)
    return h


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,x_dtype,y_dtype", [(444, 80, 80, 2048, BF16, BF16),      # 6400 pixels a thread, a block an image in two launches
                                                     (1776, 80, 80, 255, BF16, BF16),       # ... in one
                                                     (1776, 20, 20, 2048, BF16, BF16), (1776, 20, 20, 1024, F32, F32), (1776, 20, 20, 2048, F32, BF16),
                                                     (600, 40, 40, 255, F32, F32),          # images in pieces
                                                     (1, 1024, 800, 257, BF16, BF16), (1, 1024, 800, 257, F32, F32)])      # any width: 12800 pixels a thread
def test_deviations_of_many_pixels(n, h, w, c, x_dtype, y_dtype):
    x = whole_numbers(n, h, w, c, x_dtype, c + n)
    x[:, ::12800 if h * w > 12800 else h * w] = OUT
    y, mean, rstd = torch.empty(x.shape, dtype=y_dtype, device="cuda"), torch.empty(n, c, device="cuda"), torch.empty(n, c, device="cuda")
    hd = handle(c, c, x_dtype, y_dtype)
    circ.circ_gnorm_forward(hd, x, None, None, y, mean, rstd, n, h, w, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_gnorm_destroy(hd)
    for i in {0, n // 2, n - 1}:
        xd = x[i].double()
        m = xd.mean(0)
        d = xd - m
        var = (d * d).mean(0)
        r = 1 / torch.sqrt(var + EPS)
        mean_err = 375 * U * var.sqrt() + 264 * U * (xd[0] - m).abs() + U * m.abs()
        rstd_err = (850 + 4) * U * r
        assert bool(((mean[i].double() - m).abs() <= mean_err).all())
        assert bool(((rstd[i].double() - r).abs() <= rstd_err).all())
        v = d * r
        err = r * mean_err + v.abs() * 858 * U + rounding(y_dtype) * v.abs() * (1 + 2 ** -7)
        assert bool(((y[i].double() - v).abs() <= err).all())


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,w,c,x_dtype", [(444, 80, 80, 1024, BF16),      # 6400 pixels a thread, in two launches
                                             (1776, 80, 80, 255, BF16),      # ... in one
                                             (1776, 20, 20, 1024, BF16),     # 400, four channels a thread, in one
                                             (1, 1024, 800, 257, F32)])      # any width: 12800
def test_gradients_of_many_pixels(n, h, w, c, x_dtype):
    """The same gradient everywhere, one whose float32 sum drifts (6400 of them in one run: 9e-5); u = 1 everywhere.  Runs of at most 264 additions, one thread a
    channel and piece, joined in float64: 268 u."""
    value = 0.32391423
    x = torch.ones(n, h * w, c, dtype=x_dtype, device="cuda")
    grad_y = torch.full((n, h * w, c), value, device="cuda")
    mean, rstd = torch.zeros(n, c, device="cuda"), torch.ones(n, c, device="cuda")
    grad_gain, grad_bias = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    hd = handle(c, c, x_dtype, F32)
    circ.circ_gnorm_backward(hd, x, None, None, mean, rstd, grad_y, grad_y if x_dtype == F32 else x, grad_gain, grad_bias, n, h, w, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_gnorm_destroy(hd)
    g = float(torch.tensor(value))
    want = g * n * h * w
    for got in (grad_gain, grad_bias):
        assert float((got.double() - want).abs().max()) <= 268 * U * want
    # grad_x = g - A - u B, both the mean of what was summed up
    grad_x = grad_y if x_dtype == F32 else x
    for i in {0, n // 2, n - 1}:
        assert float((grad_x[i].double() + g).abs().max()) <= (2 * 268 + 4) * U * g + rounding(x_dtype) * g * (1 + 2 ** -7)
