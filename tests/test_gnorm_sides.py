"""The sides of a ReLU near 0 where the channels are walked one at a time, four at a time, or by the kernels of any width: found in float64 everywhere."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, device, rng

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("c,groups", [(35, 5), (255, 3), (64, 4), (258, 6)])
@pytest.mark.parametrize("y_dtype", [F32, BF16])
def test_sides_near_zero(c, groups, y_dtype):
    n, h, w = 2, 40, 30
    g = rng(c)
    gain, bias = 1 + 0.3 * torch.randn(c, generator=g), torch.empty(c)
    mean, rstd = 0.5 * torch.randn(n, groups, generator=g), 1 + torch.rand(n, groups, generator=g)
    mean[1], rstd[1] = mean[0], rstd[0]
    m, r = mean[0].repeat_interleave(c // groups), rstd[0].repeat_interleave(c // groups)
    base = torch.randn(c, generator=g)
    bias = -((base.double() - m.double()) * r.double() * gain.double()).float()
    steps = torch.randint(-3, 4, (n, h, w, c), generator=g)
    x = (base.view(torch.int32) + steps.int()).view(F32).clone()                     # neighbours of the value where v is 0
    x[:, ::3] += torch.randn(c, generator=g)                                         # and values far from it
    hd = circ.circ_gnorm_create(c, groups, 1e-5)
    circ.circ_gnorm_set_dtypes(hd, CODE[F32], CODE[y_dtype])
    circ.circ_gnorm_set_activation(hd, circ.CIRC_ACT_RELU)
    ones, grad_bias = torch.ones(n, h, w, c, device="cuda", dtype=y_dtype), torch.empty(c, device="cuda")
    circ.circ_gnorm_backward(hd, device(x), device(gain), device(bias), device(mean), device(rstd), ones, None, None, grad_bias, n, h, w,
                             torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_gnorm_destroy(hd)
    v = (x.double() - m.double()) * (r.double() * gain.double()) + bias.double()
    assert torch.equal(grad_bias.double().cpu(), (v > 0).double().sum((0, 1, 2)))    # whole numbers: the sum is exact
