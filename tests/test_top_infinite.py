"""Top logits of rows with scores of +inf: they come first in their order, and log sum exp is +inf (NaN where the row has a NaN too), in every way a row is
walked: by a warp, a block, in pieces, by element."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, device, rng

INF = float("inf")


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,offset", [(7, 5, 0), (7, 60, 0), (7, 500, 0), (1500, 2870, 0), (7, 2048, 0), (7, 40001, 0), (400, 30000, 0), (7, 600000, 0),
                                                 (7, 3001, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [1.0, 3.0])
def test_infinite_scores(rows, classes, offset, dtype, tau):
    count = min(20, classes)
    z = torch.randn(rows, classes, generator=rng(classes)).to(dtype)
    z[0, classes - 1] = INF
    z[1, ::2] = INF
    z[2] = INF
    z[3] = -INF
    z[3, classes // 2] = INF
    z[4] = torch.finfo(dtype).max
    z[4, 1] = INF
    z[5, 0] = INF
    z[5, classes - 1] = float("nan")
    h = circ.circ_top_create(classes, count)
    circ.circ_top_set_dtypes(h, CODE[dtype], CODE[torch.int64])
    circ.circ_top_set_temperature(h, tau)
    values, ids, lse = torch.empty(rows, count, dtype=dtype, device="cuda"), torch.empty(rows, count, dtype=torch.int64, device="cuda"), torch.empty(rows, device="cuda")
    circ.circ_top_forward(h, device(z, offset), classes, values, ids, lse, rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_top_destroy(h)
    lse = lse.cpu()
    assert bool((lse[:5] == INF).all()) and bool(lse[5].isnan()) and bool(torch.isfinite(lse[6:]).all())
    order = torch.sort(torch.where(z.isnan(), INF, z.float()), dim=1, descending=True, stable=True)
    for r in (0, 1, 2, 3, 4, rows - 1):
        assert torch.equal(ids[r].cpu(), order.indices[r, :count]) and torch.equal(values[r].float().cpu(), order.values[r, :count])
