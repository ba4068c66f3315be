"""Workspaces of the operators that train a compressed network: no call holds what it does not use; under stream capture a call whose workspace is already
as large as it needs is served, one that needs more is refused, and either way the capture and the graphs captured before stay whole."""
import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import rng

CLASSES, COUNT, TAU = 1024, 5, 2.0


def distill_inputs(rows):
    g = rng(rows)
    z = torch.randn(rows, CLASSES, generator=g)
    ids = torch.stack([torch.randperm(CLASSES, generator=g)[:COUNT] for _ in range(rows)])
    values = torch.randn(rows, COUNT, generator=g)
    p = torch.softmax(values.double() / TAU, 1)
    log_q = torch.log_softmax(z.double() / TAU, 1)
    loss = (p * (p.log() - log_q.gather(1, ids))).sum(1)
    return [t.cuda() for t in (z, values, ids)], loss


@pytest.mark.gpu
def test_captured_distillation_of_more_rows():
    h = circ.circ_distill_create(CLASSES, COUNT)
    circ.circ_distill_set_temperature(h, TAU)
    cases = {rows: (*distill_inputs(rows), torch.zeros(rows, device="cuda")) for rows in (1, 5, 5000)}

    def call(rows):
        (z, values, ids), _, out = cases[rows]
        circ.circ_distill_forward(h, z, CLASSES, values, ids, None, None, out, None, None, rows, torch.cuda.current_stream())

    call(1)
    torch.cuda.synchronize()
    graphs = {rows: torch.cuda.CUDAGraph() for rows in (1, 5, 5000)}
    for rows in (1, 5):                 # these need the same number of bytes
        with torch.cuda.graph(graphs[rows]):
            call(rows)
    counter = torch.zeros(1, device="cuda")
    with torch.cuda.graph(graphs[5000]):
        counter.add_(1)
        with pytest.raises(circ.CircError) as e:
            call(5000)
        counter.add_(1)
    assert e.value.code == circ.CIRC_ERR_UNSUPPORTED
    for _ in range(2):
        for rows in (1, 5):
            cases[rows][2].zero_()
            graphs[rows].replay()
    graphs[5000].replay()
    call(5000)                          # a larger workspace beside the one that the graphs hold
    graphs[1].replay()
    torch.cuda.synchronize()
    assert float(counter) == 2
    for rows, (_, want, out) in cases.items():
        # exponentials with (s - max) / tau above -5: (2 + 15) u, sums of 1024 by 32 lanes: (32 + 16) u, the result: u; together below 1e-5
        assert float((out.double().cpu() - want).abs().max()) <= 1e-5 * float(want.abs().max().clamp(min=1))
    del graphs
    circ.circ_distill_destroy(h)


@pytest.mark.gpu
def test_captured_group_norm_of_more_images():
    height, width, channels, groups, eps = 37, 41, 8, 2, 1e-5
    h = circ.circ_gnorm_create(channels, groups, eps)
    cases = {}
    for images in (1, 4, 300):
        x = torch.randn(images, height, width, channels, generator=rng(images))
        want = torch.nn.functional.group_norm(x.double().permute(0, 3, 1, 2), groups, eps=eps).permute(0, 2, 3, 1)
        cases[images] = x.cuda(), want, torch.zeros_like(x, device="cuda")

    def call(images):
        x, _, y = cases[images]
        circ.circ_gnorm_forward(h, x, None, None, y, None, None, images, height, width, torch.cuda.current_stream())

    call(1)
    torch.cuda.synchronize()
    graphs = {images: torch.cuda.CUDAGraph() for images in (1, 4, 300)}
    for images in (1, 4):               # these need the same number of bytes
        with torch.cuda.graph(graphs[images]):
            call(images)
    counter = torch.zeros(1, device="cuda")
    with torch.cuda.graph(graphs[300]):
        counter.add_(1)
        with pytest.raises(circ.CircError) as e:
            call(300)
        counter.add_(1)
    assert e.value.code == circ.CIRC_ERR_UNSUPPORTED
    for _ in range(2):
        for images in (1, 4):
            cases[images][2].zero_()
            graphs[images].replay()
    graphs[300].replay()
    call(300)
    graphs[1].replay()
    torch.cuda.synchronize()
    assert float(counter) == 2
    for _, want, y in cases.values():
        # values below 6 in magnitude; mean and variance from 6068 terms by 256 threads or more: (24 + 8) u of the largest difference, 12; below 5e-5
        assert float((y.double().cpu() - want).abs().max()) <= 5e-5
    del graphs
    circ.circ_gnorm_destroy(h)


@pytest.mark.gpu
def test_a_distillation_of_many_rows_holds_no_lists_that_it_does_not_use():
    rows, classes, count, some = 1 << 19, 264, 256, 1000
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    z = torch.randn(rows, classes, device="cuda", generator=g)
    values = torch.randn(rows, count, device="cuda", generator=g)
    ids = torch.arange(count, device="cuda").flip(0).expand(rows, count).contiguous()
    row_loss, mean = torch.empty(rows, device="cuda"), torch.empty(1, device="cuda")
    h = circ.circ_distill_create(classes, count)

    def forward():
        circ.circ_distill_forward(h, z, classes, values, ids, None, None, row_loss, None, mean, rows, torch.cuda.current_stream())

    def backward(offset):        # of the first rows; behind a 16-byte boundary it is done in pieces, which use the lists
        zz = torch.empty(some * classes + offset, device="cuda")[offset:].view(some, classes)
        zz.copy_(z[:some])
        grad = torch.empty_like(z[:some])
        circ.circ_distill_backward(h, zz, classes, values, ids, None, None, None, None, mean, grad, classes, float(some), some, torch.cuda.current_stream())
        return grad

    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    forward()
    torch.cuda.synchronize()
    assert free - torch.cuda.mem_get_info()[0] < 256 << 20          # the lists of all rows: 1 GB
    first = row_loss.clone()
    in_rows, in_pieces = backward(0), backward(1)
    forward()
    torch.cuda.synchronize()
    circ.circ_distill_destroy(h)
    assert torch.equal(row_loss, first)
    p, q = torch.softmax(values[:some].double(), 1), torch.softmax(z[:some].double(), 1)
    want = q.scatter_add(1, ids[:some], -p)
    for grad in (in_rows, in_pieces):      # probabilities with (2 + 3 * 12 + 264 / 32 + 16) u each, a few roundings
        assert float((grad.double() - want).abs().max()) <= 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes", [(200, 1000), (60, 300000), (3, 200000)])
def test_top_logits_that_use_no_workspace_allocate_none(rows, classes):
    z = torch.randn(rows, classes, generator=rng(rows)).cuda()
    ids = torch.empty(rows, 7, dtype=torch.int64, device="cuda")
    h = circ.circ_top_create(classes, 7)
    circ.circ_debug_fail_alloc_after(1)
    try:
        circ.circ_top_forward(h, z, classes, None, ids, None, rows, torch.cuda.current_stream())
    finally:
        circ.circ_debug_fail_alloc_after(0)
    torch.cuda.synchronize()
    assert torch.equal(ids, torch.sort(z, dim=1, descending=True, stable=True).indices[:, :7])
    circ.circ_top_destroy(h)


@pytest.mark.gpu
def test_top_logits_in_pieces_reserved_for_either_type():
    rows, classes, count = 2, 280001, 9
    z = torch.randn(rows, classes, generator=rng(3)).cuda()
    h = circ.circ_top_create(classes, count)
    circ.circ_top_set_dtypes(h, circ.CIRC_BF16, circ.CIRC_I64)
    circ.circ_top_reserve(h, rows)
    circ.circ_top_set_dtypes(h, circ.CIRC_F32, circ.CIRC_I64)
    values, ids = torch.zeros(rows, count, device="cuda"), torch.zeros(rows, count, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_top_forward(h, z, classes, values, ids, None, rows, torch.cuda.current_stream())
    graph.replay()
    torch.cuda.synchronize()
    want = torch.sort(z, dim=1, descending=True, stable=True)
    assert torch.equal(values, want.values[:, :count]) and torch.equal(ids, want.indices[:, :count])
    del graph
    circ.circ_top_destroy(h)
