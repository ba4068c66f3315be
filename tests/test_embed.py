"""Embedding lookup and its gradient by tokens against loops in 64 bits: ids of both types, padding, ids outside the table,
rows without a token, one row with all tokens, odd widths and unaligned buffers; refusals.

Bounds: the lookup is one product, rounded to float32 and then to the output type.  A gradient row is a float32 sum of n
terms in some order, |error| <= n u sum|terms|, times the scale (one rounding more), rounded once to the table's type."""
import math

import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, U, device, guarded, rng, rounding, small, within

F32, BF16 = torch.float32, torch.bfloat16


def handle(vocab, dim, table, y, ids, scale, padding=-1):
    h = circ.circ_embed_create(vocab, dim)
    circ.circ_embed_set_dtypes(h, CODE[table], CODE[y], CODE[ids])
    circ.circ_embed_set_scale(h, scale)
    circ.circ_embed_set_padding(h, padding)
    return h


def draw_ids(kind, tokens, vocab, g):
    if kind == "uniform":
        return torch.randint(vocab, (tokens,), generator=g)
    if kind == "one":                       # every token the same row
        return torch.full((tokens,), vocab - 1)
    if kind == "outside":                   # negative ids and ids behind the table among the others
        return torch.randint(-3, vocab + 3, (tokens,), generator=g)
    ids = torch.exp(torch.rand(tokens, generator=g, dtype=torch.float64) * math.log(vocab + 1)).long() - 1   # few frequent, many rare
    return ids.clamp(0, vocab - 1)


def keep_mask(ids, vocab, padding):
    return (ids >= 0) & (ids < vocab) & (ids != padding)


def plain_gradient(ids, dy, vocab, scale, padding):
    """(gradient, sum of magnitudes, tokens per row) in 64 bits."""
    keep = keep_mask(ids, vocab, padding)
    grad = torch.zeros(vocab, dy.shape[1], dtype=torch.float64)
    mag = torch.zeros_like(grad)
    for t in keep.nonzero().squeeze(1).tolist():
        grad[ids[t]] += dy[t].double()
        mag[ids[t]] += dy[t].double().abs()
    return scale * grad, abs(scale) * mag, torch.bincount(ids[keep], minlength=vocab).double()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 1, 1), (1, 1000, 4096), (7, 5, 8), (33, 100, 250), (100, 17, 1001), (300, 4000, 24)])
@pytest.mark.parametrize("table,y,ids_type,offset", [(F32, F32, torch.int64, 0), (F32, BF16, torch.int32, 0), (BF16, BF16, torch.int64, 1),
                                                     (BF16, F32, torch.int32, 3)])
def test_lookup(tokens, vocab, dim, table, y, ids_type, offset):
    g = rng(tokens * 31 + dim)
    w = torch.randn(vocab, dim, generator=g).to(table)
    ids = draw_ids("outside", tokens, vocab, g)
    scale, padding = 1.7, vocab // 2
    h = handle(vocab, dim, table, y, ids_type, scale, padding)
    out, untouched = guarded((tokens, dim), y, offset)
    circ.circ_embed_forward(h, device(w, offset), device(ids.to(ids_type)), out, tokens, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_embed_destroy(h)
    untouched()
    keep = keep_mask(ids, vocab, padding)
    s = float(torch.tensor(scale, dtype=F32))
    ref = torch.where(keep[:, None], s * w.double()[ids.clamp(0, vocab - 1)], 0.0)
    within(out, ref, (U + rounding(y)) * (1 + U) * ref.abs())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["uniform", "frequent", "one", "outside"])
@pytest.mark.parametrize("tokens,vocab,dim,table,y,ids_type,offset", [
    (1, 1, 1, F32, F32, torch.int64, 0),
    (1, 50, 64, BF16, BF16, torch.int32, 0),
    (31, 7, 40, F32, BF16, torch.int64, 0),
    (513, 1009, 100, F32, F32, torch.int32, 0),
    (700, 300, 33, BF16, F32, torch.int64, 1),       # odd width, nothing aligned
    (1000, 40, 1024, F32, BF16, torch.int64, 0),
    (257, 12, 2056, BF16, BF16, torch.int32, 0),
    (2500, 3, 16, F32, BF16, torch.int32, 0),
    (2048, 5000, 72, F32, F32, torch.int64, 0),      # the most tokens of the one-launch kernel, and one more
    (2049, 5000, 72, F32, F32, torch.int64, 0),
    (2049, 300000, 8, BF16, F32, torch.int32, 0),    # more rows than 128 classes of the sort hold
    (3000, 1009, 100, BF16, BF16, torch.int32, 0),
    (5000, 300, 33, F32, BF16, torch.int64, 1),      # odd width, nothing aligned
    (4000, 40, 1024, F32, F32, torch.int32, 0),
    (6000, 12, 2056, F32, BF16, torch.int64, 0),
    (20000, 500, 136, BF16, F32, torch.int64, 0),
])
def test_gradient(kind, tokens, vocab, dim, table, y, ids_type, offset):
    g = rng(tokens + vocab)
    ids = draw_ids(kind, tokens, vocab, g)
    dy = torch.randn(tokens, dim, generator=g).to(y)
    scale, padding = 0.3, 0 if vocab > 1 else -1
    h = handle(vocab, dim, table, y, ids_type, scale, padding)
    out, untouched = guarded((vocab, dim), table, offset)
    dyd, idd = device(dy, offset), device(ids.to(ids_type))
    circ.circ_embed_backward(h, idd, dyd, out, tokens, torch.cuda.current_stream())
    torch.cuda.synchronize()
    untouched()
    ref, mag, n = plain_gradient(ids, dy, vocab, float(torch.tensor(scale, dtype=F32)), padding)
    within(out, ref, (n[:, None] + 2) * U * mag + rounding(table) * ref.abs() + small(table))
    assert bool((out.cpu()[n == 0] == 0).all())
    again = torch.empty_like(out)                     # the order of the sums is fixed
    circ.circ_embed_backward(h, idd, dyd, again, tokens, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_embed_destroy(h)
    assert torch.equal(out, again)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,dim,share,table,y,ids_type", [(40000, 300, 24, 0.7, F32, BF16, torch.int64), (33000, 1000, 33, 1.0, F32, F32, torch.int32),
                                                                     (50000, 2, 40, 0.8, BF16, BF16, torch.int64), (60000, 3000, 136, 0.9, BF16, F32, torch.int32)])
def test_gradient_with_more_tokens_of_a_class_than_a_warp_lists(tokens, vocab, dim, share, table, y, ids_type):
    """A `share` of the tokens has one id: more of a sort block's tokens than its warps have room for (800 each at most)."""
    g = rng(tokens)
    ids = torch.where(torch.rand(tokens, generator=g) < share, min(130, vocab - 1), torch.randint(vocab, (tokens,), generator=g))
    dy = torch.randn(tokens, dim, generator=g).to(y)
    scale = 0.3
    h = handle(vocab, dim, table, y, ids_type, scale)
    out, untouched = guarded((vocab, dim), table)
    circ.circ_embed_backward(h, device(ids.to(ids_type)), device(dy), out, tokens, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_embed_destroy(h)
    untouched()
    s = float(torch.tensor(scale, dtype=F32))
    zero = torch.zeros(vocab, dim, dtype=torch.float64)
    ref, mag = s * zero.index_add(0, ids, dy.double()), s * zero.index_add(0, ids, dy.double().abs())
    n = torch.bincount(ids, minlength=vocab).double()
    within(out, ref, (n[:, None] + 2) * U * mag + rounding(table) * ref.abs() + small(table))


@pytest.mark.gpu
def test_gradient_is_the_derivative_of_the_lookup():
    tokens, vocab, dim, scale = 40, 11, 24, 1.5
    g = rng(5)
    ids = torch.randint(vocab, (tokens,), generator=g)
    w, v = (torch.randn(vocab, dim, generator=g, dtype=torch.float64) for _ in range(2))
    dy = torch.randn(tokens, dim, generator=g)
    h = handle(vocab, dim, F32, F32, torch.int64, scale)
    out = torch.empty(vocab, dim, device="cuda")
    circ.circ_embed_backward(h, device(ids), device(dy), out, tokens, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_embed_destroy(h)

    def value(table):
        return float((scale * table[ids] * dy.double()).sum())

    step = 1e-3                                       # the function is linear: central differences have rounding errors only
    slope = (value(w + step * v) - value(w - step * v)) / (2 * step)
    got = float((out.double().cpu() * v).sum())
    assert abs(got - slope) <= 1e-5 * float((out.double().cpu() * v).abs().sum())


@pytest.mark.gpu
def test_no_tokens_and_other_streams():
    vocab, dim = 100, 48
    h = handle(vocab, dim, F32, F32, torch.int32, 2.0)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    out = torch.full((vocab, dim), float("nan"), device="cuda")
    circ.circ_embed_forward(h, out, none, None, 0)
    circ.circ_embed_backward(h, none, None, out, 0, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert bool((out == 0).all())
    side = torch.cuda.Stream()
    ids = torch.arange(vocab, dtype=torch.int32, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dy = torch.randn(vocab, dim, device="cuda")
        circ.circ_embed_backward(h, ids, dy, out, vocab, side)
    side.synchronize()
    circ.circ_embed_destroy(h)
    assert torch.equal(out, 2.0 * dy)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [200, 3000])
def test_backward_in_a_captured_graph_needs_its_workspace(tokens):
    vocab, dim = 64, 32
    h = handle(vocab, dim, F32, F32, torch.int64, 1.0)
    circ.circ_embed_reserve(h, tokens)
    ids, dy = torch.randint(vocab, (tokens,), device="cuda"), torch.randn(tokens, dim, device="cuda")
    want, out = torch.empty(vocab, dim, device="cuda"), torch.zeros(vocab, dim, device="cuda")
    circ.circ_embed_backward(h, ids, dy, want, tokens, torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_embed_backward(h, ids, dy, out, tokens, torch.cuda.current_stream())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    del graph
    circ.circ_embed_destroy(h)


@pytest.mark.gpu
def test_a_captured_graph_keeps_its_workspace():
    """Calls behind the capture need more and more, and other memory takes what they leave."""
    vocab, dim, tokens = 500, 64, 3000
    h = handle(vocab, dim, F32, F32, torch.int64, 1.0)
    circ.circ_embed_reserve(h, tokens)
    ids, dy = torch.randint(vocab, (tokens,), device="cuda"), torch.randn(tokens, dim, device="cuda")
    want, out = torch.empty(vocab, dim, device="cuda"), torch.zeros(vocab, dim, device="cuda")
    circ.circ_embed_backward(h, ids, dy, want, tokens, torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_embed_backward(h, ids, dy, out, tokens, torch.cuda.current_stream())
    for more in (50000, 200000, 800000):
        ids2, dy2 = torch.randint(vocab, (more,), device="cuda"), torch.randn(more, dim, device="cuda")
        first, again = torch.empty(vocab, dim, device="cuda"), torch.empty(vocab, dim, device="cuda")
        circ.circ_embed_backward(h, ids2, dy2, first, more, torch.cuda.current_stream())
        out.zero_()
        graph.replay()
        circ.circ_embed_backward(h, ids2, dy2, again, more, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(first, again)
    del graph
    circ.circ_embed_destroy(h)


@pytest.mark.gpu
def test_a_workspace_that_cannot_be_allocated():
    vocab, dim, tokens = 300, 64, 3000
    ids, dy, out = torch.randint(vocab, (tokens,), device="cuda"), torch.randn(tokens, dim, device="cuda"), torch.empty(vocab, dim, device="cuda")
    h = handle(vocab, dim, F32, F32, torch.int64, 1.0)
    try:
        circ.circ_debug_fail_alloc_after(1)
        refused(circ.CIRC_ERR_ALLOC, circ.circ_embed_backward, h, ids, dy, out, tokens, torch.cuda.current_stream())
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_embed_backward(h, ids, dy, out, tokens, torch.cuda.current_stream())     # the handle serves the next call
        torch.cuda.synchronize()
        assert torch.allclose(out.double(), torch.zeros(vocab, dim, device="cuda", dtype=torch.float64).index_add_(0, ids, dy.double()), atol=1e-4)
        circ.circ_debug_fail_alloc_after(1)
        refused(circ.CIRC_ERR_ALLOC, circ.circ_embed_reserve, h, 1 << 20)
    finally:
        circ.circ_debug_fail_alloc_after(0)
        circ.circ_embed_destroy(h)


def refused(code, call, *args):
    with pytest.raises(circ.CircError) as e:
        call(*args)
    assert e.value.code == code


def test_refusals_before_any_device_call():
    refused(circ.CIRC_ERR_SHAPE, circ.circ_embed_create, 0, 8)
    refused(circ.CIRC_ERR_SHAPE, circ.circ_embed_create, 8, 0)
    refused(circ.CIRC_ERR_SHAPE, circ.circ_embed_create, 8, (1 << 24) + 1)
    for call, args in ((circ.circ_embed_forward, (None, 64, 64, 128, 1)), (circ.circ_embed_backward, (None, 64, 64, 128, 1)),
                       (circ.circ_embed_set_dtypes, (None, 0, 0, 0)), (circ.circ_embed_set_scale, (None, 1.0)),
                       (circ.circ_embed_set_padding, (None, 0)), (circ.circ_embed_reserve, (None, 1))):
        refused(circ.CIRC_ERR_ARG, call, *args)
    circ.circ_embed_destroy(None)


@pytest.mark.gpu
def test_refusals_of_bad_arguments():
    h = handle(10, 8, F32, F32, torch.int64, 1.0)
    a = torch.empty(64, 8, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    try:
        refused(circ.CIRC_ERR_ARG, circ.circ_embed_set_dtypes, h, circ.CIRC_E4M3, 0, 0)
        refused(circ.CIRC_ERR_ARG, circ.circ_embed_set_dtypes, h, 0, 0, 2)
        refused(circ.CIRC_ERR_ARG, circ.circ_embed_set_padding, h, 10)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_embed_forward, h, a, ids, a[32:], -1)
        refused(circ.CIRC_ERR_ARG, circ.circ_embed_forward, h, None, ids, a, 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_embed_forward, h, a, ids, a, 4)              # y is the table
        refused(circ.CIRC_ERR_ARG, circ.circ_embed_forward, h, a.data_ptr() + 2, ids, a[32:], 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_embed_backward, h, ids.data_ptr() + 4, a, a[32:], 4)
        refused(circ.CIRC_ERR_ARG, circ.circ_embed_backward, h, ids, None, a, 4)
        refused(circ.CIRC_ERR_SHAPE, circ.circ_embed_reserve, h, 1 << 31)
        with pytest.raises(AssertionError):
            circ.circ_embed_forward(h, a.t(), ids, a[32:], 4)
    finally:
        circ.circ_embed_destroy(h)
