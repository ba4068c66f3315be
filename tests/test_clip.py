"""Clipping by the global norm against the formula in 64 bits: one tensor to many, empty ones, mixed types, unaligned
addresses, in place and into copies, norms below the limit and not finite; refusals.

Bounds (u: unit roundoff of float32).  Squares are added in float32 over at most 256 values a lane and block tree (chains of at
most 300 additions), then in float64: the norm's relative error is at most 152 u, the factor's 3 u more, and every output is
rounded once more."""
import math

import pytest
import torch

import paper_1708_08917_b200 as circ
from row_helpers import CODE, U, device, guarded, rng, rounding, small

F32, BF16 = torch.float32, torch.bfloat16
NORM = 152 * U


def plain(tensors, max_norm):
    norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))
    return norm, min(1.0, max_norm / (norm + 1e-6))


def check(outs, tensors, dtypes, norm, want, factor):
    assert abs(norm - want) <= NORM * want
    for o, t, d in zip(outs, tensors, dtypes):
        ref = t.double() * factor
        assert o.dtype == d and bool(((o.double().cpu() - ref).abs() <= (NORM + 5 * U + rounding(d)) * ref.abs() + small(d)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[1], [0, 1, 0], [7, 33, 1000], [16384], [16385, 3, 70000], [4096] * 300, [5] * 1000, [1 << 20, 1, 255, 250001]])
@pytest.mark.parametrize("grads,outs,offset", [(F32, F32, 0), (BF16, F32, 0), (F32, BF16, 1), (BF16, BF16, 3), ("mixed", "mixed", 0)])
@pytest.mark.parametrize("over", [4.0, 0.5])
def test_clipped_copies(sizes, grads, outs, offset, over):
    g = rng(sum(sizes))
    gd = [F32 if i % 3 else BF16 for i in range(len(sizes))] if grads == "mixed" else [grads] * len(sizes)
    od = [BF16 if i % 4 else F32 for i in range(len(sizes))] if outs == "mixed" else [outs] * len(sizes)
    tensors = [(0.01 * torch.randn(n, generator=g)).to(d) for n, d in zip(sizes, gd)]
    max_norm = float(torch.tensor(plain(tensors, 1.0)[0] / over, dtype=F32))
    h = circ.circ_clip_create(sizes, [CODE[d] for d in gd], [CODE[d] for d in od])
    held = [device(t, offset) for t in tensors]
    results = [guarded((n,), d, offset) for n, d in zip(sizes, od)]
    circ.circ_clip_set_tensors(h, held, [r[0] for r in results], torch.cuda.current_stream())
    norm, norm_ok = guarded((1,), F32)
    circ.circ_clip_forward(h, max_norm, norm, torch.cuda.current_stream())
    torch.cuda.synchronize()
    first = [r[0].clone() for r in results]
    circ.circ_clip_forward(h, max_norm, None, torch.cuda.current_stream())        # again, without the norm: the same bits
    torch.cuda.synchronize()
    circ.circ_clip_destroy(h)
    norm_ok()
    for (o, ok), f in zip(results, first):
        ok()
        assert torch.equal(o, f)
    check([r[0] for r in results], tensors, od, float(norm), *plain(tensors, max_norm))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("over", [10.0, 0.1])
def test_in_place_and_changed_addresses(dtype, over):
    sizes = [1000, 17, 40000]
    h = circ.circ_clip_create(sizes, CODE[dtype], CODE[dtype])
    norm = torch.empty(1, device="cuda")
    for seed in (1, 2):                                                          # the second time with other tensors
        g = rng(seed)
        tensors = [torch.randn(n, generator=g).to(dtype) for n in sizes]
        max_norm = float(torch.tensor(plain(tensors, 1.0)[0] / over, dtype=F32))
        held = [device(t) for t in tensors]
        circ.circ_clip_set_tensors(h, held, held if seed == 1 else None, torch.cuda.current_stream())
        circ.circ_clip_forward(h, max_norm, norm, torch.cuda.current_stream())
        torch.cuda.synchronize()
        check(held, tensors, [dtype] * 3, float(norm), *plain(tensors, max_norm))
        if over < 1:
            assert all(torch.equal(a.cpu(), b) for a, b in zip(held, tensors))   # nothing to clip: not a bit changes
    circ.circ_clip_destroy(h)


@pytest.mark.gpu
def test_zeros_a_limit_of_zero_large_values_and_values_that_are_not_finite():
    n = 5000
    norm = torch.empty(1, device="cuda")
    h = circ.circ_clip_create([n], circ.CIRC_F32, circ.CIRC_F32)

    def clipped(t, limit):
        held, out = device(t), torch.full((n,), float("nan"), device="cuda")
        circ.circ_clip_set_tensors(h, [held], [out], torch.cuda.current_stream())
        circ.circ_clip_forward(h, limit, norm, torch.cuda.current_stream())
        torch.cuda.synchronize()
        return float(norm), out.cpu()

    x = torch.randn(n, generator=rng(6))
    got, out = clipped(torch.zeros(n), 1.0)
    assert got == 0 and bool((out == 0).all())
    got, out = clipped(x, 0.0)
    assert bool((out == 0).all())
    got, out = clipped(x * 1e17, 1.0)                      # squares of 1e34, their sum still a float32
    assert abs(got - float((x * 1e17).double().norm())) <= NORM * got and abs(float(out.norm()) - 1) < 1e-3
    y = x.clone()
    y[123] = float("nan")
    got, out = clipped(y, 1.0)
    assert math.isnan(got) and bool(out.isnan().all())
    y[123] = float("inf")
    got, out = clipped(y, 1.0)
    assert got == math.inf and bool(out[123].isnan()) and bool((out[:123] == 0).all())
    circ.circ_clip_destroy(h)


@pytest.mark.gpu
def test_nothing_but_empty_tensors_and_a_captured_graph():
    norm = torch.full((1,), float("nan"), device="cuda")
    h = circ.circ_clip_create([0, 0], circ.CIRC_F32, circ.CIRC_BF16)
    circ.circ_clip_set_tensors(h, [None, None], [None, None])
    circ.circ_clip_forward(h, 1.0, norm, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_clip_destroy(h)
    assert float(norm) == 0
    x = torch.randn(100000, device="cuda")
    out, want = torch.zeros_like(x), x * min(1.0, 2.0 / (float(x.double().norm()) + 1e-6))
    h = circ.circ_clip_create([100000], circ.CIRC_F32, circ.CIRC_F32)
    circ.circ_clip_set_tensors(h, [x], [out], torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        circ.circ_clip_forward(h, 2.0, norm, torch.cuda.current_stream())
    graph.replay()
    torch.cuda.synchronize()
    assert torch.allclose(out, want, rtol=1e-5)
    del graph
    circ.circ_clip_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first,then", [(3, 0), (0, 3), (1, 5), (0, 0)])
def test_a_captured_call_clips_the_tensors_that_were_set_last(dtype, first, then):
    """Other addresses and other alignments, which cut the tensors at other places: sizes just above 8192 and 2 x 8192 elements have a
    piece more or less."""
    sizes = [8195, 8193, 16385, 100, 0, 8192]
    h = circ.circ_clip_create(sizes, CODE[dtype], CODE[dtype])
    norm = torch.empty(1, device="cuda")
    graph = None
    kept = []                              # every tensor stays allocated, also what an old plan would reach
    for seed, offset in enumerate((first, then, first)):
        g = rng(seed)
        tensors = [torch.randn(n, generator=g).to(dtype) for n in sizes]
        held, out = [device(t, offset) for t in tensors], [guarded((n,), dtype, offset) for n in sizes]
        kept += held + [o[0] for o in out]
        max_norm = 40.0
        circ.circ_clip_set_tensors(h, held, [o[0] for o in out], torch.cuda.current_stream())
        if graph is None:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                circ.circ_clip_forward(h, max_norm, norm, torch.cuda.current_stream())
        graph.replay()
        torch.cuda.synchronize()
        for _, ok in out:
            ok()
        check([o[0] for o in out], tensors, [dtype] * len(sizes), float(norm), *plain(tensors, max_norm))
    del graph
    circ.circ_clip_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("grads,outs", [(F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("size", [1e25, 3e30, 1e19, 1e-12, 1e-20, 1e-25, 1e-38])
@pytest.mark.parametrize("alone", [False, True])
def test_values_whose_squares_are_no_float32(grads, outs, size, alone):
    """All of this size, or one element of it among smaller ones: the squares overflow or vanish in float32, the norm does not."""
    sizes = [5, 70000, 8192]
    g = rng(17)
    tensors = [torch.randn(n, generator=g) * size * (1e-6 if alone else 1.0) for n in sizes]
    if alone:
        tensors[1][12345] = size
    tensors = [t.to(grads) for t in tensors]
    want = plain(tensors, 0.0)[0]
    max_norm = float(torch.tensor(want / 3, dtype=F32))
    h = circ.circ_clip_create(sizes, CODE[grads], CODE[outs])
    held, out = [device(t) for t in tensors], [guarded((n,), outs) for n in sizes]
    norm = torch.empty(1, device="cuda")
    circ.circ_clip_set_tensors(h, held, [o[0] for o in out], torch.cuda.current_stream())
    circ.circ_clip_forward(h, max_norm, norm, torch.cuda.current_stream())
    torch.cuda.synchronize()
    circ.circ_clip_destroy(h)
    for _, ok in out:
        ok()
    _, factor = plain(tensors, max_norm)
    # a factor below float32's normal numbers has an absolute error of 2^-150
    for o, t in zip(out, tensors):
        ref = t.double() * factor
        bound = (NORM + 5 * U + rounding(outs)) * ref.abs() + 2.0 ** -150 * t.double().abs() + small(outs)
        assert bool(((o[0].double().cpu() - ref).abs() <= bound).all())
    assert abs(float(norm) - want) <= NORM * want + 2.0 ** -150


@pytest.mark.gpu
def test_the_norm_adds_few_squares_in_float32():
    """A thread adds 32 squares (33 with those in front of a boundary and behind the last vector) in four chains of at most 9 float32
    multiply-adds and joins them by 2 additions: at most 11 roundings, all terms positive, so 11 u of the sum; float64 from there on
    (2^-40 covers it).  The norm has half of that, and its own rounding: 6.5 u."""
    n = 1 << 20
    g = rng(23)
    h = circ.circ_clip_create([n, 77777], circ.CIRC_F32, circ.CIRC_F32)
    norm = torch.empty(1, device="cuda")
    for scale in (1.0, 1e-4):
        for tensors in ([scale * torch.rand(n, generator=g), scale * torch.randn(77777, generator=g)], [torch.full((n,), 0.1 * scale), torch.zeros(77777)]):
            held = [device(t) for t in tensors]
            out = [torch.empty_like(t) for t in held]
            circ.circ_clip_set_tensors(h, held, out, torch.cuda.current_stream())
            circ.circ_clip_forward(h, 1.0, norm, torch.cuda.current_stream())
            torch.cuda.synchronize()
            want = plain(tensors, 1.0)[0]
            assert abs(float(norm) - want) <= (6.5 * U + 2.0 ** -40) * want
    circ.circ_clip_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2])
def test_a_plan_that_cannot_be_allocated(n):
    try:
        circ.circ_debug_fail_alloc_after(n)
        refused(circ.CIRC_ERR_ALLOC, circ.circ_clip_create, [100, 5], circ.CIRC_F32, circ.CIRC_F32)
    finally:
        circ.circ_debug_fail_alloc_after(0)


def refused(code, call, *args):
    with pytest.raises(circ.CircError) as e:
        call(*args)
    assert e.value.code == code


def test_refusals_before_any_device_call():
    refused(circ.CIRC_ERR_ARG, circ.circ_clip_create, [], 0, 0)
    refused(circ.CIRC_ERR_SHAPE, circ.circ_clip_create, [-1], 0, 0)
    refused(circ.CIRC_ERR_SHAPE, circ.circ_clip_create, [1 << 41], 0, 0)
    refused(circ.CIRC_ERR_ARG, circ.circ_clip_create, [4], circ.CIRC_E4M3, 0)
    refused(circ.CIRC_ERR_ARG, circ.circ_clip_create, [4], 0, 5)
    refused(circ.CIRC_ERR_ARG, circ.circ_clip_set_tensors, None, [64], None)
    refused(circ.CIRC_ERR_ARG, circ.circ_clip_forward, None, 1.0, None)
    circ.circ_clip_destroy(None)


@pytest.mark.gpu
def test_refusals_of_bad_arguments():
    h = circ.circ_clip_create([8], circ.CIRC_F32, circ.CIRC_BF16)
    a, b = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda", dtype=BF16)
    try:
        refused(circ.CIRC_ERR_ARG, circ.circ_clip_forward, h, 1.0, None)                            # no tensors yet
        refused(circ.CIRC_ERR_ARG, circ.circ_clip_set_tensors, h, [a], [a])                         # in place with two types
        refused(circ.CIRC_ERR_ARG, circ.circ_clip_set_tensors, h, [a], None)
        refused(circ.CIRC_ERR_ARG, circ.circ_clip_set_tensors, h, [None], [b])
        refused(circ.CIRC_ERR_ARG, circ.circ_clip_set_tensors, h, [a.data_ptr() + 2], [b])
        circ.circ_clip_set_tensors(h, [a], [b], torch.cuda.current_stream())
        refused(circ.CIRC_ERR_ARG, circ.circ_clip_forward, h, -1.0, None)
        refused(circ.CIRC_ERR_ARG, circ.circ_clip_forward, h, float("nan"), None)
        with pytest.raises(AssertionError):
            circ.circ_clip_set_tensors(h, [a[::2]], [b])
    finally:
        torch.cuda.synchronize()
        circ.circ_clip_destroy(h)
