"""Helpers of the tests of the row operators (embedding, norm, loss, clipping): types, seeded inputs, error bounds."""
import torch

import paper_1708_08917_b200 as circ

U = 2.0 ** -24          # unit roundoff of float32
U_BF16 = 2.0 ** -8      # of bfloat16 (8 significant bits, round to nearest)
CODE = {torch.float32: circ.CIRC_F32, torch.bfloat16: circ.CIRC_BF16, torch.float8_e4m3fn: circ.CIRC_E4M3, torch.int32: circ.CIRC_I32,
        torch.int64: circ.CIRC_I64}


def rng(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def device(t, offset=0):
    """A copy on the GPU whose data starts `offset` elements behind an allocation's (256-byte aligned) start."""
    buf = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
    out = buf[offset:].view(t.shape)
    out.copy_(t)
    return out


def guarded(shape, dtype, offset=0, pad=64):
    """An output of NaN (0xFF bytes) with `pad` elements of the same on both sides, and a check that those are untouched."""
    n = 1
    for d in shape:
        n *= d
    raw = torch.full(((n + offset + 2 * pad) * torch.empty((), dtype=dtype).element_size(),), 255, dtype=torch.uint8, device="cuda")
    buf = raw.view(dtype)
    out = buf[pad + offset:pad + offset + n].view(shape)

    def untouched():
        b = raw.view(-1)
        e = buf.element_size()
        assert bool((b[:(pad + offset) * e] == 255).all()) and bool((b[(pad + offset + n) * e:] == 255).all())

    return out, untouched


def within(got, ref, bound):
    """|got - ref| <= bound element by element (float64 tensors on the CPU); reports the worst ratio."""
    got = got.double().cpu()
    assert got.shape == ref.shape and bool(torch.isfinite(got).all())
    ratio = ((got - ref).abs() / bound.clamp(min=1e-300)).max() if got.numel() else torch.zeros(())
    assert float(ratio) <= 1.0, f"error is {float(ratio):.3g} times its bound"


def rounding(dtype):
    return U_BF16 if dtype == torch.bfloat16 else U


def small(dtype):
    """Half the spacing of the smallest numbers of the type."""
    return 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149
