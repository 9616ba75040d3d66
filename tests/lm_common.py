"""Helpers of the tests of the language-model operators: types with their rounding, strided copies, comparisons."""

import torch

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}   # half a unit in the last place, relative
LEAST = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}  # smallest positive number
EPS = 2.0 ** -24


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def apart(t, ld, shift=0):
    """The matrix t with rows ld elements apart, the first `shift` elements into its memory; NaN in between."""
    rows, cols = t.shape
    buf = torch.full((max(1, rows) * ld + shift,), float("nan"), dtype=t.dtype, device=t.device)
    view = buf[shift:shift + max(1, rows) * ld].view(max(1, rows), ld)[:rows, :cols]
    view.copy_(t)
    return view


def within(got, want, tol, what=""):
    """Every |got - want| <= tol, both finite in the same places; got of any type, want and tol in 64 bits."""
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    both = torch.isfinite(got) & torch.isfinite(want)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~torch.where(both, (got - want).abs() <= tol, same)
    if bad.any():
        at = bad.nonzero()[0].tolist()
        g, w = got[tuple(at)].item(), want[tuple(at)].item()
        t = tol.expand_as(want)[tuple(at)].item() if torch.is_tensor(tol) else tol
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: {g} for {w}, allowed {t}")
