"""Shared by the tests of the operators at the vocabulary: inputs, padded and offset views, comparison with bounds an element."""
import torch

DEV = "cuda:0"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}  # the largest relative error of one rounding: 8 and 24 significant bits


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(shape, dtype, g, sigma=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def laid(t, pad, shift):
    """The matrix `t` with `pad` more elements a row, its first one `shift` elements into an allocation: any alignment."""
    if pad == 0 and shift == 0:
        return t
    rows, n = t.shape
    flat = torch.full((rows * (n + pad) + shift + 8,), 77, dtype=t.dtype, device=t.device)
    v = flat[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n]
    v.copy_(t)
    return v


def padding_untouched(v, pad, shift):
    """Whether what lies between and around the rows of laid() still holds its value."""
    rows, n = v.shape
    flat = torch.as_strided(v, (rows * (n + pad) + shift + 8,), (1,), v.storage_offset() - shift)
    keep = torch.ones_like(flat, dtype=torch.bool)
    keep[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n] = False
    return bool((flat[keep] == 77).all())


def within(got, want, bound, what):
    """Every element of `got` within `bound` (a tensor or a number) of `want`, both in 64 bits."""
    off = (got.to(F64) - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), float(off[bad].max()) if bool(bad.any()) else 0.0,
                                 torch.nonzero(bad)[:3].tolist())
