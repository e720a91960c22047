"""The norm and its gradient with their outputs in place of inputs, as the boundary allows: the bits of the call with outputs of their own on the same
layout.  Rows that are not aligned are taken in groups of which a row's last overlaps its neighbour's, so that one thread reads what another writes."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, gen, laid, normal, padding_untouched

pytestmark = pytest.mark.gpu
LAYOUTS = [(0, 0), (3, 1), (8, 8), (1, 0)]
WIDTHS = [1, 7, 64, 65, 513, 1001, 1025, 1033, 2047, 4095, 4100, 8191, 8195, 16_001]


def _same(layout, *tensors):
    return [laid(t.clone(), *layout) for t in tensors]


def _padding_untouched(t, layout):
    return layout == (0, 0) or padding_untouched(t, *layout)    # (laid() makes no padding then)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("D", WIDTHS)
def test_norm(D, layout, dtype):
    from paper_2512_00719_amd import vocab
    T, g = 37, gen(D)
    x, r = normal((T, D), dtype, g), normal((T, D), dtype, g, 3.0)
    w = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dtype)
    lx, lr, lh, lo = _same(layout, x, r, torch.zeros_like(x), torch.zeros_like(x))
    y, h, rstd = vocab.rms_norm(lx, w, residual=lr, h=lh, out=lo, need_rstd=True)
    codes, scales, _ = vocab.rms_norm_int8(lx, w, residual=lr, h=lh)
    alone = vocab.rms_norm(lx, w, out=laid(torch.zeros_like(x), *layout))[0]
    uses = []
    a, b = _same(layout, x, r)      # the sum in the residual's place, and the output in x's
    got = vocab.rms_norm(a, w, residual=b, h=b, out=a, need_rstd=True)
    uses.append((got[0], y, a)), uses.append((got[1], h, b))
    assert torch.equal(got[2], rstd)
    a, b, c = _same(layout, x, r, torch.zeros_like(x))      # the sum in x's place
    got = vocab.rms_norm(a, w, residual=b, h=a, out=c)
    uses.append((got[0], y, c)), uses.append((got[1], h, a))
    assert torch.equal(b, r)
    a, = _same(layout, x)           # no residual, the output in x's place
    uses.append((vocab.rms_norm(a, w, out=a)[0], alone, a))
    for place in (0, 1):            # the sum in x's or the residual's place beside codes
        ab = _same(layout, x, r)
        got = vocab.rms_norm_int8(ab[0], w, residual=ab[1], h=ab[place])
        assert torch.equal(got[0], codes) and torch.equal(got[1], scales)
        uses.append((got[2], h, ab[place]))
    for got, want, place in uses:
        assert got.data_ptr() == place.data_ptr() and torch.equal(got, want)
        assert _padding_untouched(place, layout)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("T", [3, 37, 2100])
def test_gradient(T, D, layout, dtype):
    from paper_2512_00719_amd import vocab
    g = gen(T + D)
    h, dy, dh = (normal((T, D), dtype, g) for _ in range(3))
    w = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dtype)
    rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-6)).float()
    lh, ldy, ldh, ldx = _same(layout, h, dy, dh, torch.zeros_like(h))
    dx, dw = vocab.rms_norm_grad(ldy, lh, w, rstd, dh=ldh, dx=ldx)
    for name in ("dy", "dh"):
        a, b = _same(layout, dy, dh)
        place = a if name == "dy" else b
        got = vocab.rms_norm_grad(a, lh, w, rstd, dh=b, dx=place)
        assert got[0].data_ptr() == place.data_ptr() and torch.equal(got[0], dx) and torch.equal(got[1], dw), name
        assert _padding_untouched(place, layout)
    a, = _same(layout, dy)
    alone = vocab.rms_norm_grad(ldy, lh, w, rstd, dx=laid(torch.zeros_like(h), *layout))
    got = vocab.rms_norm_grad(a, lh, w, rstd, dx=a)
    assert torch.equal(got[0], alone[0]) and torch.equal(got[1], alone[1]) and _padding_untouched(a, layout)
