"""The root-mean-square norm, its 8-bit form and its gradient against the formulas in 64 bits.

Bounds.  A row's sum of squares is a sum of positive float32 terms in which a term passes through at most 32 additions of its
thread and 10 of the reduction: relative error below 64 * 2^-24 = 2^-18; its square root halves that, the few products
behind it add 2^-24 each.  ARITH = 2^-17 covers them, and the output's one rounding comes on top."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, F64, HALF, gen, laid, normal, padding_untouched, within

pytestmark = pytest.mark.gpu
ARITH = 2.0 ** -17

SHAPES = [(1, 1), (3, 7), (5, 64), (1, 513), (130, 512), (9, 1000), (2, 1024), (7, 1025), (33, 2048), (4, 4095), (12, 4096),
          (3, 5078), (2, 8192), (2, 8193), (3, 16_384), (1, 32_768), (2, 32_767)]


def _inputs(T, D, dtype, residual, seed):
    g = gen(seed)
    x = normal((T, D), dtype, g)
    r = normal((T, D), dtype, g, 3.0) if residual else None
    w = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dtype)
    return x, r, w


def _codes(u):
    """rint(u * (127 / max |u|)) in float32 on the CPU.  (127.0 / tensor would be a reciprocal and a product, two roundings.)"""
    u = u.cpu()
    top = u.abs().amax(1)
    return torch.round(u * torch.div(torch.full_like(top, 127.0), top)[:, None]).to(torch.int8)


def _stream(x, r):
    return x if r is None else (x.float() + r.float()).to(x.dtype)


def _rstd(h, eps):
    return 1.0 / torch.sqrt(h.to(F64).square().mean(1) + eps)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,D", SHAPES)
def test_norm_and_codes(T, D, residual, dtype):
    from paper_2512_00719_amd import vocab
    x, r, w = _inputs(T, D, dtype, residual, T * 131 + D)
    h = _stream(x, r)
    s = _rstd(h, 1e-5)
    want = h.to(F64) * s[:, None] * w.to(F64)
    y, got_h, rstd = vocab.rms_norm(x, w, eps=1e-5, residual=r, need_rstd=True)
    assert torch.equal(got_h, h)
    within(y, want, want.abs() * (ARITH + HALF[dtype]), "y")
    within(rstd, s, s * ARITH, "rstd")
    codes, scales, got_h = vocab.rms_norm_int8(x, w, eps=1e-5, residual=r)
    assert torch.equal(got_h, h)
    # codes bit for bit: products, one division and one rounding in float32, no sum
    assert torch.equal(codes.cpu(), _codes(h.float() * w.float()))
    within(scales, want.abs().amax(1) / 127, want.abs().amax(1) / 127 * ARITH, "scales")
    codes, scales = vocab.quantize_rows(h)
    assert torch.equal(codes.cpu(), _codes(h.float()))
    top = h.to(F64).abs().amax(1) / 127
    within(scales, top, top * ARITH, "row scales")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,shift", [(1, 0), (2, 2), (8, 0), (8, 8), (3, 5)])
@pytest.mark.parametrize("D", [48, 1000, 4098])
def test_strides_and_alignments(D, pad, shift, dtype):
    from paper_2512_00719_amd import vocab
    x, r, w = _inputs(6, D, dtype, True, D + pad)
    ref = vocab.rms_norm(x, w, residual=r, need_rstd=True)
    refq = vocab.rms_norm_int8(x, w, residual=r)
    lay = lambda t: laid(t, pad, shift)  # noqa: E731
    empty = lambda dt: lay(torch.zeros(6, D, dtype=dt, device=DEV))  # noqa: E731
    h, out, q = empty(dtype), empty(dtype), empty(torch.int8)
    wide = torch.full((D + shift,), 1.0, dtype=dtype, device=DEV)
    wide[shift:] = w
    y, _, rstd = vocab.rms_norm(lay(x), wide[shift:], residual=lay(r), h=h, out=out, need_rstd=True)
    # (a row is summed by other groups of values where it is not aligned, hence not bit for bit)
    within(y, ref[0].to(F64), ref[0].to(F64).abs() * (2 * ARITH + 2 * HALF[dtype]), "y")
    assert torch.equal(h, ref[1])
    codes, scales, _ = vocab.rms_norm_int8(lay(x), w, residual=lay(r), h=h, codes=q)
    assert torch.equal(codes, refq[0])
    within(scales, refq[1].to(F64), refq[1].to(F64) * ARITH, "scales")
    for t in (h, out, q):
        assert padding_untouched(t, pad, shift)
    dy, dh = normal((6, D), dtype, gen(9)), normal((6, D), dtype, gen(10))
    dx = empty(dtype)
    a = vocab.rms_norm_grad(dy, ref[1], w, ref[2], dh=dh)
    b = vocab.rms_norm_grad(lay(dy), lay(ref[1]), w, ref[2], dh=lay(dh), dx=dx)
    assert padding_untouched(dx, pad, shift)
    size = a[0].to(F64).abs().amax(1, keepdim=True)
    within(b[0], a[0].to(F64), size * ARITH + a[0].to(F64).abs() * 2 * HALF[dtype], "dx")
    within(b[1], a[1].to(F64), 2.0 ** -20 * 6 * a[1].to(F64).abs().max(), "dweight")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,D", SHAPES + [(1030, 64), (2500, 1000), (1100, 2048)])
def test_gradient_against_the_formula(T, D, residual, dtype):
    """A token's term passes through at most 3 additions of its workgroup's rows, 32 of a group of workgroups and 32 of the groups:
    dweight is within 128 * 2^-24 = 2^-17 of the sum of its terms' magnitudes."""
    from paper_2512_00719_amd import vocab
    h, dh, w = _inputs(T, D, dtype, residual, 3 * T + D)
    dy = normal((T, D), dtype, gen(T + D))
    rstd = _rstd(h, 1e-6).float()
    dx, dw = vocab.rms_norm_grad(dy, h, w, rstd, dh=dh)
    s = rstd.to(F64)[:, None]
    n, g = h.to(F64) * s, dy.to(F64) * w.to(F64)
    m = (g * n).mean(1, keepdim=True)
    extra = 0.0 if dh is None else dh.to(F64)
    want = s * (g - n * m) + extra
    size = s * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)) + (0.0 if dh is None else dh.to(F64).abs())
    within(dx, want, size * ARITH + want.abs() * HALF[dtype], "dx")
    terms = dy.to(F64) * n
    within(dw, terms.sum(0), terms.abs().sum(0) * 2.0 ** -17, "dweight")


def test_gradient_against_differences():
    """(L(v + e d) - L(v - e d)) / 2e against <gradient, d>, L = sum of the norm's output times fixed factors, float32.  With e = 2^-7 and unit
    directions in inputs of size 1 the cubic term is below e^2 = 2^-14 of the slope's size |c| |d|, and the outputs' rounding, 2^-24 of each of
    T D terms, is 2^-24 sqrt(T D) / e = 2^-11 of it at most: 2^-9 holds both."""
    from paper_2512_00719_amd import vocab
    T, D, e = 16, 96, 2.0 ** -7
    g = gen(5)
    x, r, c, d = (normal((T, D), F32, g) for _ in range(4))
    w, dw_dir = 1 + 0.1 * normal((D,), F32, g), normal((D,), F32, g)
    ch = normal((T, D), F32, g)

    def loss(x, w):
        y, h, _ = vocab.rms_norm(x, w, residual=r)
        return float((y.to(F64) * c.to(F64)).sum() + (h.to(F64) * ch.to(F64)).sum())

    _, h, rstd = vocab.rms_norm(x, w, residual=r, need_rstd=True)
    dx, dw = vocab.rms_norm_grad(c, h, w, rstd, dh=ch)
    size = float(c.norm() * d.norm())
    assert abs((loss(x + e * d, w) - loss(x - e * d, w)) / (2 * e) - float((dx.to(F64) * d).sum())) < 2.0 ** -9 * size
    assert abs((loss(x, w + e * dw_dir) - loss(x, w - e * dw_dir)) / (2 * e) - float((dw.to(F64) * dw_dir).sum())) < 2.0 ** -9 * size


def test_rows_of_zeros_infinities_and_nan():
    from paper_2512_00719_amd import vocab
    x = normal((6, 640), F32, gen(1))
    x[1] = 0
    x[2, 17] = float("inf")
    x[3, 600] = float("nan")
    x[4] = 2.0 ** -130          # below what 127 can be divided by
    x[5, 3] = -3.0e38           # the largest magnitudes
    w = torch.ones(640, device=DEV)
    codes, scales = vocab.quantize_rows(x)
    assert not codes[1].any() and float(scales[1]) == 0 and not codes[4].any() and float(scales[4]) == 0
    assert not codes[2:4].any() and bool(scales[2:4].isnan().all())
    assert int(codes[5, 3]) == -127 and bool(scales[5].isfinite())
    codes, scales, _ = vocab.rms_norm_int8(x, w)
    assert not codes[1].any() and float(scales[1]) == 0 and bool(scales[2:4].isnan().all())
    y, _, rstd = vocab.rms_norm(x, w, eps=1e-6, need_rstd=True)
    assert not y[1].any() and bool(y[3].isnan().all()) and bool(y[0].isfinite().all())
    dx, dw = vocab.rms_norm_grad(torch.ones_like(x[:2]), x[:2], w, rstd[:2])
    assert bool(dx.isfinite().all()) and bool(dw.isfinite().all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place_and_no_rows(dtype):
    from paper_2512_00719_amd import vocab
    x, r, w = _inputs(40, 1032, dtype, True, 4)
    y, h, rstd = vocab.rms_norm(x, w, residual=r, need_rstd=True)
    r2, x2 = r.clone(), x.clone()
    y2, h2, _ = vocab.rms_norm(x2, w, residual=r2, h=r2, out=x2)
    assert y2.data_ptr() == x2.data_ptr() and h2.data_ptr() == r2.data_ptr()
    assert torch.equal(y2, y) and torch.equal(h2, h)
    dy = normal((40, 1032), dtype, gen(7))
    dx, dw = vocab.rms_norm_grad(dy, h, w, rstd, dh=r)
    dy2 = dy.clone()
    assert torch.equal(vocab.rms_norm_grad(dy2, h, w, rstd, dh=r, dx=dy2)[0], dx)
    assert torch.equal(vocab.rms_norm_grad(dy, h, w, rstd, dh=r)[1], dw)  # the same bits again
    none = x[:0]
    assert vocab.rms_norm(none, w)[0].shape == (0, 1032) and vocab.rms_norm_int8(none, w)[0].shape == (0, 1032)
    assert not vocab.rms_norm_grad(none, none, w, rstd[:0], dweight=torch.ones(1032, device=DEV))[1].any()
