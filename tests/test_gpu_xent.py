"""The cross entropy over a head's logits and its gradient against the formulas in 64 bits.

Bounds.  Products of bfloat16 values are exact in float32; a logit is a sum of D of them, off by at most
dz = (D + 8) 2^-24 sum |h w| in whatever order it is formed.  lse is off by at most the largest dz of its row, and by its own arithmetic
(a sum of at most V positive terms in blocks, an exponential and a logarithm: 2^-17, and 2^-22 of its size).  G's rounding to bfloat16 is 2^-8 of
an element, its p is off by twice dz and 2^-17; the products' sums are off by at most 2^-24 (their length / 32 + 64) of the sum of
magnitudes, and an output's own rounding comes on top."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, F64, HALF, gen, laid, normal, padding_untouched, within

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 1), (1, 7, 8), (3, 64, 16), (16, 65, 64), (17, 300, 100), (40, 1000, 72), (64, 256, 264), (65, 513, 33), (128, 777, 128), (130, 1024, 200),
          (257, 515, 96), (300, 4100, 64), (1000, 600, 520), (5, 20_000, 40), (2, 70_001, 24)]


def _inputs(T, V, D, seed, sigma=2.0):
    g = gen(seed)
    w = normal((V, D), BF16, g, sigma * D ** -0.5)
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    lean = 2.0 * torch.rand(T, 1, generator=g, device=DEV)
    h = (torch.randn(T, D, generator=g, device=DEV) + lean * w[y.long()].float()).to(BF16)
    dl = torch.randn(T, generator=g, device=DEV)
    if T > 2:   # masked in each of the ways there are
        y[1] = -1
        y[2::5] = V
        y[3::7] = -100
        dl[4::6] = 0
    return h, w, y, dl


def _formula(h, w, y, dl, c):
    h, w, dl = h.to(F64), w.to(F64), dl.to(F64)
    T, V, D = h.shape[0], w.shape[0], h.shape[1]
    z = c * (h @ w.t())
    dz = c * (D + 8) * 2.0 ** -24 * (h.abs() @ w.abs().t()) + z.abs() * 2.0 ** -24
    lse = torch.logsumexp(z, 1)
    ok = (y >= 0) & (y < V)
    at = torch.where(ok, y, torch.zeros_like(y)).long()[:, None]
    loss = torch.where(ok, lse - z.gather(1, at)[:, 0], 0.0)
    lse_off = dz.amax(1) + 2.0 ** -17 + lse.abs() * 2.0 ** -22
    loss_off = torch.where(ok, lse_off + dz.gather(1, at)[:, 0] + loss.abs() * 2.0 ** -24, 0.0)
    d = torch.where(ok, dl, 0.0)[:, None] * c
    p = (z - lse[:, None]).exp()
    g = p.clone()
    g.scatter_add_(1, at, torch.full_like(lse[:, None], -1.0))
    g = g * d
    g_off = g.abs() * (2.0 ** -8 + 2.0 ** -17) + (p * d.abs()) * (2 * dz + 2.0 ** -17)
    sums = lambda n: 2.0 ** -24 * (n / 32 + 64)  # noqa: E731
    dh, dw = g @ w, g.t() @ torch.where((d != 0), h, 0.0)
    size_h, size_w = g.abs() @ w.abs(), g.abs().t() @ h.abs()
    return {"lse": (lse, lse_off), "loss": (loss, loss_off),
            "dh": (dh, g_off @ w.abs() + size_h * sums(V) + dh.abs() * HALF[BF16]),
            "dw": (dw, g_off.t() @ h.abs() + size_w * sums(T)), "ok": ok}


def _check(got, pair, what, dtype=F32):
    want, off = pair
    within(got, want, off + want.abs() * (HALF[dtype] if what == "dw" else 0) + 1e-30, what)


@pytest.mark.parametrize("c", [1.0, 0.7])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_loss_and_gradient(T, V, D, c):
    from paper_2512_00719_amd import vocab
    h, w, y, dl = _inputs(T, V, D, T * 3 + V + D)
    want = _formula(h, w, y, dl, float(torch.tensor(c, dtype=F32)))
    loss, lse = vocab.linear_xent(h, w, y, logit_scale=c)
    _check(lse, want["lse"], "lse")
    _check(loss, want["loss"], "loss")
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse, logit_scale=c)
    _check(dh, want["dh"], "dh")
    _check(dw, want["dw"], "dw", BF16)
    # one output without the other, in float32, added to what is there; the same bits again
    assert torch.equal(vocab.linear_xent_grad(dl, h, w, y, lse, logit_scale=c, need_dweight=False)[0], dh)
    only, old = vocab.linear_xent_grad(dl, h, w, y, lse, logit_scale=c, need_dhidden=False)
    assert only is None and torch.equal(old, dw)
    full = vocab.linear_xent_grad(dl, h, w, y, lse, logit_scale=c, dweight=torch.full((V, D), 9.0, device=DEV), need_dhidden=False)[1]
    _check(full, want["dw"], "dw", F32)
    twice = vocab.linear_xent_grad(dl, h, w, y, lse, logit_scale=c, dweight=full.clone(), accumulate=True, need_dhidden=False)[1]
    assert torch.equal(twice, full + full)


@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (1, 0), (3, 5)])
@pytest.mark.parametrize("T,V,D", [(3, 70, 40), (70, 300, 136), (200, 515, 64)])
def test_strides_and_alignments(T, V, D, pad, shift):
    from paper_2512_00719_amd import vocab
    h, w, y, dl = _inputs(T, V, D, 5)
    want = _formula(h, w, y, dl, 1.0)
    lh, lw = laid(h, pad, shift), laid(w, pad, shift)
    loss, lse = vocab.linear_xent(lh, lw, y)
    _check(lse, want["lse"], "lse")
    _check(loss, want["loss"], "loss")
    dh, dw = (laid(torch.zeros(s, dtype=BF16, device=DEV), pad, shift) for s in ((T, D), (V, D)))
    vocab.linear_xent_grad(dl, lh, lw, y, lse, dhidden=dh, dweight=dw)
    _check(dh, want["dh"], "dh")
    _check(dw, want["dw"], "dw", BF16)
    assert padding_untouched(dh, pad, shift) and padding_untouched(dw, pad, shift)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,shift", [(24, 0), (24, 8), (1, 3)])
@pytest.mark.parametrize("T,D", [(5, 40), (50, 104)])
def test_few_tokens_weight_gradient_added_in_place(T, D, pad, shift, dtype):
    """Rows of whole 64 bytes (pad 24) with a short last piece, and others: the sum with zeros is the gradient bit for bit, padding stays."""
    from paper_2512_00719_amd import vocab
    V = 333
    h, w, y, dl = _inputs(T, V, D, 8)
    want = _formula(h, w, y, dl, 1.0)
    lse = vocab.linear_xent(h, w, y)[1]
    plain, added, twice = (laid(torch.zeros(V, D, dtype=dtype, device=DEV), pad, shift) for _ in range(3))
    vocab.linear_xent_grad(dl, h, w, y, lse, dweight=plain, need_dhidden=False)
    _check(plain, want["dw"], "dw", dtype)
    vocab.linear_xent_grad(dl, h, w, y, lse, dweight=added, accumulate=True, need_dhidden=False)
    assert torch.equal(added, plain)
    twice.fill_(1.0)
    vocab.linear_xent_grad(dl, h, w, y, lse, dweight=twice, accumulate=True, need_dhidden=False)
    value, off = want["dw"]
    within(twice, value + 1.0, off + (value + 1.0).abs() * HALF[dtype] + 1e-30, "dw")
    assert all(padding_untouched(t, pad, shift) for t in (plain, added, twice))


def test_pieces_of_the_vocabulary():
    """More than one piece, the last of them short: 40,000 tokens have pieces of 4096 rows."""
    from paper_2512_00719_amd import vocab
    T, V, D = 40_000, 8200, 16
    h, w, y, dl = _inputs(T, V, D, 2)
    want = _formula(h, w, y, dl, 1.0)
    loss, lse = vocab.linear_xent(h, w, y)
    _check(loss, want["loss"], "loss")
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse)
    _check(dh, want["dh"], "dh")
    _check(dw, want["dw"], "dw", BF16)


@pytest.mark.parametrize("T", [6, 100, 300])
def test_masked_tokens_keep_what_they_hold(T):
    """States of tokens that take no part may be anything: gradients are those without them, bit for bit those of zeros there."""
    from paper_2512_00719_amd import vocab
    V, D = 1000, 72
    h, w, y, dl = _inputs(T, V, D, 8)
    off = (y < 0) | (y >= V) | (dl == 0)
    assert bool(off.any())
    clean, dirty = h.clone(), h.clone()
    clean[off] = 0
    dirty[off] = float("nan")
    dirty[torch.nonzero(off)[0, 0]] = float("inf")
    a = vocab.linear_xent(clean, w, y)
    b = vocab.linear_xent(dirty, w, y)
    assert torch.equal(a[0][~off], b[0][~off]) and not b[0][(y < 0) | (y >= V)].any()
    ga, gb = vocab.linear_xent_grad(dl, clean, w, y, a[1]), vocab.linear_xent_grad(dl, dirty, w, y, b[1])
    assert torch.equal(ga[0], gb[0]) and torch.equal(ga[1], gb[1])
    assert not gb[0][off].any() and bool(gb[1].isfinite().all())
    none = torch.full_like(y, -1)   # nothing takes part
    loss, lse = vocab.linear_xent(clean, w, none)
    dh, dw = vocab.linear_xent_grad(dl, clean, w, none, lse)
    assert not loss.any() and not dh.any() and not dw.any()


def test_large_logits_and_bad_states():
    from paper_2512_00719_amd import vocab
    T, V, D = 20, 3000, 64
    h, w, y, dl = _inputs(T, V, D, 4, sigma=400.0)   # logits of thousands: one column holds all
    want = _formula(h, w, y, dl, 1.0)
    loss, lse = vocab.linear_xent(h, w, y)
    _check(lse, want["lse"], "lse")
    _check(loss, want["loss"], "loss")
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse)
    assert bool(dh.isfinite().all()) and bool(dw.isfinite().all())
    bad = h.clone()
    bad[0, 3] = float("nan")
    loss2, lse2 = vocab.linear_xent(bad, w, y)
    assert bool(lse2[0].isnan()) and torch.equal(loss2[1:], loss[1:])


def test_gradient_against_differences():
    """Central differences of the loss itself along a direction whose steps are exact in bfloat16: states are multiples of 2^-4 below 1, the step is
    2^-5 up and down.  Logits move by at most sum |d w| / 32 < 0.25, so the cubic term is below 0.25^2 / 6 < 2^-6 of the slope's size
    sum |G| |dz|; the losses' float32 error, 2^-18 each at their size, is below 2^-8 of it, G's and the output's rounding 2^-7."""
    from paper_2512_00719_amd import vocab
    T, V, D = 24, 500, 32
    g = gen(9)
    h = (torch.randint(-15, 16, (T, D), generator=g, device=DEV) / 16).to(BF16)
    d = torch.randint(-1, 2, (T, D), generator=g, device=DEV).to(BF16) / 32
    w = normal((V, D), BF16, g, 0.3)
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    dl = torch.rand(T, generator=g, device=DEV) + 0.5
    loss = lambda x: float((vocab.linear_xent(x.to(BF16), w, y)[0].to(F64) * dl.to(F64)).sum())  # noqa: E731
    up, down = h.float() + d.float(), h.float() - d.float()
    assert torch.equal(up.to(BF16).float(), up) and torch.equal(down.to(BF16).float(), down)
    _, lse = vocab.linear_xent(h, w, y)
    dh, _ = vocab.linear_xent_grad(dl, h, w, y, lse)
    slope = float((dh.to(F64) * d.to(F64)).sum())
    z, step = h.to(F64) @ w.to(F64).t(), (d.to(F64) @ w.to(F64).t()).abs()
    p = torch.softmax(z, 1)
    size = float((dl.to(F64)[:, None] * p * step).sum() + (dl.to(F64) * step.gather(1, y.long()[:, None])[:, 0]).sum())
    assert float(step.max()) < 0.25
    assert abs((loss(up) - loss(down)) / 2 - slope) < (2.0 ** -6 + 2.0 ** -8 + 2.0 ** -7) * size


def test_no_tokens():
    from paper_2512_00719_amd import vocab
    w = torch.ones(300, 24, dtype=BF16, device=DEV)
    h, f, y = w[:0], torch.zeros(0, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV)
    loss, lse = vocab.linear_xent(h, w, y)
    assert loss.shape == (0,) and lse.shape == (0,)
    dh, dw = vocab.linear_xent_grad(f, h, w, y, f, dweight=w.clone())
    assert dh.shape == (0, 24) and not dw.any()
    assert torch.equal(vocab.linear_xent_grad(f, h, w, y, f, dweight=w.clone(), accumulate=True)[1], w)


def test_copies_with_aligned_rows_in_more_than_one_piece():
    """More than 512 tokens and 65,536 rows of 19 values: the weights are copied a piece at a time, forward and for the gradient."""
    from paper_2512_00719_amd import vocab
    h, w, y, dl = _inputs(530, 66_000, 19, 6)
    want = _formula(h, w, y, dl, 1.0)
    loss, lse = vocab.linear_xent(h, w, y)
    _check(lse, want["lse"], "lse")
    _check(loss, want["loss"], "loss")
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse)
    _check(dh, want["dh"], "dh")
    _check(dw, want["dw"], "dw", BF16)


@pytest.mark.parametrize("T", [3, 40])
def test_few_tokens_against_more_than_one_piece(T):
    """A vocabulary of more than 2^20 rows, which is taken in two pieces."""
    from paper_2512_00719_amd import vocab
    h, w, y, dl = _inputs(T, 1_100_000, 8, T)
    y[0] = 1_099_999
    want = _formula(h, w, y, dl, 1.0)
    loss, lse = vocab.linear_xent(h, w, y)
    _check(loss, want["loss"], "loss")
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse)
    _check(dh, want["dh"], "dh")
    _check(dw, want["dw"], "dw", BF16)
