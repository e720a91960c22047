"""How many bits the cross entropy's gradients keep, element by element (the bounds are xent_bounds.formula's).  With one bfloat16 value for G, 2^-8, each
test here fails but that of large logits, whose sums' own errors are larger."""
import math

import pytest
import torch

from vocab_util import BF16, DEV, F32, F64, gen, normal, within
from xent_bounds import formula

pytestmark = pytest.mark.gpu


def _check(h, w, y, dl, c=1.0):
    from paper_2512_00719_amd import vocab
    want = formula(h, w, y, dl, float(torch.tensor(c, dtype=F32)))
    lse = vocab.linear_xent(h, w, y, logit_scale=c)[1]
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse, logit_scale=c, dweight=torch.empty(w.shape, dtype=F32, device=DEV))
    within(dh, want["dh"][0], want["dh"][1] + 1e-37, "dh")
    within(dw, want["dw"][0], want["dw"][1] + 1e-37, "dw")
    return want, dh, dw


def _inputs(T, V, D, seed, lean):
    """Weights whose first column is 1, before states of 0: there dH is the sum of a row of G, which is 0 but for G's errors, and no rounding of an output
    covers them.  Targets are all different where there are enough of them, so that a row of dW is one token's for the most part."""
    g = gen(seed)
    w = normal((V, D), BF16, g, 2.0 * D ** -0.5)
    y = torch.randperm(V, generator=g, device=DEV)[:T].to(torch.int32) if T <= V else torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    h = (torch.randn(T, D, generator=g, device=DEV) + lean * w[y.long()].float()).to(BF16)
    w[:, 0], h[:, 0] = 1.0, 0.0
    return h, w, y


SHAPES = [(3, 200, 64), (16, 1000, 72), (33, 515, 136), (64, 4100, 64), (65, 700, 64), (130, 1024, 200), (300, 4100, 96), (777, 1500, 100), (1000, 600, 264)]


@pytest.mark.parametrize("c", [1.0, 0.7])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_bits_of_ordinary_rows(T, V, D, c):
    h, w, y = _inputs(T, V, D, T + V, torch.rand(T, 1, generator=gen(7), device=DEV) * 2)
    dl = torch.randn(T, generator=gen(8), device=DEV)
    _check(h, w, y, dl, c)


@pytest.mark.parametrize("T,V,D", SHAPES)
def test_bits_of_rows_that_are_nearly_certain(T, V, D):
    """Targets of probability 1/2 to 1 - 2^-20: a row's power of two is its own."""
    h, w, y = _inputs(T, V, D, T + V + 1, torch.linspace(2.0, 7.0, T, device=DEV)[:, None])
    want, _, _ = _check(h, w, y, torch.rand(T, generator=gen(9), device=DEV) + 0.5)
    assert float(want["left"].min()) < 2.0 ** -12 and float(want["left"].max()) > 2.0 ** 8 * float(want["left"].min())


@pytest.mark.parametrize("T,V,D", SHAPES[1:])
def test_bits_where_the_losses_weights_differ(T, V, D):
    """dloss from 1 to 2^-24 in one call, of either sign."""
    h, w, y = _inputs(T, V, D, T + V + 2, 1.0)
    sign = torch.where(torch.arange(T, device=DEV) % 2 == 0, 1.0, -1.0)
    _check(h, w, y, sign * 2.0 ** -torch.linspace(0, 24, T, device=DEV).floor())


@pytest.mark.parametrize("scale", [2.0 ** -40, 2.0 ** 40])
@pytest.mark.parametrize("T", [40, 200])
def test_bits_where_all_weights_of_the_loss_are_small_or_large(T, scale):
    h, w, y = _inputs(T, 900, 72, T, 1.5)
    _check(h, w, y, (torch.rand(T, generator=gen(3), device=DEV) + 0.5) * scale)


@pytest.mark.parametrize("T", [20, 200, 600])
def test_large_logits(T):
    """Logits of hundreds: rows in which one column holds all, most of them not the target's, where p is 0 or 1 but for 2^-24."""
    g = gen(4)
    V, D = 3000, 64
    w, h = normal((V, D), BF16, g, 50.0), normal((T, D), BF16, g)
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    z = h.to(F64) @ w.to(F64).t()
    y[::3] = z.argmax(1)[::3].to(torch.int32)
    _check(h, w, y, torch.ones(T, device=DEV))


@pytest.mark.parametrize("T", [40, 200])
def test_a_column_that_is_improbable_under_every_token(T):
    """Its row of dW is as small as its probability: with p about 2^-27 of 1 - p_y it has the bits of the others, with 2^-35 (steps of 2^-38) three or
    four.  Up to 64 tokens it always has them."""
    V, D = 300, 64
    h, w, y = _inputs(T, V, D, T, 0.5)
    y = torch.where(y < 2, y + 2, y)
    h[:, 1], w[:, 1] = 1.0, 0.0
    for column, down in ((0, 16), (1, 24)):
        w[column, 1:] = 0.0
        w[column, 1] = -down * math.log(2.0)
    want, _, dw = _check(h, w, y, torch.ones(T, device=DEV))
    exact = want["dw"][0]
    off = ((dw.to(F64) - exact).norm(dim=1) / exact.norm(dim=1)).tolist()
    assert off[0] < 2.0 ** -10 and off[1] < (2.0 ** -10 if T <= 64 else 2.0 ** -3), off[:2]
