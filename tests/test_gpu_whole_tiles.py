"""The matrix kernels at sizes that take whole 256 x 256 tiles over several steps of k, in rounds and with loads that run on from tile to tile (tile_cases.py;
test_tile_plans_host.py holds the library to these plans), against sums in 64 bits."""
import pytest
import torch

from tile_cases import GRAD, HEAD, HEAD_K, LOSS, LOSS_D
from vocab_util import BF16, DEV, F32, F64, HALF, gen, normal, within
from xent_bounds import formula

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", HEAD_K)
@pytest.mark.parametrize("T,V", HEAD)
def test_head(T, V, K):
    """Sums are exact; three float32 roundings behind them, and the output's."""
    from paper_2512_00719_amd import vocab
    g = gen(T + K)
    a, b = (torch.randint(-128, 128, (n, K), generator=g, device=DEV).to(torch.int8) for n in (T, V))
    sa, sb = torch.rand(T, generator=g, device=DEV) + 0.01, torch.rand(V, generator=g, device=DEV) + 0.01
    want = (a.to(F64) @ b.to(F64).t()) * sa.to(F64)[:, None] * sb.to(F64)
    for dtype in (F32, BF16):
        out = vocab.linear_int8(a, sa, b, sb, out=torch.full((T, V), 77.0, dtype=dtype, device=DEV))
        within(out, want, want.abs() * (3 * 2.0 ** -24 + (HALF[BF16] if dtype == BF16 else 0) + 2.0 ** -45), "logits")


def _inputs(T, V, D, seed):
    g = gen(seed)
    w = normal((V, D), BF16, g, 2.0 * D ** -0.5)
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    h = (torch.randn(T, D, generator=g, device=DEV) + 2.0 * torch.rand(T, 1, generator=g, device=DEV) * w[y.long()].float()).to(BF16)
    w[:, 0], h[:, 0] = 1.0, 0.0    # (dH's first column is the sum of a row of G: no rounding of the output covers G's)
    y[3::7], y[-1] = -1, V - 1
    return h, w, y, torch.rand(T, generator=g, device=DEV) + 0.5


@pytest.mark.parametrize("D", LOSS_D)
@pytest.mark.parametrize("T,V", LOSS)
def test_loss(T, V, D):
    """Products are exact in float32, a logit's sum off by D + 8 roundings; lse by the largest of its row, 2^-17 and 2^-22 of itself."""
    from paper_2512_00719_amd import vocab
    h, w, y, _ = _inputs(T, V, D, T + D)
    loss, lse = vocab.linear_xent(h, w, y, loss=torch.full((T,), 77.0, device=DEV), lse=torch.full((T,), 77.0, device=DEV))
    h, w = h.to(F64), w.to(F64)
    z = h @ w.t()
    dz = (D + 8) * 2.0 ** -24 * (h.abs() @ w.abs().t()) + z.abs() * 2.0 ** -24
    want = torch.logsumexp(z, 1)
    off = dz.amax(1) + 2.0 ** -17 + want.abs() * 2.0 ** -22
    within(lse, want, off, "lse")
    at = y.clamp(min=0).long()[:, None]
    each = torch.where(y >= 0, want - z.gather(1, at)[:, 0], 0.0)
    within(loss, each, torch.where(y >= 0, off + dz.gather(1, at)[:, 0] + each.abs() * 2.0 ** -24, 0.0), "loss")


@pytest.mark.parametrize("T,V,D", GRAD)
def test_gradient(T, V, D):
    from paper_2512_00719_amd import vocab
    h, w, y, dl = _inputs(T, V, D, T + V)
    want = formula(h, w, y, dl, 1.0)
    lse = vocab.linear_xent(h, w, y)[1]
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse)
    within(dh, want["dh"][0], want["dh"][1], "dh")
    exact, off = want["dw"]
    within(dw, exact, off + exact.abs() * HALF[BF16], "dw")
    full = vocab.linear_xent_grad(dl, h, w, y, lse, dweight=torch.full((V, D), 77.0, device=DEV), need_dhidden=False)[1]
    within(full, exact, off, "dw")
    assert torch.equal(full.to(BF16), dw)
    twice = vocab.linear_xent_grad(dl, h, w, y, lse, dweight=full.clone(), accumulate=True)[1]
    assert torch.equal(twice, full + full)
    added = vocab.linear_xent_grad(dl, h, w, y, lse, dweight=dw.clone(), accumulate=True, need_dhidden=False)[1]
    assert torch.equal(added, (full + dw.float()).to(BF16))
    torch.cuda.empty_cache()


def test_unaligned_gradient():
    """Copies with aligned rows ahead of whole tiles: more than 512 tokens, rows of 1001 values."""
    from paper_2512_00719_amd import vocab
    h, w, y, dl = _inputs(3000, 33_000, 1001, 6)
    want = formula(h, w, y, dl, 1.0)
    lse = vocab.linear_xent(h, w, y)[1]
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse, dweight=torch.full(w.shape, 77.0, device=DEV))
    within(dh, want["dh"][0], want["dh"][1], "dh")
    within(dw, want["dw"][0], want["dw"][1], "dw")
