"""A row's gradient is summed in an order that depends on the ids and their number alone: neither on the width, nor on how rows lie, nor on whether
the tokens are sorted.  So a table's gradient formed by blocks of columns has the bits of the whole one."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, gen, laid, normal

pytestmark = pytest.mark.gpu


def _ids(T, V, kind, g):
    if kind == "one":
        return torch.full((T,), V // 2, dtype=torch.int32, device=DEV)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    if kind == "runs":
        return ids % 5 * (V // 5)
    if kind == "skewed":
        ids = torch.where(torch.rand(T, generator=g, device=DEV) < 0.5, ids % 3, ids)
    if kind == "invalid":
        ids = torch.where(torch.rand(T, generator=g, device=DEV) < 0.5, ids % 3, ids)
        ids[::3] = -1
        ids[1::7] = V
    return ids


@pytest.mark.parametrize("types", [(BF16, F32), (F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("kind", ["one", "runs", "skewed", "invalid"])
@pytest.mark.parametrize("T,D", [(40, 1024), (150, 9000), (300, 1031), (512, 1024), (512, 8200), (513, 1024), (2000, 520), (5000, 300)])
def test_blocks_of_columns_have_the_bits_of_the_whole(T, D, kind, types):
    from paper_2512_00719_amd import vocab
    g = gen(T + D)
    V = 61
    ids, dout = _ids(T, V, kind, g), normal((T, D), types[0], g)
    whole = vocab.embed_grad(ids, dout, V, scale=0.7, dtable=torch.empty(V, D, dtype=types[1], device=DEV))
    for c0, c1 in ((0, 1), (3, 70), (64, 128), (0, 288)):
        block = vocab.embed_grad(ids, dout[:, c0:c1], V, scale=0.7, dtable=torch.empty(V, c1 - c0, dtype=types[1], device=DEV))
        assert torch.equal(block, whole[:, c0:c1]), (c0, c1)
    other = vocab.embed_grad(ids, laid(dout, 3, 1), V, scale=0.7, dtable=laid(torch.empty_like(whole), 5, 3))
    assert torch.equal(other, whole)
