"""Calls whose workgroups times their threads pass 2^32, more than one launch takes: every row is there, the last ones too."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, F64, gen, within

pytestmark = pytest.mark.gpu


def _room(nbytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < nbytes:
        pytest.skip(f"wants {nbytes >> 30} GiB of device memory")


def test_norm_of_more_rows_than_a_launch_has_waves():
    """2^26 and some rows of one value, a wave each: y = x / sqrt(x^2 + eps) * w."""
    from paper_2512_00719_amd import vocab
    T = 2 ** 26 + 1003
    x = torch.randn(T, 1, generator=gen(1), device=DEV).to(BF16)
    x[x == 0] = 1.0
    w = torch.full((1,), 1.5, dtype=BF16, device=DEV)
    out = torch.full_like(x, 77)
    _, _, rstd = vocab.rms_norm(x, w, eps=1e-3, out=out, need_rstd=True)
    s = 1.0 / torch.sqrt(x[:, 0].to(F64).square() + 1e-3)
    within(rstd, s, s * 2.0 ** -17, "rstd")
    want = x[:, 0].to(F64) * s * 1.5
    within(out[:, 0], want, want.abs() * (2.0 ** -17 + 2.0 ** -8), "y")
    codes, scales = vocab.quantize_rows(x, codes=torch.zeros(T, 1, dtype=torch.int8, device=DEV), scales=torch.zeros(T, device=DEV))
    assert torch.equal(codes[:, 0].float(), 127 * x[:, 0].float().sign())
    top = x[:, 0].to(F64).abs() / 127
    within(scales, top, top * 2.0 ** -23, "scales")
    codes, scales, _ = vocab.rms_norm_int8(x, w, eps=1e-3, codes=torch.zeros_like(codes), scales=torch.zeros_like(scales))
    assert torch.equal(codes[:, 0].float(), 127 * x[:, 0].float().sign())
    within(scales, want.abs() / 127, want.abs() / 127 * 2.0 ** -17, "scales")


def test_lookup_of_more_rows_than_a_launch_has_threads_for():
    """2^26 and some rows of 129 float32 values, four by a workgroup of 256."""
    from paper_2512_00719_amd import vocab
    T, D = 2 ** 26 + 77, 129
    _room(T * D * 4 + (4 << 30))
    table = torch.randn(50, D, generator=gen(2), device=DEV)
    ids = torch.randint(0, 50, (T,), generator=gen(3), device=DEV, dtype=torch.int32)
    out = torch.empty(T, D, device=DEV)
    out[-1000:] = 77
    vocab.embed(ids, table, out=out)
    for rows in (slice(0, 1000), slice(2 ** 25 - 500, 2 ** 25 + 500), slice(T - 1000, T)):
        assert torch.equal(out[rows], table[ids[rows].long()])
    del out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T", [5, 600, 5000])
def test_zeros_of_more_rows_than_a_launch_has_threads_for(T):
    """2^22 and some rows of 8208 bytes, with others' bytes between them: a workgroup's share of zeros is one row."""
    from paper_2512_00719_amd import vocab
    V, D, stride = 2 ** 22 + 9, 2052, 2053
    _room(V * stride * 4 + (4 << 30))
    whole = torch.full((V, stride), 77.0, device=DEV)
    table = whole[:, :D]
    ids = torch.randint(0, V, (T,), generator=gen(4), device=DEV, dtype=torch.int32)
    ids[0] = V - 1
    dout = torch.ones(T, D, device=DEV)
    vocab.embed_grad(ids, dout, V, dtable=table)
    counts = torch.bincount(ids.long(), minlength=V).float()
    for v0 in range(0, V, 2 ** 19):
        rows = whole[v0:v0 + 2 ** 19]
        assert bool((rows[:, :D] == counts[v0:v0 + 2 ** 19, None]).all()) and bool((rows[:, D:] == 77).all())
    del whole, table, rows
    torch.cuda.empty_cache()


def test_cross_entropy_of_more_tiles_than_a_launch_has_workgroups_for():
    """2^20 tokens against 2^19 + 300 rows of 8 values: T V is a quarter of what the call takes.  Bounds as in the cross entropy's own tests."""
    from paper_2512_00719_amd import vocab
    T, V, D = 2 ** 20, 2 ** 19 + 300, 8
    _room(24 << 30)
    g = gen(5)
    h, w = torch.randn(T, D, generator=g, device=DEV).to(BF16), torch.randn(V, D, generator=g, device=DEV).to(BF16)
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    y[-1], y[5] = V - 1, -1
    loss, lse = vocab.linear_xent(h, w, y, loss=torch.full((T,), 77.0, device=DEV), lse=torch.full((T,), 77.0, device=DEV))
    for at in (slice(0, 64), slice(T // 2 - 32, T // 2 + 32), slice(T - 64, T)):
        hs, ws, ys = h[at].to(F64), w.to(F64), y[at]
        z = hs @ ws.t()
        dz = (D + 8) * 2.0 ** -24 * (hs.abs() @ ws.abs().t()) + z.abs() * 2.0 ** -24
        want = torch.logsumexp(z, 1)
        off = dz.amax(1) + 2.0 ** -17 + want.abs() * 2.0 ** -22
        within(lse[at], want, off, "lse")
        at_y = ys.clamp(min=0).long()[:, None]
        each = torch.where(ys >= 0, want - z.gather(1, at_y)[:, 0], 0.0)
        within(loss[at], each, off + dz.gather(1, at_y)[:, 0] + each.abs() * 2.0 ** -24, "loss")
    torch.cuda.empty_cache()
