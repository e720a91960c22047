"""Operands and outputs of more than 2^31 elements: rows behind that place, and at the start, against the formulas in 64 bits (bounds as in each operator's own tests)."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, F64, HALF, gen, within
from xent_bounds import formula

pytestmark = pytest.mark.gpu
N, D = 530_000, 4104      # 2.18e9 elements
ROWS = [0, 1, N // 2, 523_263, 523_264, 523_265, N - 2, N - 1]   # 2^31 elements end in row 523,266


@pytest.fixture(autouse=True)
def _room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("wants 40 GiB of device memory")
    yield
    torch.cuda.empty_cache()


def _big(g, rows=N, width=D):
    t = torch.empty(rows, width, dtype=BF16, device=DEV)
    for part in t.split(50_000):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV))
    return t


def test_norm_and_its_gradient():
    from paper_2512_00719_amd import vocab
    g = gen(1)
    x, w = _big(g), (1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(BF16)
    y, _, rstd = vocab.rms_norm(x, w, eps=1e-5, need_rstd=True)
    h = x[ROWS].to(F64)
    s = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-5)
    want = h * s * w.to(F64)
    within(y[ROWS], want, want.abs() * (2.0 ** -17 + HALF[BF16]), "y")
    codes, scales, _ = vocab.rms_norm_int8(x, w, eps=1e-5)
    step = want.abs().amax(1, keepdim=True) / 127
    within(codes[ROWS].to(F64) * scales[ROWS].to(F64)[:, None], want, step * (0.5 + 2.0 ** -8), "codes times scales")
    del codes
    dx, dw = vocab.rms_norm_grad(y, x, w, rstd)
    dy = y[ROWS].to(F64)
    n, gg = h * s, dy * w.to(F64)
    m = (gg * n).mean(1, keepdim=True)
    want = s * (gg - n * m)
    size = s * (gg.abs() + n.abs() * (gg * n).abs().mean(1, keepdim=True))
    within(dx[ROWS], want, size * 2.0 ** -16 + want.abs() * HALF[BF16], "dx")
    terms, sizes = torch.zeros(D, dtype=F64, device=DEV), torch.zeros(D, dtype=F64, device=DEV)
    for a, b, r in zip(x.split(50_000), y.split(50_000), rstd.split(50_000)):
        t = a.to(F64) * b.to(F64) * r.to(F64)[:, None]
        terms += t.sum(0)
        sizes += t.abs().sum(0)
    # a term passes through ceil(530,000 / 1024) additions of its workgroup's rows and 64 of the workgroups
    within(dw, terms, sizes * (518 + 64 + 4) * 2.0 ** -24, "dweight")


def test_embedding_and_its_gradient():
    from paper_2512_00719_amd import vocab
    g = gen(2)
    table = _big(g)
    ids = torch.tensor(ROWS + [-1, N], dtype=torch.int32, device=DEV).repeat(70)
    out = vocab.embed(ids, table, scale=2.0)
    live = (ids >= 0) & (ids < N)
    assert torch.equal(out[live], table[ids[live].long()] * 2) and not out[~live].any()
    for n in (len(ROWS) + 2, 700):
        dtable = vocab.embed_grad(ids[:n], torch.ones(n, D, dtype=BF16, device=DEV), N, dtable=table)
        assert bool((dtable[ROWS] == n // (len(ROWS) + 2)).all())
        assert sum(int(part.any(1).sum()) for part in dtable.split(50_000)) == len(ROWS)
    rows = torch.randint(0, N, (N,), generator=g, device=DEV, dtype=torch.int32)
    dout = vocab.embed(rows, table, out=torch.empty_like(table))     # more than 2^31 elements of output, and then of what is summed
    assert torch.equal(dout[ROWS], table[rows[ROWS].long()])
    back = vocab.embed_grad(torch.arange(N, device=DEV, dtype=torch.int32).flip(0), dout.fill_(1.0), N, dtable=table)
    assert all(bool((part == 1).all()) for part in back.split(50_000))


def test_head():
    from paper_2512_00719_amd import vocab
    g = gen(3)
    T, V, K = 16_500, 131_072, 64      # 2.16e9 logits
    a, b = (torch.randint(-127, 128, (n, K), generator=g, device=DEV).to(torch.int8) for n in (T, V))
    sa, sb = torch.rand(T, generator=g, device=DEV) + 0.01, torch.rand(V, generator=g, device=DEV) + 0.01
    out = vocab.linear_int8(a, sa, b, sb, out_dtype=BF16)
    at = [0, 16_383, 16_384, T - 1]
    want = (a[at].to(F64) @ b.to(F64).t()) * sa[at].to(F64)[:, None] * sb.to(F64)
    within(out[at], want, want.abs() * (3 * 2.0 ** -24 + HALF[BF16]), "logits")
    del out
    b = torch.randint(-127, 128, (V, 16_400), generator=g, device=DEV, dtype=torch.int8)      # 2.15e9 codes
    a = torch.randint(-127, 128, (3, 16_400), generator=g, device=DEV, dtype=torch.int8)
    out = vocab.linear_int8(a, sa[:3], b, sb)
    want = torch.cat([a.to(F64) @ part.to(F64).t() for part in b.split(16_384)], 1) * sa[:3].to(F64)[:, None] * sb.to(F64)
    within(out, want, want.abs() * 3 * 2.0 ** -24, "logits")


@pytest.mark.parametrize("T", [2, 80])
def test_cross_entropy(T):
    """A vocabulary whose weights, and their gradient, are more than 2^31 elements: loss, dH and the rows of dW at its start and its end."""
    from paper_2512_00719_amd import vocab
    g = gen(T)
    w = _big(g)
    for part in w.split(50_000):
        part.mul_(2.0 * D ** -0.5)
    y = torch.tensor(ROWS, dtype=torch.int32, device=DEV).repeat(10)[:T] if T > 2 else torch.tensor([N - 1, 523_265], dtype=torch.int32, device=DEV)
    h = (torch.randn(T, D, generator=g, device=DEV) + 2.0 * w[y.long()].float()).to(BF16)
    loss, lse = vocab.linear_xent(h, w, y)
    z = torch.cat([h.to(F64) @ part.to(F64).t() for part in w.split(50_000)], 1)
    want = torch.logsumexp(z, 1)
    dz = max(float((h.to(F64).abs() @ w[v:v + 20_000].to(F64).abs().t()).max()) for v in range(0, N, 20_000)) * (D + 8) * 2.0 ** -24
    within(lse, want, dz + 2.0 ** -17, "lse")
    each = want - z.gather(1, y.long()[:, None])[:, 0]
    within(loss, each, 2 * dz + 2.0 ** -17, "loss")
    dl = torch.rand(T, generator=g, device=DEV) + 0.5
    dh, dw = vocab.linear_xent_grad(dl, h, w, y, lse)
    G = (z - want[:, None]).exp()
    G.scatter_add_(1, y.long()[:, None], torch.full((T, 1), -1.0, dtype=F64, device=DEV))
    G *= dl.to(F64)[:, None]
    rows = sorted(set(ROWS + list(range(523_200, 523_330)) + list(range(N - 300, N))))
    bits = 2.0 ** -10 if T > 64 else 2.0 ** -14
    size = G[:, rows].abs().t() @ h.to(F64).abs()
    exact = G[:, rows].t() @ h.to(F64)
    within(dw[rows], exact, size * (bits + 2 * dz + 2.0 ** -17) + exact.abs() * HALF[BF16] + 2.0 ** -34 * float(h.abs().max()), "dw")
    exact, size = torch.zeros(T, D, dtype=F64, device=DEV), torch.zeros(T, D, dtype=F64, device=DEV)
    for v in range(0, N, 50_000):
        part = w[v:v + 50_000].to(F64)
        exact += G[:, v:v + 50_000] @ part
        size += G[:, v:v + 50_000].abs() @ part.abs()
    within(dh, exact, size * (bits + 2 * dz + 2.0 ** -17 + 2.0 ** -24 * (N / 32 + 64)) + exact.abs() * HALF[BF16], "dh")
