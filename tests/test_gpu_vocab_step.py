"""The operators at the vocabulary together: the example's training and decoding steps, refusals of operands that do not fit, other
streams, and a graph that is replayed."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, F64, gen, normal

pytestmark = pytest.mark.gpu


def test_the_example_learns_and_decodes():
    from paper_2512_00719_amd import vocab_step
    model = vocab_step.TiedModel(1000, 128, seed=1)
    ids = torch.arange(0, 300, device=DEV, dtype=torch.int32)
    targets = ids + 1
    targets[::10] = -1
    first = float(model.train_step(ids, targets, rate=1.0))
    for _ in range(15):
        last = float(model.train_step(ids, targets, rate=1.0))
    assert 6.0 < first < 9.0 and last < 0.5 * first, (first, last)
    drawn = vocab_step.decode(model, ids[:5], 3)
    assert drawn.shape == (5, 3) and bool(((drawn >= 0) & (drawn < 1000)).all())


def test_the_whole_step_against_automatic_differentiation():
    """Loss and gradients of embed -> norm -> cross entropy with one tied table against torch's own, in 64 bits from the same bfloat16 values.
    Rounded to bfloat16 on the way are the embedding's rows, the norm's output and dy, dx: each rounding is 2^-8 of its size, a gradient's elements are
    sums over them, and their norms agree to 2^-8 times a small number of roundings, 2^-5 with room."""
    from paper_2512_00719_amd import vocab
    g = gen(2)
    V, D, T = 700, 96, 130
    table, w = normal((V, D), BF16, g, 0.3), (1 + 0.1 * torch.randn(D, generator=g, device=DEV)).to(BF16)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    y[::7] = -1
    live = (y >= 0).float()
    x = vocab.embed(ids, table, scale=2.0)
    n, h, rstd = vocab.rms_norm(x, w, need_rstd=True)
    loss, lse = vocab.linear_xent(n, table, y)
    dtable = torch.zeros(V, D, device=DEV)
    dn, _ = vocab.linear_xent_grad(live, n, table, y, lse, dweight=dtable)
    dx, dw = vocab.rms_norm_grad(dn, h, w, rstd)
    vocab.embed_grad(ids, dx, V, scale=2.0, dtable=dtable, accumulate=True)
    t64, w64 = table.to(F64).requires_grad_(), w.to(F64).requires_grad_()
    e = 2.0 * t64[ids.long()]
    m = e / torch.sqrt(e.square().mean(1, keepdim=True) + 1e-6) * w64
    z = m @ t64.t().contiguous()
    each = torch.logsumexp(z, 1) - z.gather(1, y.clamp(min=0).long()[:, None])[:, 0]
    (each * live).sum().backward()
    off = lambda a, b: float((a.to(F64) - b).norm() / b.norm())  # noqa: E731
    assert off(loss, (each * live).detach()) < 2.0 ** -5
    assert off(dtable, t64.grad) < 2.0 ** -5 and off(dw, w64.grad) < 2.0 ** -5


def test_refusals_of_operands_that_do_not_fit():
    from paper_2512_00719_amd import vocab
    x, w = torch.ones(4, 64, device=DEV), torch.ones(64, device=DEV)
    ids = torch.zeros(4, dtype=torch.int32, device=DEV)
    cases = [
        (TypeError, lambda: vocab.rms_norm(x, w.to(BF16))),
        (TypeError, lambda: vocab.rms_norm(x.half(), w.half())),
        (ValueError, lambda: vocab.rms_norm(x, w[:32])),
        (ValueError, lambda: vocab.rms_norm(x, w, residual=x[:2])),
        (ValueError, lambda: vocab.rms_norm(x.t(), torch.ones(4, device=DEV))),
        (ValueError, lambda: vocab.rms_norm(x, w, h=x)),
        (ValueError, lambda: vocab.rms_norm(x, w, out=x.cpu())),
        (TypeError, lambda: vocab.embed(ids.long(), x)),
        (ValueError, lambda: vocab.embed_grad(ids, x, 9, accumulate=True)),
        (TypeError, lambda: vocab.embed_grad(ids, x, 9, dtable=torch.ones(9, 64, device=DEV, dtype=torch.float16))),
        (ValueError, lambda: vocab.embed_grad(ids, x, 9, dtable=torch.ones(8, 64, device=DEV))),
        (TypeError, lambda: vocab.linear_int8(x.to(torch.int8), w[:4], x, w[:4])),
        (ValueError, lambda: vocab.linear_int8(x.to(torch.int8), w[:4], x[:, :32].to(torch.int8), w[:4])),
        (TypeError, lambda: vocab.linear_int8(x.to(torch.int8), w[:4], x.to(torch.int8), w[:4], out_dtype=torch.float16)),
        (TypeError, lambda: vocab.linear_xent(x, x, ids)),
        (TypeError, lambda: vocab.linear_xent(x.to(BF16), x.to(BF16), ids.long())),
        (ValueError, lambda: vocab.linear_xent(x.to(BF16), x[:, :32].to(BF16), ids)),
        (ValueError, lambda: vocab.linear_xent_grad(w[:4], x.to(BF16), x.to(BF16), ids, w[:4], accumulate=True)),
    ]
    for error, call in cases:
        with pytest.raises(error):
            call()
    from paper_2512_00719_amd import binding
    with pytest.raises(binding.SimpleError) as e:
        vocab.linear_xent(x.to(BF16), x.to(BF16), ids, logit_scale=0.0)
    assert e.value.code == binding.SIMPLE_EINVAL


def _chain(table, codes, scales, w, ids, y, dl):
    from paper_2512_00719_amd import vocab
    x = vocab.embed(ids, table, scale=3.0)
    c, s, h = vocab.rms_norm_int8(x, w, residual=x)
    logits = vocab.linear_int8(c, s, codes, scales, out_dtype=BF16)
    n, _, rstd = vocab.rms_norm(h, w, need_rstd=True)
    loss, lse = vocab.linear_xent(n, table, y)
    dn, dtable = vocab.linear_xent_grad(dl, n, table, y, lse)
    dx, dw = vocab.rms_norm_grad(dn, h, w, rstd)
    vocab.embed_grad(ids, dx, table.shape[0], scale=3.0, dtable=dtable, accumulate=True)
    return logits, loss, lse, dtable, dw


def _chain_inputs(T, V, D, seed):
    from paper_2512_00719_amd import vocab
    g = gen(seed)
    table, w = normal((V, D), BF16, g, 0.2), torch.ones(D, device=DEV, dtype=BF16)
    ids = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    y = torch.randint(-1, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    return [table, *vocab.quantize_rows(table), w, ids, y, torch.rand(T, generator=g, device=DEV)]


@pytest.mark.parametrize("T", [3, 200])
def test_on_a_stream_of_their_own(T):
    inputs = _chain_inputs(T, 900, 136, T)
    want = _chain(*inputs)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    fresh = [t.clone() for t in inputs]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _chain(*fresh)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [3, 200, 5000])
def test_graph_replays(T):
    """The chain in a graph, replayed on new values in the same buffers with eager work between: each replay is what the eager calls give."""
    inputs = _chain_inputs(T, 900, 72, 1)
    _chain(*inputs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _chain(*inputs)
    for seed in range(2, 6):
        for held, new in zip(inputs, _chain_inputs(T, 900, 72, seed)):
            held.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, _chain(*inputs)):
            assert torch.equal(a, b)
