"""The cross entropy's calls write nothing beside the workspace that they ask for, and a call on aligned operands allocates no room for copies."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, gen, laid, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("T,V,D", [(1, 70_000, 24), (40, 1000, 64), (64, 66_000, 104), (65, 3000, 136), (600, 5000, 72), (700, 66_000, 40)])
def test_nothing_is_written_beside_the_workspace(T, V, D, pad):
    from paper_2512_00719_amd import binding, vocab
    lib, g = vocab._lib, gen(T)
    h, w = laid(normal((T, D), BF16, g), pad, pad), laid(normal((V, D), BF16, g, D ** -0.5), pad, pad)
    y, dl = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32), torch.rand(T, generator=g, device=DEV)
    f = "_aligned" if pad == 0 else ""
    want = vocab.linear_xent(h, w, y)
    grads = vocab.linear_xent_grad(dl, h, w, y, want[1])
    stream = binding._current_stream()

    def with_workspace(n, call):
        room = torch.full((n + 8192,), 77, dtype=torch.uint8, device=DEV)
        assert room.data_ptr() % 16 == 0
        assert call(room.data_ptr() + 4096, n) == binding.SIMPLE_OK
        assert bool((room[:4096] == 77).all()) and bool((room[4096 + n:] == 77).all())

    loss, lse = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    with_workspace(getattr(lib, "simple_xent_workspace" + f)(T, V, D), lambda ws, n: lib.simple_xent(
        h.data_ptr(), h.stride(0) if T > 1 else D + pad, w.data_ptr(), w.stride(0), y.data_ptr(), T, V, D, 1.0, loss.data_ptr(), lse.data_ptr(), ws, n, stream))
    assert torch.equal(loss, want[0]) and torch.equal(lse, want[1])
    for need_h, need_w in ((1, 1), (1, 0), (0, 1)):
        dh, dw = torch.empty(T, D, dtype=BF16, device=DEV), torch.empty(V, D, dtype=BF16, device=DEV)
        with_workspace(getattr(lib, "simple_xent_grad_workspace" + f)(T, V, D, need_h, need_w), lambda ws, n: lib.simple_xent_grad(
            dl.data_ptr(), h.data_ptr(), h.stride(0) if T > 1 else D + pad, w.data_ptr(), w.stride(0), y.data_ptr(), lse.data_ptr(), T, V, D, 1.0,
            dh.data_ptr() if need_h else 0, D, dw.data_ptr() if need_w else 0, D, binding.SIMPLE_BF16, 0, ws, n, stream))
        assert not need_h or torch.equal(dh, grads[0])
        assert not need_w or torch.equal(dw, grads[1])


@pytest.mark.parametrize("T", [1, 600])
def test_aligned_operands_have_no_room_for_copies(T):
    from paper_2512_00719_amd import vocab
    V, D, g = 66_000, 2048, gen(1)
    h, w = normal((T, D), BF16, g), normal((V, D), BF16, g, D ** -0.5)
    y = torch.zeros(T, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()

    def peak(call):
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        out = call()
        return out, torch.cuda.max_memory_allocated() - before

    (_, lse), n = peak(lambda: vocab.linear_xent(h, w, y))
    assert n < 32 << 20
    out, n = peak(lambda: vocab.linear_xent_grad(torch.ones(T, device=DEV), h, w, y, lse))
    pieces = 2 * T * 66_048 * 2 + D * 66_048 * 2 if T > 64 else 0      # G in both orders and the turned weights, which the large path works on
    sums = 64 << 20
    assert n < w.numel() * 2 + pieces + sums
