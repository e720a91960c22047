"""Sizes of the cross entropy's workspaces: what a call needs follows the operands' alignment, and too little is refused before anything is enqueued."""
import pytest

from paper_2512_00719_amd import binding, vocab

lib, CAPACITY, INVALID = vocab._lib, binding.SIMPLE_ECAPACITY, binding.SIMPLE_EINVAL
X = 4096


def _sizes(T, V, D):
    return [(lib.simple_xent_workspace_aligned(T, V, D), lib.simple_xent_workspace(T, V, D))] + [
        (lib.simple_xent_grad_workspace_aligned(T, V, D, h, w), lib.simple_xent_grad_workspace(T, V, D, h, w)) for h, w in ((1, 1), (1, 0), (0, 1))]


def test_sizes_of_aligned_operands():
    """Copies of operands are no part of them: the largest loss's pairs, and a token's G in a few forms."""
    assert lib.simple_xent_workspace_aligned(8192, 128_256, 4096) <= 501 * 8192 * 8 + 8192 * 4 + (1 << 16)
    assert lib.simple_xent_grad_workspace_aligned(1, 128_256, 4096, 1, 1) < 16 << 20
    for T in (0, 1, 64, 65, 512, 513, 5000, 2 ** 20):
        for V in (1, 300, 128_256, 2 ** 28):
            for D in (8, 64, 4096, 65_536):
                for least, most in _sizes(T, V, D):
                    assert 0 <= least <= most and least % 65_536 == most % 65_536 == 0
    for bad in ((-1, 5, 8), (2, 0, 8), (2, 5, 0)):
        assert lib.simple_xent_workspace_aligned(*bad) == lib.simple_xent_grad_workspace_aligned(*bad, 1, 1) == INVALID
    assert lib.simple_xent_workspace_aligned(2, 5, 65_537) == lib.simple_xent_grad_workspace_aligned(2, 5, 65_537, 1, 1) == CAPACITY


@pytest.mark.parametrize("T", [2, 64, 65, 600])
def test_too_little_is_refused(T):
    V, D = 100_000, 512
    xent = lambda n, h=X, s=D, ws=D: lib.simple_xent(h, s, X, ws, X, T, V, D, 1.0, X, X, X, n, 0)  # noqa: E731
    grad = lambda n, h=X, s=D, ws=D, dh=X, dw=X: lib.simple_xent_grad(X, h, s, X, ws, X, X, T, V, D, 1.0, dh, D, dw, D, binding.SIMPLE_BF16, 0, X, n, 0)  # noqa: E731
    (least, most), (both, both_most), (dh, dh_most), (dw, dw_most) = _sizes(T, V, D)
    assert xent(least - 1) == CAPACITY and grad(both - 1) == grad(dh - 1, dw=0) == grad(dw - 1, dh=0) == CAPACITY
    # an address, a stride of either operand that is not a multiple of 16 bytes, a stride beyond what is addressed directly: copies are wanted
    for other in (dict(h=X + 2), dict(s=D + 4), dict(ws=D + 1), dict(ws=(1 << 21) + 8)):
        assert xent(most - 1, **other) == CAPACITY and grad(both_most - 1, **other) == CAPACITY
        assert grad(dh_most - 1, dw=0, **other) == grad(dw_most - 1, dh=0, **other) == CAPACITY
