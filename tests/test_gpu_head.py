"""The 8-bit head against whole-number sums: the sum is exact, so an output is off by three float32 roundings (the sum's
conversion, two scales) and that of its type."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, F64, HALF, gen, laid, padding_untouched, within

pytestmark = pytest.mark.gpu


def _inputs(T, V, K, seed, lowest=-127):
    g = gen(seed)
    a = torch.randint(lowest, 128, (T, K), generator=g, device=DEV).to(torch.int8)
    b = torch.randint(lowest, 128, (V, K), generator=g, device=DEV).to(torch.int8)
    return a, torch.rand(T, generator=g, device=DEV) + 0.01, b, torch.rand(V, generator=g, device=DEV) + 0.01


def _want(a, sa, b, sb):
    return (a.to(F64) @ b.to(F64).t()) * sa.to(F64)[:, None] * sb.to(F64)


def _check(out, want, dtype):
    within(out, want, want.abs() * (3 * 2.0 ** -24 + (HALF[BF16] if dtype == BF16 else 0) + 2.0 ** -45), "logits")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,K", [(1, 1), (5, 16), (63, 15), (64, 64), (65, 100), (260, 128), (130, 130), (1000, 1000), (300, 4112), (2052, 257)])
@pytest.mark.parametrize("T", [1, 2, 16, 17, 33, 64, 65, 128, 129, 257, 600])
def test_sizes(T, V, K, dtype):
    from paper_2512_00719_amd import vocab
    a, sa, b, sb = _inputs(T, V, K, T + V * 7 + K, -128)
    _check(vocab.linear_int8(a, sa, b, sb, out_dtype=dtype), _want(a, sa, b, sb), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pads", [(16, 0, 16, 32), (1, 0, 0, 0), (0, 0, 3, 1), (16, 8, 16, 16), (0, 0, 0, 0)])
@pytest.mark.parametrize("T,V,K", [(3, 70, 144), (40, 130, 272), (300, 514, 160), (129, 257, 1008)])
def test_strides_and_alignments(T, V, K, pads, dtype):
    from paper_2512_00719_amd import vocab
    a, sa, b, sb = _inputs(T, V, K, 5)
    pa, sha, pb, shb = pads
    for pad, shift in ((0, 0), (1, 0), (4, 4), (7, 3)):
        out = laid(torch.zeros(T, V, dtype=dtype, device=DEV), pad, shift)
        vocab.linear_int8(laid(a, pa, sha), sa, laid(b, pb, shb), sb, out=out)
        _check(out, _want(a, sa, b, sb), dtype)
        assert padding_untouched(out, pad, shift) if pad or shift else True


def test_what_lies_beside_the_operands_is_not_read_into_the_sums():
    """Rows of every length modulo 16 inside a larger allocation of other codes: chunks at a row's end, and rows behind the last."""
    from paper_2512_00719_amd import vocab
    for K in list(range(113, 130)) + [250, 255, 256, 257]:
        a, sa, b, sb = _inputs(20, 70, K, K)
        va, vb = laid(a, 16 - K % 16, 16), laid(b, 16 - K % 16, 16)
        _check(vocab.linear_int8(va, sa, vb, sb), _want(a, sa, b, sb), F32)


def test_largest_sums_and_scales_of_bad_rows():
    from paper_2512_00719_amd import vocab
    K = 131_071
    a, b = torch.full((2, K), -128, dtype=torch.int8, device=DEV), torch.full((5, K), -128, dtype=torch.int8, device=DEV)
    one = torch.ones(5, device=DEV)
    _check(vocab.linear_int8(a, one[:2], b, one), _want(a, one[:2], b, one), F32)
    scales = torch.tensor([float("nan"), 1.0], device=DEV)
    out = vocab.linear_int8(a * 0, scales, b, one)
    assert bool(out[0].isnan().all()) and not out[1].any()
    assert vocab.linear_int8(a[:0], one[:0], b, one).shape == (0, 5)


def test_norm_head_and_sampling_call_together():
    """Codes of the norm through the head give the logits of the norm's output and the quantised weights, and the sampling call reads them."""
    from paper_2512_00719_amd import binding, synth, vocab
    g = gen(11)
    T, V, D = 12, 4104, 512
    x, r = torch.randn(T, D, generator=g, device=DEV).to(BF16), torch.randn(T, D, generator=g, device=DEV).to(BF16)
    w = torch.ones(D, device=DEV).to(BF16)
    head = (torch.randn(V, D, generator=g, device=DEV) * D ** -0.5).to(BF16)
    w_codes, w_scales = vocab.quantize_rows(head)
    codes, scales, h = vocab.rms_norm_int8(x, w, residual=r)
    logits = vocab.linear_int8(codes, scales, w_codes, w_scales)
    _check(logits, _want(codes, scales, w_codes, w_scales), F32)
    params = torch.from_numpy(synth.make_params(T, temperature=0.0).view("u1").reshape(T, 32)).to(DEV)
    s = binding.Sampler(V, 0)
    ids = s.sample(logits, params, seed=1, step=0)
    assert torch.equal(ids.long(), logits.argmax(1))
    s.close()


def test_copies_with_aligned_rows_in_more_than_one_piece():
    """More than 512 tokens and 65,536 channels, rows of 33 codes: the weights are copied a piece at a time."""
    from paper_2512_00719_amd import vocab
    a, sa, b, sb = _inputs(520, 66_000, 33, 3)
    _check(vocab.linear_int8(a, sa, b, sb), _want(a, sa, b, sb), F32)
