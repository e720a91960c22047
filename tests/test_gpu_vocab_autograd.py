"""What the operators at the vocabulary do beside automatic differentiation: they record nothing, and say so rather than lose a gradient silently."""
import pytest
import torch

from vocab_util import BF16, DEV, F32, gen, normal

pytestmark = pytest.mark.gpu


def _calls():
    from paper_2512_00719_amd import vocab
    g = gen(1)
    x, w, table = normal((6, 64), BF16, g), normal((64,), BF16, g), normal((90, 64), BF16, g)
    ids = torch.arange(6, device=DEV, dtype=torch.int32)
    f = torch.ones(6, device=DEV)
    codes, scales = vocab.quantize_rows(x)
    return [(vocab.rms_norm, [x, w], {"residual": x.clone()}), (vocab.rms_norm_int8, [x, w], {"residual": x.clone()}), (vocab.quantize_rows, [x], {}),
            (vocab.rms_norm_grad, [x, x.clone(), w, f], {"dh": x.clone()}), (vocab.embed, [ids, table], {}), (vocab.embed_grad, [ids, x, 90], {}),
            (vocab.linear_int8, [codes, scales, codes, scales], {}), (vocab.linear_xent, [x, table, ids], {}),
            (vocab.linear_xent_grad, [f, x, table, ids, f], {})]


def test_operands_that_want_a_gradient_are_refused():
    for call, args, named in _calls():
        places = [(args, i) for i in range(len(args))] + [(named, k) for k in named]
        for holder, at in places:
            t = holder[at]
            if not (isinstance(t, torch.Tensor) and t.is_floating_point()):
                continue
            holder[at] = t.clone().requires_grad_()
            with pytest.raises(ValueError, match="gradient"):
                call(*args, **named)
            with torch.no_grad():
                call(*args, **named)
            with torch.inference_mode():
                call(*args, **named)
            holder[at] = holder[at].detach()
            call(*args, **named)
            holder[at] = t
        call(*args, **named)


def test_tensors_that_are_written_have_another_version():
    """A tensor that torch has saved for a backward pass, and that a call then writes in place, is found to have changed."""
    from paper_2512_00719_amd import vocab
    g = gen(2)
    x, r, w = normal((6, 64), F32, g), normal((6, 64), F32, g), normal((64,), F32, g)
    factor = torch.ones(6, 64, device=DEV, requires_grad=True)
    product = (factor * x).sum()      # x is saved
    vocab.rms_norm(x, w, residual=r, h=r, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()
    ids, y = torch.arange(6, device=DEV, dtype=torch.int32), torch.zeros(90, 64, dtype=BF16, device=DEV)
    f, b = torch.ones(6, device=DEV), x.to(BF16)
    e = lambda *shape, dtype=F32: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    q, s = vocab.quantize_rows(x)
    for call, args, outs in [
            (vocab.rms_norm, (x, w), {"residual": r, "h": e(6, 64), "out": e(6, 64), "rstd": e(6)}),
            (vocab.rms_norm_int8, (x, w), {"codes": e(6, 64, dtype=torch.int8), "scales": e(6)}),
            (vocab.quantize_rows, (x,), {"codes": e(6, 64, dtype=torch.int8), "scales": e(6)}),
            (vocab.rms_norm_grad, (x, r, w, f), {"dx": e(6, 64), "dweight": e(64)}), (vocab.embed, (ids, x), {"out": e(6, 64)}),
            (vocab.embed_grad, (ids, x, 6), {"dtable": e(6, 64)}), (vocab.linear_int8, (q, s, q, s), {"out": e(6, 6)}),
            (vocab.linear_xent, (b, y, ids), {"loss": e(6), "lse": e(6)}),
            (vocab.linear_xent_grad, (f, b, y, ids, f), {"dhidden": e(6, 64, dtype=BF16), "dweight": e(90, 64)})]:
        written = {k: v for k, v in outs.items() if k != "residual"}
        before = {k: v._version for k, v in written.items()}
        call(*args, **outs)
        for k, v in written.items():
            assert v._version > before[k], (call.__name__, k)
    with torch.inference_mode():      # tensors without a version
        z = torch.empty(6, 64, device=DEV)
        vocab.rms_norm(x, w, out=z)
