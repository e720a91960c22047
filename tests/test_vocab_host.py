"""Checks of the operators at the vocabulary that need no GPU: exports, refusals at the C boundary and in the wrappers, workspace sizes."""
import os
import re

import pytest
import torch

from paper_2512_00719_amd import binding, vocab

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
lib, INVALID, CAPACITY, OK = vocab._lib, binding.SIMPLE_EINVAL, binding.SIMPLE_ECAPACITY, binding.SIMPLE_OK
F32, BF16 = binding.SIMPLE_F32, binding.SIMPLE_BF16
X = 4096  # an address that is not NULL: what is refused is refused before anything is enqueued


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "simple_vocab.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    assert set(re.findall(r"\b(simple_[a-z0-9_]+)\s*\(", header)) == set(vocab.EXPORTS)
    for name in vocab.EXPORTS:
        assert getattr(lib, name) is not None


def _norm(x=X, xs=8, r=0, rs=0, w=X, T=2, D=8, t=F32, eps=1e-6, h=0, hs=0, out=X, os_=8):
    return lib.simple_rms_norm(x, xs, r, rs, w, T, D, t, eps, h, hs, out, os_, 0, 0)


def test_norm_refusals():
    for bad in (dict(x=0), dict(w=0), dict(out=0), dict(xs=7), dict(os_=7), dict(T=-1), dict(D=0), dict(t=2), dict(eps=-1.0), dict(eps=float("nan")),
                dict(r=X, rs=8), dict(r=X, rs=7, h=X, hs=8), dict(h=X, hs=7)):
        assert _norm(**bad) == INVALID, bad
    assert _norm(D=32_769, xs=32_769, os_=32_769) == CAPACITY
    assert _norm(T=0, x=0, w=0, out=0) == OK
    assert lib.simple_rms_norm_int8(X, 8, 0, 0, X, 2, 8, F32, 1e-6, 0, 0, X, 8, 0, 0) == INVALID      # no scales
    assert lib.simple_rms_norm_int8(X, 8, 0, 0, X, 2, 8, F32, 1e-6, 0, 0, X, 7, X, 0) == INVALID      # code stride
    assert lib.simple_quantize_rows(0, 8, 2, 8, F32, X, 8, X, 0) == INVALID
    assert lib.simple_quantize_rows(X, 8, 0, 8, F32, 0, 8, 0, 0) == OK
    need = lib.simple_rms_norm_grad_workspace(2, 8)
    assert need >= 8 * 4 and lib.simple_rms_norm_grad_workspace(-1, 8) == INVALID and lib.simple_rms_norm_grad_workspace(2, 0) == INVALID
    grad = lambda ws=X, n=need, dw=X, dhs=8, dy=X: lib.simple_rms_norm_grad(dy, 8, X, 8, X, X, X, dhs, 2, 8, F32, X, 8, dw, ws, n, 0)  # noqa: E731
    assert grad(n=need - 1) == CAPACITY
    assert grad(ws=0) == grad(ws=X + 4) == grad(dw=0) == grad(dhs=7) == grad(dy=0) == INVALID


def test_embedding_refusals():
    embed = lambda ids=X, tab=X, ts=8, T=2, V=5, D=8, t=F32, out=X, os_=8: lib.simple_embed(ids, tab, ts, T, V, D, t, 1.0, out, os_, 0)  # noqa: E731
    assert embed(ids=0) == embed(tab=0) == embed(out=0) == embed(ts=7) == embed(os_=7) == embed(T=-1) == embed(V=0) == embed(D=0) == embed(t=5) == INVALID
    assert embed(V=2 ** 31 - 1) == embed(T=2 ** 31) == CAPACITY
    assert embed(T=0, ids=0, tab=0, out=0) == OK
    need = lib.simple_embed_grad_workspace(2, 5, 8)
    assert need > 0 and lib.simple_embed_grad_workspace(2, 0, 8) == INVALID
    grad = lambda ids=X, d=X, ds=8, T=2, V=5, D=8, t=F32, o=X, os_=8, ot=F32, acc=0, ws=X, n=need: lib.simple_embed_grad(  # noqa: E731
        ids, d, ds, T, V, D, t, 1.0, o, os_, ot, acc, ws, n, 0)
    assert grad(ids=0) == grad(d=0) == grad(ds=7) == grad(t=2) == grad(o=0) == grad(os_=7) == grad(ot=2) == grad(ws=0) == grad(ws=X + 2) == INVALID
    assert grad(n=need - 1) == CAPACITY
    assert grad(T=0, acc=1, ids=0, d=0, ws=0) == OK


def test_head_refusals():
    head = lambda a=X, as_=8, sa=X, b=X, bs=8, sb=X, T=2, V=5, K=8, o=X, os_=5, t=F32, ws=0, n=0: lib.simple_linear_int8(  # noqa: E731
        a, as_, sa, b, bs, sb, T, V, K, o, os_, t, ws, n, 0)
    assert (head(a=0) == head(sa=0) == head(b=0) == head(sb=0) == head(o=0) == head(as_=7) == head(bs=7) == head(os_=4) == head(T=-1) == head(V=0) ==
            head(K=0) == head(t=2) == head(ws=X + 8) == INVALID)
    need = lib.simple_linear_int8_workspace(600, 5, 8)
    assert need > 0 and head(T=600, ws=X, n=need - 1) == CAPACITY and lib.simple_linear_int8_workspace(200, 0, 8) == INVALID
    assert head(K=131_072, as_=131_072, bs=131_072) == CAPACITY
    assert head(T=0, a=0, o=0) == OK


def test_cross_entropy_refusals():
    need = lib.simple_xent_workspace(2, 5, 8)
    xent = lambda h=X, hs=8, w=X, wst=8, y=X, T=2, V=5, D=8, c=1.0, l=X, e=X, ws=X, n=need: lib.simple_xent(h, hs, w, wst, y, T, V, D, c, l, e, ws, n, 0)  # noqa: E731,E741
    assert (xent(h=0) == xent(hs=7) == xent(w=0) == xent(wst=7) == xent(y=0) == xent(T=-1) == xent(V=0) == xent(D=0) == xent(l=0) == xent(e=0) ==
            xent(ws=0) == xent(ws=X + 8) == xent(c=0.0) == xent(c=-1.0) == xent(c=float("nan")) == xent(c=float("inf")) == INVALID)
    assert xent(n=need - 1) == xent(T=2 ** 20 + 1) == xent(D=65_537, hs=65_537, wst=65_537) == CAPACITY
    assert xent(T=0, h=0, w=0, ws=0) == OK
    need = lib.simple_xent_grad_workspace(2, 5, 8, 1, 1)
    grad = lambda dl=X, h=X, hs=8, w=X, wst=8, y=X, e=X, T=2, V=5, D=8, c=1.0, dh=X, dhs=8, dw=X, dws=8, t=BF16, acc=0, ws=X, n=need: lib.simple_xent_grad(  # noqa: E731
        dl, h, hs, w, wst, y, e, T, V, D, c, dh, dhs, dw, dws, t, acc, ws, n, 0)
    assert (grad(dl=0) == grad(h=0) == grad(hs=7) == grad(w=0) == grad(wst=7) == grad(y=0) == grad(e=0) == grad(dhs=7) == grad(dws=7) == grad(t=2) ==
            grad(c=0.0) == grad(ws=0) == grad(ws=X + 8) == INVALID)
    assert grad(n=need - 1) == CAPACITY
    assert grad(dh=0, dw=0) == OK and grad(T=0, acc=1, ws=0) == OK and grad(T=0, dw=0, ws=0) == OK


def test_workspaces_over_the_whole_range():
    for T in (0, 1, 16, 17, 64, 65, 128, 129, 5000, 2 ** 20):
        for V in (1, 300, 128_256, 2 ** 28):
            for D in (1, 64, 4096, 65_536):
                both = lib.simple_xent_grad_workspace(T, V, D, 1, 1)
                assert both >= max(lib.simple_xent_grad_workspace(T, V, D, 1, 0), lib.simple_xent_grad_workspace(T, V, D, 0, 1)) >= 0
                assert lib.simple_xent_workspace(T, V, D) >= 0 and lib.simple_embed_grad_workspace(T, V, D) >= 0
                assert lib.simple_rms_norm_grad_workspace(T, D) >= 0


def test_the_wrappers_take_tensors_of_the_current_gpu_alone():
    x, w = torch.ones(3, 8), torch.ones(8)
    ids = torch.zeros(3, dtype=torch.int32)
    for call in (lambda: vocab.rms_norm(x, w), lambda: vocab.rms_norm_int8(x, w), lambda: vocab.quantize_rows(x),
                 lambda: vocab.rms_norm_grad(x, x, w, torch.ones(3)), lambda: vocab.embed(ids, x), lambda: vocab.embed_grad(ids, x, 5),
                 lambda: vocab.linear_int8(x.to(torch.int8), torch.ones(3), x.to(torch.int8), torch.ones(3)),
                 lambda: vocab.linear_xent(x.bfloat16(), x.bfloat16(), ids)):
        with pytest.raises(ValueError, match="current GPU"):
            call()
    with pytest.raises(TypeError):
        vocab.rms_norm(x.to(torch.float16), w)
    with pytest.raises(TypeError):
        vocab.linear_xent(x, x, ids)
    with pytest.raises(ValueError):
        vocab.rms_norm(torch.ones(8), w)
