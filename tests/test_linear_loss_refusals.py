"""Host-side refusals of the output layer's losses and of the top logits, and the plain 64-bit gradient against differences
(no GPU needed: a call that fails validation launches nothing)."""
import ctypes

import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64_loss as pl
from test_operator_refusals import ALIAS, ALIGN, DTYPE, MB, NULL, SHAPE, VALUE, WORKSPACE, arr

R = ctypes.byref
B, H16, F, Q, Q2 = sc.BF16, sc.F16, sc.F32, sc.E4M3, sc.E5M2
NAN, INF = float("nan"), float("inf")
p = lambda a: None if a is None else R(a)  # noqa: E731
h, w, t, g = arr(1, B, (4, 64)), arr(2, B, (100, 64)), arr(3, F, (4, 8)), arr(13, F, (4,))
dh, dw = arr(14, B, (4, 64)), arr(15, B, (100, 64))
IDS, LOSS, LSE, MEAN, WS, NB = 8 * MB, 9 * MB, 10 * MB, 11 * MB, 64 * MB, 256 * MB


def ce(H=h, W=w, ids=IDS, z=0.0, loss=LOSS, lse=LSE, mean=MEAN, ws=WS, nb=NB):
    return sc.lib().scalify_scaled_linear_cross_entropy(p(H), p(W), ids, -1, z, loss, lse, mean, ws, nb, None)


def ce_bwd(H=h, W=w, ids=IDS, z=0.0, lse=LSE, grad=g, dH=dh, dW=dw, ws=WS, nb=NB):
    return sc.lib().scalify_scaled_linear_cross_entropy_bwd(p(H), p(W), ids, -1, z, lse, p(grad), p(dH), p(dW), ws, nb, None)


def kd(H=h, W=w, T=t, ids=IDS, tl=None, temp=1.0, loss=LOSS, lse=LSE, mean=MEAN, ws=WS, nb=NB):
    return sc.lib().scalify_scaled_linear_distill(p(H), p(W), p(T), ids, -1, tl, temp, loss, lse, mean, ws, nb, None)


def kd_bwd(H=h, W=w, T=t, ids=IDS, tl=None, temp=1.0, lse=LSE, grad=g, dH=dh, dW=dw, ws=WS, nb=NB):
    return sc.lib().scalify_scaled_linear_distill_bwd(p(H), p(W), p(T), ids, -1, tl, temp, lse, p(grad), p(dH), p(dW), ws, nb, None)


@pytest.mark.parametrize("call", [ce, ce_bwd, kd, kd_bwd])
def test_operands(call):
    assert call(H=None) == NULL and call(W=None) == NULL and call(ids=None) == NULL
    assert call(H=arr(1, H16, (4, 64))) == DTYPE                      # not W's type
    assert call(H=arr(1, F, (4, 64)), W=arr(2, F, (100, 64))) == DTYPE
    assert call(H=arr(1, Q, (4, 64))) == DTYPE                        # 8-bit with 16-bit
    assert call(H=arr(1, 7, (4, 64))) == DTYPE
    assert call(H=arr(1, B, (4, 72))) == SHAPE
    assert call(H=arr(1, B, (4, 1, 64))) == SHAPE
    assert call(H=arr(1, B, (4, 0)), W=arr(2, B, (100, 0))) == SHAPE
    assert call(W=arr(2, B, (0, 64))) == SHAPE
    assert call(W=arr(2, B, ((1 << 24) + 1, 64))) == SHAPE
    assert call(H=arr(1, B, (4, 65544)), W=arr(2, B, (100, 65544))) == SHAPE
    assert call(H=arr(1, B, ((1 << 24) + 1, 64))) == SHAPE
    assert call(H=arr(1, B, (4, 64), offset=8)) == ALIGN
    assert call(H=arr(1, B, (4, 64), (68, 1))) == ALIGN
    assert call(W=arr(2, B, (100, 64), (64, 2))) == ALIGN
    assert call(H=arr(1, B, (4, 64), (0, 1))) == SHAPE and call(W=arr(2, B, (100, 64), (56, 1))) == SHAPE   # overlapping rows
    assert call(ws=None) == WORKSPACE and call(nb=4095) == WORKSPACE and call(ws=WS + 128) == WORKSPACE


@pytest.mark.parametrize("call", [kd, kd_bwd])
def test_teacher(call):
    assert call(T=None) == NULL
    assert call(T=arr(3, Q, (4, 16))) == DTYPE
    assert call(T=arr(3, F, (5, 8))) == SHAPE and call(T=arr(3, F, (4, 260))) == SHAPE and call(T=arr(3, F, (32,))) == SHAPE
    assert call(T=arr(3, F, (4, 0))) in (SHAPE, ALIGN)
    assert call(T=arr(3, F, (4, 8), offset=4)) == ALIGN
    for temp in (0.0, -1.0, NAN, INF, 1e-45, 3e38):                   # (the reciprocal has to be a normal number too)
        assert call(temp=temp) == VALUE


@pytest.mark.parametrize("call", [ce, ce_bwd])
def test_penalty(call):
    for z in (-1e-4, NAN, INF):
        assert call(z=z) == VALUE


@pytest.mark.parametrize("call", [ce, kd])
def test_forward_outputs(call):
    assert call(loss=None) == NULL and call(lse=None) == NULL
    assert call(loss=LSE) == ALIAS and call(mean=LSE + 4) == ALIAS and call(mean=LOSS + 12) == ALIAS
    assert call(loss=1 * MB + 64) == ALIAS                            # over H
    assert call(lse=2 * MB + 100 * 128 - 4) == ALIAS                  # over the end of W
    assert call(loss=IDS + 16) == ALIAS


def test_teacher_aliases():
    assert kd(loss=3 * MB) == ALIAS and kd(loss=12 * MB, tl=12 * MB) == ALIAS and kd(mean=IDS + 4 * 8 * 8 - 4) == ALIAS


@pytest.mark.parametrize("call", [ce_bwd, kd_bwd])
def test_backward_outputs(call):
    assert call(dH=None, dW=None) == NULL and call(lse=None) == NULL
    assert call(dH=arr(14, F, (4, 64))) == DTYPE and call(dW=arr(15, Q, (100, 64))) == DTYPE
    assert call(dH=arr(14, B, (5, 64))) == SHAPE and call(dW=arr(15, B, (100, 72))) == SHAPE
    assert call(dW=arr(15, B, (100, 64), (56, 1))) == SHAPE           # rows over one another
    assert call(dW=arr(15, B, (100, 64), (68, 1))) == ALIGN
    assert call(dH=arr(1, B, (4, 64))) == ALIAS and call(dW=arr(2, B, (100, 64))) == ALIAS   # in place
    assert call(dH=arr(15, B, (4, 64), offset=16)) == ALIAS           # over dW
    assert call(dH=arr(10, B, (4, 64))) == ALIAS and call(dW=arr(8, B, (100, 64))) == ALIAS  # over lse, ids
    assert call(dH=arr(13, B, (4, 64))) == ALIAS                      # over grad
    assert call(grad=arr(13, B, (4,))) == DTYPE and call(grad=arr(13, F, (5,))) == SHAPE and call(grad=arr(13, F, (1, 4))) == SHAPE
    assert call(dH=arr(14, B, (4, 64), scale=64), dW=arr(15, B, (100, 64), scale=64)) == ALIAS
    assert call(H=arr(1, B, (4, 64), scale=64), dH=arr(14, B, (4, 64), scale=64)) == ALIAS
    assert call(grad=arr(13, F, (4,), scale=64), dW=arr(15, B, (100, 64), scale=64)) == ALIAS


def test_workspace_sizes():
    size = lambda H, W, k, b: sc.lib().scalify_linear_loss_workspace_bytes(p(H), p(W), k, b)  # noqa: E731
    assert size(h, w, 0, 0) >= 4096 and size(h, w, 8, 1) >= size(h, w, 0, 1) >= 4096
    assert size(None, w, 0, 0) == 0 and size(h, arr(2, H16, (100, 64)), 0, 0) == 0 and size(h, w, 257, 0) == 0 and size(h, w, -1, 0) == 0
    big = size(arr(1, B, (8192, 768)), arr(2, B, (50257, 768)), 0, 1)
    assert big < 8192 * 50257                                         # less than half of the logits in 16 bits
    for call, k, b in ((ce, 0, 0), (kd, 8, 0), (ce_bwd, 0, 1), (kd_bwd, 8, 1)):
        assert call(nb=size(h, w, k, b) - 1) == WORKSPACE


def test_top_logits_refusals():
    x, v = arr(1, B, (4, 100)), arr(2, B, (4, 8))

    def top(X=arr(1, B, (4, 104)), V=v, temp=1.0, ids=IDS, lse=LSE):
        return sc.lib().scalify_scaled_top_logits(p(X), temp, p(V), ids, lse, None)

    assert top(X=None) == NULL and top(V=None) == NULL and top(ids=None) == NULL
    assert top(X=arr(1, Q, (4, 112))) == DTYPE and top(V=arr(2, F, (4, 8))) == DTYPE
    assert top(V=arr(2, B, (5, 8))) == SHAPE and top(V=arr(2, B, (4, 264))) == SHAPE and top(V=arr(2, B, (4, 0))) in (SHAPE, ALIGN)
    assert top(X=arr(1, B, (4, 8)), V=arr(2, B, (4, 16))) == SHAPE      # more than there are
    assert top(X=arr(1, B, (4, (1 << 24) + 8))) == SHAPE
    assert top(V=arr(2, B, (4, 16), (8, 1))) == SHAPE
    assert top(X=x) == ALIGN and top(X=arr(1, B, (4, 104), offset=2)) == ALIGN
    for temp in (0.0, -1.0, NAN, INF, 1e-45, 3e38):
        assert top(temp=temp) == VALUE
    assert top(V=arr(1, B, (4, 8))) == ALIAS and top(ids=1 * MB + 8) == ALIAS and top(lse=1 * MB) == ALIAS
    assert top(lse=IDS) == ALIAS and top(V=arr(8, B, (4, 8))) == ALIAS and top(V=arr(10, B, (4, 8))) == ALIAS
    assert top(X=arr(1, B, (4, 104), scale=64), V=arr(2, B, (4, 8), scale=64)) == ALIAS


def test_python_checks():
    T = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    A = lambda *s, dtype=torch.bfloat16: sc.ScaledTensor(T(*s, dtype=dtype))  # noqa: E731
    H, W = A(4, 64), A(100, 64)
    with pytest.raises(ValueError):
        sc.scalify_linear_loss_workspace_bytes(H, A(100, 64, dtype=torch.float16))
    ws = type("W", (), {"buf": T(8), "ptr": 0, "nbytes": 0})()
    with pytest.raises(ValueError, match="ids"):
        sc.scalify_scaled_linear_cross_entropy(H, W, T(4, dtype=torch.int32), T(4), T(4), ws)
    with pytest.raises(ValueError, match="loss"):
        sc.scalify_scaled_linear_cross_entropy(H, W, T(4, dtype=torch.int64), T(5), T(4), ws)
    with pytest.raises(ValueError, match="mean"):
        sc.scalify_scaled_linear_cross_entropy(H, W, T(4, dtype=torch.int64), T(4), T(4), ws, mean=T(2))
    with pytest.raises(ValueError, match="ids"):
        sc.scalify_scaled_linear_distill(H, W, A(4, 8), T(4, 7, dtype=torch.int64), T(4), T(4), ws)
    with pytest.raises(ValueError, match="teacher_lse"):
        sc.scalify_scaled_linear_distill(H, W, A(4, 8), T(4, 8, dtype=torch.int64), T(4), T(4), ws, teacher_lse=T(3))
    with pytest.raises(ValueError, match="CUDA"):
        sc.scalify_scaled_linear_cross_entropy(H, W, T(4, dtype=torch.int64), T(4), T(4), ws)
    with pytest.raises(ValueError, match="lse"):
        sc.scalify_scaled_top_logits(A(4, 104), A(4, 8), T(4, 8, dtype=torch.int64), lse=T(4, dtype=torch.float64))


@pytest.mark.parametrize("k", [0, 5])
def test_plain_gradient_against_differences(k):
    g_ = torch.Generator().manual_seed(k)
    n, vocab, d = 7, 23, 6
    H, W = (torch.randn(*s, generator=g_, dtype=torch.float64) for s in ((n, d), (vocab, d)))
    ids = torch.randint(0, vocab, (n, k) if k else (n,), generator=g_)
    ids.view(-1)[3] = -1
    T = torch.randn(n, k, generator=g_, dtype=torch.float64) * 2 if k else None
    tl = torch.logsumexp(T / 1.7, 1) + 0.2 if k else None
    up = torch.randn(n, generator=g_, dtype=torch.float64)
    opt = dict(padding_id=-1, T=T, teacher_lse=tl, temp=1.7 if k else 1.0, z_loss=0.0 if k else 0.05, gs=0.5)
    value = lambda a, b: float((pl.linear_loss(a, 0.5, b, 2.0, ids, **opt)["loss"] * up * 0.5).sum())  # noqa: E731
    out = pl.linear_loss(H, 0.5, W, 2.0, ids, grad=up, **opt)
    for X, name, s in ((H, "dH", 0.5), (W, "dW", 2.0)):
        step = torch.randn(X.shape, generator=g_, dtype=torch.float64) * 1e-5
        pair = [(X + q * step, W) if name == "dH" else (H, X + q * step) for q in (1, -1)]
        want = float((out[name] * out[name + "_s"] * step * s).sum())
        assert abs((value(*pair[0]) - value(*pair[1])) / 2 - want) < 1e-8 * abs(want) + 1e-12
