"""Gradients of the output layer's losses for few rows: their error is that of rounding them, D's own being that of two halves."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64_loss as pl
from test_gpu_linear_loss import BF16, E4M3, E5M2, F16, F32, check, ids_of, layer, rand, teacher

pytestmark = pytest.mark.gpu
KINDS = [(BF16, BF16), (F16, F16), (E4M3, E4M3), (E5M2, E4M3)]


def near(H, W, ids, dH, dW, D_abs, top, hs, ws, half, quantum, **opt):
    """The norm of the error.  dH is the nearest value of its type to (exact + e), so it is at most as far from the exact one as
    the nearest to that is, plus twice |e|.  e: the 64-bit form's bound for a D of 32 bits, and D's two halves: the second one
    rounds what the first left out, half a step of half a step, at its type's smallest step at least (FP16 at the scale that
    brings the largest coefficient to 2^13 at least)."""
    fine = pl.linear_loss(H, hs, W, ws, ids, d_type=F32, **opt)
    h, w = H.double(), W.double()
    exact = dict(dH=fine["dH"], dW=fine["dW"])
    e = half * half * D_abs + quantum / 2 * top * 2.0 ** -13
    more = dict(dH=e @ w.abs() / pl.kf(W.shape[0]), dW=e.T @ h.abs() / pl.kf(H.shape[0]))
    for name, got in (("dH", dH.data), ("dW", dW.data)):
        x = exact[name]
        bar = (x.to(got.dtype).double() - x).norm() + 2 * (fine["e_" + name] + more[name]).norm()
        err = (got.double() - x).norm()
        assert bool(err <= bar), (name, float(err / x.norm()), float(bar / x.norm()))


def sizes(H, hs, W, ws, ids):
    """|D| of a cross entropy's mean and its rows' coefficient, in units of the gradient's scale."""
    n, vocab = H.shape[0], W.shape[0]
    p = torch.softmax(H.double() @ W.double().T * (hs * ws), 1)
    valid = ids >= 0
    p[torch.arange(n, device="cuda")[valid], ids[valid]] -= 1
    top = 1.0 / max(1, int(valid.sum())) / pl.p2(1.0 / n)
    return torch.where(valid[:, None], p.abs(), 0.0) * top, top


@pytest.mark.parametrize("ht,wt", KINDS)
@pytest.mark.parametrize("n,vocab,d", [(1, 300, 64), (2, 1646, 136), (3, 40, 24), (5, 1745, 158), (11, 129, 80), (16, 300, 72)])
def test_gradients_are_rounded_once(n, vocab, d, ht, wt):
    H, W = layer(n, vocab, d, ht, wt, seed=n + d, pad=8 * (n % 2))
    ids = ids_of(n, vocab)
    _, _, _, dH, dW, _ = check(H, W, ids, out=BF16 if ht == BF16 else F16, pad=d % 2)
    d_type = BF16 if ht == BF16 else F16
    near(H, W, ids, dH, dW, *sizes(H, 0.5, W, 0.125, ids), 0.5, 0.125, torch.finfo(d_type).eps / 2, pl.QUANTUM[d_type], padding_id=-1)


@pytest.mark.parametrize("ht", [BF16, F16, E4M3])
@pytest.mark.parametrize("n", [1, 4, 15, 16, 17])
@pytest.mark.parametrize("vocab", [1, 31, 33, 257, 9001])
def test_ends_of_rows_and_of_tiles(n, vocab, ht):
    H, W = layer(n, vocab, 72, ht, seed=n + vocab, pad=n % 3)
    check(H, W, ids_of(n, vocab), grad=rand((n,), 5), z_loss=1e-3 if n % 2 else 0.0, out=F16 if ht == F16 else BF16, out2=F16, pad=1)
    T, ids = teacher(n, min(vocab, 9), vocab, BF16)
    check(H, W, ids, T=T, grad=rand((n,), 6), out=BF16, pad=3)


@pytest.mark.parametrize("n", [2, 16])
def test_either_side_alone(n):
    H, W = layer(n, 5003, 200, BF16, seed=n)
    ids = ids_of(n, 5003)
    Hs, Ws = sc.ScaledTensor.make(H, 0.5), sc.ScaledTensor.make(W, 0.125)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ws = sc.Workspace(sc.scalify_linear_loss_workspace_bytes(Hs, Ws))
    sc.scalify_scaled_linear_cross_entropy(Hs, Ws, ids, loss, lse, ws, padding_id=-1)
    got = []
    for sides in ((1, 1), (1, 0), (0, 1)):
        dH = sc.ScaledTensor.empty((n, 200), BF16) if sides[0] else None
        dW = sc.ScaledTensor.empty((5003, 200), BF16) if sides[1] else None
        sc.scalify_scaled_linear_cross_entropy_bwd(Hs, Ws, ids, lse, dH, dW, ws, padding_id=-1)
        got.append((dH, dW))
    assert torch.equal(got[0][0].data, got[1][0].data) and torch.equal(got[0][1].data, got[2][1].data)
