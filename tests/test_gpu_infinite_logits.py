"""Infinite and NaN logits: log sum exp of a row that holds +inf is +inf, of one of -inf throughout -inf, of one with NaN NaN."""
import pytest
import torch

import plain64_loss as pl
from test_gpu_linear_loss import check, ids_of, layer, rand
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu
BF16, F16, F32, E5M2, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e5m2, torch.float8_e4m3fn
INF, NAN = float("inf"), float("nan")


def same(got, want, bar):
    """Non-finite values alike, finite ones within the bar."""
    fine = want.isfinite()
    assert bool((got.isfinite() == fine).all())
    assert torch.equal(got.double()[~fine].nan_to_num(nan=5.0, posinf=INF, neginf=-INF), want[~fine].nan_to_num(nan=5.0, posinf=INF, neginf=-INF))
    assert bool(((got.double() - want).abs()[fine] <= bar[fine]).all())


def losses(H, W, ids, lse, z_loss=0.0, T=None):
    """The definition term by term (hs 0.5, ws 0.125): a term that is not there is not 0 times infinity."""
    z = H.double() @ W.double().T / 16
    q, neg, counts = pl.targets(ids, W.shape[0], -1, T)
    loss = neg - torch.where(q > 0, q * z, 0.0).sum(1) + q.sum(1) * lse
    return torch.where(counts, loss + z_loss * lse ** 2 if z_loss else loss, 0.0)


@pytest.mark.parametrize("ht,wt", [(BF16, BF16), (F16, F16), (E5M2, E4M3)])
@pytest.mark.parametrize("n,vocab,d", [(12, 300, 64), (12, 9001, 64), (300, 9001, 72), (40, 2100, 1608), (300, 700, 3208)])
def test_losses(n, vocab, d, ht, wt):
    H, W = layer(n, vocab, d, ht, wt, seed=n + d)
    W[:, 3] = 1.0                      # a row of H with +-inf there has it in all logits, but for these classes
    for v in (0, 255, 256, vocab - 1):
        W[v, 3] = -1.0
    H[1, 3] = INF                      # +inf, four classes -inf
    H[2, 3] = -INF                     # -inf, four classes +inf
    W[:, 5] = 1.0
    H[4, 5] = -INF                     # -inf throughout
    H[5, 3], H[5, 5] = INF, -INF       # NaN in most, -inf in four
    H[6, 7] = NAN
    ids = ids_of(n, vocab, some=False)
    ids[1], ids[2], ids[4] = 0, 7, 9   # the target's logit is -inf, -inf, -inf
    ids[8] = -1
    for z_loss in (0.0, 1e-3):
        loss, lse, m, dH, _, want = check(H, W, ids, z_loss=z_loss, bars=False)
        same(lse, want["lse"], want["e_lse"])
        same(loss, losses(H, W, ids, want["lse"], z_loss), want["e_loss"])
        assert float(lse[1]) == INF and float(lse[2]) == INF and float(lse[4]) == -INF
        assert float(loss[1]) == INF and float(loss[2]) == INF and bool(m.isnan())
        bad = torch.zeros(n, dtype=torch.bool, device="cuda")
        bad[torch.tensor([1, 2, 4, 5, 6], device="cuda")] = True
        assert bool((dH.data.isfinite().all(1) == ~bad).all())
    ids[1], ids[2] = 1, 256            # the target's logit is +inf: inf - inf
    loss, lse, _, _, _, want = check(H, W, ids, bars=False)
    same(loss, losses(H, W, ids, want["lse"]), want["e_loss"])
    assert bool(loss[1].isnan()) and bool(loss[2].isnan()) and float(lse[1]) == INF


def test_mean_of_an_infinite_loss():
    H, W = layer(200, 1000, 64, BF16)
    W[:, 3] = 1.0
    W[17, 3] = -1.0
    H[:, 3] = 0.0
    H[150, 3] = INF
    ids = ids_of(200, 1000)
    ids[150] = 17
    loss, _, m, _, _, _ = check(H, W, ids, bars=False)
    assert float(m) == INF and float(loss[150]) == INF and bool(loss[:150].isfinite().all())


@pytest.mark.parametrize("n", [12, 300])
def test_divergence(n):
    vocab, k = 3000, 8
    H, W = layer(n, vocab, 64, BF16)
    W[:, 3] = 1.0
    W[40:60, 3] = -1.0
    H[1, 3], H[2, 3] = INF, INF
    T = 4 * rand((n, k), 4)
    ids = (100 + torch.rand(n, vocab - 100, generator=gen(5), device="cuda").argsort(1)[:, :k]).contiguous()
    ids[1] = torch.arange(40, 48, device="cuda")      # the teacher's entries are all at -inf: the divergence is infinite
    loss, lse, _, _, _, want = check(H, W, ids, T=T, bars=False)
    same(lse, want["lse"], want["e_lse"])
    same(loss, losses(H, W, ids, want["lse"], T=T.double() * 0.5), want["e_loss"])
    assert float(loss[1]) == INF and bool(loss[2].isnan())
    # entries without any mass: nothing, whatever the student's row holds
    tl = torch.full((n,), 1e4, device="cuda")
    loss, lse, _, _, _, _ = check(H, W, ids, T=T, teacher_lse=tl, bars=False)
    assert float(lse[1]) == INF and not loss.any()
