"""The output layer's losses and the top logits past 32-bit element offsets, and for very long batches."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64
import plain64_loss as pl
from test_gpu_linear_loss import check, ids_of, layer
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu
BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


@pytest.mark.parametrize("n,vocab,d", [(140001, 600, 16), (70000, 900, 40)])
def test_long_batches(n, vocab, d):
    H, W = layer(n, vocab, d, F16)
    check(H, W, ids_of(n, vocab), out=F16, grad=torch.randn(n, generator=gen(1), device="cuda"))


@pytest.mark.parametrize("n,k", [(5, 0), (120, 0), (120, 30)])
def test_large_vocabularies(n, k):
    """Single-CTA tiles over several pieces, more tiles than the entries' table has bins."""
    vocab, d = 600011, 16
    H, W = layer(n, vocab, d, F16)
    if k:
        T = torch.randn(n, 32, generator=gen(3), device="cuda")[:, :k]
        ids = torch.randint(0, vocab, (n, k), generator=gen(4), device="cuda")
        ids[:, ::3] = torch.randint(0, 3000, (n, k // 3), generator=gen(5), device="cuda")   # many in few bins
        check(H, W, ids, T=T, temp=2.0, out=F16)
    else:
        check(H, W, ids_of(n, vocab), out=F16)


def test_weights_past_2_31_elements():
    n, vocab, d = 70, 70003, 32768
    assert vocab * d > 1 << 31
    H = torch.randn(n, d, generator=gen(1), device="cuda").to(E4M3)
    W = torch.empty(vocab, d, dtype=E4M3, device="cuda")
    for i in range(0, vocab, 8192):
        W[i:i + 8192] = torch.randn(min(8192, vocab - i), d, generator=gen(2 + i), device="cuda").to(E4M3)
    ids = ids_of(n, vocab)
    hs, ws = 2.0 ** -4, 2.0 ** -3
    Hs, Ws = sc.ScaledTensor.make(H, hs), sc.ScaledTensor.make(W, ws)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    wsp = sc.Workspace(max(sc.scalify_linear_loss_workspace_bytes(Hs, Ws, backward=b) for b in (False, True)))
    dH, dW = sc.ScaledTensor.empty((n, d), BF16), sc.ScaledTensor.empty((vocab, d), BF16)
    sc.scalify_scaled_linear_cross_entropy(Hs, Ws, ids, loss, lse, wsp, padding_id=-1)
    sc.scalify_scaled_linear_cross_entropy_bwd(Hs, Ws, ids, lse, dH, dW, wsp, padding_id=-1)
    assert wsp.check_status() == 0
    # the last rows of the vocabulary in 64 bits, given the logsumexp of all of them
    tail = 300
    Wt = W[-tail:]
    z = torch.empty(n, vocab, device="cuda", dtype=torch.float64)
    for i in range(0, vocab, 4096):
        z[:, i:i + 4096] = H.double() @ W[i:i + 4096].double().T * (hs * ws)
    want = torch.logsumexp(z, 1)
    steps = d // 32
    ez = float((H.double().abs() @ Wt.double().abs().T).max()) * hs * ws * (steps + 1) * 2.0 ** -23
    assert float((lse.double() - want).abs().max()) <= ez + 2.0 ** -16 + 2.0 ** -21 * float(1 + want.abs().max() + z.abs().max())
    known = ids >= 0
    m = int(known.sum())
    unit = pl.p2(1.0 / n)
    D = torch.exp(z[:, -tail:] - want[:, None]) * known[:, None] / m / unit
    at = ids - (vocab - tail)
    for t in (known & (at >= 0)).nonzero()[:, 0].tolist():
        D[t, at[t]] -= 1.0 / m / unit
    kn = pl.kf(n)
    ref, mag = D.T @ H.double() / kn, D.abs().T @ H.double().abs() / kn
    rel = 2.0 ** -11 + 2 * ez + 2.0 ** -14     # rounding of D; its exponent; sums
    assert dW.scale_value() == unit * hs * kn
    assert bool(p64.close(dW.data[-tail:], ref, rel * mag + 2.0 ** -36 * H.double().abs().sum(0) / kn).all())
    assert bool(dW.data.isfinite().all()) and bool(dH.data.isfinite().all())


def test_top_logits_past_2_31_elements():
    n, vocab, k = 40000, 60008, 8
    X = torch.empty(n, vocab, dtype=BF16, device="cuda")
    for i in range(0, n, 4000):
        X[i:i + 4000] = torch.randn(4000, vocab, generator=gen(i), device="cuda")
    V, ids = sc.ScaledTensor.empty((n, k), BF16), torch.empty(n, k, dtype=torch.int64, device="cuda")
    lse = torch.empty(n, device="cuda")
    sc.scalify_scaled_top_logits(sc.ScaledTensor.make(X, 1.0), V, ids, lse=lse)
    for r in (slice(0, 20), slice(n - 40, n)):
        want, places = pl.top_logits(X[r], k)
        assert torch.equal(ids[r], places) and torch.equal(V.data[r], want)
        assert bool(((lse[r].double() - torch.logsumexp(X[r].double(), 1)).abs() < 1e-4).all())
