"""The top logits' logsumexp of rows with infinities and NaN: exactly the infinity or NaN that the definition has."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64_loss as pl
from test_gpu_infinite_logits import BF16, F16, F32, INF, NAN, same
from test_gpu_rmsnorm import gen, put, rows_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("n,vocab,k", [(12, 9000, 3), (12, 50257, 200), (400, 9001, 16), (400, 5003, 200), (12, 11, 5)])
def test_top_logits(n, vocab, k, dt):
    X, _ = put(3 * torch.randn(n, vocab, generator=gen(n + vocab), device="cuda"), dt)
    last = vocab - 1
    X[0, last] = INF
    X[1, 0], X[1, 3] = INF, INF
    X[2] = INF
    X[3] = -INF
    X[4, 5], X[4, last - 1] = INF, NAN
    X[5, 2] = NAN
    X[6, ::2] = -INF
    X[7] = torch.finfo(dt).min
    X[7, last // 2] = INF
    X[8] = torch.finfo(dt).max
    X[8, 1] = INF
    X[9] = -INF
    X[9, last] = INF
    X[10] = -INF
    X[10, last] = 1.5
    V, ids, lse = sc.ScaledTensor(rows_of(n, k, dt)[0], torch.zeros(1, device="cuda")), torch.zeros(n, k, dtype=torch.int64, device="cuda"), torch.zeros(n, device="cuda")
    for s, temp in ((1.0, 1.0), (0.5, 2.0), (2.0 ** -30, 0.7)):
        sc.scalify_scaled_top_logits(sc.ScaledTensor.make(X, s), V, ids, lse=lse, temperature=temp)
        want, places = pl.top_logits(X, k)
        assert torch.equal(ids, places) and torch.equal(V.data.nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))
        ref = torch.logsumexp(X.double() * (s / temp), 1)
        # (exponents in base 2, rounded three times at their size; sums of at most vocab/4096 + 32 sequential additions)
        same(lse, ref, 2.0 ** -20 * (1 + torch.where(X.isfinite(), X.double().abs() * (s / temp), 0.0).amax(1)) + (vocab / 4096 + 32) * 2.0 ** -24)
