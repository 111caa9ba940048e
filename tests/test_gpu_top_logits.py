"""The top logits of a row against a stable 64-bit sort (values and places exactly), and their logsumexp.

Bar of the logsumexp: exponents in base 2 are rounded in fp32 at sizes up to |x| log2(e) (2^-22 of it, three roundings), ex2
2^-22; a thread adds its elements one vector's sum after the other, at most vocab/4096 + 8 sequential additions, 13 more
across the block."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64_loss as pl
from test_gpu_rmsnorm import gap_untouched, gen, put, rows_of

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")


def check(X, k, s=0.5, temp=1.0, pad=0, lse=True):
    n, vocab = X.shape
    V, base = rows_of(max(n, 1), k, X.dtype, pad)
    V = V[:n]
    Vs = sc.ScaledTensor(V, torch.zeros(1, device="cuda"))
    ids = torch.full((n, k), -7, dtype=torch.int64, device="cuda")
    out = torch.zeros(n, device="cuda") if lse else None
    sc.scalify_scaled_top_logits(sc.ScaledTensor.make(X, s), Vs, ids, lse=out, temperature=temp)
    want, places = pl.top_logits(X, k)
    assert Vs.scale_value() == s and gap_untouched(base, k)
    assert torch.equal(ids, places)
    assert torch.equal(V.nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))
    if lse and n:
        z = X.double() * s / temp
        ref = torch.logsumexp(z, 1)
        fine = ref.isfinite()
        big = torch.where(z.isfinite(), z.abs(), 0.0).amax(1)
        bar = 2.0 ** -20 * (1 + big) + (vocab / 4096 + 32) * 2.0 ** -24
        assert bool(((out.double() - ref).abs()[fine] <= bar[fine]).all())
        assert bool((out.isnan() | (out.double() == ref))[~fine].all())
    return V, ids


@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("n,vocab,k", [(1, 1, 1), (3, 7, 7), (2, 256, 256), (5, 511, 100), (4, 2047, 255), (3, 2049, 256), (37, 5003, 16),
                                       (2, 50257, 64), (300, 1000, 1), (2, 200003, 256)])
def test_random_rows(n, vocab, k, dt):
    X, _ = put(3 * torch.randn(n, vocab, generator=gen(n + vocab), device="cuda"), dt, vocab % 2)
    check(X, k, temp=[1.0, 0.7, 2.0][k % 3], pad=k % 2, lse=n != 3)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_ties(dt):
    X = torch.zeros(6, 6000, device="cuda")
    X[1] = -0.0
    X[1, ::2] = 0.0                                    # equal to -0
    X[2, 5000:] = 1.0
    X[3] = torch.randint(0, 3, (6000,), generator=gen(1), device="cuda").float()
    X[4, 17] = 2.0
    X[5] = -INF
    for k in (1, 64, 256):
        check(X.to(dt), k)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_infinities_nan_and_lowest_values(dt):
    X = torch.randn(7, 9000, generator=gen(2), device="cuda").to(dt)
    X[0, 4000:] = -INF
    X[1, :8999] = -INF
    X[2, 5], X[2, 77] = INF, INF
    X[3, 100], X[3, 8000] = float("nan"), float("nan")
    X[4, ::2] = torch.finfo(dt).min
    X[5] = float("nan")
    X[6] = INF
    for k in (3, 200):
        check(X, k, s=1.0)


@pytest.mark.parametrize("dt", [BF16, F16, F32])
def test_rows_of_the_lowest_value(dt):
    """What an additive mask leaves of a row: the lowest finite value throughout, or but for one place; and the largest."""
    low = torch.finfo(dt).min
    X = torch.full((5, 5000), low, device="cuda", dtype=dt)
    X[1, 4321] = 2.0
    X[2] = -low
    X[3, ::2] = low / 2
    X[4, 7:] = -INF
    V, ids = sc.ScaledTensor.empty((5, 8), dt), torch.zeros(5, 8, dtype=torch.int64, device="cuda")
    lse = torch.zeros(5, device="cuda")
    for temp in (1.0, 2.0):
        sc.scalify_scaled_top_logits(sc.ScaledTensor.make(X, 1.0), V, ids, lse=lse, temperature=temp)
        want, places = pl.top_logits(X, 8)
        assert torch.equal(V.data, want) and torch.equal(ids, places)
        ref = torch.logsumexp(X.double() / temp, 1)
        assert bool(((lse.double() - ref).abs() <= 2.0 ** -22 * ref.abs() + 2.0 ** -18).all())


def test_subnormal_and_huge_values():
    for dt in (BF16, F16, F32):
        tiny = torch.finfo(dt).smallest_normal
        X = (torch.randn(3, 3000, generator=gen(3), device="cuda").double() * tiny / 4).to(dt)
        check(X, 50, s=1.0)
        Y = (torch.randn(3, 3000, generator=gen(4), device="cuda").clamp(-3.9, 3.9).double() * torch.finfo(dt).max / 4).to(dt)
        check(Y, 50, s=2.0 ** -100 if dt != F16 else 2.0 ** -10)


def test_no_rows():
    check(torch.empty(0, 100, dtype=BF16, device="cuda"), 5)


def test_replayed():
    X = torch.randn(64, 4000, generator=gen(5), device="cuda").to(BF16)
    V, ids = sc.ScaledTensor.empty((64, 32), BF16), torch.zeros(64, 32, dtype=torch.int64, device="cuda")
    lse = torch.zeros(64, device="cuda")
    Xs = sc.ScaledTensor.make(X, 0.5)
    sc.scalify_scaled_top_logits(Xs, V, ids, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sc.scalify_scaled_top_logits(Xs, V, ids, lse=lse)
    X.copy_(torch.randn(64, 4000, generator=gen(6), device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    want, places = pl.top_logits(X, 32)
    assert torch.equal(ids, places) and torch.equal(V.data, want)
