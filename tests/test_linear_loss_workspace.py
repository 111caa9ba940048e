"""A workspace of the output layer's losses that was sized for the longest batch serves every shorter one."""
import ctypes

import pytest
import torch

import paper_2407_17353_b200 as sc
from test_operator_refusals import WORKSPACE, arr

R = ctypes.byref


def size(n, vocab, d, dtype, k, backward):
    return sc.lib().scalify_linear_loss_workspace_bytes(R(arr(1, dtype, (n, d))), R(arr(2, dtype, (vocab, d))), k, backward)


def lengths(longest):
    """Every length up to 300, then steps that meet the borders of row tiles, contraction blocks and pieces, on both sides."""
    yield from range(min(longest, 300) + 1)
    n = 320
    while n <= longest:
        yield from (n - 1, n, n + 1)
        n += 32 if n < 40000 else n // 32 // 32 * 32
    yield longest


@pytest.mark.parametrize("k,backward", [(0, 0), (7, 0), (0, 1), (256, 1)])
@pytest.mark.parametrize("vocab,d,dtype", [(50257, 768, sc.BF16), (50257, 768, sc.E4M3), (128000, 4096, sc.BF16), (32003, 1204, sc.F16),
                                           (500, 64, sc.E4M3), (1, 8, sc.BF16), (1 << 24, 64, sc.F16), (300, 65536, sc.BF16),
                                           (115392, 672, sc.BF16), (1 << 21, 16, sc.F16)])
def test_sizes_never_fall(vocab, d, dtype, k, backward):
    before, at = 0, -1
    for n in lengths(1 << 24 if backward == 0 or vocab < 1000 else 70000):
        s = size(n, vocab, d, dtype, k, backward)
        assert s >= before, (at, before, n, s)
        before, at = s, n


@pytest.mark.parametrize("vocab,d", [(50257, 768), (300, 64)])
def test_a_gradients_workspace_serves_its_forward_call(vocab, d):
    for n in (0, 1, 16, 17, 128, 129, 1000, 2600, 12032, 16384):
        for k in (0, 20):
            assert size(n, vocab, d, sc.BF16, k, 1) >= size(n, vocab, d, sc.BF16, k, 0)


def test_a_longer_batchs_size_is_no_waste():
    """At most what two pieces of D can take (2 x 128 MiB) and the longest of the parts' sums above the batch's own arrays."""
    for n, vocab, d in ((8192, 50257, 768), (4096, 50257, 768), (1531, 32003, 1204), (100, 50257, 768)):
        pieces = 2 * n * -(-vocab // 256) * 256
        assert size(n, vocab, d, sc.BF16, 0, 1) <= min(2 * pieces, 2 << 27) + 4 * n * d * 33 + (48 << 20)


def test_too_small_is_refused():
    H, W = arr(1, sc.BF16, (2600, 768)), arr(64, sc.BF16, (50257, 768))
    need = size(2600, 50257, 768, sc.BF16, 0, 0)
    call = lambda nb: sc.lib().scalify_scaled_linear_cross_entropy(R(H), R(W), 200 << 20, -1, 0.0, 210 << 20, 220 << 20, None,  # noqa: E731
                                                                   256 << 20, nb, None)
    assert call(need // 2) == WORKSPACE and call(4095) == WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("k", [0, 9])
def test_one_workspace_for_all_lengths(k, dtype):
    vocab, d, longest = 50257, 64, 4096
    g = torch.Generator(device="cuda")
    g.manual_seed(k)
    H = torch.randn(longest, d, generator=g, device="cuda").to(dtype)
    W = sc.ScaledTensor.make(torch.randn(vocab, d, generator=g, device="cuda").to(dtype), 0.125)
    ids = torch.randint(0, vocab, (longest, k) if k else (longest,), generator=g, device="cuda")
    T = torch.randn(longest, 2 * 8, generator=g, device="cuda")[:, :k]
    shared = sc.Workspace(sc.scalify_linear_loss_workspace_bytes(sc.ScaledTensor.make(H, 0.5), W, k=k))
    for n in (4096, 2600, 1331, 17, 16, 3, 129, 2700, 0):
        Hs = sc.ScaledTensor.make(H[:n], 0.5)
        outs = []
        for ws in (shared, sc.Workspace(sc.scalify_linear_loss_workspace_bytes(Hs, W, k=k))):
            loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            dH, dW = sc.ScaledTensor.empty((n, d), torch.bfloat16), sc.ScaledTensor.empty((vocab, d), torch.bfloat16)
            if k:
                a = (Hs, W, sc.ScaledTensor.make(T[:n], 0.5), ids[:n])
                sc.scalify_scaled_linear_distill(*a, loss, lse, ws)
                sc.scalify_scaled_linear_distill_bwd(*a, lse, dH, dW, ws)
            else:
                sc.scalify_scaled_linear_cross_entropy(Hs, W, ids[:n], loss, lse, ws)
                sc.scalify_scaled_linear_cross_entropy_bwd(Hs, W, ids[:n], lse, dH, dW, ws)
            assert ws.check_status() == 0
            outs.append([t.clone() for t in (loss, lse, dH.data, dW.data)])
        assert all(torch.equal(a, b) for a, b in zip(*outs))
