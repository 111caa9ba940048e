"""scalify_scaled_embedding_lookup and scalify_scaled_embedding_grad against the plain 64-bit form (tests/plain64.py).

Bars: the lookup multiplies by the fp32 rest of c (its own rounding U, the product's U): 2 U.  The gradient adds at most
`count` rows in fp32 in sequence, whatever the split, then multiplies (rest of c: 2 U) and adds the addend (U): the
error is below (count + 4) U of the sum of the magnitudes."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64
from test_gpu_rmsnorm import gap_untouched, gen, put, rows_of

pytestmark = pytest.mark.gpu
U = p64.U
BF16, F16, F32, E4M3, E5M2 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.float8_e5m2
ALL = [BF16, F16, F32, E4M3, E5M2]


def zipf(n, vocab, seed):
    u = torch.rand(n, generator=gen(seed), device="cuda", dtype=torch.float64)
    return (vocab ** u - 1).long().clamp(0, vocab - 1)


def lookup(ids, vocab, d, wt, yt, c, padding_id=None, pad=0, seed=0):
    W, _ = put(torch.randn(vocab, d, generator=gen(seed), device="cuda"), wt, pad)
    Y, base = rows_of(max(ids.numel(), 1), d, yt, pad)
    Y = Y[: ids.numel()]
    Yt = sc.ScaledTensor(Y, torch.zeros(1, device="cuda"))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sc.scalify_scaled_embedding_lookup(ids, sc.ScaledTensor.make(W, 0.25), Yt, c=c, padding_id=padding_id, status=status)
    want = p64.embedding_lookup(ids, W, c, -(1 << 63) if padding_id is None else padding_id, vocab)
    if ids.numel():
        assert Yt.scale_value() == 0.25 * p64.p2(c)
    assert bool(p64.close(Y, want, 2 * U * want.abs()).all()) and gap_untouched(base, d)
    return int(status.item())


@pytest.mark.parametrize("wt", ALL)
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (37, 50, 7), (5, 300, 100), (130, 1000, 768), (33, 500, 1032), (9, 40, 5004)])
def test_lookup(n, vocab, d, wt):
    ids = torch.randint(0, vocab, (n,), generator=gen(n), device="cuda")
    yt = ALL[(n + d) % 5]
    assert lookup(ids, vocab, d, wt, yt, float(d) ** 0.5, pad=n % 2) == 0


def test_lookup_padding_and_unknown_tokens():
    ids = torch.tensor([3, -1, 0, 7, -1, 9], device="cuda")
    assert lookup(ids, 10, 64, BF16, BF16, 3.0, padding_id=-1) == 0
    assert lookup(ids, 10, 64, BF16, F32, 0.3, padding_id=7) == sc.DEV_BAD_INDEX   # -1 is unknown then
    assert lookup(ids, 9, 64, BF16, F32, 1.0, padding_id=-1) == sc.DEV_BAD_INDEX   # 9 is past the table
    assert lookup(torch.tensor([1 << 40, -(1 << 40)], device="cuda"), 9, 64, BF16, F32, 1.0) == sc.DEV_BAD_INDEX
    assert lookup(torch.empty(0, dtype=torch.int64, device="cuda"), 9, 64, BF16, F32, 1.0) == 0


def grad(ids, vocab, d, gt, ot, c=1.0, padding_id=None, tied=False, pad=0, seed=0, in_place=False, status=0):
    n = ids.numel()
    G, _ = put(torch.randn(max(n, 1), d, generator=gen(seed), device="cuda"), gt, pad)
    G = G[:n]
    A, abase = put(torch.randn(vocab, d, generator=gen(seed + 1), device="cuda"), ot, pad) if tied else (None, None)
    W, base = (A, abase) if in_place else rows_of(vocab, d, ot, pad)
    gs, as_ = 2.0 ** -10, 2.0 ** -9
    want, scale, mag, count = p64.embedding_grad(ids, G, gs, vocab, c, -(1 << 63) if padding_id is None else padding_id,
                                                 A.clone() if tied else None, as_)
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, n, d))
    Wt = sc.ScaledTensor(W, torch.zeros(1, device="cuda"))
    sc.scalify_scaled_embedding_grad(ids, sc.ScaledTensor.make(G, gs), Wt, ws, c=c, padding_id=padding_id,
                                     addend=sc.ScaledTensor.make(A, as_) if tied else None)
    assert ws.check_status() == status
    assert Wt.scale_value() == scale
    assert bool(p64.close(W, want, (count + 4) * U * mag).all()) and gap_untouched(base, d)
    return W


@pytest.mark.parametrize("gt", ALL)
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (2, 3, 7), (31, 5, 40), (32, 5, 256), (33, 5, 264), (64, 1, 8), (65, 2, 100),
                                       (500, 37, 768), (700, 300, 520), (1000, 70000, 16)])
def test_grad(n, vocab, d, gt):
    ids = torch.randint(0, vocab, (n,), generator=gen(n + d), device="cuda")
    grad(ids, vocab, d, gt, [F32, BF16, F16][(n + d) % 3], c=float(d) ** 0.5, tied=n % 2 == 0, pad=d % 2, seed=n)


@pytest.mark.parametrize("n,vocab,d,ot", [(4096, 50257, 64, F32), (5000, 300, 64, F32), (8192, 50257, 768, F32),
                                          (8191, 20, 72, F32), (20000, 300, 72, F32), (40000, 100000, 40, BF16),
                                          (131072, 40, 16, F32), (70001, 65535, 16, F32), (70001, 65536, 16, F32),
                                          (3000, 1 << 24, 8, BF16)])
def test_grad_frequent_tokens_and_long_batches(n, vocab, d, ot):
    grad(zipf(n, vocab, n), vocab, d, BF16, ot, c=2.5, seed=n)
    grad(zipf(n, vocab, n + 1), vocab, d, BF16, ot, c=2.5, seed=n, tied=True, padding_id=0)


def test_grad_one_token_only():
    """Every row of the batch belongs to one token: a run over all chunks."""
    for n in (32, 64, 96, 1000, 32768):
        grad(torch.full((n,), 3, device="cuda"), 5, 264, F32, F32, seed=n)


def test_grad_padding_unknown_and_no_tokens():
    ids = torch.tensor([3, -1, 0, 7, -1, 9, 3, 3], device="cuda")
    grad(ids, 10, 64, BF16, F32, padding_id=-1)
    grad(ids, 10, 64, BF16, F32, padding_id=3, status=sc.DEV_BAD_INDEX)
    grad(ids, 8, 64, BF16, F32, padding_id=-1, tied=True, status=sc.DEV_BAD_INDEX)
    grad(torch.full((100,), -1, device="cuda"), 40, 64, BF16, F32, padding_id=-1, tied=True)
    grad(torch.full((100,), 1 << 35, device="cuda"), 40, 64, BF16, F32, status=sc.DEV_BAD_INDEX)
    grad(torch.empty(0, dtype=torch.int64, device="cuda"), 40, 64, BF16, F32)
    grad(torch.empty(0, dtype=torch.int64, device="cuda"), 40, 64, BF16, F32, tied=True)


def test_grad_accumulates_in_place():
    ids = zipf(5000, 900, 4)
    out = grad(ids, 900, 264, BF16, F32, tied=True, seed=5)
    assert torch.equal(out, grad(ids, 900, 264, BF16, F32, tied=True, seed=5, in_place=True))


def test_grad_is_the_same_every_time():
    ids = zipf(30000, 50257, 2)
    first = grad(ids, 50257, 128, BF16, F32, seed=6)
    for _ in range(4):
        assert torch.equal(first, grad(ids, 50257, 128, BF16, F32, seed=6))


def test_offsets_past_32_bits():
    """Rows 2^27 elements apart: table, batch and gradient reach past 2^31 elements."""
    base = torch.empty(20 * (1 << 27), dtype=BF16, device="cuda")
    rows = base.view(20, 1 << 27)
    ids = torch.tensor([19, 3, 19, 0, 18, 5, 5, 19, 7, 1, 1, 1, 1, 12, 19, 2, 2, 4, 19, 19], device="cuda")
    W = torch.randn(20, 40, generator=gen(8), device="cuda").to(BF16)
    rows[:, :40] = W
    zeros = lambda: torch.zeros(1, device="cuda")
    near, far = sc.ScaledTensor.empty((20, 40), BF16), sc.ScaledTensor(rows[:, 64:104], zeros())
    sc.scalify_scaled_embedding_lookup(ids, sc.ScaledTensor.make(W, 1.0), near, c=1.5)
    sc.scalify_scaled_embedding_lookup(ids, sc.ScaledTensor.make(rows[:, :40], 1.0), far, c=1.5)
    assert torch.equal(near.data, far.data) and torch.equal(near.data, (W[ids].double() * 1.5).to(BF16))
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, 20, 40))
    a, b = sc.ScaledTensor.empty((20, 40), BF16), sc.ScaledTensor(rows[:, 128:168], zeros())
    sc.scalify_scaled_embedding_grad(ids, near, a, ws)
    sc.scalify_scaled_embedding_grad(ids, far, b, ws)
    assert torch.equal(a.data, b.data) and torch.equal(rows[:, :40], W)
    want, _, mag, count = p64.embedding_grad(ids, near.data, 1.0, 20, 1.0, -1)
    assert bool(p64.close(b.data, want, (count + 4) * U * mag).all())


def test_calls_on_two_streams_at_once():
    """Two calls beside each other, each with its own workspace."""
    ids = [zipf(20000, 5000, k) for k in (1, 2)]
    G = [sc.ScaledTensor.make(torch.randn(20000, 264, generator=gen(k), device="cuda").to(BF16), 1.0) for k in (1, 2)]
    ws = [sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, 20000, 264)) for _ in (1, 2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[sc.ScaledTensor.empty((5000, 264), F32) for _ in (1, 2)] for _ in range(5)]
    # once alone, every buffer: the first result, and what the bounds-checking build learns of it while nothing runs
    for stream in (None, streams):
        for k, out in enumerate(outs):
            for i in (0, 1):
                if stream is None or k:
                    sc.scalify_scaled_embedding_grad(ids[i], G[i], out[i], ws[i], stream=None if stream is None else stream[i])
                if stream is None:
                    torch.cuda.synchronize()
                    if k:
                        out[i].data.fill_(float("nan"))
        torch.cuda.synchronize()
    assert all(torch.equal(a.data, b.data) for out in outs[1:] for a, b in zip(outs[0], out))
    assert ws[0].check_status() == 0 == ws[1].check_status()


def test_grad_agrees_with_the_atomic_form():
    n, T, vocab, d = 512, 64, 100, 64
    ids = torch.randint(0, vocab, (n,), device="cuda")
    G = sc.ScaledTensor.make(torch.randn(n, d, device="cuda").to(BF16), 1.0)
    a, b = sc.ScaledTensor.empty((vocab, d), F32), sc.ScaledTensor.empty((vocab, d), F32)
    sc.scalify_scaled_embedding_bwd(ids, T, G, a, None)
    sc.scalify_scaled_embedding_grad(ids, G, b, sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, n, d)))
    _, _, mag, count = p64.embedding_grad(ids, G.data, 1.0, vocab, 1.0, -1)
    assert bool(((a.data - b.data).abs() <= 2 * (count + 4) * U * mag).all())


def test_lookup_and_grad_in_a_graph_with_new_tokens():
    n, vocab, d = 3000, 700, 264
    ids = zipf(n, vocab, 1)
    W = sc.ScaledTensor.make(torch.randn(vocab, d, device="cuda").to(BF16), 1.0)
    Y, dW = sc.ScaledTensor.empty((n, d), BF16), sc.ScaledTensor.empty((vocab, d), F32)
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, n, d))

    def step():
        sc.scalify_scaled_embedding_lookup(ids, W, Y, c=2.0)
        sc.scalify_scaled_embedding_grad(ids, Y, dW, ws, c=2.0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    ids.copy_(zipf(n, vocab, 9))
    graph.replay()
    torch.cuda.synchronize()
    got = Y.data.clone(), dW.data.clone()
    step()
    torch.cuda.synchronize()
    assert torch.equal(got[0], Y.data) and torch.equal(got[1], dW.data)
    want, _, mag, count = p64.embedding_grad(ids, Y.data, 1.0, vocab, 2.0, -1)
    assert bool(p64.close(dW.data, want, (count + 4) * U * mag).all())
