"""Long sums of the output layer's losses: no accumulator of the tensor cores takes more of them than its truncation allows.

An addition there takes 32 bytes of products along K (16 of 16-bit operands, 32 of 8-bit ones; a K block is four additions).  By
measurement (sums of 2^16 to 2^22 products of one sign in one accumulator: 4.3e-4, 1.3e-2, 2.6e-2 too small) every product loses what
lies below 2^-25 of the sum so far, and every addition what lies below 2^-23 of it.  So `a` additions of `t` products in a row
lose at most (t 2^-25 + 2^-23) sum_i S i/a = (a + 1)/2 (t/4 + 1) 2^-23 S; parts joined in fp32 lose half a step of 2^-23 each, at
most parts 2^-24 S.  Everything in one accumulator would lose half of the former on average, with a the whole length: more than the
bars here allow, wherever products have more digits than the 8 of 8-bit operands (those lose next to nothing one by one)."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64_loss as pl
from test_gpu_linear_loss import check, ids_of, layer, rand
from test_gpu_rmsnorm import gen, put

pytestmark = pytest.mark.gpu
BF16, F16, F32, E4M3, E5M2 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.float8_e5m2


def lost(additions, longest, terms=16):
    """Relative loss of a sum of that many additions in parts of at most `longest`."""
    return (min(additions, longest) + 1) / 2 * (terms / 4 + 1) * 2.0 ** -23 + -(-additions // longest) * 2.0 ** -24


def positive(shape, dtype, seed):
    return put(rand(shape, seed).abs().clamp(min=2.0 ** -6), dtype)[0]


def exponents(lse, z):
    """Roundings of the exponentials and of their sum, absolute in lse (derived in plain64_loss)."""
    return 2.0 ** -16 + 2.0 ** -21 * (1 + float(lse.abs().max()) + float(z.abs().max()))


@pytest.mark.parametrize("ht,wt,d", [(BF16, BF16, 16384), (F16, F16, 16384), (E4M3, E4M3, 32768), (E5M2, E4M3, 32768), (BF16, BF16, 4104)])
@pytest.mark.parametrize("n", [40, 200])
def test_logits_of_long_rows(n, ht, wt, d):
    vocab = 300
    H, W = positive((n, d), ht, 1), positive((vocab, d), wt, 2)
    hs, ws = 2.0 ** -4, 2.0 ** -5 if d < 30000 else 2.0 ** -6
    ids = ids_of(n, vocab)
    Hs, Ws = sc.ScaledTensor.make(H, hs), sc.ScaledTensor.make(W, ws)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    wsp = sc.Workspace(sc.scalify_linear_loss_workspace_bytes(Hs, Ws, backward=False))
    sc.scalify_scaled_linear_cross_entropy(Hs, Ws, ids, loss, lse, wsp, padding_id=-1)
    z = H.double() @ W.double().T * (hs * ws)
    want = torch.logsumexp(z, 1)
    # (parts of at most 48 additions)
    ez = lost(-(-d * H.element_size() // 32), 48, 32 // H.element_size()) * float(z.max())
    bar = ez + exponents(want, z)
    assert float((lse.double() - want).abs().max()) <= bar
    there = ids >= 0
    at = torch.where(there, want - z.gather(1, ids.clamp(min=0)[:, None])[:, 0], 0.0)
    assert float((loss.double() - at).abs().max()) <= bar + ez + 2.0 ** -22 * float(want.max())


def relative(got, want):
    return float((got.double() - want).norm() / want.norm())


# The penalty on the logsumexp outweighs the targets, so that D = a p - g q is positive nearly everywhere.
PENALTY = 100.0


@pytest.mark.parametrize("dtype,d", [(F16, 65536), (E4M3, 65536)])
@pytest.mark.parametrize("n", [64, 200])
def test_gradients_of_long_rows(n, dtype, d):
    """The logits computed again for the gradients meet the logsumexp of the forward call's: parts of 64 K blocks there."""
    vocab, hs, ws = 300, 2.0 ** -5, 2.0 ** -5
    H, W = positive((n, d), dtype, 3), positive((vocab, d), dtype, 4)
    ids = ids_of(n, vocab)
    _, _, _, dH, dW, _ = check(H, W, ids, hs=hs, ws=ws, z_loss=PENALTY, out=F16, bars=False)
    fine = pl.linear_loss(H, hs, W, ws, ids, padding_id=-1, z_loss=PENALTY, d_type=F32)
    z = H.double() @ W.double().T * (hs * ws)
    additions, terms = d * H.element_size() // 32, 32 // H.element_size()
    # relative in p: the logits, the logsumexp, the exponentials; D's rounding and the result's (half a step each)
    bar = (lost(additions, 256, terms) + lost(additions, 48, terms)) * float(z.max()) + 2 * exponents(fine["lse"], z) + 2 * 2.0 ** -11
    assert relative(dH.data, fine["dH"]) <= bar and relative(dW.data, fine["dW"]) <= bar


@pytest.mark.parametrize("dtype", [F16, E4M3])
def test_weight_gradient_of_a_long_batch(dtype):
    """dW's contraction is over the rows: parts of 256 K blocks of 64."""
    n, vocab, d, hs, ws, gs = 1 << 22, 64, 64, 2.0 ** -2, 2.0 ** -2, 2.0 ** -7
    H, W = positive((n, d), dtype, 5), positive((vocab, d), dtype, 6)
    ids = torch.randint(0, vocab, (n,), generator=gen(7), device="cuda")
    G = torch.ones(n, device="cuda")
    Hs, Ws = sc.ScaledTensor.make(H, hs), sc.ScaledTensor.make(W, ws)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    wsp = sc.Workspace(sc.scalify_linear_loss_workspace_bytes(Hs, Ws))
    dW = sc.ScaledTensor.empty((vocab, d), F16)
    sc.scalify_scaled_linear_cross_entropy(Hs, Ws, ids, loss, lse, wsp, z_loss=PENALTY)
    sc.scalify_scaled_linear_cross_entropy_bwd(Hs, Ws, ids, lse, None, dW, wsp, z_loss=PENALTY, grad=sc.ScaledTensor.make(G, gs))
    want, step, big = 0.0, 1 << 18, 0.0
    for i in range(0, n, step):
        part = pl.linear_loss(H[i:i + step], hs, W, ws, ids[i:i + step], z_loss=PENALTY, grad=G[i:i + step], gs=gs, d_type=F32)
        want = want + part["dW"] * (pl.kf(step) / pl.kf(n))
        big = max(big, exponents(part["lse"], part["lse"]))
    bar = lost(n // 16, 1024) + 2 * big + 2 * 2.0 ** -11
    assert relative(dW.data, want) <= bar


@pytest.mark.parametrize("n,vocab", [(16, 1 << 22), (20, 1 << 22), (20, 1 << 20)])
def test_hidden_gradient_of_a_large_vocabulary(n, vocab):
    """dH's contraction is over the vocabulary: parts of 256 K blocks of 64, whether a piece has one part or several."""
    d, hs, ws = 16, 2.0 ** -2, 2.0 ** -2
    H, W = positive((n, d), F16, 8), positive((vocab, d), F16, 9)
    ids = torch.randint(0, vocab, (n,), generator=gen(7), device="cuda")
    _, _, _, dH, _, _ = check(H, W, ids, hs=hs, ws=ws, z_loss=PENALTY, out=F16, bars=False)
    fine = pl.linear_loss(H, hs, W, ws, ids, z_loss=PENALTY, d_type=F32)
    # (at most sixteen rows: D in two halves; more: rounded once)
    bar = lost(vocab // 16, 1024) + 2 * exponents(fine["lse"], fine["lse"]) + (2 if n > 16 else 1) * 2.0 ** -11
    assert relative(dH.data, fine["dH"]) <= bar


@pytest.mark.parametrize("ht,wt", [(BF16, BF16), (F16, F16), (E5M2, E4M3)])
@pytest.mark.parametrize("n,vocab,d", [(16385, 300, 72), (33000, 257, 264), (100, 530000, 24), (200, 500, 8200), (33, 300, 8232)])
def test_parts_at_ragged_sizes(n, vocab, d, ht, wt):
    """Every element, either sign: one K block more than a part has, ends of tiles inside and outside."""
    H, W = layer(n, vocab, d, ht, wt, seed=n, pad=n % 2)
    check(H, W, ids_of(n, vocab), ws=2.0 ** -5, grad=rand((n,), 9), out=BF16 if ht == BF16 else F16, pad=1)
    T = 4 * rand((n, 24), 1)
    ids = torch.randint(0, vocab, (n, 24), generator=gen(2), device="cuda")
    check(H, W, ids, ws=2.0 ** -5, T=T, temp=2.0, out=BF16 if ht == BF16 else F16)


@pytest.mark.parametrize("dtype", [F16, E4M3])
@pytest.mark.parametrize("n,vocab,d", [(7, 20011, 24), (20, 20011, 24), (100, 20011, 264), (300, 20011, 72), (5000, 20011, 72), (2500, 30000, 40),
                                       (17000, 1000, 72)])
def test_every_block_of_a_contraction_counts(n, vocab, d, dtype):
    """Terms of one sign and about one size: a K block of 64 left out or taken twice, at the border of a part, a piece or an
    accumulator, changes a gradient by 64 / n or 64 / vocab of itself, more than the bar."""
    hs, ws = 2.0 ** -3, 2.0 ** -3
    H, W = positive((n, d), dtype, 8), positive((vocab, d), dtype, 9)
    ids = torch.randint(0, vocab, (n,), generator=gen(7), device="cuda")
    _, _, _, dH, dW, _ = check(H, W, ids, hs=hs, ws=ws, z_loss=PENALTY, out=F16, bars=False)
    fine = pl.linear_loss(H, hs, W, ws, ids, z_loss=PENALTY, d_type=F32)
    most = 2 * exponents(fine["lse"], fine["lse"]) + 2 * 2.0 ** -11   # (D rounded, and the result)
    for got, name, terms in ((dH, "dH", vocab), (dW, "dW", n)):
        bar = most + lost(-(-terms // 16), 1024)
        assert terms < 256 or 64 / terms > 1.5 * bar
        assert relative(got.data, fine[name]) <= bar


def test_hidden_gradient_of_weights_past_2_31_elements():
    """dH of weights beyond 32-bit offsets, all of it (logits of one sign, as above)."""
    n, vocab, d, hs, ws = 70, 70003, 32768, 2.0 ** -5, 2.0 ** -6
    assert vocab * d > 1 << 31
    H = positive((n, d), E4M3, 1)
    W = torch.empty(vocab, d, dtype=E4M3, device="cuda")
    for i in range(0, vocab, 8192):
        W[i:i + 8192] = positive((min(8192, vocab - i), d), E4M3, 2 + i)
    ids = ids_of(n, vocab)
    Hs, Ws = sc.ScaledTensor.make(H, hs), sc.ScaledTensor.make(W, ws)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    wsp = sc.Workspace(sc.scalify_linear_loss_workspace_bytes(Hs, Ws))
    dH = sc.ScaledTensor.empty((n, d), F16)
    sc.scalify_scaled_linear_cross_entropy(Hs, Ws, ids, loss, lse, wsp, padding_id=-1, z_loss=PENALTY)
    sc.scalify_scaled_linear_cross_entropy_bwd(Hs, Ws, ids, lse, dH, None, wsp, padding_id=-1, z_loss=PENALTY)
    assert wsp.check_status() == 0
    z = torch.cat([H.double() @ W[i:i + 4096].double().T * (hs * ws) for i in range(0, vocab, 4096)], 1)
    want = torch.logsumexp(z, 1)
    there = ids >= 0
    m, unit = int(there.sum()), pl.p2(1.0 / n)
    D = torch.exp(z - want[:, None]) * (1 + 2 * PENALTY * want)[:, None] * there[:, None]
    D[torch.arange(n, device="cuda")[there], ids[there]] -= 1.0
    ref = sum(D[:, i:i + 4096] @ W[i:i + 4096].double() for i in range(0, vocab, 4096)) / m / unit / pl.kf(vocab)
    assert dH.scale_value() == unit * ws * pl.kf(vocab)
    bar = (lost(d // 32, 256, 32) + lost(d // 32, 48, 32)) * float(z.max()) + 2 * exponents(want, z) + 2 * 2.0 ** -11 + lost(vocab // 16, 1024)
    assert relative(dH.data, ref) <= bar
