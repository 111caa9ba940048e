"""The order of the embedding gradient's sums: the token ids alone fix it."""
import pytest
import torch

import paper_2407_17353_b200 as sc
from test_gpu_embedding_sorted import zipf
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [4000, 16383, 16384, 20000, 65536])
def test_a_column_does_not_depend_on_the_others(n):
    """The same ids with rows of 64 and of 2048 elements: the same bits in the columns they share, frequent tokens included."""
    ids = zipf(n, 300, n)
    G = torch.randn(n, 2048, generator=gen(n), device="cuda").to(torch.bfloat16)
    out = []
    for d in (64, 520, 2048):
        W = sc.ScaledTensor.empty((300, d), torch.float32)
        ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, n, d))
        sc.scalify_scaled_embedding_grad(ids, sc.ScaledTensor.make(G[:, :d], 1.0), W, ws)
        out.append(W.data)
    assert torch.equal(out[0], out[2][:, :64]) and torch.equal(out[1], out[2][:, :520])


def test_one_workspace_for_batches_of_any_length():
    """A workspace of the longest batch, used for shorter ones in between."""
    d = 264
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, 17000, d))
    G = torch.randn(17000, d, generator=gen(1), device="cuda").to(torch.bfloat16)
    ids = zipf(17000, 500, 1)
    for n in (17000, 16383, 3, 16384, 12000, 0):
        out = []
        for w in (ws, sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, n, d))):
            W = sc.ScaledTensor.empty((500, d), torch.float32)
            sc.scalify_scaled_embedding_grad(ids[:n], sc.ScaledTensor.make(G[:n], 1.0), W, w)
            assert w.check_status() == 0
            out.append(W.data)
        assert torch.equal(*out)
