"""The embedding gradient of batches whose sort takes more than one tile of 8192 keys per block (beyond 131072 tokens with
the 16 blocks of the cluster): counts from a sweep of their own, first slots carried from tile to tile."""
import pytest
import torch

import paper_2407_17353_b200 as sc
from test_gpu_embedding_sorted import grad, zipf
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("vocab", [200, 50257, 100000])   # one, two and three passes of 8 bits
@pytest.mark.parametrize("n", [131073, 139264, 300001])   # keys per block: 8193, 8704, 18751
def test_several_tiles(n, vocab):
    ids = zipf(n, vocab, n)
    ids[torch.rand(n, generator=gen(1), device="cuda") < 0.03] = -1                  # padding
    ids[torch.rand(n, generator=gen(2), device="cuda") < 0.2] = vocab - 1            # one token in a fifth of the batch
    grad(ids, vocab, 16, BF16, F32, c=2.5, padding_id=-1, seed=n, tied=True)
    ids[::1001] = vocab + 5                                                            # unknown ones: left out, reported
    first = grad(ids, vocab, 16, BF16, F32, padding_id=-1, seed=n, status=sc.DEV_BAD_INDEX)
    for _ in range(2):
        assert torch.equal(first, grad(ids, vocab, 16, BF16, F32, padding_id=-1, seed=n, status=sc.DEV_BAD_INDEX))


def test_the_sort_is_stable_over_tiles():
    """Rows whose fp32 sum depends on the order: 2^24, then ones that are each lost beside it (ties, to even), then -2^24, for
    tokens that occur 13 or 14 times: a run of at most 16 is summed whole, in the order of the batch."""
    n, vocab = 270000, 20000
    ids = (torch.arange(n, device="cuda") % vocab).contiguous()
    G = torch.zeros(n, 8, device="cuda")
    for token, count in ((3, 14), (7777, 14), (19999, 13)):
        at = (ids == token).nonzero()[:, 0]
        assert at.numel() == count
        G[at] = 1.0
        G[at[0]], G[at[-1]] = 2.0 ** 24, -2.0 ** 24
    W = sc.ScaledTensor.empty((vocab, 8), F32)
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, n, 8))
    sc.scalify_scaled_embedding_grad(ids, sc.ScaledTensor.make(G, 1.0), W, ws)
    assert ws.check_status() == 0 and bool((W.data == 0).all())


def test_all_padding_and_one_token():
    n = 140000
    grad(torch.full((n,), -1, device="cuda"), 300, 16, BF16, F32, padding_id=-1, tied=True)
    grad(torch.full((n,), 299, device="cuda"), 300, 16, BF16, F32, seed=3)
