"""A padding id that does not fit the ids' type is refused instead of standing for another one (its lowest 64 bits)."""
import pytest
import torch

import paper_2407_17353_b200 as sc


@pytest.mark.parametrize("padding_id", [1 << 64, (1 << 64) - 1, 1 << 63, -(1 << 63) - 1])
def test_refused(padding_id):
    H, W, T = (sc.ScaledTensor(torch.zeros(*s, dtype=torch.bfloat16)) for s in ((4, 64), (100, 64), (4, 8)))
    ids, v = torch.zeros(4, dtype=torch.int64), [torch.zeros(4), torch.zeros(4)]
    ws = type("W", (), {"buf": torch.zeros(8), "ptr": 0, "nbytes": 0})()
    for call, args in ((sc.scalify_scaled_linear_cross_entropy, (H, W, ids, *v, ws)),
                       (sc.scalify_scaled_linear_cross_entropy_bwd, (H, W, ids, v[0], H, W, ws)),
                       (sc.scalify_scaled_linear_distill, (H, W, T, torch.zeros(4, 8, dtype=torch.int64), *v, ws)),
                       (sc.scalify_scaled_linear_distill_bwd, (H, W, T, torch.zeros(4, 8, dtype=torch.int64), v[0], H, W, ws))):
        with pytest.raises(ValueError, match="padding_id"):
            call(*args, padding_id=padding_id)
    Y = sc.ScaledTensor(torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="padding_id"):
        sc.scalify_scaled_embedding_lookup(ids, W, Y, padding_id=padding_id)
