"""Calls without rows write the output scale words, as calls with rows do, and nothing else."""
import ctypes

import pytest
import torch

import paper_2407_17353_b200 as sc

pytestmark = pytest.mark.gpu


def test_lookup_of_no_tokens():
    Y = sc.ScaledTensor(torch.empty(0, 64, device="cuda"), torch.full((1,), 7.0, device="cuda"))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    W = sc.ScaledTensor.make(torch.randn(10, 64, device="cuda"), 0.5)
    sc.scalify_scaled_embedding_lookup(torch.empty(0, dtype=torch.int64, device="cuda"), W, Y, c=6.0, status=status)
    assert Y.scale_value() == 2.0 and int(status) == 0


@pytest.mark.parametrize("d", [96, 1024])
def test_norm_of_no_rows(d):
    """(torch gives empty tensors no address, so the descriptors are made from buffers.)"""
    data = torch.full((4, 4, d), 7.0, device="cuda")
    words = torch.tensor([0.5, 4.0, 0.0, 0.0, 2.0], device="cuda")
    gamma = torch.ones(d, device="cuda")

    def desc(k, t, shape):
        a = sc.scalify_array()
        a.data, a.dtype, a.ndim, a.scale = t.data_ptr(), sc.F32, len(shape), words.data_ptr() + 4 * k
        for i, s in enumerate(shape):
            a.shape[i], a.stride[i] = s, d if i + 1 < len(shape) else 1
        return a
    X, R, H, Y = (desc(k, data[k], (0, d)) for k in range(4))
    g = desc(4, gamma, (d,))
    rinv = torch.full((4,), 7.0, device="cuda")
    r = ctypes.byref
    rc = sc.lib().scalify_scaled_add_rmsnorm(r(X), r(R), r(g), 1e-5, r(H), r(Y), None, rinv.data_ptr(), None,
                                             torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert words.tolist() == [0.5, 4.0, 4.0, 2.0, 2.0]
    assert bool((data == 7.0).all()) and bool((rinv == 7.0).all())
