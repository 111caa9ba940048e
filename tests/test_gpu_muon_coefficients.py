"""Newton-Schulz coefficients near the border of what FP16 holds: finite results, one step inside the element-wise bar of
plain64.newton_schulz_bar."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def inputs(r, c):
    """Gaussian; one singular value of 1 in a corner (an entry of A and of D of its own); all singular values equal."""
    one = torch.zeros(r, c, device="cuda")
    one[r - 1, c - 1] = -3.0
    flat = torch.linalg.qr(torch.randn(c, r, generator=gen(r), device="cuda"))[0].T.contiguous()
    return torch.stack([torch.randn(r, c, generator=gen(c), device="cuda"), one, flat])


@pytest.mark.parametrize("coef", [(15.4, -30.0, 15.0), (-15.4, 0.0, 0.0), (0.0, 0.0, 13.5), (8.25, -23.5, 17.25)])
@pytest.mark.parametrize("r,c", [(40, 96), (300, 400)])
def test_one_step_at_the_border(r, c, coef):
    X = sc.ScaledTensor.make(inputs(r, c), 1.0)
    O = sc.ScaledTensor.empty((3, r, c), BF16)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([X]))
    sc.scalify_orthogonalize(X, O, ws, steps=1, coef=coef)
    unit = 1.0 / p64.kf(c)
    want, bar = p64.newton_schulz(X.data, 1, coef) / unit, p64.newton_schulz_bar(X.data, 1, coef) / unit
    assert ws.check_status() == 0 and bool(p64.close(O.data, want, bar).all())


@pytest.mark.parametrize("coef,steps", [((1.09, 0.0, 0.0), 11), ((3.4445, -4.7750, 2.0315), 16), ((2.0, -1.5, 0.5), 16)])
def test_many_steps_stay_finite(coef, steps):
    X = sc.ScaledTensor.make(inputs(130, 200), 1.0)
    O = sc.ScaledTensor.empty((3, 130, 200), BF16)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([X]))
    sc.scalify_orthogonalize(X, O, ws, steps=steps, coef=coef)
    assert ws.check_status() == 0 and bool(O.data.float().isfinite().all())


def test_coefficients_out_of_range_are_refused():
    X, O = sc.ScaledTensor.make(inputs(40, 96), 1.0), sc.ScaledTensor.empty((3, 40, 96), BF16)
    O.data.fill_(7.0)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([X]))
    with pytest.raises(sc.ScalifyError):
        sc.scalify_orthogonalize(X, O, ws, coef=(20.0, -30.0, 12.0))
    torch.cuda.synchronize()
    assert bool((O.data == 7.0).all())
