"""The norm gradient of rows beyond 6144 columns with several rows per block: column sums and statistic carried over rows, the
next row requested ahead, the residual gradient read again where dX is written over it.  Bars as in test_gpu_rmsnorm."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64
from test_gpu_rmsnorm import U, gen, put, rows_of, run_backward, scaled

pytestmark = pytest.mark.gpu
BF16, F16, F32, E4M3, E5M2 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.float8_e5m2


@pytest.mark.parametrize("gt,ht", [(BF16, BF16), (BF16, F32), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("rows,d", [(700, 8200), (1000, 6152), (613, 6145), (310, 16384)])
def test_rows_in_turn(rows, d, gt, ht):
    """Two resident blocks per SM at 6152 columns, one above: up to five rows for a block, the last round ragged."""
    ws, *_ = run_backward(rows, d, gt, ht, qt=E5M2, seed=rows, stat=sc.STAT_AMAX, stat_in=torch.full((1,), 3.7, device="cuda"))
    assert ws.check_status() == 0
    run_backward(rows, d, gt, ht, qt=E4M3, seed=d, pad=3, stat=sc.STAT_L2, residual=False, gamma_dt=BF16, dg_dt=BF16)


@pytest.mark.parametrize("alias,gt,ht", [("Gr", BF16, BF16), ("Gr", BF16, F32), ("G", F32, F32), ("G", BF16, BF16)])
@pytest.mark.parametrize("rows,d", [(700, 8200), (1000, 6152)])
def test_in_place(alias, gt, ht, rows, d):
    run_backward(rows, d, gt, ht, qt=E5M2, seed=6, alias=alias, stat=sc.STAT_AMAX)
    run_backward(rows, d, gt, ht, seed=7, pad=1, alias=alias, stat=sc.STAT_L2)


@pytest.mark.parametrize("rows,d", [(700, 8200), (1000, 6152)])
def test_the_same_every_time_and_broadcast_rows(rows, d):
    first = run_backward(rows, d, BF16, F32, qt=E5M2, seed=9, stat=sc.STAT_AMAX)
    again = run_backward(rows, d, BF16, F32, qt=E5M2, seed=9, stat=sc.STAT_AMAX)
    assert torch.equal(first[3].data, again[3].data) and torch.equal(first[1].data, again[1].data)
    H, _ = put(torch.randn(rows, d, generator=gen(d), device="cuda"), F32)
    one = torch.randn(d, generator=gen(d + 1), device="cuda").to(BF16)
    G = one.as_strided((rows, d), (0, 1))
    rinv = ((H.double().square().mean(1) + 1e-5) ** -0.5).float()
    dX = sc.ScaledTensor(rows_of(rows, d, F32)[0], torch.empty(1, device="cuda"))
    dg = sc.ScaledTensor.empty((d,), F32)
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_RMSNORM_BWD, rows, d))
    sc.scalify_scaled_add_rmsnorm_bwd(scaled(G, 1.0), None, scaled(H, 1.0), None, rinv, dX, ws, dgamma=dg)
    want = p64.add_rmsnorm_bwd(G, 1.0, None, 0.0, H, 1.0, None, 1.0, rinv)
    assert ws.check_status() == 0 and bool(p64.close(dX.data, want["dX"], U * want["mag"]).all())
    assert bool(p64.close(dg.data, want["dgamma"], (rows + 16) * U * want["dgamma_mag"]).all())
