"""scalify_scaled_add_rmsnorm and its gradient against the plain 64-bit form (tests/plain64.py).

Bars: the sum of squares of a row of d elements is added in fp32 by at most 32 sequential adds per lane, five shuffles
and at most five more across warps, so its relative error is below 48 U and that of its inverse root below 24 U + 3 U
(division, addition of eps, root); two multiplications follow.  30 U on n * gamma covers it.  In the gradient every term
of the row's dot product carries the same 48 sequential adds plus the roundings of its factors, hence 64 U of the mean
magnitude; the other operations are 8 U of the terms they combine.  dgamma adds `rows` terms in fp32 at worst."""
import math

import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64

pytestmark = pytest.mark.gpu
U = p64.U
BF16, F16, F32, E4M3, E5M2 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.float8_e5m2
PAIRS = [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (F32, F32)]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows_of(rows, d, dtype, pad=0):
    """[rows, d] view with a row stride that is a multiple of 16 bytes (`pad` more vectors between the rows); the gap
    is filled with a value the kernels must neither use nor change."""
    step = 16 // torch.empty(0, dtype=dtype).element_size()
    ld = (-(-d // step) + pad) * step
    base = torch.full((rows, ld), 7.0, device="cuda").to(dtype)
    return base[:, :d], base


def put(x, dtype, pad=0):
    v, base = rows_of(*x.shape, dtype, pad)
    v.copy_(p64.saturate(x, dtype))
    return v, base


def gap_untouched(base, d):
    gap = base[:, d:].float()
    return bool((gap == 7.0).all())


def make(rows, d, xt, ht, seed, gamma_dt=F32):
    g = gen(seed)
    x, r = torch.randn(rows, d, generator=g, device="cuda"), 3 * torch.randn(rows, d, generator=g, device="cuda")
    gamma = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(gamma_dt) if gamma_dt else None
    return x, r, gamma


def scaled(t, s):
    return None if t is None else sc.ScaledTensor.make(t, s)


def run_forward(rows, d, xt, ht, yt, *, seed=0, pad=0, gamma_dt=F32, residual=True, eps=1e-5, mx=False):
    x, r, gamma = make(rows, d, xt, ht, seed, gamma_dt)
    X, _ = put(x, xt, pad)
    R, _ = put(r, ht, pad) if residual else (None, None)
    H, hbase = rows_of(rows, d, ht, pad) if residual else (None, None)
    Y, ybase = rows_of(rows, d, yt, pad)
    rinv = torch.full((rows,), -1.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    xs, rs = 0.5, 4.0
    Ht = None if H is None else sc.ScaledTensor(H, torch.zeros(1, device="cuda"))
    Yt = sc.MxTensor(rows, d, yt) if mx else sc.ScaledTensor(Y, torch.zeros(1, device="cuda"))
    sc.scalify_scaled_add_rmsnorm(scaled(X, xs), scaled(R, rs), scaled(gamma, 2.0), Ht, Yt, eps=eps, rinv=rinv, status=status)
    assert int(status.item()) == 0
    total, hs, norm = p64.add_rmsnorm(X, xs, R, rs, gamma, eps)
    if residual:
        assert Ht.scale_value() == hs
        assert bool(p64.close(H, total, U * total.abs()).all()) and gap_untouched(hbase, d)
    y, ri = norm(H if residual else X)
    assert Yt.scale_value() == (2.0 if gamma_dt else 1.0)
    assert bool(p64.close(rinv, ri, 27 * U * ri).all())
    if not mx:
        assert bool(p64.close(Y, y, 30 * U * y.abs()).all()) and gap_untouched(ybase, d)
    return dict(X=X, R=R, gamma=gamma, H=H if residual else X, Y=Yt, rinv=rinv, y=y, hs=hs if residual else xs)


@pytest.mark.parametrize("xt,ht", PAIRS)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (5, 64), (37, 100), (2, 264), (9, 768), (6, 1000), (4, 1024), (3, 1032),
                                    (5, 5004), (2, 8200), (1, 16384)])
def test_forward(rows, d, xt, ht):
    yt = [E4M3, E5M2, BF16, F16, F32][(rows + d) % 5]
    run_forward(rows, d, xt, ht, yt, seed=rows * d, pad=rows % 3)


@pytest.mark.parametrize("yt", [E4M3, E5M2, BF16, F16, F32])
@pytest.mark.parametrize("gamma_dt", [None, F32, BF16, F16])
def test_forward_output_and_gamma_types(yt, gamma_dt):
    run_forward(130, 776, BF16, BF16, yt, seed=3, gamma_dt=gamma_dt)
    run_forward(11, 2056, BF16, F32, yt, seed=4, gamma_dt=gamma_dt, residual=False)


def test_equals_the_separate_add():
    """H is scalify_scaled_add's output bit for bit."""
    r = run_forward(300, 768, BF16, BF16, E4M3, seed=8)
    Y = sc.ScaledTensor.empty((300, 768), BF16)
    sc.scalify_scaled_add(sc.ScaledTensor.make(r["X"].contiguous(), 0.5), sc.ScaledTensor.make(r["R"].contiguous(), 4.0), Y)
    assert torch.equal(Y.data.view(torch.int16), r["H"].contiguous().view(torch.int16)) and Y.scale_value() == r["hs"]


@pytest.mark.parametrize("yt", [E4M3, E5M2])
@pytest.mark.parametrize("rows,d", [(1, 128), (3, 256), (129, 768), (256, 1024), (300, 1152), (70, 4096), (2, 16384)])
def test_block_scaled_output_equals_quantising_the_wide_output(rows, d, yt):
    """The fused quantisation is scalify_mx_quantize of the fp32 output: same bytes, same exponents, padding included."""
    wide = run_forward(rows, d, BF16, F32, F32, seed=d)
    got = run_forward(rows, d, BF16, F32, yt, seed=d, mx=True)["Y"]
    want = sc.MxTensor(rows, d, yt)
    sc.scalify_mx_quantize(sc.ScaledTensor.make(wide["Y"].data.contiguous(), 2.0), want)
    assert torch.equal(got.data.view(torch.uint8), want.data.view(torch.uint8))
    assert torch.equal(got.sf, want.sf)


def test_rows_of_zeros_and_of_infinities_stay_their_own():
    rows, d = 9, 768
    x = torch.randn(rows, d, device="cuda").to(BF16)
    x[2] = 0
    x[4, 5] = float("inf")
    x[6, 7] = float("nan")
    for dd, xx in ((d, x), (1536, x.repeat(1, 2))):
        rinv = torch.empty(rows, device="cuda")
        Y = sc.ScaledTensor.empty((rows, dd), BF16)
        M = sc.MxTensor(rows, 1536)
        sc.scalify_scaled_add_rmsnorm(sc.ScaledTensor.make(xx, 1.0), None, None, None, Y, eps=1e-5, rinv=rinv)
        ok = [0, 1, 2, 3, 5, 7, 8]
        want, _ = p64.add_rmsnorm(xx, 1.0, None, 1.0, None, 1e-5)[2](xx)
        assert bool(p64.close(Y.data, want, 30 * U * want.abs())[ok].all())
        assert bool((Y.data[2] == 0).all()) and bool(Y.data[6].isnan().any())
    sc.scalify_scaled_add_rmsnorm(sc.ScaledTensor.make(xx, 1.0), None, None, None, M, eps=0.0)
    assert bool((M.exponents()[2] == 127).all()) and bool((M.data[2].float().isnan() | (M.data[2].float() == 0)).all())


def test_in_place_residual_stream():
    """H in R's buffer and H in X's buffer give the bits of the call with buffers of their own."""
    for ht, where in ((F32, "R"), (BF16, "R"), (BF16, "X")):
        a = run_forward(133, 1032, BF16, ht, E4M3, seed=5)
        x, r = a["X"].clone(), a["R"].clone()
        H = r if where == "R" else x
        Y = sc.ScaledTensor.empty((133, 1032 + 8), E4M3)
        Y.data = Y.data[:, :1032]
        sc.scalify_scaled_add_rmsnorm(sc.ScaledTensor.make(x, 0.5), sc.ScaledTensor.make(r, 4.0), sc.ScaledTensor.make(a["gamma"], 2.0),
                                      sc.ScaledTensor(H, torch.empty(1, device="cuda")), Y, eps=1e-5)
        assert torch.equal(H.float(), a["H"].float())
        assert torch.equal(Y.data.float(), a["Y"].data.float())


def run_backward(rows, d, gt, ht, *, qt=None, seed=0, pad=0, gamma_dt=F32, residual=True, stat=None, dg_dt=F32, stat_in=None,
                 alias=None):
    g = gen(seed)
    rnd = lambda: torch.randn(rows, d, generator=g, device="cuda")  # noqa: E731
    H, _ = put(2 * rnd(), ht, pad)
    G, gb = put(rnd(), gt, pad)
    Gr, rb = put(rnd(), ht, pad) if residual else (None, None)
    gamma = (1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(gamma_dt) if gamma_dt else None
    rinv = ((H.double().square().mean(1) + 1e-5) ** -0.5).float()
    gs, grs, hs = 2.0 ** -9, 2.0 ** -12, 2.0
    want = p64.add_rmsnorm_bwd(G, gs, Gr, grs, H, hs, gamma, 1.0 if gamma is None else 4.0, rinv)
    dX, base = rows_of(rows, d, ht, pad) if alias is None else ((Gr, rb) if alias == "Gr" else (G, gb))
    dXq, qbase = rows_of(rows, d, qt, pad) if qt else (None, None)
    word = lambda: torch.zeros(1, device="cuda")  # noqa: E731
    T = sc.ScaledTensor
    dg = T(torch.full((d,), 9.0, device="cuda").to(dg_dt), word()) if dg_dt else None
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_RMSNORM_BWD, rows, d))
    dXt, dQt = T(dX, word()), (T(dXq, word()) if qt else None)
    sc.scalify_scaled_add_rmsnorm_bwd(scaled(G, gs), scaled(Gr, grs), scaled(H, hs), scaled(gamma, 4.0), rinv, dXt, ws, dXq=dQt,
                                      stat_in=stat_in, stat_dx=stat or sc.STAT_NONE, dgamma=dg)
    assert dXt.scale_value() == want["dX_s"]
    assert bool(p64.close(dX, want["dX"], U * want["mag"]).all()) and gap_untouched(base, d)
    r = 1.0
    if stat_in is not None and math.isfinite(float(stat_in)) and float(stat_in) >= 2.0 ** -126:
        r = p64.p2(float(stat_in))
    if qt:  # a cast of the stored gradient: exact up to that one rounding
        assert dQt.scale_value() == want["dX_s"] * r
        cast = p64.saturate(dX.float() / r, qt).to(qt)
        assert torch.equal(cast.view(torch.uint8), dXq.contiguous().view(torch.uint8)) and gap_untouched(qbase, d)
    if dg is not None:
        assert dg.scale_value() == want["dgamma_s"]
        assert bool(p64.close(dg.data, want["dgamma"], (rows + 16) * U * want["dgamma_mag"]).all())
    if stat == sc.STAT_AMAX:
        assert float(ws.statistic()) == float(dX.float().abs().max())
    if stat == sc.STAT_L2:  # sums in fp64, one rounding to fp32
        assert math.isclose(float(ws.statistic()), float(dX.double().square().mean().sqrt()), rel_tol=2 * U)
    return ws, dXt, dQt, dg


@pytest.mark.parametrize("gt,ht", PAIRS)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (5, 64), (37, 100), (2, 264), (700, 768), (6, 1000), (9, 1024), (3, 1032),
                                    (5, 5004), (700, 2048), (2, 8200), (3, 16384)])
def test_backward(rows, d, gt, ht):
    ws, *_ = run_backward(rows, d, gt, ht, qt=[E4M3, E5M2, None][rows % 3], seed=rows + d, pad=d % 2, stat=sc.STAT_AMAX,
                          residual=rows % 2 == 1, dg_dt=[F32, BF16, F16][d % 3])
    assert ws.check_status() == 0


def test_backward_options():
    word = lambda v: torch.full((1,), v, device="cuda")  # noqa: E731
    run_backward(3000, 776, BF16, BF16, qt=E5M2, seed=1, stat=sc.STAT_L2, stat_in=word(3.7))
    run_backward(300, 776, BF16, F32, qt=E4M3, seed=2, stat_in=word(2.0 ** -7), dg_dt=None, gamma_dt=None)
    run_backward(300, 2056, BF16, F32, seed=3, dg_dt=F32, gamma_dt=BF16, stat=sc.STAT_L2)
    ws, *_ = run_backward(20, 776, BF16, BF16, qt=E5M2, seed=4, stat_in=word(float("nan")))
    assert ws.check_status() == sc.DEV_NONFINITE_STAT
    run_backward(20, 776, BF16, BF16, qt=E5M2, seed=5, stat_in=word(0.0))


@pytest.mark.parametrize("alias,gt,ht", [("Gr", BF16, F32), ("Gr", BF16, BF16), ("G", F32, F32)])
def test_backward_in_place(alias, gt, ht):
    run_backward(700, 1000, gt, ht, qt=E5M2, seed=6, alias=alias)
    run_backward(70, 3000, gt, ht, qt=E5M2, seed=7, alias=alias)


def test_backward_is_the_same_every_time():
    first = run_backward(5000, 1024, BF16, BF16, qt=E5M2, seed=9, stat=sc.STAT_AMAX)
    for _ in range(3):
        again = run_backward(5000, 1024, BF16, BF16, qt=E5M2, seed=9, stat=sc.STAT_AMAX)
        assert torch.equal(first[3].data, again[3].data) and torch.equal(first[1].data, again[1].data)


def test_without_workspace_and_on_a_side_stream():
    rows, d = 64, 768
    H = sc.ScaledTensor.make(torch.randn(rows, d, device="cuda").to(BF16), 1.0)
    G = sc.ScaledTensor.make(torch.randn(rows, d, device="cuda").to(BF16), 1.0)
    rinv = (H.data.double().square().mean(1) + 1e-5).rsqrt().float()
    outs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        dX = sc.ScaledTensor.empty((rows, d), BF16)
        if stream is not None:
            side.wait_stream(torch.cuda.current_stream())
        sc.scalify_scaled_add_rmsnorm_bwd(G, None, H, None, rinv, dX, stream=stream)
        torch.cuda.synchronize()
        outs.append(dX.data)
    assert torch.equal(outs[0], outs[1])


def test_replayed_from_a_graph():
    rows, d = 513, 768
    X = sc.ScaledTensor.make(torch.randn(rows, d, device="cuda").to(BF16), 1.0)
    R = sc.ScaledTensor.make(torch.randn(rows, d, device="cuda").to(BF16), 1.0)
    H, Y, dX, dg = (sc.ScaledTensor.empty((rows, d), t) for t in (BF16, E4M3, BF16, F32))
    dg = sc.ScaledTensor.empty((d,), F32)
    rinv = torch.empty(rows, device="cuda")
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_RMSNORM_BWD, rows, d))

    def step():
        sc.scalify_scaled_add_rmsnorm(X, R, None, H, Y, rinv=rinv)
        sc.scalify_scaled_add_rmsnorm_bwd(X, R, H, None, rinv, dX, ws, stat_dx=sc.STAT_AMAX, dgamma=dg)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    X.data.copy_(torch.randn(rows, d, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (H.data, dX.data, dg.data, ws.statistic())]
    for t in (H, dX, dg):
        t.data.zero_()
    step()
    torch.cuda.synchronize()
    for a, b in zip(got, (H.data, dX.data, dg.data, ws.statistic())):
        assert torch.equal(a, b)


def test_bad_scale_word_is_reported():
    X = sc.ScaledTensor.make(torch.randn(4, 64, device="cuda").to(BF16), 3.0)
    Y = sc.ScaledTensor.empty((4, 64), BF16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    sc.scalify_scaled_add_rmsnorm(X, None, None, None, Y, status=status)
    assert int(status.item()) == sc.DEV_BAD_SCALE


def test_broadcast_rows():
    """Inputs whose rows are one row (stride 0), ragged and not."""
    for d in (100, 776, 1500, 5004):
        rows = 9
        H, _ = put(torch.randn(rows, d, generator=gen(d), device="cuda"), F32)
        one = torch.zeros((-(-d // 8)) * 8, device="cuda", dtype=BF16)
        one[:d] = torch.randn(d, generator=gen(d + 1), device="cuda").to(BF16)
        G = one[:d].as_strided((rows, d), (0, 1))
        rinv = ((H.double().square().mean(1) + 1e-5) ** -0.5).float()
        dX = sc.ScaledTensor(rows_of(rows, d, F32)[0], torch.empty(1, device="cuda"))
        sc.scalify_scaled_add_rmsnorm_bwd(scaled(G, 1.0), None, scaled(H, 1.0), None, rinv, dX)
        want = p64.add_rmsnorm_bwd(G, 1.0, None, 0.0, H, 1.0, None, 1.0, rinv)
        assert bool(p64.close(dX.data, want["dX"], U * want["mag"]).all())


def test_offsets_past_32_bits():
    """Rows 2^27 elements apart: every array of both directions reaches past 2^31 elements."""
    rows, d = 20, 264
    base = torch.empty(rows * (1 << 27), dtype=BF16, device="cuda")
    wide = base.view(rows, 1 << 27)
    x, r, g = (torch.randn(rows, d, generator=gen(k), device="cuda").to(BF16) for k in (1, 2, 3))
    results = []
    for far in (False, True):
        def place(k, src=None):
            v = wide[:, 512 * k:512 * k + d] if far else torch.empty(rows, d, dtype=BF16, device="cuda")
            if src is not None:
                v.copy_(src)
            return sc.ScaledTensor(v, torch.ones(1, device="cuda"))
        X, R, G, H, Y, dX = place(0, x), place(1, r), place(2, g), place(3), place(4), place(5)
        rinv = torch.empty(rows, device="cuda")
        sc.scalify_scaled_add_rmsnorm(X, R, None, H, Y, rinv=rinv)
        sc.scalify_scaled_add_rmsnorm_bwd(G, None, H, None, rinv, dX)
        results.append([t.data.clone() for t in (H, Y, dX)])
        assert torch.equal(X.data, x) and torch.equal(R.data, r) and torch.equal(G.data, g)
    assert all(torch.equal(a, b) for a, b in zip(*results))
