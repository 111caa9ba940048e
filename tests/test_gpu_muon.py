"""scalify_orthogonalize and scalify_scaled_muon_step against the plain 64-bit form (tests/plain64.py).

One step is held element by element to plain64.newton_schulz_bar, which carries the FP16 roundings of Z, A and D and the
fp32 accumulation through the products.  After five steps such a worst-case bound says nothing (every step multiplies it by
about thirty while the roundings themselves are independent), so five steps are held in the norm: with independent roundings
of h/sqrt(3) each, h = 2^-11, a step adds about 3.5 h/sqrt(3) = 1e-3 of the norm (A's rounding enters D with a factor of up
to 3), which later steps multiply by at most 1.64 (the largest s p'(s)/p(s) on the interval); five of them: sqrt(5) 1.64 1e-3
= 3.7e-3.  The BF16 output adds 2^-8/sqrt(3) = 2.3e-3 at most.  Bar: 6e-3."""
import math

import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64
from test_gpu_rmsnorm import gap_untouched, gen

pytestmark = pytest.mark.gpu
U = p64.U
BF16, F16, F32, E4M3, E5M2 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.float8_e5m2
FIVE = 6e-3


def strided(b, r, c, dtype, pad=0, fill=7.0):
    """[b, r, c] view (2-D for b == 0) with rows a multiple of 16 bytes apart and `pad` vectors between them."""
    step = 16 // torch.empty(0, dtype=dtype).element_size()
    ld = (-(-c // step) + pad) * step
    base = torch.full((max(b, 1), r, ld), fill, device="cuda").to(dtype)
    return (base if b else base[0])[..., :c], base


def matrices(b, r, c, dtype, seed, pad=0, scale=1.0):
    v, base = strided(b, r, c, dtype, pad)
    x = torch.randn(max(b, 1), r, c, generator=gen(seed), device="cuda") * scale
    v.copy_(p64.saturate(x if b else x[0], dtype))
    return v, base


def orth(b, r, c, xt, ot, steps, seed=0, pad=0, scale=1.0, eps=1e-7):
    X, _ = matrices(b, r, c, xt, seed, pad, scale)
    O, base = strided(b, r, c, ot, pad)
    Xs, Os = sc.ScaledTensor.make(X, 2.0 ** -10), sc.ScaledTensor(O, torch.zeros(1, device="cuda"))
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([Xs]))
    sc.scalify_orthogonalize(Xs, Os, ws, steps=steps, eps=eps)
    assert ws.check_status() == 0
    unit = 1.0 / p64.kf(max(r, c))
    assert Os.scale_value() == unit and gap_untouched(base.reshape(-1, base.shape[-1]), c)
    x3 = X if b else X[None]
    return (O if b else O[None]), x3, unit


@pytest.mark.parametrize("ot", [F16, BF16])
@pytest.mark.parametrize("b,r,c", [(0, 1, 1), (0, 1, 37), (2, 37, 1), (3, 5, 9), (1, 64, 64), (2, 128, 200), (0, 129, 130), (2, 200, 128),
                                   (0, 256, 256), (2, 300, 700), (0, 700, 300), (1, 513, 257), (0, 1030, 90), (3, 257, 1100)])
def test_one_step(b, r, c, ot):
    xt = [BF16, F32, F16, E5M2, E4M3][(r + c) % 5]
    O, X, unit = orth(b, r, c, xt, ot, 1, seed=r + c, pad=r % 2)
    want, bar = p64.newton_schulz(X, 1) / unit, p64.newton_schulz_bar(X, 1) / unit
    assert bool(p64.close(O, want, bar).all())


@pytest.mark.parametrize("b,r,c,xt", [(4, 256, 320, BF16), (0, 768, 768, F32), (2, 1000, 333, BF16), (0, 640, 2304, BF16),
                                      (130, 40, 30, F32), (1, 2048, 2048, BF16), (2, 64, 5000, F16), (0, 3, 2000, F32), (1, 3333, 3400, BF16),
                                      (24, 700, 760, BF16)])
def test_five_steps(b, r, c, xt):
    O, X, unit = orth(b, r, c, xt, BF16, 5, seed=r)
    want = p64.newton_schulz(X, 5) / unit
    err = (O.double() - want).flatten(1).norm(dim=1) / want.flatten(1).norm(dim=1)
    assert float(err.max()) < FIVE, float(err.max())


def test_result_does_not_depend_on_scale():
    """Data of any magnitude: the norm is taken before anything is rounded to FP16."""
    base = None
    for scale in (2.0 ** -20, 1.0, 2.0 ** 40):
        O, _, _ = orth(1, 200, 300, F32, BF16, 5, seed=3, scale=scale, eps=0.0)
        base = O if base is None else base
        assert torch.equal(O, base)


def test_zeros_and_nan_stay_in_their_matrix():
    X = torch.randn(3, 150, 304, device="cuda").to(BF16)
    X[1] = 0
    good = sc.ScaledTensor.make(X.clone(), 1.0)
    X[2, 3, 4] = float("nan")
    out = []
    for x, eps in ((good, 0.0), (sc.ScaledTensor.make(X, 1.0), 0.0)):
        O = sc.ScaledTensor.empty((3, 150, 304), BF16)
        ws = sc.Workspace(sc.scalify_muon_workspace_bytes([x]))
        sc.scalify_orthogonalize(x, O, ws, eps=eps)
        out.append((O.data, ws.check_status()))
    (a, sa), (b, sb) = out
    assert sa == 0 and sb == sc.DEV_NONFINITE_STAT
    assert bool((a[1] == 0).all()) and torch.equal(a[:2], b[:2]) and bool(b[2].isnan().all())


def test_norms_beyond_the_range_of_fp32_squares():
    """A norm below 2^-60 counts as zero and one above 2^63 as infinite, with eps = 0 as well; nothing in between is lost."""
    X = torch.randn(4, 150, 304, generator=gen(5), device="cuda")
    plain = X[1].clone()
    for k, e in enumerate((-75, -40, 40, 62)):
        X[k] = plain * 2.0 ** e
    x, O = sc.ScaledTensor.make(X, 1.0), sc.ScaledTensor.empty((4, 150, 304), BF16)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([x]))
    sc.scalify_orthogonalize(x, O, ws, eps=0.0)
    assert ws.check_status() == sc.DEV_NONFINITE_STAT
    o, o1 = O.data, sc.ScaledTensor.empty((150, 304), BF16)
    sc.scalify_orthogonalize(sc.ScaledTensor.make(plain, 1.0), o1, ws, eps=0.0)
    assert bool((o[0] == 0).all()) and torch.equal(o[1], o1.data) and torch.equal(o[2], o1.data) and bool(o[3].isnan().all())


def test_calls_on_several_streams_at_once():
    """Calls that run beside each other, each with its own workspace, give what they give one after the other."""
    sizes = [(6, 500, 900), (40, 120, 90), (1, 1030, 700)]
    Xs = [sc.ScaledTensor.make(matrices(*s, BF16, seed=i)[0], 1.0) for i, s in enumerate(sizes)]
    streams = [torch.cuda.Stream() for _ in Xs]
    work = [sc.Workspace(sc.scalify_muon_workspace_bytes([x])) for x in Xs]
    outs = [[sc.ScaledTensor(strided(*s, BF16)[0], torch.zeros(1, device="cuda")) for s in sizes] for _ in range(5)]
    # once alone, every buffer: the first result, and what the bounds-checking build learns of it while nothing runs
    for beside in (False, True):
        for k, O in enumerate(outs):
            for x, o, ws, st in zip(Xs, O, work, streams):
                if k or not beside:
                    sc.scalify_orthogonalize(x, o, ws, stream=st if beside else None)
                if not beside:
                    torch.cuda.synchronize()
                    if k:
                        o.data.fill_(float("nan"))
        torch.cuda.synchronize()
    for O in outs[1:]:
        assert all(torch.equal(a.data, b.data) for a, b in zip(outs[0], O))
    assert all(ws.check_status() == 0 for ws in work)


def test_offsets_past_32_bits():
    """Rows 2^27 elements apart: the last one lies past 2^31 elements, for the gradient as for the weights."""
    base = torch.empty(20 * (1 << 27), dtype=BF16, device="cuda")
    rows = base.view(20, 1 << 27)
    X = torch.randn(20, 48, generator=gen(3), device="cuda").to(BF16)
    rows[:, :48] = X
    far, near = sc.ScaledTensor.make(rows[:, :48], 1.0), sc.ScaledTensor.make(X, 1.0)
    O = sc.ScaledTensor.empty((20, 48), BF16)
    P = sc.ScaledTensor(rows[:, 64:112], torch.zeros(1, device="cuda"))
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([near]))
    sc.scalify_orthogonalize(near, O, ws)
    out = sc.ScaledTensor.empty((20, 48), BF16)
    sc.scalify_orthogonalize(far, out, ws)
    assert torch.equal(out.data, O.data)
    sc.scalify_orthogonalize(near, P, ws)
    assert torch.equal(P.data, O.data) and torch.equal(rows[:, :48], X)


def test_other_coefficients():
    X = sc.ScaledTensor.make(torch.randn(300, 400, device="cuda"), 1.0)
    O = sc.ScaledTensor.empty((300, 400), BF16)
    coef = (2.0, -1.5, 0.5)
    sc.scalify_orthogonalize(X, O, sc.Workspace(sc.scalify_muon_workspace_bytes([X])), steps=1, coef=coef)
    unit = 1.0 / p64.kf(400)
    want, bar = p64.newton_schulz(X.data[None], 1, coef)[0] / unit, p64.newton_schulz_bar(X.data[None], 1, coef)[0] / unit
    assert bool(p64.close(O.data, want, bar).all())


def make_list(shapes, gt, mt, wt, ct, seed):
    lists = [[], [], [], []]
    for i, (r, c) in enumerate(shapes):
        for k, (dt, s, amp) in enumerate(((gt, 2.0 ** -8, 1.0), (mt, 2.0 ** -9, 1.0), (wt, 2.0 ** -6, 1.0))):
            lists[k].append(sc.ScaledTensor.make(matrices(0, r, c, dt, seed + 10 * i + k, pad=i % 2, scale=amp)[0], s))
        lists[3].append(sc.ScaledTensor(strided(0, r, c, ct, i % 2)[0], torch.zeros(1, device="cuda")) if ct else None)
    return lists[0], lists[1], lists[2], (lists[3] if ct else None)


@pytest.mark.parametrize("gt,mt,wt,ct,nesterov,momentum,factor", [
    (E5M2, F16, F16, E4M3, True, 0.95, 1), (BF16, F32, F32, BF16, False, 0.9, 2), (F32, F16, BF16, None, True, 0.0, 0),
    (E4M3, F32, BF16, E5M2, True, 0.75, 1), (F16, F16, F32, F16, False, 0.95, 2)])
def test_step(gt, mt, wt, ct, nesterov, momentum, factor):
    shapes = [(100, 260), (33, 65), (260, 100), (300, 300), (100, 260), (1, 50), (400, 130)]
    g, m, w, wc = make_list(shapes, gt, mt, wt, ct, seed=11)
    lr, decay = 0.03, 0.1
    before = [(a.data.clone(), b.data.clone(), c.data.clone()) for a, b, c in zip(g, m, w)]
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes(w))
    sc.scalify_scaled_muon_step(sc.MuonTensors(g, m, w, wc), ws, lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=decay,
                                steps=1, factor=factor)
    assert ws.check_status() == 0
    mu, lrf = (float(torch.tensor(v, dtype=torch.float32)) for v in (momentum, lr))
    for i, (r, c) in enumerate(shapes):
        gd, md, wd = before[i]
        ref = p64.muon_step(gd, 2.0 ** -8, md, 2.0 ** -9, wd, 2.0 ** -6, lr=lrf, momentum=mu, nesterov=nesterov, decay=lrf * 0.1,
                            steps=1, factor=factor)
        assert m[i].scale_value() == ref["m_s"] and w[i].scale_value() == ref["w_s"]
        terms = mu * md.double().abs() * (2.0 ** -9 / ref["m_s"]) + gd.double().abs() * (2.0 ** -8 / ref["m_s"])
        assert bool(p64.close(m[i].data, ref["m"], 4 * U * terms).all())
        bar = p64.newton_schulz_bar(ref["u"][None], 1)[0] + 16 * U * ref["o"].abs()
        err = ref["step"] / ref["w_s"] * bar + 4 * U * (wd.double().abs() + ref["w"].abs())
        assert bool(p64.close(w[i].data, ref["w"], err).all())
        if ct:  # a cast of the stored weight
            assert wc[i].scale_value() == ref["w_s"]
            want = p64.saturate(w[i].data.float(), ct).to(ct)
            assert torch.equal(want.float(), wc[i].data.float())


def test_step_agrees_with_orthogonalize():
    """momentum 0, no decay: w' = w - lr O(g), with O from scalify_orthogonalize of the gradient."""
    g, m, w, _ = make_list([(256, 512)], BF16, F16, F32, None, seed=5)
    w0 = w[0].data.double() * 2.0 ** -6
    O = sc.ScaledTensor.empty((256, 512), F16)
    sc.scalify_orthogonalize(g[0], O, sc.Workspace(sc.scalify_muon_workspace_bytes(g)), eps=0.0)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes(w))
    sc.scalify_scaled_muon_step(sc.MuonTensors(g, m, w), ws, lr=0.5, momentum=0.0, nesterov=False, eps=0.0, factor=sc.MUON_UNIT)
    want = w0 - 0.5 * O.data.double() * O.scale_value()
    assert bool(((w[0].data.double() * w[0].scale_value() - want).abs() <= 4 * U * (w0.abs() + want.abs())).all())


def test_five_step_update_in_the_norm_and_many_tensors():
    """More matrices of one shape than one batch holds, two orientations, one workspace for two steps in a row."""
    shapes = [(48, 80) if i % 2 else (80, 48) for i in range(110)]
    g, m, w, _ = make_list(shapes, BF16, F16, F32, None, seed=2)
    before = [(b.data.clone(), c.data.clone()) for b, c in zip(m, w)]
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes(w))
    T = sc.MuonTensors(g, m, w)
    sc.scalify_scaled_muon_step(T, ws, lr=0.1, weight_decay=0.0)
    assert ws.check_status() == 0
    mu, lrf = (float(torch.tensor(v, dtype=torch.float32)) for v in (0.95, 0.1))
    for i in range(len(shapes)):
        ref = p64.muon_step(g[i].data, 2.0 ** -8, before[i][0], 2.0 ** -9, before[i][1], 2.0 ** -6, lr=lrf, momentum=mu, nesterov=True,
                            decay=0.0, steps=5, factor=1)
        moved = (w[i].data.double() * w[i].scale_value() - before[i][1].double() * 2.0 ** -6)
        want = -ref["step"] * ref["o"]
        assert float((moved - want).norm() / want.norm()) < FIVE
    sc.scalify_scaled_muon_step(T, ws, lr=0.1)
    assert ws.check_status() == 0


def test_the_same_bits_every_time_and_in_a_graph():
    shapes = [(300, 700), (700, 300), (128, 128)]
    first = None
    for mode in ("eager", "eager", "graph"):
        g, m, w, wc = make_list(shapes, E5M2, F16, F16, E4M3, seed=7)
        ws = sc.Workspace(sc.scalify_muon_workspace_bytes(w))
        T = sc.MuonTensors(g, m, w, wc)
        if mode == "graph":
            keep = [(a.data.clone(), a.scale.clone()) for a in m + w]
            sc.scalify_scaled_muon_step(T, ws, lr=0.02)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                sc.scalify_scaled_muon_step(T, ws, lr=0.02)
            for a, (d, s) in zip(m + w, keep):
                a.data.copy_(d)
                a.scale.copy_(s)
            graph.replay()
        else:
            sc.scalify_scaled_muon_step(T, ws, lr=0.02)
        torch.cuda.synchronize()
        assert ws.check_status() == 0
        got = [t.data.float().clone() for t in m + w + wc] + [t.scale.clone() for t in m + w + wc]
        first = got if first is None else first
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_bad_scale_word_is_reported():
    g, m, w, _ = make_list([(40, 50)], BF16, F16, F16, None, seed=1)
    m[0].scale.fill_(3.0)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes(w))
    sc.scalify_scaled_muon_step(sc.MuonTensors(g, m, w), ws, lr=0.02)
    assert ws.check_status() == sc.DEV_BAD_SCALE


def test_orthogonal_rows():
    """Five steps bring the singular values of a full-rank matrix near 1."""
    O, _, unit = orth(0, 200, 500, F32, BF16, 5, seed=9)
    s = torch.linalg.svdvals(O[0].double() * unit)
    assert 0.6 < float(s.min()) and float(s.max()) < 1.3 and math.isfinite(float(s.sum()))
