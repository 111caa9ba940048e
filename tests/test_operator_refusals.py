"""Host-side refusals of the norm, embedding and optimiser entry points, and the plain 64-bit gradients against
differences (no GPU needed: a call that fails validation launches nothing)."""
import ctypes

import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64

R = ctypes.byref
NULL, DTYPE, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED, ALIAS, VALUE = -1, -2, -3, -4, -5, -6, -8, -9
MB = 1 << 20


def arr(mb, dtype, shape, stride=None, scale=None, offset=0):
    """Descriptor of a made-up array that begins `mb` megabytes into the address space."""
    a = sc.scalify_array()
    a.data, a.dtype, a.ndim = mb * MB + offset, dtype, len(shape)
    if stride is None:
        stride, n = [], 1
        for s in reversed(shape):
            stride.insert(0, n)
            n *= s
    for i, (s, t) in enumerate(zip(shape, stride)):
        a.shape[i], a.stride[i] = s, t
    a.scale = scale
    return a


def mx(mb, dtype, rows, K, transposed=0):
    return sc.scalify_mx_array(mb * MB, dtype, rows, K, mb * MB + (MB >> 1), None, transposed)


def norm_call(X=None, Rr=None, gamma=None, eps=1e-5, H=None, Y=None, Ymx=None):
    p = lambda a: None if a is None else R(a)  # noqa: E731
    return sc.lib().scalify_scaled_add_rmsnorm(p(X), p(Rr), p(gamma), eps, p(H), p(Y),
                                               None if Ymx is None else ctypes.addressof(Ymx), None, None, None)


def test_norm_refusals():
    B, F, Q = sc.BF16, sc.F32, sc.E4M3
    x, r, h, y = arr(1, B, (4, 128)), arr(2, B, (4, 128)), arr(3, B, (4, 128)), arr(4, Q, (4, 128))
    assert norm_call(None, r, None, 1e-5, h, y) == NULL
    assert norm_call(x, r, None, 1e-5, None, y) == NULL          # a residual without the sum
    assert norm_call(x, None, None, 1e-5, h, y) == NULL          # a sum without a residual
    assert norm_call(x, r, None, 1e-5, h, None) == NULL          # no output
    assert norm_call(x, r, None, 1e-5, h, y, mx(5, Q, 4, 128)) == UNSUPPORTED
    assert norm_call(x, r, None, 1e-5, h, None, mx(5, Q, 16, 128, 1)) == UNSUPPORTED
    assert norm_call(x, r, None, 1e-5, h, None, mx(5, Q, 5, 128)) == SHAPE
    assert norm_call(arr(1, B, (4, 64)), None, None, 1e-5, None, None, mx(5, Q, 4, 64)) == SHAPE
    assert norm_call(arr(1, Q, (4, 128)), r, None, 1e-5, h, y) == DTYPE
    assert norm_call(x, arr(2, sc.F16, (4, 128)), None, 1e-5, arr(3, sc.F16, (4, 128)), y) == DTYPE
    assert norm_call(x, arr(2, F, (4, 128)), None, 1e-5, h, y) == DTYPE
    assert norm_call(arr(1, F, (4, 128)), r, None, 1e-5, h, y) == DTYPE
    assert norm_call(x, arr(2, B, (4, 120)), None, 1e-5, h, y) == SHAPE
    assert norm_call(x, r, None, 1e-5, h, arr(4, Q, (5, 128))) == SHAPE
    assert norm_call(arr(1, B, (1, 16392)), None, None, 1e-5, None, arr(4, B, (1, 16392))) == SHAPE
    assert norm_call(x, r, arr(5, F, (127,)), 1e-5, h, y) == SHAPE
    assert norm_call(x, r, arr(5, Q, (128,)), 1e-5, h, y) == DTYPE
    assert norm_call(x, r, None, -1.0, h, y) == VALUE
    assert norm_call(x, r, None, float("nan"), h, y) == VALUE
    assert norm_call(x, r, None, float("inf"), h, y) == VALUE
    assert norm_call(x, r, None, 1e-5, h, arr(4, Q, (4, 128), offset=8)) == ALIGN
    assert norm_call(x, r, None, 1e-5, h, arr(4, Q, (4, 128), (136, 1))) == ALIGN
    assert norm_call(x, r, None, 1e-5, arr(1, B, (4, 128), offset=16), y) == ALIAS   # overlaps X, not the same rows
    assert norm_call(x, r, None, 1e-5, arr(2, B, (4, 128), (136, 1)), y) == ALIAS    # R's buffer, other stride
    assert norm_call(x, r, None, 1e-5, h, arr(1, B, (4, 128))) == ALIAS              # Y over X
    assert norm_call(x, r, None, 1e-5, h, arr(3, B, (4, 128))) == ALIAS              # Y over H
    assert norm_call(arr(1, B, (4, 128), scale=64), r, None, 1e-5, arr(3, B, (4, 128), scale=64), y) == ALIAS
    assert norm_call(x, r, None, 1e-5, arr(3, B, (4, 128), scale=64), arr(4, Q, (4, 128), scale=64)) == ALIAS


def norm_bwd(G=None, Gr=None, H=None, gamma=None, rinv=8 * MB, dX=None, dXq=None, stat_in=None, stat=0, dg=None, ws=None, nb=0):
    p = lambda a: None if a is None else R(a)  # noqa: E731
    return sc.lib().scalify_scaled_add_rmsnorm_bwd(p(G), p(Gr), p(H), p(gamma), rinv, p(dX), p(dXq), stat_in, stat, p(dg), ws,
                                                   nb, None)


def test_norm_backward_refusals():
    B, F, Q = sc.BF16, sc.F32, sc.E5M2
    g, h, dx = arr(1, B, (4, 128)), arr(2, B, (4, 128)), arr(3, B, (4, 128))
    ok = dict(G=g, H=h, dX=dx)
    assert norm_bwd(**{**ok, "G": None}) == NULL
    assert norm_bwd(**ok, rinv=None) == NULL
    assert norm_bwd(**ok, stat_in=64) == NULL                          # a rescale without the copy it applies to
    assert norm_bwd(**{**ok, "dX": arr(3, F, (4, 128))}) == DTYPE
    assert norm_bwd(**{**ok, "H": arr(2, sc.F16, (4, 128)), "dX": arr(3, sc.F16, (4, 128))}) == DTYPE
    assert norm_bwd(**ok, Gr=arr(4, F, (4, 128))) == DTYPE
    assert norm_bwd(**ok, dXq=arr(4, B, (4, 128))) == DTYPE
    assert norm_bwd(**ok, dXq=arr(4, Q, (4, 112))) == SHAPE
    assert norm_bwd(**{**ok, "G": arr(1, B, (3, 128))}) == SHAPE
    assert norm_bwd(G=arr(1, B, (0, 128)), H=arr(2, B, (0, 128)), dX=arr(3, B, (0, 128))) == SHAPE
    assert norm_bwd(**ok, stat=3) == VALUE
    assert norm_bwd(**ok, dg=arr(4, F, (128,))) == WORKSPACE
    assert norm_bwd(**ok, stat=1) == WORKSPACE
    assert norm_bwd(**ok, stat=1, ws=16 * MB, nb=300) == WORKSPACE
    assert norm_bwd(**ok, stat=1, ws=16 * MB + 64, nb=64 * MB) == WORKSPACE
    assert norm_bwd(**{**ok, "dX": arr(2, B, (4, 128))}) == ALIAS        # dX over H
    assert norm_bwd(**ok, dXq=arr(1, Q, (4, 128))) == ALIAS              # the copy over G
    assert norm_bwd(**ok, Gr=arr(3, B, (4, 128), offset=16)) == ALIAS
    assert norm_bwd(**ok, dXq=arr(4, Q, (4, 128)), stat_in=16 * MB + 16, stat=1, ws=16 * MB, nb=64 * MB) == ALIAS
    assert norm_bwd(**{**ok, "dX": arr(3, B, (4, 128), scale=64), "H": arr(2, B, (4, 128), scale=64)}) == ALIAS


def test_arrays_of_different_devices_are_refused_by_the_binding():
    x = sc.ScaledTensor(torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        sc.scalify_scaled_add_rmsnorm(x, None, None, None, sc.ScaledTensor(torch.zeros(4, 64, dtype=torch.bfloat16)))
    with pytest.raises(ValueError):
        sc.scalify_scaled_add_rmsnorm(x, None, None, None, sc.ScaledTensor(torch.zeros(4, 64, dtype=torch.bfloat16, device="meta")))
    with pytest.raises(ValueError):
        sc.scalify_scaled_add_rmsnorm(x, None, None, None, x, rinv=torch.zeros(3))


def test_plain_norm_gradient_against_differences():
    torch.manual_seed(0)
    rows, d, eps = 3, 10, 1e-3
    x, r, gam, up = (torch.randn(*s, dtype=torch.float64) for s in ((rows, d), (rows, d), (d,), (rows, d)))
    res = torch.randn(rows, d, dtype=torch.float64)
    xs, rs = 0.5, 2.0

    def loss(x, gam):
        total, hs, norm = p64.add_rmsnorm(x, xs, r, rs, gam, eps)
        return float((norm(total)[0] * up).sum() + (total * hs * res).sum())
    total, hs, norm = p64.add_rmsnorm(x, xs, r, rs, gam, eps)
    _, rinv = norm(total)
    got = p64.add_rmsnorm_bwd(up, 1.0, res, 1.0, total, hs, gam, 1.0, rinv)
    dx, step = got["dX"] * got["dX_s"], 1e-6
    for i, j in ((0, 0), (1, 4), (2, 9)):
        e = torch.zeros_like(x)
        e[i, j] = step
        # the derivative with respect to the VALUE of x: its data move by step / xs
        diff = (loss(x + e / xs, gam) - loss(x - e / xs, gam)) / (2 * step)
        assert abs(diff - float(dx[i, j])) < 1e-6 * max(1.0, abs(diff))
    dg = got["dgamma"] * got["dgamma_s"]
    for j in (0, 5):
        e = torch.zeros_like(gam)
        e[j] = step
        diff = (loss(x, gam + e) - loss(x, gam - e)) / (2 * step)
        assert abs(diff - float(dg[j])) < 1e-6 * max(1.0, abs(diff))


def test_embedding_refusals():
    B, F, Q = sc.BF16, sc.F32, sc.E4M3
    L = sc.lib()
    w, y, ids = arr(1, B, (50, 64)), arr(2, B, (7, 64)), 8 * MB

    def look(ids=ids, n=7, w=w, c=1.0, y=y):
        return L.scalify_scaled_embedding_lookup(ids, n, -1, None if w is None else R(w), c, None if y is None else R(y), None, None)
    assert look(ids=None) == NULL and look(w=None) == NULL and look(y=None) == NULL
    assert look(n=6) == SHAPE and look(n=-1) == SHAPE and look(y=arr(2, B, (7, 56))) == SHAPE
    assert look(w=arr(1, B, (64,))) == SHAPE and look(w=arr(1, B, (0, 64))) == SHAPE
    for c in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        assert look(c=c) == VALUE
    assert look(y=arr(1, B, (7, 64), offset=64)) == ALIAS
    assert look(w=arr(1, B, (50, 64), scale=64), y=arr(2, B, (7, 64), scale=64)) == ALIAS
    assert look(w=arr(1, B, (50, 60))) == ALIGN

    g, dw = arr(2, B, (7, 64)), arr(1, F, (50, 64))
    big = 64 * MB

    def grad(ids=ids, n=7, g=g, c=1.0, a=None, dw=dw, ws=16 * MB, nb=big):
        p = lambda t: None if t is None else R(t)  # noqa: E731
        return L.scalify_scaled_embedding_grad(ids, n, -1, p(g), c, p(a), p(dw), ws, nb, None)
    assert grad(ids=None) == NULL and grad(g=None) == NULL and grad(dw=None) == NULL
    assert grad(dw=arr(1, Q, (50, 64))) == DTYPE
    assert grad(g=arr(2, B, (6, 64))) == SHAPE and grad(g=arr(2, B, (7, 56))) == SHAPE and grad(n=-1) == SHAPE
    assert grad(a=arr(3, B, (50, 64))) == DTYPE and grad(a=arr(3, F, (49, 64))) == SHAPE
    assert grad(a=arr(1, F, (50, 64), offset=256)) == ALIAS and grad(g=arr(1, B, (7, 64), offset=256)) == ALIAS
    assert grad(dw=arr(1, F, (50, 64), scale=64), g=arr(2, B, (7, 64), scale=64)) == ALIAS
    assert grad(c=0.0) == VALUE
    assert grad(ws=None) == WORKSPACE and grad(nb=4095) == WORKSPACE and grad(ws=16 * MB + 16) == WORKSPACE
    assert sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, 1 << 20, 64) > (1 << 24)
    assert grad(n=1, g=arr(1000, B, (1, 1 << 24)), dw=arr(2000, F, (1, 1 << 24)), ws=4000 * MB, nb=1 << 40) == SHAPE   # too many columns
    assert grad(dw=arr(1, F, ((1 << 24) + 1, 64)), g=arr(1 << 20, B, (7, 64))) == SHAPE                            # too many tokens


def test_token_ids_are_checked_by_the_binding():
    w, y = sc.ScaledTensor(torch.zeros(4, 64)), sc.ScaledTensor(torch.zeros(2, 64))
    for ids in (torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError):
            sc.scalify_scaled_embedding_lookup(ids, w, y)


def test_plain_embedding_gradient_against_differences():
    torch.manual_seed(1)
    ids = torch.tensor([2, 0, 2, -1, 4, 2])
    w, up = torch.randn(5, 3, dtype=torch.float64), torch.randn(6, 3, dtype=torch.float64)
    c = 3.3
    got, scale, _, count = p64.embedding_grad(ids, up, 1.0, 5, c, -1)
    f = lambda w: float((p64.embedding_lookup(ids, w, c, -1, 5) * p64.p2(c) * up).sum())  # noqa: E731
    for i in range(5):
        for j in range(3):
            e = torch.zeros_like(w)
            e[i, j] = 1e-6
            assert abs((f(w + e) - f(w - e)) / 2e-6 - float(got[i, j]) * scale) < 1e-6
    assert count == 3


def test_orthogonalize_refusals():
    B, F = sc.BF16, sc.F32
    L = sc.lib()
    coef = (ctypes.c_float * 3)(2.0, -1.5, 0.5)
    x, o, big = arr(1, F, (64, 96)), arr(2, B, (64, 96)), 256 * MB

    def call(x=x, steps=5, coef=None, eps=1e-7, o=o, ws=16 * MB, nb=big):
        p = lambda a: None if a is None else R(a)  # noqa: E731
        return L.scalify_orthogonalize(p(x), steps, coef, eps, p(o), ws, nb, None)
    assert call(x=None) == NULL and call(o=None) == NULL
    assert call(o=arr(2, F, (64, 96))) == DTYPE and call(o=arr(2, sc.E4M3, (64, 96))) == DTYPE
    assert call(o=arr(2, B, (96, 64))) == SHAPE and call(x=arr(1, F, (96,)), o=arr(2, B, (96,))) == SHAPE
    assert call(x=arr(1, F, (32776, 8)), o=arr(2, B, (32776, 8))) == SHAPE
    assert call(x=arr(1, F, (0, 8)), o=arr(2, B, (0, 8))) == SHAPE
    assert call(steps=0) == VALUE and call(steps=17) == VALUE and call(eps=-1.0) == VALUE and call(eps=float("nan")) == VALUE
    for i in range(3):
        bad = (ctypes.c_float * 3)(*coef)
        bad[i] = float("inf")
        assert call(coef=bad) == VALUE
    assert call(o=arr(1, B, (64, 96), offset=256)) == ALIAS
    assert call(x=arr(1, F, (64, 96), scale=64), o=arr(2, B, (64, 96), scale=64)) == ALIAS
    assert call(ws=None) == WORKSPACE and call(nb=4096) == WORKSPACE and call(ws=16 * MB + 16) == WORKSPACE
    need = L.scalify_muon_workspace_bytes(1, R(x))
    assert need > 2 * 2 * 64 * 96 and call(nb=need - 1) == WORKSPACE
    assert L.scalify_muon_workspace_bytes(1, R(arr(1, F, (96,)))) == 0
    assert L.scalify_muon_workspace_bytes(-1, None) == 0 and L.scalify_muon_workspace_bytes(0, None) >= 4096


def test_muon_refusals():
    L = sc.lib()
    H, Q = sc.F16, sc.E4M3
    words = iter(range(64, 100000, 4))

    def lists(n=2, g=sc.E5M2, m=H, w=H, c=Q, shape=(64, 96), **over):
        out = []
        for k, dt in enumerate((g, m, w, c)):
            a = (sc.scalify_array * n)()
            for i in range(n):
                a[i] = arr(1 + 8 * k + i, dt, shape, scale=next(words))
            out.append(a)
        for key, v in over.items():
            out["gmwc".index(key[0])][int(key[1])] = v
        return out

    def call(ls, n=2, lr=0.02, mu=0.95, wd=0.0, steps=5, eps=1e-7, factor=1, ws=64 * MB, nb=256 * MB):
        return L.scalify_scaled_muon_step(n, *ls, lr, mu, 1, wd, steps, None, eps, factor, ws, nb, None)
    assert call([None] * 4, n=0) == 0 and call([None] * 4) == NULL and call(lists(), n=-1) == SHAPE
    for lr, mu, wd in ((-1.0, 0.9, 0.0), (0.1, 1.0, 0.0), (0.1, -0.1, 0.0), (0.1, 0.9, -1.0), (0.5, 0.9, 2.0), (float("nan"), 0.9, 0.0)):
        assert call(lists(), lr=lr, mu=mu, wd=wd) == VALUE
    assert call(lists(), factor=3) == VALUE and call(lists(), steps=0) == VALUE and call(lists(), eps=-1.0) == VALUE
    assert call(lists(m=sc.BF16)) == DTYPE and call(lists(w=Q)) == DTYPE and call(lists(c=sc.F32)) == DTYPE
    assert call(lists(g1=arr(2, sc.BF16, (64, 96), scale=next(words)))) == DTYPE          # one dtype per list
    assert call(lists(g1=arr(2, sc.E5M2, (96, 64), scale=next(words)))) == SHAPE
    assert call(lists(w0=arr(17, H, (64 * 96,), scale=next(words)))) == SHAPE
    assert call(lists(m0=arr(9, H, (64, 96)))) == NULL and call(lists(c1=arr(26, Q, (64, 96)))) == NULL  # no scale word
    same = next(words)
    assert call(lists(m0=arr(9, H, (64, 96), scale=same), w1=arr(18, H, (64, 96), scale=same))) == ALIAS
    assert call(lists(g0=arr(1, sc.E5M2, (64, 96), scale=same), w1=arr(18, H, (64, 96), scale=same))) == ALIAS
    assert call(lists(m0=arr(17, H, (64, 96), scale=next(words)))) == ALIAS               # m over w
    assert call(lists(c0=arr(17, Q, (64, 96), scale=next(words)))) == ALIAS               # the copy over w
    assert call(lists(), ws=None) == WORKSPACE and call(lists(), nb=4096) == WORKSPACE


def test_plain_newton_schulz_against_the_singular_values():
    torch.manual_seed(2)
    for shape in ((5, 8), (8, 5)):
        u = torch.randn(1, *shape, dtype=torch.float64)
        a, s, b = torch.linalg.svd(u[0], full_matrices=False)
        s = s / s.square().sum().sqrt()
        for _ in range(5):
            s = p64.COEF[0] * s + p64.COEF[1] * s ** 3 + p64.COEF[2] * s ** 5
        assert float((p64.newton_schulz(u, eps=0.0)[0] - a @ torch.diag(s) @ b).abs().max()) < 1e-10


def test_muon_binding_checks():
    t = sc.ScaledTensor(torch.zeros(4, 8))
    with pytest.raises(ValueError):
        sc.MuonTensors([t], [t, t], [t])
    with pytest.raises(ValueError):
        sc.scalify_muon_workspace_bytes([sc.ScaledTensor(torch.zeros(8))])


def test_overlapping_output_rows_are_refused():
    B, F = sc.BF16, sc.F32
    L = sc.lib()
    x, over = arr(1, B, (4, 128)), lambda mb, dt=B: arr(mb, dt, (4, 128), (64, 1))  # noqa: E731
    assert norm_call(x, None, None, 1e-5, None, over(4)) == SHAPE
    assert norm_call(x, arr(2, B, (4, 128)), None, 1e-5, over(3), arr(4, B, (4, 128))) == SHAPE
    assert norm_bwd(G=x, H=arr(2, B, (4, 128)), dX=over(3)) == SHAPE
    assert norm_bwd(G=x, H=arr(2, B, (4, 128)), dX=arr(3, B, (4, 128)), dXq=over(4, sc.E5M2)) == SHAPE
    assert L.scalify_scaled_embedding_lookup(8 * MB, 4, -1, R(arr(1, B, (50, 128))), 1.0, R(over(2)), None, None) == SHAPE
    assert L.scalify_scaled_embedding_grad(8 * MB, 4, -1, R(arr(2, B, (4, 128))), 1.0, None, R(over(1, F)), 16 * MB, 64 * MB, None) == SHAPE
    assert L.scalify_orthogonalize(R(arr(1, F, (4, 128))), 5, None, 0.0, R(over(2)), 16 * MB, 64 * MB, None) == SHAPE
    assert L.scalify_orthogonalize(R(arr(1, F, (2, 4, 128))), 5, None, 0.0, R(arr(2, B, (2, 4, 128), (256, 128, 1))), 16 * MB,
                                   64 * MB, None) == SHAPE


def test_overlapping_column_slices_are_refused():
    """Slices of one buffer may lie side by side (the GPU tests do that), not across one another or a row's end."""
    B = sc.BF16
    L = sc.lib()
    cols = lambda mb, first, n=128, ld=512, dt=B, rows=4: arr(mb, dt, (rows, n), (ld, 1), offset=2 * first)  # noqa: E731
    x = cols(1, 128)
    for first in (8, 128, 136, 248):
        assert norm_call(x, None, None, 1e-5, None, cols(1, first)) == ALIAS, first
    assert norm_call(x, None, None, 1e-5, None, cols(1, 512 + 120)) == ALIAS     # begins a row later
    assert norm_call(x, None, None, 1e-5, None, cols(1, 384, n=128, ld=504)) == ALIAS  # rows that drift
    assert norm_call(cols(1, 0), None, None, 1e-5, None, cols(1, 400, n=128)) == ALIAS  # runs into the next row
    assert L.scalify_scaled_embedding_lookup(8 * MB, 4, -1, R(cols(1, 0, rows=50)), 1.0, R(cols(1, 120)), None, None) == ALIAS
    assert L.scalify_orthogonalize(R(cols(1, 0)), 5, None, 0.0, R(cols(1, 64)), 16 * MB, 64 * MB, None) == ALIAS


def test_muon_factors():
    """Every documented factor passes the checks of arguments (the call then lacks its workspace); no other value does."""
    L = sc.lib()
    ls = [(sc.scalify_array * 1)(arr(1 + k, dt, (64, 96), scale=64 + 4 * k)) for k, dt in enumerate((sc.E5M2, sc.F16, sc.F16, sc.E4M3))]
    call = lambda f: L.scalify_scaled_muon_step(1, *ls, 0.02, 0.95, 1, 0.0, 5, None, 1e-7, f, None, 0, None)  # noqa: E731
    assert all(call(f) == WORKSPACE for f in (sc.MUON_UNIT, sc.MUON_SPECTRAL, sc.MUON_RMS, sc.MUON_SPECTRAL_IN_OUT))
    assert all(call(f) == VALUE for f in (-1, 3, 5, 8))


def test_newton_schulz_coefficients_that_leave_fp16_are_refused():
    """The iterate's products are held in FP16 at a scale of 2^12.  The rule of the header, here by brute force over x, at both
    sides of its border; a call that passes it lacks its workspace."""
    L = sc.lib()
    x, o = arr(1, sc.F32, (64, 96)), arr(2, sc.BF16, (64, 96))
    words = [(sc.scalify_array * 1)(arr(1 + k, dt, (64, 96), scale=64 + 4 * k)) for k, dt in enumerate((sc.E5M2, sc.F16, sc.F16))]

    def call(coef, steps):
        c = (ctypes.c_float * 3)(*coef)
        a = L.scalify_orthogonalize(R(x), steps, c, 1e-7, R(o), None, 0, None)
        b = L.scalify_scaled_muon_step(1, *words, None, 0.02, 0.95, 1, 0.0, steps, c, 1e-7, 1, None, 0, None)
        assert a == b and a in (VALUE, WORKSPACE)
        return a == WORKSPACE

    assert call((3.4445, -4.7750, 2.0315), 5) and call((3.4445, -4.7750, 2.0315), 16) and call((2.0, -1.5, 0.5), 16)
    assert call((8.25, -23.5, 17.25), 1) and call((0.0, 0.0, 0.0), 3) and call((15.4, 0.0, -15.4), 1)
    assert not call((20.0, -30.0, 12.0), 1)       # the diagonal of D
    assert not call((-16.0, 0.0, 0.0), 1) and not call((0.0, 0.0, 16.0), 1)
    assert call((15.4, -30.0, 15.0), 1) and not call((15.4, -30.0, 15.0), 2)   # the iterate grows to 4.5
    assert call((1.5, 0.0, 0.0), 3) and not call((1.5, 0.0, 0.0), 16)
    g = torch.Generator().manual_seed(0)
    seen = [0, 0]
    for i in range(400):
        steps = 1 + i % 6
        coef = [float(torch.tensor(v, dtype=torch.float32)) for v in (torch.randn(3, generator=g, dtype=torch.float64) * torch.tensor([5.0, 8.0, 5.0])).tolist()]
        m, ok, near = 33 / 32, True, False
        for _ in range(steps):
            xs = torch.linspace(0, m, 20001, dtype=torch.float64)
            d = coef[0] + coef[1] * xs ** 2 + coef[2] * xs ** 4
            ok = ok and m <= 3.875 and float(d.abs().max()) <= 15.5
            near = near or abs(m - 3.875) < 1e-3 or abs(float(d.abs().max()) - 15.5) < 1e-3
            m = min(33 / 32 * float((xs * d).abs().max()), 1e6)
        if not near:
            assert call(coef, steps) == ok, (coef, steps)
            seen[ok] += 1
    assert min(seen) > 50, seen


def test_embedding_workspace_of_the_largest_batch_serves_smaller_ones():
    for d in (8, 768, 2048):
        sizes = [sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, n, d) for n in sorted({*range(0, 300000, 511), 16383, 16384, 16385,
                                                                                         18943, 18944, 37887, 37888, 151551, 151552})]
        assert sizes == sorted(sizes), d


def test_outputs_over_the_plain_vectors_of_a_call_are_refused():
    """rinv, the exponent bytes and the token ids are memory like any other: no output may lie over them, nor they over an input."""
    B, F, Q = sc.BF16, sc.F32, sc.E4M3
    L = sc.lib()
    x, r, h, y, gam = arr(1, B, (4, 128)), arr(2, B, (4, 128)), arr(3, B, (4, 128)), arr(4, Q, (4, 128)), arr(5, F, (128,))

    def fwd(rinv, Ymx=None):
        return L.scalify_scaled_add_rmsnorm(R(x), R(r), R(gam), 1e-5, R(h), None if Ymx else R(y), ctypes.addressof(Ymx) if Ymx else None,
                                            rinv, None, None)
    for mb in (1, 2, 3, 4, 5):
        assert fwd(mb * MB) == ALIAS and fwd(mb * MB - 12) == ALIAS and fwd(mb * MB + 500) == ALIAS, mb
    m = lambda data, sf: sc.scalify_mx_array(data, Q, 4, 128, sf, None, 0)  # noqa: E731
    assert fwd(4 * MB, m(4 * MB, 6 * MB)) == ALIAS and fwd(6 * MB + 1000, m(4 * MB, 6 * MB)) == ALIAS   # over data, exponents
    for mb in (1, 2, 3, 4, 5):
        assert fwd(8 * MB, m(4 * MB, mb * MB)) == ALIAS, mb
    g, dx = arr(1, B, (4, 128)), arr(3, B, (4, 128))
    for over in (dict(rinv=3 * MB), dict(rinv=4 * MB + 16, dXq=arr(4, sc.E5M2, (4, 128))), dict(rinv=6 * MB, dg=arr(6, F, (128,)))):
        assert norm_bwd(G=g, H=r, dX=dx, **over) == ALIAS
    # in the gap between the rows of dX it touches nothing: the call gets as far as its missing workspace
    wide = arr(3, B, (4, 128), (512, 1))
    assert norm_bwd(G=g, H=r, dX=wide, rinv=3 * MB + 256, stat=1) == WORKSPACE
    assert norm_bwd(G=g, H=r, dX=wide, rinv=3 * MB + 1024 - 16, stat=1) == WORKSPACE
    for off in (-4, 0, 252, 1024 - 12, 1024, 3 * 1024 + 252):
        assert norm_bwd(G=g, H=r, dX=wide, rinv=3 * MB + off, stat=1) == ALIAS, off
    w = arr(1, B, (50, 64))
    assert L.scalify_scaled_embedding_lookup(2 * MB, 7, -1, R(w), 1.0, R(arr(2, B, (7, 64))), None, None) == ALIAS
    assert L.scalify_scaled_embedding_grad(1 * MB + 64, 7, -1, R(arr(2, B, (7, 64))), 1.0, None, R(arr(1, F, (50, 64))), 16 * MB, 64 * MB,
                                           None) == ALIAS


def test_muon_lists_whose_matrices_overlap_are_refused():
    """Outputs of one entry over anything of another entry (the same matrix twice among them); gradients may be shared, and
    column slices of one buffer lie beside each other."""
    L = sc.lib()
    H, Q, G = sc.F16, sc.E4M3, sc.E5M2

    def call(make, n=3):
        ls, word = [], iter(range(64, 4096, 4))
        for k, dt in enumerate((G, H, H, Q)):
            a = (sc.scalify_array * n)()
            for i in range(n):
                a[i] = make("gmwc"[k], i, dt, next(word)) or arr(1 + 8 * k + i, dt, (64, 96), scale=next(word))
            ls.append(a)
        return L.scalify_scaled_muon_step(n, *ls, 0.02, 0.95, 1, 0.0, 5, None, 1e-7, 1, None, 0, None)
    at = lambda which, index, mb, off=0: (lambda k, i, dt, word: arr(mb, dt, (64, 96), scale=word, offset=off) if (k, i) == (which, index) else None)  # noqa: E731,E501
    assert call(lambda *a: None) == WORKSPACE
    for which, base in (("m", 9), ("w", 17), ("c", 25)):
        for other in (1, 9, 17, 25):       # entry 2's output over entry 0's gradient, momentum, weight, copy
            assert call(at(which, 2, other)) == ALIAS, (which, other)
        assert call(at(which, 2, base, 4096)) == ALIAS and call(at(which, 0, base + 2, -16)) == ALIAS
    assert call(at("g", 2, 9)) == ALIAS                 # a gradient over another entry's momentum
    assert call(at("g", 2, 1)) == WORKSPACE             # one gradient for two entries
    cols = lambda first: (lambda k, i, dt, word: arr(17, dt, (64, 96), (512, 1), scale=word, offset=2 * first(i)) if k == "w" else None)  # noqa: E731,E501
    assert call(cols(lambda i: 96 * i)) == WORKSPACE    # three slices side by side
    assert call(cols(lambda i: 88 * i)) == ALIAS


def test_slices_whose_row_strides_are_multiples_of_each_other():
    """Every row of one half of a buffer's columns beside every other row of the other half: no overlap; across it: one."""
    B = sc.BF16
    g, h = arr(1, B, (8, 128)), arr(2, B, (8, 128))
    dX = arr(3, B, (8, 128), (256, 1))

    def call(offset, width, ld):
        q = arr(3, sc.E5M2, (8, width), (ld, 1), offset=offset)   # (bytes; dX has rows of 256 bytes every 512)
        return norm_bwd(G=arr(1, B, (8, width)), H=arr(2, B, (8, width)), dX=arr(3, B, (8, width), (256, 1)), dXq=q, stat=1)
    assert norm_bwd(G=g, H=h, dX=dX, stat=1) == WORKSPACE
    assert call(256, 128, 1024) == WORKSPACE and call(256 + 512, 128, 1024) == WORKSPACE and call(256 + 128, 128, 1024) == WORKSPACE
    assert call(256, 128, 512) == WORKSPACE and call(256 - 16, 128, 1024) == ALIAS and call(512 - 16, 128, 1024) == ALIAS
    assert call(256, 128, 768) == ALIAS   # rows that drift
    assert norm_bwd(G=g, H=h, dX=arr(3, B, (8, 128), (1024, 1)), dXq=arr(3, sc.E5M2, (8, 128), (512, 1), offset=256), stat=1) == WORKSPACE
    assert norm_bwd(G=g, H=h, dX=arr(3, B, (8, 128), (1024, 1)), dXq=arr(3, sc.E5M2, (8, 128), (512, 1), offset=128), stat=1) == ALIAS
