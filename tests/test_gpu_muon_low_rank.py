"""The orthogonalisation of matrices with directions in which they have nothing: low rank (the gradient of few tokens),
decaying singular values, few occupied rows.

Z, A and D are rounded to FP16.  What a rounding leaves in an empty direction the steps multiply by a = 3.4445 each, while the
occupied directions settle near 1, so the error is absolute, not relative to the result:
  * FP16's roundings are 0.85 2^-12 of the value in the root mean square (uniform within a step of 2^-10 2^e, over mantissas
    that are uniform in the logarithm).  The rounding of Z_t, whose norm is at most a^t (|p(s)| <= a s), ends as
    0.85 2^-12 a^steps at most, for t = 0 .. steps - 1; independent, five of them make sqrt(5) 0.85 = 1.9 times 2^-12 a^steps;
  * the roundings of A and D meet Z in sums over a row, in which independent ones average out; those of the diagonal of D do
    not: all its entries are close to a and err alike, by at most 4 in 14109 (2.8e-4), which shifts the occupied directions
    by up to 2.8e-4 a step and, through the steps behind it, by about twice that: 5 x 2 x 2.8e-4 = 2.8e-3 of the norm;
  * the F16 output adds 2^-11.
Bar: 2^-11 a^steps + (2.8e-3 + 2^-11) |O| in the Frobenius norm, for O with singular values near 1."""
import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu
BF16, F16, F32, E4M3, E5M2 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.float8_e5m2
A = p64.COEF[0]


def bar(want, steps):
    return 2.0 ** -11 * A ** steps + (2.8e-3 + 2.0 ** -11) * float(want.norm())


def matrix(kind, r, c, seed):
    g = gen(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    if isinstance(kind, int):
        return rnd(r, kind) @ rnd(kind, c)
    if kind == "rows":  # a few rows and columns, the rest zeros
        x = torch.zeros(r, c, device="cuda")
        x[5:21, 32:96] = rnd(16, 64)
        return x
    k = min(r, c)
    i = torch.arange(1, k + 1, device="cuda", dtype=torch.float32)
    s = i ** -2 if kind == "1/i^2" else torch.exp2(-i / 2)
    return (torch.linalg.qr(rnd(r, k))[0] * s) @ torch.linalg.qr(rnd(c, k))[0].T


@pytest.mark.parametrize("xt", [F32, BF16, E5M2])
@pytest.mark.parametrize("kind", [1, 2, 16, 64, "1/i^2", "2^-i/2", "rows"])
@pytest.mark.parametrize("r,c", [(256, 320), (304, 128), (768, 2304), (1104, 208), (2048, 512)])
def test_few_directions(r, c, kind, xt):
    x = matrix(kind, r, c, seed=r + c)
    x = x * (100.0 / float(x.abs().max()))
    X, O = sc.ScaledTensor.make(x.to(xt), 1.0), sc.ScaledTensor.empty((r, c), F16)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([X]))
    for steps in (1, 3, 5):
        sc.scalify_orthogonalize(X, O, ws, steps=steps, eps=0.0)
        want = p64.newton_schulz(X.data.double()[None], steps, eps=0.0)[0]
        err = float((O.data.double() * O.scale_value() - want).norm())
        assert ws.check_status() == 0 and err <= bar(want, steps), (steps, err, bar(want, steps))
    if kind == "rows":  # zeros stay zeros
        assert bool((O.data[:5] == 0).all()) and bool((O.data[21:] == 0).all()) and bool((O.data[:, :32] == 0).all())


@pytest.mark.parametrize("tokens", [1, 8, 100])
def test_step_on_the_gradient_of_few_tokens(tokens):
    """dW = X^T dY of a few tokens has no more directions than tokens; the weight moves by the step of the 64-bit form."""
    n_in, n_out, lr = 320, 768, 0.0625
    put = lambda *s, dt: sc.ScaledTensor.make(torch.randn(*s, generator=gen(s[1]), device="cuda").to(dt), 1.0)  # noqa: E731
    pad = 16 - tokens % 16 if tokens % 16 else 0
    X, dY = put(tokens + pad, n_in, dt=E4M3), put(tokens + pad, n_out, dt=E5M2)
    X.data.view(torch.uint8)[tokens:] = 0
    dW = sc.ScaledTensor.empty((n_in, n_out), BF16)
    sc.scalify_scaled_matmul(X, dY, dW, sc.Workspace(sc.scalify_workspace_bytes(sc.OP_MATMUL, n_in, n_out)), transA=True)
    w = sc.ScaledTensor.make(torch.zeros(n_in, n_out, device="cuda"), 2.0 ** -12)
    m = sc.ScaledTensor.make(torch.zeros(n_in, n_out, device="cuda"), 2.0 ** -20)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([w]))
    sc.scalify_scaled_muon_step(sc.MuonTensors([dW], [m], [w]), ws, lr=lr, momentum=0.0, nesterov=False, eps=0.0,
                                factor=sc.MUON_UNIT)
    assert ws.check_status() == 0
    want = p64.newton_schulz(dW.data.double()[None], 5, eps=0.0)[0]
    assert float((w.data.double() * w.scale_value() / -lr - want).norm()) <= bar(want, 5)
