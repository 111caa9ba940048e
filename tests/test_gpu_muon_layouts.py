"""The Muon step of a linear layer whose weight is stored [inputs, outputs] or [outputs, inputs]: the same update, with the
step length of the layer's shape (sqrt(max(1, outputs/inputs)) for the spectral factors)."""
import math

import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu
U = p64.U
BF16, F32, E4M3, E5M2 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.float8_e5m2


def layer(n_in, n_out, seed):
    """Weight and its gradient X^T dY of Y = X W, from the library's matmul, [inputs, outputs]."""
    g, tokens = gen(seed), 512
    put = lambda *s, dtype: sc.ScaledTensor.make(torch.randn(*s, generator=g, device="cuda").to(dtype), 1.0)  # noqa: E731
    X, W, dY = put(tokens, n_in, dtype=E4M3), put(n_in, n_out, dtype=E4M3), put(tokens, n_out, dtype=E5M2)
    ws = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_MATMUL, max(tokens, n_in), n_out))
    Y, dW = sc.ScaledTensor.empty((tokens, n_out), BF16), sc.ScaledTensor.empty((n_in, n_out), BF16)
    sc.scalify_scaled_matmul(X, W, Y, ws)  # the layout [inputs, outputs]: a plain B operand
    sc.scalify_scaled_matmul(X, dY, dW, ws, transA=True)
    want = X.data.double() @ W.data.double()
    got = Y.data.double() * Y.scale_value()
    assert float((got - want).norm() / want.norm()) < 2.0 ** -8
    return W.data.float(), dW


def update(w, g, factor, lr, steps):
    """The change of the value of a weight [rows, cols] of zeros by one step on the gradient g."""
    w = sc.ScaledTensor.make(w.contiguous(), 2.0 ** -6)
    before = w.data.double() * w.scale_value()
    m = sc.ScaledTensor.make(torch.zeros_like(w.data), 2.0 ** -20)
    ws = sc.Workspace(sc.scalify_muon_workspace_bytes([w]))
    sc.scalify_scaled_muon_step(sc.MuonTensors([sc.ScaledTensor(g.data.contiguous(), g.scale)], [m], [w]), ws, lr=lr, momentum=0.0,
                                nesterov=False, steps=steps, eps=0.0, factor=factor)
    assert ws.check_status() == 0
    return w.data.double() * w.scale_value() - before, before, w.scale_value()


@pytest.mark.parametrize("n_in,n_out", [(128, 512), (512, 128), (192, 448), (448, 192), (256, 256)])
def test_both_layouts_give_the_same_update(n_in, n_out):
    """One Newton-Schulz step, element by element: the bar of the orthogonalisation (plain64.newton_schulz_bar) at this step's
    length, plus 4 U of the weight before and after (two multiplications, a subtraction and the fp32 rounding)."""
    W, dW = layer(n_in, n_out, seed=n_in)
    lr = 0.0625
    length = lr * math.sqrt(max(1.0, n_out / n_in))
    g64 = dW.data.double()
    want, bar = -length * p64.newton_schulz(g64[None], 1, eps=0.0)[0], length * p64.newton_schulz_bar(g64[None], 1, eps=0.0)[0]
    got = []
    for layout in ("in_out", "out_in"):
        turn = (lambda t: t) if layout == "in_out" else (lambda t: t.T)
        d, before, _ = update(turn(W), sc.ScaledTensor(turn(dW.data), dW.scale),
                              sc.MUON_SPECTRAL_IN_OUT if layout == "in_out" else sc.MUON_SPECTRAL, lr, 1)
        d, before = turn(d), turn(before)
        err = bar + 4 * U * (before.abs() + (before + want).abs() + want.abs())
        assert bool(((d - want).abs() <= err).all()), (layout, float((d / want).median()))
        got.append(d)
    assert bool(((got[0] - got[1]).abs() <= 2 * err).all())


@pytest.mark.parametrize("n_in,n_out", [(128, 512), (192, 448), (256, 256)])
def test_the_output_changes_by_the_learning_rate(n_in, n_out):
    """Five steps bring the singular values of a full-rank gradient to 0.6 .. 1.3 (the quintic's band, 0.68 .. 1.21, with room
    for the FP16 iterates), so the largest change of the output's root mean square, over all inputs of root mean square 1, is
    lr times that: sigma_max(dW) sqrt(inputs/outputs)."""
    W, dW = layer(n_in, n_out, seed=n_out)
    lr = 0.0625
    for layout in ("in_out", "out_in"):
        turn = (lambda t: t) if layout == "in_out" else (lambda t: t.T)
        d, _, _ = update(turn(W) * 0, sc.ScaledTensor(turn(dW.data), dW.scale),
                         sc.MUON_SPECTRAL_IN_OUT if layout == "in_out" else sc.MUON_SPECTRAL, lr, 5)
        gain = float(torch.linalg.matrix_norm(d, 2)) * math.sqrt(n_in / n_out)
        assert 0.6 * lr < gain < 1.3 * lr, (layout, gain / lr)
