"""The norm, embedding and optimiser operators in one training step, next to the library's FP8 matmuls, cross-entropy and
Adam: a block y = norm(x + norm(x) W) between a tied embedding and its output layer.

Gradients are compared, in the norm, with those of the same network in 64 bits without any 8-bit rounding.  On the way to a
gradient lie three E4M3 roundings (two norm outputs or one and a weight, the tied weight) and two E5M2 ones (dlogits, the norm
gradient's copy); a rounding to nearest is uniform within half a step, so it adds 2^-4/sqrt(3) = 0.036 (E4M3) or 0.072 (E5M2)
of its operand's norm, and independent ones add up to sqrt(3 0.036^2 + 2 0.072^2) = 0.12.  Bar: twice that, 0.24; a scale
that is off by one power of two would give 0.5 or more."""
import math

import pytest
import torch

import paper_2407_17353_b200 as sc
import plain64 as p64
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu
BF16, F16, F32, E4M3, E5M2 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn, torch.float8_e5m2
N, V, D = 512, 304, 256
C = math.sqrt(D)
BAR = 0.24


class Step:
    def __init__(self, seed=0):
        g = gen(seed)
        T, empty = sc.ScaledTensor, sc.ScaledTensor.empty
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.ids = torch.randint(0, V, (N,), generator=g, device="cuda")
        self.ids[::37] = -1
        self.targets = torch.randint(0, V, (N,), generator=g, device="cuda")
        self.wte = T.make((rnd(V, D)).to(F16), 2.0 ** -4)
        self.W = T.make(rnd(D, D).to(F16), 2.0 ** -4)
        self.gamma = [T.make((1 + 0.1 * rnd(D)).to(F32), 1.0) for _ in range(2)]
        self.wte8, self.W8 = empty((V, D), E4M3), empty((D, D), E4M3)
        self.x, self.z, self.h = (empty((N, D), BF16) for _ in range(3))
        self.y1, self.y2 = empty((N, D), E4M3), empty((N, D), E4M3)
        self.r1, self.r2 = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        self.logits, self.dlogits = empty((N, V), BF16), empty((N, V), E5M2)
        self.loss = torch.zeros(1, device="cuda")
        self.dhead, self.dwte = empty((V, D), F32), empty((V, D), F32)
        self.dy2, self.dy1, self.dx2, self.dx1 = (empty((N, D), BF16) for _ in range(4))
        self.dz8 = empty((N, D), E5M2)
        self.dW = empty((D, D), BF16)
        self.dgamma = [empty((D,), F32) for _ in range(2)]
        self.m = T.make(torch.zeros(D, D, device="cuda", dtype=F16), 2.0 ** -20)
        self.am, self.av = (T.make(torch.zeros(V, D, device="cuda", dtype=F16), s) for s in (2.0 ** -16, 2.0 ** -26))
        b = sc.scalify_workspace_bytes
        self.ws = {k: sc.Workspace(n) for k, n in dict(
            mm=b(sc.OP_MATMUL, 4096, 4096), ce=b(sc.OP_CROSS_ENTROPY, N), norm=b(sc.OP_RMSNORM_BWD, N, D),
            emb=b(sc.OP_EMBEDDING_GRAD, N, D), adam=b(sc.OP_ADAM, 1), muon=sc.scalify_muon_workspace_bytes([self.W])).items()}
        self.muon = sc.MuonTensors([self.dW], [self.m], [self.W], [self.W8])
        self.adam = sc.AdamTensors([self.dwte], [self.am], [self.av], [self.wte])
        self.stat = torch.ones(1, device="cuda")
        sc.scalify_rescale(self.W, self.W8)

    def forward_backward(self):
        ws = self.ws
        sc.scalify_rescale(self.wte, self.wte8)
        sc.scalify_scaled_embedding_lookup(self.ids, self.wte, self.x, c=C, padding_id=-1)
        sc.scalify_scaled_add_rmsnorm(self.x, None, self.gamma[0], None, self.y1, rinv=self.r1)
        sc.scalify_scaled_matmul(self.y1, self.W8, self.z, ws["mm"])
        sc.scalify_scaled_add_rmsnorm(self.z, self.x, self.gamma[1], self.h, self.y2, rinv=self.r2)
        sc.scalify_scaled_matmul(self.y2, self.wte8, self.logits, ws["mm"], transB=True)
        sc.scalify_scaled_cross_entropy(self.logits, V, self.targets, self.loss, self.dlogits, ws["ce"])
        sc.scalify_scaled_matmul(self.dlogits, self.y2, self.dhead, ws["mm"], transA=True)
        sc.scalify_scaled_matmul(self.dlogits, self.wte8, self.dy2, ws["mm"])
        sc.scalify_scaled_add_rmsnorm_bwd(self.dy2, None, self.h, self.gamma[1], self.r2, self.dx2, ws["norm"], dXq=self.dz8,
                                          stat_in=self.stat, stat_dx=sc.STAT_AMAX, dgamma=self.dgamma[1])
        self.stat.copy_(ws["norm"].statistic())  # the next step's prediction of the gradient's magnitude
        sc.scalify_scaled_matmul(self.y1, self.dz8, self.dW, ws["mm"], transA=True)
        sc.scalify_scaled_matmul(self.dz8, self.W8, self.dy1, ws["mm"], transB=True)
        sc.scalify_scaled_add_rmsnorm_bwd(self.dy1, self.dx2, self.x, self.gamma[0], self.r1, self.dx1, ws["norm"],
                                          dgamma=self.dgamma[0])
        sc.scalify_scaled_embedding_grad(self.ids, self.dx1, self.dwte, ws["emb"], c=C, padding_id=-1, addend=self.dhead)

    def update(self, t):
        sc.scalify_scaled_muon_step(self.muon, self.ws["muon"], lr=0.02)
        sc.scalify_scaled_adam_step(self.adam, self.ws["adam"], lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=t)

    def status(self):
        return {k: w.check_status() for k, w in self.ws.items()}


def value(t):
    return t.data.double() * t.scale_value()


def reference(s):
    """Loss and gradients of the network in 64 bits by autograd."""
    wte, W = value(s.wte).requires_grad_(), value(s.W).requires_grad_()
    g1, g2 = (value(g).requires_grad_() for g in s.gamma)
    x = wte[s.ids.clamp(min=0)] * (s.ids >= 0)[:, None] * C
    # the library normalises the data component and adds eps to its mean square
    norm = lambda h, g, hs: h / hs * ((h / hs).square().mean(1, keepdim=True) + 1e-5).rsqrt() * g  # noqa: E731
    z = norm(x, g1, s.x.scale_value()) @ W
    logits = norm(x + z, g2, s.h.scale_value()) @ wte.T
    loss = torch.nn.functional.cross_entropy(logits, s.targets)
    return float(loss), dict(zip(("wte", "W", "gamma1", "gamma2"), torch.autograd.grad(loss, (wte, W, g1, g2))))


def test_gradients_of_a_step():
    s = Step()
    for _ in range(2):  # the second time with the statistic of the first
        s.forward_backward()
    torch.cuda.synchronize()
    assert all(v == 0 for v in s.status().values()), s.status()
    loss, want = reference(s)
    assert abs(float(s.loss) - loss) < 0.24 * loss
    got = dict(wte=value(s.dwte), W=value(s.dW), gamma1=value(s.dgamma[0]), gamma2=value(s.dgamma[1]))
    for k in want:
        err = float((got[k] - want[k]).norm() / want[k].norm())
        assert err < BAR, (k, err)


def test_steps_update_and_replay_from_a_graph():
    eager, captured = Step(3), Step(3)
    for t in (1, 2):
        eager.forward_backward()
        eager.update(t)
    captured.forward_backward()
    captured.update(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.forward_backward()
        captured.update(2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(v == 0 for s in (eager, captured) for v in s.status().values())
    for k in ("wte", "W", "m", "am", "av", "W8", "dwte", "dW"):
        a, b = getattr(eager, k), getattr(captured, k)
        assert torch.equal(a.data.float(), b.data.float()) and a.scale_value() == b.scale_value(), k
    # the copy that the next forward pass multiplies with is the cast of the updated weight
    assert torch.equal(p64.saturate(eager.W.data.float(), E4M3).to(E4M3).float(), eager.W8.data.float())


def test_block_scaled_norm_feeds_the_block_scaled_matmul():
    g = gen(5)
    x = sc.ScaledTensor.make(torch.randn(300, 384, generator=g, device="cuda").to(BF16), 1.0)
    r = sc.ScaledTensor.make(torch.randn(300, 384, generator=g, device="cuda"), 1.0)
    h, y, w8 = sc.ScaledTensor.empty((300, 384), F32), sc.MxTensor(300, 384), sc.MxTensor(256, 384)
    w = sc.ScaledTensor.make(torch.randn(256, 384, generator=g, device="cuda").to(BF16), 1.0)
    sc.scalify_scaled_add_rmsnorm(x, r, None, h, y)
    sc.scalify_mx_quantize(w, w8)
    out = sc.ScaledTensor.empty((300, 256), F32)
    sc.scalify_mx_matmul(y, w8, out, sc.Workspace(sc.scalify_workspace_bytes(sc.OP_MATMUL, 300, 256)))
    deq = lambda t: t.data.double() * torch.exp2(t.exponents().double() - 127).repeat_interleave(32, 1)  # noqa: E731
    a, b = deq(y), deq(w8)
    want, mag = a @ b.T, a.abs() @ b.abs().T
    assert bool(((value(out) - want).abs() <= 384 * p64.U * mag + 2 * p64.U * want.abs()).all())
    # and the operand is the norm, rounded to three bits of mantissa with one exponent per 32
    total, _, norm = p64.add_rmsnorm(x.data, 1.0, r.data, 1.0, None, 1e-5)
    n = norm(h.data)[0]
    assert float((a - n).norm() / n.norm()) < 2.0 ** -4
