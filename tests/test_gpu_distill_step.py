"""A student's training step with the output layer's losses: a teacher's logits from an FP8 matmul, their top ones, the student's
cross entropy and distillation losses on one output layer tied to its embedding, the gradients through the norm into the
embedding (whose gradient takes the output layer's as an addend), and the Adam step.

Gradients are compared, in the norm, with those of the same network in 64 bits without any 8-bit rounding.  Two E4M3 roundings
lie on the way, of the norm's output and of the tied weight: each is 2^-4/sqrt(3) = 0.036 of its operand.  They move a logit by
sqrt(2) 0.036 of its size, 0.08 for logits of at most 1.5 in the mean, hence every probability by as much, and enter the two
products once more: sqrt(0.08^2 + 2 0.036^2) = 0.095.  Bar: twice that; a scale off by one power of two would give 0.5."""
import math

import pytest
import torch

import paper_2407_17353_b200 as sc
from test_gpu_rmsnorm import gen

pytestmark = pytest.mark.gpu
BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
N, V, D, K, TEMP = 300, 1003, 256, 24, 2.0
BAR = 0.19


class Step:
    def __init__(self):
        g = gen(7)
        T, empty = sc.ScaledTensor, sc.ScaledTensor.empty
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        vec = lambda: torch.empty(N, device="cuda")  # noqa: E731
        self.tokens = torch.randint(0, V, (N,), generator=g, device="cuda")
        self.targets = torch.randint(0, V, (N,), generator=g, device="cuda")
        self.targets[::29] = -1
        self.wte = T.make(rnd(V, D).to(F16), 2.0 ** -4)
        self.gamma = T.make((1 + 0.1 * rnd(D)).to(F32), 1.0)
        self.wte8, self.x, self.y = empty((V, D), E4M3), empty((N, D), BF16), empty((N, D), E4M3)
        self.rinv = vec()
        # the teacher: wider, with logits of its own
        self.th, self.tw = T.make(rnd(N, 512).to(E4M3), 0.25), T.make(rnd(V, 512).to(E4M3), 0.25)
        buf = torch.empty(N, 1008, dtype=BF16, device="cuda")   # rows of a multiple of 16 bytes
        self.t_logits = T(buf[:, :V], torch.empty(1, device="cuda"))
        self.t_top, self.t_ids, self.t_lse = empty((N, K), BF16), torch.empty(N, K, dtype=torch.int64, device="cuda"), vec()
        self.ce, self.ce_lse, self.kd, self.kd_lse = vec(), vec(), vec(), vec()
        self.ce_mean, self.kd_mean = (torch.empty(1, device="cuda") for _ in range(2))
        self.dy = [empty((N, D), BF16) for _ in range(3)]
        self.dw = [empty((V, D), BF16) for _ in range(3)]
        self.dx, self.dgamma, self.dwte = empty((N, D), BF16), empty((D,), F32), empty((V, D), BF16)
        self.m, self.v = (T.make(torch.zeros(V, D, device="cuda", dtype=F16), s) for s in (2.0 ** -16, 2.0 ** -26))
        b = sc.scalify_workspace_bytes
        self.ws = sc.Workspace(max([b(sc.OP_MATMUL, 4096, 4096), b(sc.OP_RMSNORM_BWD, N, D), b(sc.OP_EMBEDDING_GRAD, N, D), b(sc.OP_ADAM, 1)]
                                   + [sc.scalify_linear_loss_workspace_bytes(self.y, self.wte8, k=k, backward=w) for k in (0, K) for w in (0, 1)]))
        self.adam = sc.AdamTensors([self.dwte], [self.m], [self.v], [self.wte])

    def gradients(self):
        ws = self.ws
        sc.scalify_scaled_matmul(self.th, self.tw, self.t_logits, ws, transB=True)
        sc.scalify_scaled_top_logits(self.t_logits, self.t_top, self.t_ids, lse=self.t_lse, temperature=TEMP)
        sc.scalify_rescale(self.wte, self.wte8)
        sc.scalify_scaled_embedding_lookup(self.tokens, self.wte, self.x, c=math.sqrt(D))
        sc.scalify_scaled_add_rmsnorm(self.x, None, self.gamma, None, self.y, eps=1e-5, rinv=self.rinv)
        kd = dict(teacher_lse=self.t_lse, temperature=TEMP)
        sc.scalify_scaled_linear_cross_entropy(self.y, self.wte8, self.targets, self.ce, self.ce_lse, ws, padding_id=-1, mean=self.ce_mean)
        sc.scalify_scaled_linear_distill(self.y, self.wte8, self.t_top, self.t_ids, self.kd, self.kd_lse, ws, mean=self.kd_mean, **kd)
        sc.scalify_scaled_linear_cross_entropy_bwd(self.y, self.wte8, self.targets, self.ce_lse, self.dy[0], self.dw[0], ws, padding_id=-1)
        sc.scalify_scaled_linear_distill_bwd(self.y, self.wte8, self.t_top, self.t_ids, self.kd_lse, self.dy[1], self.dw[1], ws, **kd)
        sc.scalify_scaled_add(self.dy[0], self.dy[1], self.dy[2])
        sc.scalify_scaled_add(self.dw[0], self.dw[1], self.dw[2])
        sc.scalify_scaled_add_rmsnorm_bwd(self.dy[2], None, self.x, self.gamma, self.rinv, self.dx, ws, dgamma=self.dgamma)
        sc.scalify_scaled_embedding_grad(self.tokens, self.dx, self.dwte, ws, c=math.sqrt(D), addend=self.dw[2])

    def plain(self):
        """(losses, gradients of wte and gamma) in 64 bits; the teacher as stored."""
        value = lambda t: t.data.double() * t.scale_value()  # noqa: E731
        wte, gamma = value(self.wte).requires_grad_(), value(self.gamma).requires_grad_()
        x = wte[self.tokens] * math.sqrt(D)
        y = x / (x.square().mean(1, keepdim=True) + 1e-5 * float(self.x.scale_value()) ** 2).sqrt() * gamma
        z = y @ wte.T
        known = self.targets >= 0
        ce = torch.nn.functional.cross_entropy(z[known], self.targets[known])
        logp = torch.log_softmax(z / TEMP, 1).gather(1, self.t_ids)
        logq = value(self.t_logits).div(TEMP).log_softmax(1).gather(1, self.t_ids)
        kd = (logq.exp() * (logq - logp)).sum(1).mean()
        return (float(ce.detach()), float(kd.detach())), torch.autograd.grad(ce + kd, (wte, gamma))


def test_gradients_and_replay():
    s = Step()
    s.gradients()
    assert s.ws.check_status() == 0
    (ce, kd), (dwte, dgamma) = s.plain()
    # the teacher's top logits are those of the stored logits
    order = s.t_logits.data.float().sort(dim=1, descending=True, stable=True).indices[:, :K]
    assert torch.equal(order, s.t_ids)
    # a logit is moved by 0.08 at most in the mean: so is a mean loss
    assert abs(float(s.ce_mean) - ce) < 0.08 and abs(float(s.kd_mean) - kd) < 0.08
    for got, want in ((s.dwte, dwte), (s.dgamma, dgamma)):
        err = (got.data.double() * got.scale_value() - want).norm() / want.norm()
        assert float(err) < BAR, float(err)
    outs = [s.ce, s.kd, s.ce_mean, s.kd_mean, s.dwte.data, s.dgamma.data, s.dwte.scale]
    first = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.gradients()
    for t in outs:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
    sc.scalify_scaled_adam_step(s.adam, s.ws, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    graph.replay()                     # the next step, on the updated weights
    assert s.ws.check_status() == 0 and bool(s.dwte.data.isfinite().all()) and not torch.equal(first[4], s.dwte.data)


def test_two_graphs_on_one_workspace_and_two_streams_on_two():
    a, b = Step(), Step()
    b.tokens.copy_((a.tokens + 5) % V)
    b.ws = a.ws
    for s in (a, b):
        s.gradients()
    torch.cuda.synchronize()
    want = [s.dwte.data.clone() for s in (a, b)]
    graphs = []
    for s in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.gradients()
    for i in (1, 0, 0, 1, 0):
        graphs[i].replay()
    torch.cuda.synchronize()
    assert torch.equal(a.dwte.data, want[0]) and torch.equal(b.dwte.data, want[1])
    b.ws = sc.Workspace(a.ws.nbytes)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                s.gradients()
    torch.cuda.synchronize()
    assert torch.equal(a.dwte.data, want[0]) and torch.equal(b.dwte.data, want[1])
