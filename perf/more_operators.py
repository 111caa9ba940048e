"""Timed cases of the losses that a language model's output layer is trained with, without its logits in memory:

* ``ce`` / ``ce_step``: softmax cross entropy of H W^T over a large vocabulary, alone (scoring, validation) and with its
  gradients with respect to H and W (a training step);
* ``distill`` / ``distill_step``: the divergence from a teacher's top logits, alone and with its gradients;
* ``top_logits``: a row's largest logits with their places, and the row's logsumexp: what a teacher hands on.

Every array is a scaled array: data in a low-precision type and one fp32 power of two, value = data * scale.
Where ``own`` is false, ``run`` computes the operators with elementary torch operations in 32 bits; where it is true
it makes the calls a user of the library makes.
"""
import math

import torch

own = False

E4M3, E5M2, F16, BF16, F32 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float16, torch.bfloat16, torch.float32
DTYPES = {"e4m3": E4M3, "e5m2": E5M2, "f16": F16, "bf16": BF16, "f32": F32}
LARGEST = {E4M3: 448.0, E5M2: 57344.0}
VOCAB = 50257  # GPT-2's vocabulary, the one of this repository's training step
PAD = -1


def listed():
    return [
        # the score of one token of a small model, FP8 operands: the weights are read once, latency
        {"name": "ce 1 token", "op": "ce", "n": 1, "vocab": VOCAB, "d": 768, "h": "e4m3", "w": "e4m3", "z_loss": 0.0},
        # validation loss of the 8 x 1024 token batch of the 12-layer, d = 768 model, FP8 operands
        {"name": "ce 8192x768", "op": "ce", "n": 8192, "vocab": VOCAB, "d": 768, "h": "e4m3", "w": "e4m3", "z_loss": 0.0},
        # the output layer of that model's training step, FP8 operands, mean over the tokens that count
        {"name": "ce step 8192x768 fp8", "op": "ce_step", "n": 8192, "vocab": VOCAB, "d": 768, "h": "e4m3", "w": "e4m3",
         "out": "bf16", "z_loss": 0.0, "rows": False},
        # the same with 16-bit operands, a weight for every token, and the penalty on the logsumexp
        {"name": "ce step 8192x768 bf16", "op": "ce_step", "n": 8192, "vocab": VOCAB, "d": 768, "h": "bf16", "w": "bf16",
         "out": "bf16", "z_loss": 1e-4, "rows": True},
        # ragged sizes of a mid-sized model
        {"name": "ce step 1531x1204", "op": "ce_step", "n": 1531, "vocab": 32003, "d": 1204, "h": "f16", "w": "f16",
         "out": "f16", "z_loss": 0.0, "rows": False},
        # a wide model with a large vocabulary
        {"name": "ce step 4096x4096", "op": "ce_step", "n": 4096, "vocab": 128000, "d": 4096, "h": "bf16", "w": "bf16",
         "out": "bf16", "z_loss": 1e-4, "rows": False},
        # the divergence of one short answer from its teacher
        {"name": "distill 37x768", "op": "distill", "n": 37, "vocab": VOCAB, "d": 768, "h": "bf16", "w": "bf16", "k": 16,
         "t": "bf16", "lse": True, "temperature": 1.0},
        # the output layer of a small student's step on stored top logits, FP8 operands, softened
        {"name": "distill step 8192x768", "op": "distill_step", "n": 8192, "vocab": VOCAB, "d": 768, "h": "e4m3",
         "w": "e4m3", "out": "bf16", "k": 64, "t": "bf16", "lse": False, "temperature": 2.0, "rows": False},
        # a wider student, the teacher's own probabilities
        {"name": "distill step 2047x2048", "op": "distill_step", "n": 2047, "vocab": 32003, "d": 2048, "h": "bf16",
         "w": "bf16", "out": "bf16", "k": 100, "t": "f32", "lse": True, "temperature": 1.0, "rows": True},
        # the candidates for one token
        {"name": "top logits 1x50257", "op": "top_logits", "n": 1, "vocab": VOCAB, "x": "bf16", "k": 16, "temperature": 1.0},
        # a teacher's batch, 16-bit logits
        {"name": "top logits 8192x50257", "op": "top_logits", "n": 8192, "vocab": VOCAB, "x": "bf16", "k": 64,
         "temperature": 2.0},
        # a large vocabulary, fp32 logits
        {"name": "top logits 1001x128000", "op": "top_logits", "n": 1001, "vocab": 128000, "x": "f32", "k": 200,
         "temperature": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ce", "ce_step", "ce_step", "distill", "distill_step", "top_logits"])
    vocab = _log(rng, 500, 128000)
    if op == "top_logits":
        return {"op": op, "n": _log(rng, 1, min(8192, 200_000_000 // vocab)), "vocab": vocab,
                "x": rng.choice(["bf16", "f16", "f32"]), "k": _log(rng, 1, 256), "temperature": rng.choice([0.7, 1.0, 2.0])}
    d = _log(rng, 64, 4096)
    n = _log(rng, 1, min(16384, 400_000_000 // vocab, 1_000_000_000_000 // (vocab * d)))
    kind = rng.choice(["bf16", "f16", "fp8"])
    c = {"op": op, "n": n, "vocab": vocab, "d": d}
    if kind == "fp8":
        c["h"], c["w"] = rng.choice(["e4m3", "e4m3", "e5m2"]), "e4m3"
    else:
        c["h"] = c["w"] = kind
    if op.startswith("distill"):
        c.update(k=_log(rng, 1, 256), t=rng.choice(["bf16", "f16", "f32"]), lse=rng.random() < 0.5,
                 temperature=rng.choice([1.0, 2.0, 3.3]))
    else:
        c["z_loss"] = rng.choice([0.0, 1e-4])
    if op.endswith("step"):
        c.update(out="bf16" if kind == "bf16" else rng.choice(["bf16", "f16"]), rows=rng.random() < 0.5)
    return c


# ---------------------------------------------------------------------------------------------------- inputs
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=F32)


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda", dtype=F32)


def _padded(rows, d, dtype):
    """An empty [rows, d] view whose row stride is a multiple of 16 bytes, as the library's arrays have."""
    step = 16 // torch.empty(0, dtype=dtype).element_size()
    return torch.empty(rows, -(-d // step) * step, dtype=dtype, device="cuda")[:, :d]


def _put(x, dtype):
    out = _padded(x.shape[-2], x.shape[-1], dtype)
    if dtype in LARGEST:
        x = x.clamp(-LARGEST[dtype], LARGEST[dtype])
    out.copy_(x)
    return out


def _word(v):
    return torch.full((1,), float(v), dtype=F32, device="cuda")


def _ids(g, n, vocab):
    """Token ids by log-uniform rank (word frequencies)."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab)) - 1).long().clamp(0, vocab - 1)


def _teacher(g, s, c, first):
    """Distinct ids by word frequency, logits that fall with the rank; some rows shorter, a few without any."""
    n, vocab, k = c["n"], c["vocab"], c["k"]
    weight = -torch.log(torch.arange(1, vocab + 1, device="cuda", dtype=F32))
    ids = torch.empty(n, k, dtype=torch.int64, device="cuda")
    step = max(1, 200_000_000 // vocab)
    for i in range(0, n, step):
        m = min(step, n - i)
        score = weight - torch.log(-torch.log(_uniform(g, m, vocab).clamp(1e-20, 1 - 1e-7)))
        score[torch.arange(m, device="cuda"), first[i:i + m]] = float("inf")
        ids[i:i + m] = score.topk(k, 1).indices
    t = 9 - 1.5 * torch.log(torch.arange(1, k + 1, device="cuda", dtype=F32)) + 0.3 * _normal(g, n, k)
    t = t.sort(1, descending=True).values
    s["T"], s["T_s"] = _put(t * 2, DTYPES[c["t"]]), _word(0.5)
    length = torch.where(_uniform(g, n) < 1 / 8, 1 + (_uniform(g, n) * k).long(), k)
    length = torch.where(_uniform(g, n) < 1 / 30, 0, length)
    s["ids"] = torch.where(torch.arange(k, device="cuda") < length[:, None], ids, PAD)
    if c["lse"]:  # of the whole row: the entries that were kept hold 75 to 98 percent
        v = s["T"].double() * 0.5 / c["temperature"]
        v = torch.where(s["ids"] != PAD, v, -float("inf"))
        s["t_lse"] = torch.where(length > 0, torch.logsumexp(v, 1) + 0.02 + 0.28 * _uniform(g, n), 1.0).to(F32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    c, s = dict(case), {}
    n, vocab = c["n"], c["vocab"]
    s["case"] = c
    if c["op"] == "top_logits":
        c["k"] = min(c["k"], vocab)
        s["X"], s["X_s"] = _put(_normal(g, n, vocab) * 3, DTYPES[c["x"]]), _word(0.5)
        s["V"], s["V_s"] = _padded(n, c["k"], DTYPES[c["x"]]), _word(0)
        s["ids"] = torch.empty(n, c["k"], dtype=torch.int64, device="cuda")
        s["lse"] = torch.empty(n, device="cuda")
        if own:
            _library(s)
        return s
    d = c["d"]
    if "k" in c:
        c["k"] = min(c["k"], vocab)
    # logits of standard deviation 1 to 2, the right token's lifted by up to about ten
    unit = 2.0 ** -math.ceil(math.log2(math.sqrt(d)) - 1)
    w = _normal(g, vocab, d)
    target = _ids(g, n, vocab)
    h = _normal(g, n, d) + w[target] * (6 * _uniform(g, n, 1) / math.sqrt(d))
    s["H"], s["H_s"] = _put(h, DTYPES[c["h"]]), _word(0.5)
    s["W"], s["W_s"] = _put(w, DTYPES[c["w"]]), _word(2 * unit)
    if "k" in c:
        _teacher(g, s, c, target)
    else:
        s["ids"] = torch.where(_uniform(g, n) < 1 / 30, PAD, target)
    s["loss"], s["lse"], s["mean"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), _word(0)
    if "out" in c:
        s["dH"], s["dH_s"] = _padded(n, d, DTYPES[c["out"]]), _word(0)
        s["dW"], s["dW_s"] = _padded(vocab, d, DTYPES[c["out"]]), _word(0)
        if c["rows"]:
            s["G"], s["G_s"] = _normal(g, n), _word(2.0 ** -math.ceil(math.log2(n)))
    if own:
        _library(s)
    return s


def _library(s):
    """The library's handles of the state's arrays, and the workspace that a training program keeps."""
    import paper_2407_17353_b200 as sc
    c, T = s["case"], sc.ScaledTensor
    s["sc"] = sc
    if c["op"] == "top_logits":
        s["args"] = [T(s["X"], s["X_s"]), T(s["V"], s["V_s"])]
        return
    s["args"] = [T(s["H"], s["H_s"]), T(s["W"], s["W_s"])]
    if "k" in c:
        s["teacher"] = T(s["T"], s["T_s"])
    step = "out" in c
    if step:
        s["outs"] = [T(s["dH"], s["dH_s"]), T(s["dW"], s["dW_s"])]
        s["grad"] = T(s["G"], s["G_s"]) if c["rows"] else None
    s["ws"] = sc.Workspace(sc.scalify_linear_loss_workspace_bytes(*s["args"], k=c.get("k", 0), backward=step))


# ---------------------------------------------------------------------------------------------------- one pass
OUTPUTS = {"ce": ("loss", "lse", "mean"), "distill": ("loss", "lse", "mean"),
           "ce_step": ("loss", "lse", "mean", "dH", "dH_s", "dW", "dW_s"),
           "distill_step": ("loss", "lse", "mean", "dH", "dH_s", "dW", "dW_s"), "top_logits": ("V", "V_s", "ids", "lse")}


def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        sc = s["sc"]
        if op == "top_logits":
            sc.scalify_scaled_top_logits(*s["args"], s["ids"], lse=s["lse"], temperature=c["temperature"])
        elif "k" in c:
            opt = {"teacher_lse": s.get("t_lse"), "temperature": c["temperature"], "padding_id": PAD}
            sc.scalify_scaled_linear_distill(*s["args"], s["teacher"], s["ids"], s["loss"], s["lse"], s["ws"],
                                             mean=s["mean"], **opt)
            if "out" in c:
                sc.scalify_scaled_linear_distill_bwd(*s["args"], s["teacher"], s["ids"], s["lse"], *s["outs"], s["ws"],
                                                     grad=s["grad"], **opt)
        else:
            opt = {"padding_id": PAD, "z_loss": c["z_loss"]}
            sc.scalify_scaled_linear_cross_entropy(*s["args"], s["ids"], s["loss"], s["lse"], s["ws"], mean=s["mean"], **opt)
            if "out" in c:
                sc.scalify_scaled_linear_cross_entropy_bwd(*s["args"], s["ids"], s["lse"], *s["outs"], s["ws"],
                                                           grad=s["grad"], **opt)
    elif op == "top_logits":
        _plain_top_logits(s)
    else:
        _plain_loss(s)
    return {k: s[k] for k in OUTPUTS[op]}


def _kf(k):
    """sqrt(k) rounded down to a power of two."""
    return 2.0 ** ((int(k).bit_length() - 1) // 2)


def _p2(c):
    """The largest power of two that is at most c > 0."""
    return 2.0 ** (math.frexp(c)[1] - 1)


def _plain_top_logits(s):
    c = s["case"]
    x = s["X"].float()
    v, i = x.sort(dim=1, descending=True, stable=True)  # ties: the lowest index first
    s["V"].copy_(v[:, :c["k"]])
    s["ids"].copy_(i[:, :c["k"]])
    s["V_s"].copy_(s["X_s"])
    z = x * (s["X_s"] / c["temperature"])
    top = z.amax(1, keepdim=True)
    s["lse"].copy_(torch.log(torch.exp(z - top).sum(1)) + top[:, 0])


def _plain_teacher(s):
    """The teacher's probabilities of its entries (0 where there is none), and their negative entropy."""
    c = s["case"]
    there = s["ids"] != PAD
    t = torch.where(there, s["T"].float() * (s["T_s"] / c["temperature"]), -float("inf"))
    if c["lse"]:
        norm = s["t_lse"][:, None]
    else:
        top = t.amax(1, keepdim=True)
        top = torch.where(top == -float("inf"), 0.0, top)
        norm = torch.log(torch.exp(t - top).sum(1, keepdim=True)) + top
    q = torch.where(there, torch.exp(t - norm), 0.0)
    return there, q, torch.where(q > 0, q * (t - norm), 0.0).sum(1)


def _plain_loss(s):
    """Loss and, for a step, gradients: L = sum q log q - sum q z / T + Q lse (cross entropy: one q = 1)."""
    c = s["case"]
    n, vocab = c["n"], c["vocab"]
    temp, zl = c.get("temperature", 1.0), c.get("z_loss", 0.0)
    h, w = s["H"].float(), s["W"].float()
    z = torch.mm(h, w.t()).mul_(s["H_s"] * s["W_s"] / temp)
    top = z.amax(1)
    s["lse"].copy_(torch.log(torch.exp(z - top[:, None]).sum(1)) + top)
    lse = s["lse"]
    if "k" in c:
        ids = s["ids"]
        there, q, neg = _plain_teacher(s)
        counts = there.any(1)
    else:
        ids = s["ids"][:, None]
        there, neg = ids != PAD, 0.0
        q, counts = there.float(), there[:, 0]
    total = q.sum(1)
    zq = z.gather(1, ids.clamp(min=0))
    row = neg - (q * torch.where(there, zq, 0.0)).sum(1) + total * lse + zl * lse.square()
    s["loss"].copy_(torch.where(counts, row, 0.0))
    many = counts.sum().clamp(min=1)
    s["mean"].copy_(s["loss"].double().sum() / many)
    if "out" not in c:
        return
    if c["rows"]:
        grad, unit = s["G"], s["G_s"]
    else:
        unit = _p2(1.0 / n)
        grad = (1.0 / many.float() / unit).expand(n)
    unit = unit * _p2(1.0 / temp)
    grad = torch.where(counts, grad, 0.0) * ((1.0 / temp) / _p2(1.0 / temp))
    p = z.sub_(lse[:, None]).exp_().mul_((grad * (total + 2 * zl * lse))[:, None])
    p.scatter_add_(1, ids.clamp(min=0), -grad[:, None] * q)
    s["dH"].copy_(torch.mm(p, w) / _kf(vocab))
    s["dW"].copy_(torch.mm(p.t(), h) / _kf(n))
    s["dH_s"].copy_(unit * s["W_s"] * _kf(vocab))
    s["dW_s"].copy_(unit * s["H_s"] * _kf(n))


# ---------------------------------------------------------------------------------------------------- the least work
def _size(name):
    return torch.empty(0, dtype=DTYPES[name]).element_size()


def work(case):
    c = case
    n, vocab = c["n"], c["vocab"]
    k = min(c.get("k", 1), vocab)
    if c["op"] == "top_logits":
        return {"bytes": n * (vocab * _size(c["x"]) + k * (_size(c["x"]) + 8) + 4), "flops": 4 * n * vocab}
    per = 8 * k + 8 + (k * _size(c["t"]) + (4 if c["lse"] else 0) if "k" in c else 0)
    size = n * c["d"] * _size(c["h"]) + vocab * c["d"] * _size(c["w"]) + n * per
    if not c["op"].endswith("step"):
        return {"bytes": size, "flops": 2 * n * vocab * c["d"]}
    size += (n + vocab) * c["d"] * _size(c["out"]) + (4 * n if c["rows"] else 0)
    return {"bytes": size, "flops": 8 * n * vocab * c["d"]}  # logits twice (they are not kept), and two gradients


# ---------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """From the definitions in 64 bits."""
    s = prepare(case, seed)
    c = s["case"]
    f = lambda k: s[k].to(torch.float64)  # noqa: E731
    if c["op"] == "top_logits":
        value = f("X") * f("X_s")
        top = f("X").topk(c["k"], 1).values  # (the places are whole numbers: the plain form's, ties to the lowest)
        return {"V": top, "V_s": f("X_s"), "ids": None, "lse": torch.logsumexp(value / c["temperature"], 1)}
    n, vocab, temp = c["n"], c["vocab"], c.get("temperature", 1.0)
    hv, wv = f("H") * f("H_s"), f("W") * f("W_s")
    logp = (hv @ wv.T).div_(temp)
    lse = torch.logsumexp(logp, 1)
    logp -= lse[:, None]
    # the target distribution as a dense matrix's non-zero entries
    if "k" in c:
        valid = s["ids"] >= 0
        tv = f("T") * f("T_s") / temp
        tv[~valid] = -float("inf")
        logq = tv - f("t_lse")[:, None] if c["lse"] else torch.log_softmax(tv, 1)
        q = torch.where(valid, logq.exp(), 0.0)
        logq = torch.where(q > 0, logq, 0.0)
        idx = torch.where(valid, s["ids"], 0)
        counted = valid.sum(1) > 0
    else:
        counted = s["ids"] >= 0
        idx = torch.where(counted, s["ids"], 0)[:, None]
        q = counted.to(torch.float64)[:, None]
        logq = torch.zeros_like(q)
    zeta = c.get("z_loss", 0.0)
    loss = (q * (logq - logp.gather(1, idx))).sum(1) + torch.where(counted, zeta * lse ** 2, 0.0)
    m = max(1, int(counted.sum()))
    out = {"loss": loss, "lse": lse, "mean": loss.sum().reshape(1) / m}
    if "out" not in c:
        return out
    up = torch.where(counted, f("G") * f("G_s") if c["rows"] else torch.full_like(lse, 1.0 / m), 0.0)
    # d/dz of sum q (log q - log p) + zeta lse^2
    dz = logp.exp_()
    dz *= (up * (q.sum(1) + (2 * zeta) * lse) / temp)[:, None]
    dz.scatter_add_(1, idx, -up[:, None] * q / temp)
    scale = (float(s["G_s"]) if c["rows"] else _p2(1 / n)) * _p2(1 / temp)
    sh, sw = scale * float(s["W_s"]) * _kf(vocab), scale * float(s["H_s"]) * _kf(n)
    return {**out, "dH": dz @ wv / sh, "dH_s": sh, "dW": dz.T @ hv / sw, "dW_s": sw}
