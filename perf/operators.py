"""Timed cases of the operators that feed, normalise and optimise a transformer's training step:

* ``add_rmsnorm`` / ``add_rmsnorm_bwd``: residual addition and root-mean-square norm with an 8-bit output (one scale
  per tensor, or one exponent per 32 elements), and its gradient;
* ``lookup`` / ``lookup_grad``: embedding lookup with a constant factor, and its gradient by sorted tokens;
* ``orthogonalize`` / ``muon``: Newton-Schulz orthogonalisation of a batch of matrices, and the optimiser step on it.

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
COEF = (3.4445, -4.7750, 2.0315)  # quintic of the Newton-Schulz iteration


def listed():
    return [
        # one token through one norm of a small model (decode, or a validation step on one sequence): latency only
        {"name": "norm 1 token", "op": "add_rmsnorm", "rows": 1, "d": 768, "x": "bf16", "h": "bf16", "y": "e4m3"},
        # the norm of a 12-layer, d = 768 model on 8 x 1024 tokens, FP8 operand of the next matmul
        {"name": "norm 8192x768", "op": "add_rmsnorm", "rows": 8192, "d": 768, "x": "bf16", "h": "bf16", "y": "e4m3"},
        # a wider model: fp32 residual stream, block-scaled operand, a row count that ends inside an exponent tile
        {"name": "norm mx 10000x4096", "op": "add_rmsnorm", "rows": 10000, "d": 4096, "x": "bf16", "h": "f32",
         "y": "mx_e4m3"},
        # its gradient in the small model: residual gradient added, E5M2 copy for the weight-gradient matmuls
        {"name": "norm bwd 8192x768", "op": "add_rmsnorm_bwd", "rows": 8192, "d": 768, "x": "bf16", "h": "bf16",
         "q": "e5m2"},
        # and in a wider model whose row is no multiple of a vector, fp32 residual stream
        {"name": "norm bwd 4099x5004", "op": "add_rmsnorm_bwd", "rows": 4099, "d": 5004, "x": "bf16", "h": "f32",
         "q": "e5m2"},
        # token embeddings of one short prompt
        {"name": "lookup 37x768", "op": "lookup", "n": 37, "vocab": VOCAB, "d": 768, "w": "bf16", "y": "bf16"},
        # and of a long-context batch of a wider model, FP16 master weights
        {"name": "lookup 65536x2048", "op": "lookup", "n": 65536, "vocab": VOCAB, "d": 2048, "w": "f16", "y": "bf16"},
        # the embedding's gradient in the 8 x 1024 token step: tied weights, added to the output layer's gradient
        {"name": "lookup grad 8192x768", "op": "lookup_grad", "n": 8192, "vocab": VOCAB, "d": 768, "g": "bf16",
         "o": "f32", "tied": True},
        # a long-context batch, untied: a few tokens make up much of it (log-uniform ranks)
        {"name": "lookup grad 65536x1024", "op": "lookup_grad", "n": 65536, "vocab": VOCAB, "d": 1024, "g": "bf16",
         "o": "bf16", "tied": False},
        # a few small matrices (a probe model's attention projections)
        {"name": "orthogonalize 4x256x320", "op": "orthogonalize", "batch": 4, "rows": 256, "cols": 320, "x": "bf16"},
        # the optimiser step on the query/key/value projections of twelve layers
        {"name": "muon 12x768x2304", "op": "muon", "batch": 12, "rows": 768, "cols": 2304, "w": "f16"},
        # the tall projections of a wide model
        {"name": "muon 4x8192x2048", "op": "muon", "batch": 4, "rows": 8192, "cols": 2048, "w": "f16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["add_rmsnorm", "add_rmsnorm_bwd", "lookup", "lookup_grad", "orthogonalize", "muon"])
    if op in ("add_rmsnorm", "add_rmsnorm_bwd"):
        d = _log(rng, 64, 8192)
        x = rng.choice(["bf16", "f16"])
        c = {"op": op, "x": x, "h": rng.choice([x, "f32"])}
        if op == "add_rmsnorm":
            c["y"] = rng.choice(["e4m3", "e5m2", "bf16", "mx_e4m3", "mx_e5m2"])
            if c["y"].startswith("mx"):
                d = max(128, d // 128 * 128)
        else:
            c["q"] = rng.choice(["e4m3", "e5m2"])
        return {**c, "rows": _log(rng, 1, min(20000, 30_000_000 // d)), "d": d}
    if op == "lookup":
        d = _log(rng, 64, 4096)
        return {"op": op, "n": _log(rng, 1, min(65536, 100_000_000 // d)), "vocab": _log(rng, 500, 100000), "d": d,
                "w": rng.choice(["bf16", "f16", "f32", "e4m3"]), "y": rng.choice(["bf16", "f16"])}
    if op == "lookup_grad":
        d = _log(rng, 64, 2048)
        return {"op": op, "n": _log(rng, 1, min(65536, 60_000_000 // d)), "vocab": _log(rng, 500, 60000), "d": d,
                "g": rng.choice(["bf16", "f16", "f32", "e5m2"]), "o": rng.choice(["f32", "bf16"]),
                "tied": rng.random() < 0.5}
    a, b = _log(rng, 64, 2048), _log(rng, 64, 2048)
    batch = max(1, min(_log(rng, 1, 16), int(1.2e10 / (a * b * min(a, b)))))
    c = {"op": op, "batch": batch, "rows": a, "cols": b}
    return {**c, "x": rng.choice(["bf16", "f32"])} if op == "orthogonalize" else {**c, "w": rng.choice(["f16", "bf16"])}


# ---------------------------------------------------------------------------------------------------- inputs
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=F32)


def _activations(g, rows, d):
    """Roughly unit Gaussian with a few channels that are ten times larger, as residual streams have."""
    x = _normal(g, rows, d)
    return x * torch.where(torch.rand(d, generator=g, device="cuda") < 0.01, 10.0, 1.0)


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
    """Token ids by log-uniform rank (word frequencies), a thirtieth of them padding (id -1)."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(vocab)) - 1).long().clamp(0, vocab - 1)
    return torch.where(torch.rand(n, generator=g, device="cuda") < 1 / 30, -1, ids)


def _gradients(g, batch, rows, cols):
    """Matrices with a decaying spectrum on a noise floor, as weight gradients have."""
    rank = max(1, min(rows, cols) // 8)
    low = torch.bmm(_normal(g, batch, rows, rank) * torch.linspace(1, 0.1, rank, device="cuda"),
                    _normal(g, batch, rank, cols)) / math.sqrt(rank / 3)
    return low + 0.5 * _normal(g, batch, rows, cols)


def _matrices(x, dtype):
    """[batch, rows, cols] with rows padded to 16 bytes."""
    b, r, c = x.shape
    out = _padded(b * r, c, dtype)
    if dtype in LARGEST:
        x = x.clamp(-LARGEST[dtype], LARGEST[dtype])
    out = out.as_strided((b, r, c), (r * out.stride(0), out.stride(0), 1))
    out.copy_(x)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    c, s = dict(case), {}
    op = c["op"]
    if op in ("add_rmsnorm", "add_rmsnorm_bwd"):
        rows, d = c["rows"], c["d"]
        xt, ht = DTYPES[c["x"]], DTYPES[c["h"]]
        s["gamma"], s["gamma_s"] = (1 + 0.1 * _normal(g, d)).to(F32), _word(1.0)
    if op == "add_rmsnorm":
        s["X"], s["X_s"] = _put(_normal(g, rows, d), xt), _word(0.5)
        s["R"], s["R_s"] = _put(_activations(g, rows, d), ht), _word(2.0)
        s["H"], s["H_s"], s["rinv"], s["Y_s"] = _padded(rows, d, ht), _word(0), torch.empty(rows, device="cuda"), _word(0)
        if not c["y"].startswith("mx"):
            s["Y"] = _padded(rows, d, DTYPES[c["y"]])
        else:
            s["Y"] = torch.empty(rows, d, dtype=DTYPES[c["y"][3:]], device="cuda")
            s["sf"] = torch.empty(-(-rows // 256) * 256 * (d // 32), dtype=torch.uint8, device="cuda")
    elif op == "add_rmsnorm_bwd":
        h = _put(_activations(g, rows, d), ht)
        s["H"], s["H_s"] = h, _word(2.0)
        s["rinv"] = torch.rsqrt(h.float().square().mean(1) + 1e-5)
        s["G"], s["G_s"] = _put(_normal(g, rows, d), xt), _word(2.0 ** -12)
        s["Gr"], s["Gr_s"] = _put(_normal(g, rows, d), ht), _word(2.0 ** -13)
        s["stat_in"] = _word(3.7)  # the largest magnitude of an earlier step's gradient
        s["dX"], s["dX_s"], s["dXq"], s["dXq_s"] = _padded(rows, d, ht), _word(0), _padded(rows, d, DTYPES[c["q"]]), _word(0)
        s["dgamma"], s["dgamma_s"], s["stat"] = torch.empty(d, device="cuda"), _word(0), _word(0)
    elif op == "lookup":
        s["ids"] = _ids(g, c["n"], c["vocab"])
        s["W"], s["W_s"] = _put(_normal(g, c["vocab"], c["d"]), DTYPES[c["w"]]), _word(2.0 ** -6)
        s["Y"], s["Y_s"], s["factor"] = _padded(c["n"], c["d"], DTYPES[c["y"]]), _word(0), math.sqrt(c["d"])
    elif op == "lookup_grad":
        s["ids"] = _ids(g, c["n"], c["vocab"])
        s["G"], s["G_s"] = _put(_normal(g, c["n"], c["d"]), DTYPES[c["g"]]), _word(2.0 ** -10)
        s["W"], s["W_s"], s["factor"] = _padded(c["vocab"], c["d"], DTYPES[c["o"]]), _word(0), math.sqrt(c["d"])
        if c["tied"]:
            s["A"], s["A_s"] = _put(_normal(g, c["vocab"], c["d"]), DTYPES[c["o"]]), _word(2.0 ** -11)
    elif op == "orthogonalize":
        s["X"], s["X_s"] = _matrices(_gradients(g, c["batch"], c["rows"], c["cols"]), DTYPES[c["x"]]), _word(2.0 ** -10)
        s["O"], s["O_s"] = _matrices(torch.zeros(c["batch"], c["rows"], c["cols"], device="cuda"), BF16), _word(0)
    else:
        shape = (c["batch"], c["rows"], c["cols"])
        n = c["batch"]
        s["G"], s["G_s"] = _matrices(_gradients(g, *shape), E5M2), torch.full((n,), 2.0 ** -10, device="cuda")
        s["M"], s["M_s"] = _matrices(_gradients(g, *shape), F16), torch.full((n,), 2.0 ** -12, device="cuda")
        s["W"], s["W_s"] = _matrices(_normal(g, *shape), DTYPES[c["w"]]), torch.full((n,), 2.0 ** -6, device="cuda")
        s["Wq"], s["Wq_s"] = _matrices(torch.zeros(shape, device="cuda"), E4M3), torch.zeros(n, device="cuda")
    s["case"] = c
    if own:
        _library(s)
    return s


def _library(s):
    """The library's handles of the state's arrays, and the workspace that a training program keeps."""
    import paper_2407_17353_b200 as sc
    c, T = s["case"], sc.ScaledTensor
    s["sc"] = sc
    op = c["op"]
    if op == "add_rmsnorm":
        s["args"] = [T(s[k], s[k + "_s"]) for k in ("X", "R", "gamma", "H")]
        if "sf" in s:
            mx = sc.MxTensor(c["rows"], c["d"], s["Y"].dtype)
            s["Y"], s["sf"], s["Y_s"] = mx.data, mx.sf, mx.scale
            s["args"].append(mx)
        else:
            s["args"].append(T(s["Y"], s["Y_s"]))
    elif op == "add_rmsnorm_bwd":
        s["args"] = [T(s[k], s[k + "_s"]) for k in ("G", "Gr", "H", "gamma")]
        s["outs"] = [T(s[k], s[k + "_s"]) for k in ("dX", "dXq", "dgamma")]
        s["ws"] = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_RMSNORM_BWD, c["rows"], c["d"]))
    elif op == "lookup":
        s["args"] = [T(s["W"], s["W_s"]), T(s["Y"], s["Y_s"])]
    elif op == "lookup_grad":
        s["args"] = [T(s["G"], s["G_s"]), T(s["W"], s["W_s"])]
        s["addend"] = T(s["A"], s["A_s"]) if c["tied"] else None
        s["ws"] = sc.Workspace(sc.scalify_workspace_bytes(sc.OP_EMBEDDING_GRAD, c["n"], c["d"]))
    elif op == "orthogonalize":
        s["args"] = [T(s["X"], s["X_s"]), T(s["O"], s["O_s"])]
        s["ws"] = sc.Workspace(sc.scalify_muon_workspace_bytes([s["args"][0]]))
    else:
        lists = [[T(s[k][i], s[k + "_s"][i:i + 1]) for i in range(c["batch"])] for k in ("G", "M", "W", "Wq")]
        s["tensors"] = sc.MuonTensors(*lists)
        s["ws"] = sc.Workspace(sc.scalify_muon_workspace_bytes(lists[2]))


# ---------------------------------------------------------------------------------------------------- one pass
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.1


def run(s):
    op = s["case"]["op"]
    if own:
        sc = s["sc"]
        if op == "add_rmsnorm":
            sc.scalify_scaled_add_rmsnorm(*s["args"], eps=1e-5, rinv=s["rinv"])
        elif op == "add_rmsnorm_bwd":
            sc.scalify_scaled_add_rmsnorm_bwd(*s["args"], s["rinv"], s["outs"][0], s["ws"], dXq=s["outs"][1],
                                              stat_in=s["stat_in"], stat_dx=sc.STAT_AMAX, dgamma=s["outs"][2])
            s["stat"] = s["ws"].statistic()
        elif op == "lookup":
            sc.scalify_scaled_embedding_lookup(s["ids"], *s["args"], c=s["factor"], padding_id=-1)
        elif op == "lookup_grad":
            sc.scalify_scaled_embedding_grad(s["ids"], *s["args"], s["ws"], c=s["factor"], padding_id=-1,
                                             addend=s["addend"])
        elif op == "orthogonalize":
            sc.scalify_orthogonalize(*s["args"], s["ws"], steps=5, coef=COEF, eps=1e-7)
        else:
            sc.scalify_scaled_muon_step(s["tensors"], s["ws"], lr=LR, momentum=MOMENTUM, nesterov=True,
                                        weight_decay=DECAY, steps=5, coef=COEF, eps=1e-7, factor=sc.MUON_SPECTRAL)
    elif op == "add_rmsnorm":
        _plain_norm(s)
    elif op == "add_rmsnorm_bwd":
        _plain_norm_bwd(s)
    elif op == "lookup":
        _plain_lookup(s)
    elif op == "lookup_grad":
        _plain_lookup_grad(s)
    elif op == "orthogonalize":
        _plain_orthogonalize(s)
    else:
        _plain_muon(s)
    out = {k: s[k] for k in OUTPUTS[op]}
    if "sf" in s:
        out["sf"] = s["sf"].view(torch.float8_e8m0fnu)  # the powers of two that the exponent bytes stand for
    return out


OUTPUTS = {"add_rmsnorm": ("H", "H_s", "Y", "Y_s", "rinv"),
           "add_rmsnorm_bwd": ("dX", "dX_s", "dXq", "dXq_s", "dgamma", "dgamma_s", "stat"),
           "lookup": ("Y", "Y_s"), "lookup_grad": ("W", "W_s"), "orthogonalize": ("O", "O_s"),
           "muon": ("M", "M_s", "W", "W_s", "Wq", "Wq_s")}


def _store(out, x):
    out.copy_(x.clamp(-LARGEST[out.dtype], LARGEST[out.dtype]) if out.dtype in LARGEST else x)


def _p2(c):
    """The largest power of two that is at most c > 0."""
    return 2.0 ** (math.frexp(c)[1] - 1)


def _kf(k):
    """sqrt(k) rounded down to a power of two."""
    return 2.0 ** ((int(k).bit_length() - 1) // 2)


def _tile_exponents(codes, rows, kb):
    """Plain [rows, K/32] exponent codes -> the tiles the block-scaled matmul reads (padding rows: code 127)."""
    pr = -(-rows // 256) * 256
    full = torch.full((pr, kb), 127, dtype=torch.uint8, device=codes.device)
    full[:rows] = codes
    return full.view(pr // 128, 4, 32, kb // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _plain_norm(s):
    torch.maximum(s["X_s"], s["R_s"], out=s["H_s"])
    s["H"].copy_(s["X"].float() * (s["X_s"] / s["H_s"]) + s["R"].float() * (s["R_s"] / s["H_s"]))
    h = s["H"].float()
    torch.rsqrt(h.square().mean(1) + 1e-5, out=s["rinv"])
    y = h * s["rinv"][:, None] * s["gamma"]
    s["Y_s"].copy_(s["gamma_s"])
    if "sf" not in s:
        return _store(s["Y"], y)
    rows, d = y.shape
    blocks = y.view(rows, d // 32, 32)
    amax = blocks.abs().amax(2)
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 1 - (8 if s["Y"].dtype == E4M3 else 15), 0).clamp(-127, 127)
    _store(s["Y"], torch.ldexp(blocks, -e[..., None]).reshape(rows, d))
    s["sf"].copy_(_tile_exponents((e + 127).to(torch.uint8), rows, d // 32))


def _plain_norm_bwd(s):
    rows, d = s["H"].shape
    r = s["rinv"][:, None]
    n = s["H"].float() * r
    gf = s["G"].float()
    gh = gf * s["gamma"]
    dh = r * (gh - n * (gh * n).mean(1, keepdim=True))
    branch = s["G_s"] * s["gamma_s"] / s["H_s"]
    torch.maximum(branch, s["Gr_s"], out=s["dX_s"])
    s["dX"].copy_(dh * (branch / s["dX_s"]) + s["Gr"].float() * (s["Gr_s"] / s["dX_s"]))
    stored = s["dX"].float()
    s["stat"] = stored.abs().amax().reshape(1)
    f = torch.exp2(torch.frexp(s["stat_in"]).exponent.float() - 1)  # rounded down to a power of two
    _store(s["dXq"], stored / f)
    torch.mul(s["dX_s"], f, out=s["dXq_s"])
    torch.div((gf * n).sum(0), _kf(rows), out=s["dgamma"])
    torch.mul(s["G_s"], _kf(rows), out=s["dgamma_s"])


def _plain_lookup(s):
    ids, p = s["ids"], _p2(s["factor"])
    rows = s["W"][ids.clamp(min=0)].float() * (s["factor"] / p)
    _store(s["Y"], rows * (ids >= 0)[:, None])
    torch.mul(s["W_s"], p, out=s["Y_s"])


def _plain_lookup_grad(s):
    ids, p = s["ids"], _p2(s["factor"])
    vocab, d = s["W"].shape
    acc = torch.zeros(vocab + 1, d, device="cuda")
    acc.index_add_(0, torch.where(ids >= 0, ids, vocab), s["G"].float())  # row `vocab` takes the padding
    acc = acc[:vocab] * (s["factor"] / p)
    if "A" in s:
        gs = s["G_s"] * p
        torch.maximum(gs, s["A_s"], out=s["W_s"])
        _store(s["W"], acc * (gs / s["W_s"]) + s["A"].float() * (s["A_s"] / s["W_s"]))
    else:
        torch.mul(s["G_s"], p, out=s["W_s"])
        _store(s["W"], acc)


def _newton_schulz(x):
    a, b, c = COEF
    gram = torch.bmm(x, x.transpose(1, 2))
    return a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)


def _plain_iterate(u):
    """Five steps on [batch, rows, cols] of any scale, on the side with the smaller Gram matrix."""
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    x = _newton_schulz(_newton_schulz(_newton_schulz(_newton_schulz(_newton_schulz(x)))))
    return x.transpose(1, 2) if tall else x


def _plain_orthogonalize(s):
    unit = 1.0 / _kf(max(s["X"].shape[1:]))
    s["O"].copy_(_plain_iterate(s["X"].float()) / unit)
    s["O_s"].fill_(unit)


def _plain_muon(s):
    rows, cols = s["W"].shape[1:]
    m_s = torch.maximum(_p2(MOMENTUM) * s["M_s"], _p2(1 - MOMENTUM) * s["G_s"])
    wide = lambda v: v[:, None, None]  # noqa: E731
    g = s["G"].float() * wide(s["G_s"] / m_s)
    m = s["M"].float() * (MOMENTUM * wide(s["M_s"] / m_s)) + g * (1 - MOMENTUM)
    o = _plain_iterate(m * MOMENTUM + g * (1 - MOMENTUM))
    s["M"].copy_(m)
    s["M_s"].copy_(m_s)
    step = LR * math.sqrt(max(1.0, rows / cols))
    w_s = torch.clamp(s["W_s"], min=_p2(step) / _kf(max(rows, cols)))
    w = s["W"].float() * ((1 - LR * DECAY) * wide(s["W_s"] / w_s)) - o * (step / wide(w_s))
    s["W"].copy_(w)
    s["W_s"].copy_(w_s)
    _store(s["Wq"], s["W"].float())
    s["Wq_s"].copy_(w_s)


# ---------------------------------------------------------------------------------------------------- the least work
def _size(name):
    return torch.empty(0, dtype=DTYPES[name]).element_size()


def work(case):
    c = case
    op = c["op"]
    if op == "add_rmsnorm":
        per = _size(c["x"]) + 2 * _size(c["h"]) + (1 + 1 / 32 if c["y"].startswith("mx") else _size(c["y"]))
        return {"bytes": c["rows"] * (c["d"] * per + 4) + 4 * c["d"], "flops": 7 * c["rows"] * c["d"]}
    if op == "add_rmsnorm_bwd":
        per = _size(c["x"]) + 3 * _size(c["h"]) + 1
        return {"bytes": c["rows"] * (c["d"] * per + 4) + 8 * c["d"], "flops": 14 * c["rows"] * c["d"]}
    if op == "lookup":
        rows = c["vocab"] * -math.expm1(-c["n"] / c["vocab"])  # at most so many different rows are read
        return {"bytes": c["n"] * (c["d"] * _size(c["y"]) + 8) + min(rows, c["n"]) * c["d"] * _size(c["w"]),
                "flops": c["n"] * c["d"]}
    if op == "lookup_grad":
        out = c["vocab"] * c["d"] * _size(c["o"]) * (2 if c["tied"] else 1)
        return {"bytes": c["n"] * (c["d"] * _size(c["g"]) + 8) + out, "flops": c["n"] * c["d"]}
    k, l = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    n = c["batch"] * k * l
    # a step: the Gram matrix and its square are symmetric (half of 2 k k l and 2 k k k), then 2 k k l
    flops = 5.0 * c["batch"] * (k * k * l + k * k * k + 2 * k * k * l)
    if op == "orthogonalize":
        return {"bytes": n * (_size(c["x"]) + 2), "flops": flops}
    return {"bytes": n * (1 + 2 * 2 + 2 * _size(c["w"]) + 1), "flops": flops}


# ---------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """From the definitions in 64 bits; 8-bit outputs, and what is computed from a stored output, after its rounding."""
    s = prepare(case, seed)
    c = s["case"]
    op = c["op"]
    f = lambda k: s[k].to(torch.float64)  # noqa: E731
    value = lambda k: f(k) * f(k + "_s")  # noqa: E731

    def stored(x, dtype):
        return (x.clamp(-LARGEST[dtype], LARGEST[dtype]) if dtype in LARGEST else x).to(dtype).to(torch.float64)

    if op == "add_rmsnorm":
        hs = max(float(s["X_s"]), float(s["R_s"]))
        total = (value("X") + value("R")) / hs
        h = stored(total, s["H"].dtype)
        rms = ((h * h).sum(1) / c["d"] + 1e-5).sqrt()
        y = (h / rms[:, None]) * f("gamma")
        out = {"H": total, "H_s": hs, "rinv": 1 / rms, "Y_s": 1.0}
        if "sf" not in s:
            return {**out, "Y": stored(y, s["Y"].dtype)}
        blocks = y.reshape(c["rows"], -1, 32)
        top = blocks.abs().max(2).values
        e = torch.where(top > 0, torch.floor(torch.log2(top.clamp(min=1e-300))) - (8 if s["Y"].dtype == E4M3 else 15), 0.0)
        code = _tile_exponents((e + 127).to(torch.uint8), c["rows"], c["d"] // 32)
        return {**out, "Y": stored((blocks / torch.exp2(e)[..., None]).reshape(y.shape), s["Y"].dtype),
                "sf": torch.exp2(code.to(torch.float64) - 127)}
    if op == "add_rmsnorm_bwd":
        h, r, g, gam = f("H"), f("rinv")[:, None], f("G"), f("gamma")
        up = g * gam * float(s["G_s"]) * float(s["gamma_s"])
        # d/dh of (h r) . up with r = (mean(h^2) + eps)^(-1/2), in units of the data of H, then of its values
        dv = (up * r - h * r ** 3 * (up * h).sum(1, keepdim=True) / c["d"]) / float(s["H_s"]) + value("Gr")
        ds = max(float(s["G_s"]) * float(s["gamma_s"]) / float(s["H_s"]), float(s["Gr_s"]))
        dx = stored(dv / ds, s["dX"].dtype)
        fac = _p2(float(s["stat_in"]))
        k = _kf(c["rows"])
        return {"dX": dv / ds, "dX_s": ds, "dXq": stored(dx / fac, s["dXq"].dtype), "dXq_s": ds * fac,
                "dgamma": (g * (h * r)).sum(0) / k, "dgamma_s": float(s["G_s"]) * k, "stat": dx.abs().max().reshape(1)}
    if op == "lookup":
        ids, p = s["ids"], _p2(s["factor"])
        out = torch.zeros(c["n"], c["d"], dtype=torch.float64, device="cuda")
        known = (ids != -1).nonzero()[:, 0]
        out[known] = f("W")[ids[known]] * s["factor"] / p
        return {"Y": out, "Y_s": float(s["W_s"]) * p}
    if op == "lookup_grad":
        ids, p = s["ids"], _p2(s["factor"])
        known = (ids != -1).nonzero()[:, 0]
        acc = torch.zeros(c["vocab"], c["d"], dtype=torch.float64, device="cuda")
        acc.index_put_((ids[known],), value("G")[known] * s["factor"], accumulate=True)
        ws = float(s["G_s"]) * p
        if c["tied"]:
            acc, ws = acc + value("A"), max(ws, float(s["A_s"]))
        return {"W": acc / ws, "W_s": ws}

    def polar(u):  # Newton-Schulz through the smaller Gram matrix, 64 bits
        x = u / (torch.linalg.norm(u.flatten(1), dim=1)[:, None, None] + 1e-7)
        left = u.shape[1] <= u.shape[2]
        eye = torch.eye(min(u.shape[1:]), dtype=torch.float64, device="cuda")
        for _ in range(5):
            q = x @ x.mT if left else x.mT @ x
            q = COEF[0] * eye + q @ (COEF[1] * eye + COEF[2] * q)
            x = q @ x if left else x @ q
        return x

    rows, cols = c["rows"], c["cols"]
    unit = 1.0 / _kf(max(rows, cols))
    if op == "orthogonalize":
        return {"O": polar(f("X")) / unit, "O_s": unit}
    each = lambda k: f(k)[:, None, None]  # noqa: E731
    gv, mv = f("G") * each("G_s"), f("M") * each("M_s")
    ms = torch.maximum(_p2(MOMENTUM) * f("M_s"), _p2(1 - MOMENTUM) * f("G_s"))
    m = MOMENTUM * mv + (1 - MOMENTUM) * gv
    o = polar((MOMENTUM * m + (1 - MOMENTUM) * gv) / ms[:, None, None])
    step = LR * math.sqrt(max(1.0, rows / cols))
    ws = torch.clamp(f("W_s"), min=_p2(step) * unit)
    w = (1 - LR * DECAY) * f("W") * each("W_s") - step * o
    wd = w / ws[:, None, None]
    return {"M": m / ms[:, None, None], "M_s": ms, "W": wd, "W_s": ws, "Wq": stored(stored(wd, s["W"].dtype), E4M3),
            "Wq_s": ws}
