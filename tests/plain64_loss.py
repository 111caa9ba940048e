"""Plain 64-bit forms of the output layer's losses and of the top logits, with the magnitudes their error bounds are made of.

Bounds.  A logit is a sum of d products in fp32 on the tensor cores, `steps` accumulations (32 bytes of K each), every one
off by at most one step of 2^-23 of the magnitudes summed so far: ez = (steps + 1) 2^-23 sum_k |h w| (values, over T).  An
exponent in base 2 is rounded three times near |z| log2(e) (product with the scale, fused multiply-add, the shift), 2^-22 of
its size, ex2 itself 2^-22; sums of up to 2^17 terms in at most 2^11 sequential additions per partial result: 2^-13 at the
very worst for terms of one sign, taken as 2^-18 (the additions of one partial result are at most 160 sequential ones of
ascending totals, 160 U < 2^-16.6; a run of tiles adds one group of four chunk sums at a time).  So
  e_lse = max_v ez + 2^-16 + 2^-21 (1 + |lse| + max|z|)
which is also the absolute error of log p, hence the relative one of p."""
import torch

U = 2.0 ** -24
QUANTUM = {torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133, torch.float32: 2.0 ** -149}


def p2(c):
    return float(2.0 ** (torch.frexp(torch.tensor(float(c), dtype=torch.float64)).exponent.item() - 1))


def kf(n):
    return 2.0 ** ((int(max(n, 1)).bit_length() - 1) // 2)


def targets(ids, vocab, padding_id, T=None, teacher_lse=None, temp=1.0):
    """(dense q [n, vocab], sum q log q, counts [n]); T: values of the teacher's logits."""
    n = ids.shape[0]
    q = torch.zeros(n, vocab, dtype=torch.float64, device=ids.device)
    if T is None:
        ids = ids[:, None]
    there = (ids >= 0) & (ids < vocab) & (ids != padding_id)
    if T is None:
        qe, lq = there.double(), torch.zeros_like(there, dtype=torch.float64)
    else:
        there = there & (T != -float("inf"))
        t = torch.where(there, T.double() / temp, -float("inf"))
        norm = torch.logsumexp(t, 1) if teacher_lse is None else teacher_lse.double()
        lq = torch.where(there, t - torch.where(there.any(1), norm, 0.0)[:, None], 0.0)
        qe = torch.where(there, lq.exp(), 0.0)
    q.scatter_add_(1, torch.where(there, ids, 0), qe)
    return q, torch.where(qe > 0, qe * lq, 0.0).sum(1), there.any(1)


def linear_loss(H, hs, W, ws, ids, padding_id=None, T=None, teacher_lse=None, temp=1.0, z_loss=0.0, grad=None, gs=1.0,
                d_type=torch.float16):
    """dict: loss, lse, mean, dH, dW (data) and their scales; e_*: the bounds (without the output's own rounding)."""
    pad = -(1 << 63) if padding_id is None else padding_id
    n, d = H.shape
    vocab = W.shape[0]
    h, w = H.double(), W.double()
    s = hs * ws / temp
    z = h @ w.T * s
    steps = -(-d * H.element_size() // 32)
    ez = ((h.abs() @ w.abs().T * s).amax(1) if n else torch.zeros(0, dtype=torch.float64, device=H.device)) * (steps + 1) * 2.0 ** -23
    lse = torch.logsumexp(z, 1)
    q, neg, counts = targets(ids, vocab, pad, T, teacher_lse, temp)
    Q = q.sum(1)
    qz = torch.where(q > 0, q * z, 0.0).sum(1)
    loss = torch.where(counts, neg - qz + Q * lse + z_loss * lse ** 2, 0.0)
    e_lse = ez + 2.0 ** -16 + 2.0 ** -21 * (1 + lse.abs() + (z.abs().amax(1) if n else 0))
    # q: an exponential of t/T - norm, whose sizes are rounded in fp32; every product with it, and their sum
    t_big = 0.0 if T is None or not n else torch.where(T.isfinite(), T.double().abs() / temp, 0.0).amax(1)
    e_q = 2.0 ** -21 * (2 + t_big) if T is not None else 0.0
    e_loss = (Q + 2 * z_loss * lse.abs()) * e_lse + Q * ez + (e_q + 2.0 ** -20) * (neg.abs() + (q * z.abs()).sum(1) + Q * lse.abs() + Q) \
        + 2.0 ** -21 * loss.abs()
    m = max(1, int(counts.sum()))
    out = dict(loss=loss, lse=lse, mean=loss.sum() / m, e_lse=e_lse, e_loss=torch.where(counts, e_loss, 0.0), counts=counts)
    out["e_mean"] = out["e_loss"].sum() / m + U * abs(out["mean"])
    unit = gs if grad is not None else p2(1.0 / max(n, 1))
    g = grad.double() if grad is not None else torch.full((n,), 1.0 / m / unit, dtype=torch.float64, device=H.device)
    g = torch.where(counts, g, 0.0) / temp / p2(1.0 / temp)
    unit *= p2(1.0 / temp)
    a = g * (Q + 2 * z_loss * lse)
    p = torch.exp(z - lse[:, None])
    D = a[:, None] * p - g[:, None] * q
    # rounded once to d_type (half a step; FP16 at a power of two that brings the largest coefficient to 2^13 at least)
    top = float(torch.maximum(a.abs(), (g * Q).abs()).max()) if n else 0.0
    eD = torch.finfo(d_type).eps / 2 * D.abs() + QUANTUM[d_type] / 2 * top * 2.0 ** -13 \
        + (a.abs() * (e_lse + 2.0 ** -20))[:, None] * p + (g.abs() * (e_q + 2.0 ** -20))[:, None] * q + (g.abs() * 2 * z_loss * e_lse)[:, None] * p
    kv, kn = kf(vocab), kf(n)
    out["dH"], out["dW"] = D @ w / kv, D.T @ h / kn
    aD = D.abs() + eD
    out["e_dH"] = (eD @ w.abs() + (vocab / 16 + 8) * 2.0 ** -23 * (aD @ w.abs())) / kv
    out["e_dW"] = (eD.T @ h.abs() + (n / 16 + 8) * 2.0 ** -23 * (aD.T @ h.abs())) / kn
    out["dH_s"], out["dW_s"] = unit * ws * kv, unit * hs * kn
    return out


def top_logits(x, k):
    """(values, places) of the k largest of every row, equal ones by place; NaN above everything."""
    key = torch.where(x.isnan(), float("inf"), x.double() + 0.0)
    key = torch.where(x.isnan(), torch.finfo(torch.float64).max, torch.where(x == float("inf"), 1e300, key))
    order = key.sort(dim=1, descending=True, stable=True).indices[:, :k]
    return x.gather(1, order), order
