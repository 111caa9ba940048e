"""Plain 64-bit implementations of the norm, embedding and orthogonalising operators (torch float64, any device), and
the elementwise bar the GPU tests hold the kernels to.

``close`` accepts |got - want| <= eps(dtype)/2 * |want| + quantum/2 + err, where the first two terms are the one
rounding to the stored type (half a step; half the subnormal step near zero) and ``err`` is what the caller derives for
the fp32 arithmetic before it (a tensor or a number, absolute).
"""
import math

import torch

U = 2.0 ** -24  # half a step of fp32, relative
LARGEST = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
QUANTUM = {torch.float8_e4m3fn: 2.0 ** -9, torch.float8_e5m2: 2.0 ** -16, torch.float16: 2.0 ** -24,
           torch.bfloat16: 2.0 ** -133, torch.float32: 2.0 ** -149}


def saturate(x, dtype):
    return x.clamp(-LARGEST[dtype], LARGEST[dtype]) if dtype in LARGEST else x


def close(got, want, err=0.0):
    """Boolean mask of the acceptable elements of `got` (as stored) against `want` (float64)."""
    dt = got.dtype
    want = saturate(want, dt)
    bound = (torch.finfo(dt).eps / 2 * want.abs() + QUANTUM[dt] / 2 + err) * (1 + 1e-9)
    d = (got.double() - want).abs()
    return (d <= bound) | (got.double() == want) | (got.double().isnan() & want.isnan())


def p2(c):
    return 2.0 ** (math.frexp(c)[1] - 1)


def kf(n):
    return 2.0 ** ((int(n).bit_length() - 1) // 2)


def add_rmsnorm(x, xs, r, rs, gamma, eps):
    """(H data before rounding, H scale, function of the stored H -> (n * gamma, rinv))."""
    if r is None:
        total, hs = x.double(), xs
    else:
        hs = max(xs, rs)
        total = x.double() * (xs / hs) + r.double() * (rs / hs)

    def norm(h):
        h = h.double()
        rinv = (h.square().mean(1) + eps) ** -0.5
        n = h * rinv[:, None]
        return (n if gamma is None else n * gamma.double()), rinv
    return total, hs, norm


def add_rmsnorm_bwd(g, gs, gr, grs, h, hs, gamma, gammas, rinv):
    """dict: dX data and scale, dgamma data and scale, and the magnitudes the rounding bounds are made of."""
    rows, d = h.shape
    g, h, rinv = g.double(), h.double(), rinv.double()[:, None]
    gam = torch.ones(d, dtype=torch.float64, device=h.device) if gamma is None else gamma.double()
    n = h * rinv
    up = g * gam
    dot = (up * n).mean(1, keepdim=True)
    dh = rinv * (up - n * dot)
    branch = gs * gammas / hs
    ds = branch if gr is None else max(branch, grs)
    dx = dh * (branch / ds)
    mag = rinv * (up.abs() + (n * dot).abs()) * 8 + rinv * n.abs() * (up * n).abs().mean(1, keepdim=True) * 64
    mag = mag * (branch / ds)
    if gr is not None:
        res = gr.double() * (grs / ds)
        dx, mag = dx + res, mag + 2 * res.abs()
    k = kf(rows)
    return {"dX": dx, "dX_s": ds, "mag": mag, "dgamma": (g * n).sum(0) / k, "dgamma_s": gs * k,
            "dgamma_mag": (g * n).abs().sum(0) / k}


def embedding_lookup(ids, w, c, padding_id, vocab):
    """Data of the looked-up rows (scale: the table's times p2(c)); padding and unknown tokens are rows of zeros."""
    known = (ids >= 0) & (ids < vocab) & (ids != padding_id)
    return w.double()[ids.clamp(0, vocab - 1)] * known[:, None] * (c / p2(c))


def embedding_grad(ids, g, gs, vocab, c, padding_id, addend=None, addend_s=0.0):
    """(data, scale, magnitude of the terms of the sums, largest number of terms of a row)."""
    known = (ids >= 0) & (ids < vocab) & (ids != padding_id)
    out = torch.zeros(vocab, g.shape[1], dtype=torch.float64, device=g.device)
    mag = torch.zeros_like(out)
    count = torch.zeros(vocab, dtype=torch.int64, device=g.device)
    for i in range(ids.numel()) if ids.numel() < 4096 else ():
        if bool(known[i]):
            out[ids[i]] += g[i].double()
            mag[ids[i]] += g[i].double().abs()
    if ids.numel() >= 4096:
        out.index_put_((ids[known],), g[known].double(), accumulate=True)
        mag.index_put_((ids[known],), g[known].double().abs(), accumulate=True)
    count.index_put_((ids[known],), torch.ones_like(ids[known]), accumulate=True)
    scale, f = gs * p2(c), c / p2(c)
    out, mag = out * f, mag * f
    if addend is not None:
        s = max(scale, addend_s)
        out = out * (scale / s) + addend.double() * (addend_s / s)
        mag = mag * (scale / s) + addend.double().abs() * (addend_s / s)
        scale = s
    return out, scale, mag, int(count.max()) if count.numel() else 0


COEF = (3.4445, -4.7750, 2.0315)


def newton_schulz(u, steps=5, coef=COEF, eps=1e-7):
    """[batch, rows, cols] float64 -> the iterate after `steps`, by the definition on the shorter side."""
    tall = u.shape[1] > u.shape[2]
    z = u.double()
    z = z.transpose(1, 2) if tall else z
    z = z / (z.square().sum((1, 2), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        a = z @ z.transpose(1, 2)
        z = coef[0] * z + (coef[1] * a + coef[2] * (a @ a)) @ z
    return z.transpose(1, 2) if tall else z


def newton_schulz_bar(u, steps=1, coef=COEF, eps=1e-7):
    """A bound, element by element and to first order, on the error of the iterate when Z, A and D are rounded to FP16
    (h = 2^-11 relative, and half the smallest subnormal at the scale each is held at) and products are accumulated in
    fp32 (k terms: k 2^-24 of their magnitudes).  The magnitudes are carried along in absolute values."""
    tall = u.shape[1] > u.shape[2]
    z = u.double()
    z = z.transpose(1, 2) if tall else z
    z = z / (z.square().sum((1, 2), keepdim=True).sqrt() + eps)
    n, k = z.shape[1], z.shape[2]
    h, sub = 2.0 ** -11, 2.0 ** -25
    eye = torch.eye(n, dtype=torch.float64, device=u.device)
    ez = (h + 8 * U) * z.abs() + sub / kf(k)
    for _ in range(steps):
        a = z @ z.transpose(1, 2)
        za = z.abs()
        mag = za @ za.transpose(1, 2)
        ea = (h + 2 * U) * a.abs() + (k * U) * mag + 2 * (ez @ za.transpose(1, 2)) + sub / 4096
        ea = torch.maximum(ea, ea.transpose(1, 2))
        d = coef[0] * eye + coef[1] * a + coef[2] * (a @ a)
        aa = a.abs()
        ed = (h + 4 * U) * d.abs() + abs(coef[1]) * ea + abs(coef[2]) * (n * U * (aa @ aa) + 2 * (ea @ aa)) + sub / 4096
        ed = torch.maximum(ed, ed.transpose(1, 2))
        new = d @ z
        ez = (h + 2 * U) * new.abs() + ed @ za + d.abs() @ ez + n * U * (d.abs() @ za) + sub / kf(k)
        z = new
    return ez.transpose(1, 2) * 1.02 if tall else ez * 1.02  # 2 %: the products of two errors


def muon_step(g, gs, m, ms, w, ws, *, lr, momentum, nesterov, decay, steps, factor, coef=COEF, eps=1e-7):
    """Data and scales of m' and w' before rounding, u (in units of m'_s), the orthogonalised u, and w's step length."""
    rows, cols = w.shape
    m_s = gs * p2(1 - momentum)
    if momentum > 0:
        m_s = max(m_s, p2(momentum) * ms)
    gd, md = g.double() * (gs / m_s), m.double() * (ms / m_s)
    new_m = momentum * md + (1 - momentum) * gd
    u = momentum * new_m + (1 - momentum) * gd if nesterov else new_m
    o = newton_schulz(u[None], steps, coef, eps)[0]
    kappa = {0: 1.0, 1: math.sqrt(max(1.0, rows / cols)), 2: 0.2 * math.sqrt(max(rows, cols))}[factor]
    step = lr * kappa
    w_s = max(ws, p2(step) / kf(max(rows, cols))) if step > 0 else ws
    new_w = (1 - decay) * (ws / w_s) * w.double() - (step / w_s) * o
    return dict(m=new_m, m_s=m_s, w=new_w, w_s=w_s, u=u, o=o, step=step)
