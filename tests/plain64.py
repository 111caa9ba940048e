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
