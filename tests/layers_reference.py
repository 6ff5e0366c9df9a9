"""The operators of hr_layers.h in 64 bits, written from their definitions, and how far 32-bit arithmetic may lie from them."""
import math

import torch

from scores_reference import EPS, TINY, U, close  # noqa: F401


# ---- layer norm.  A sum over a row of n is at most 96 + n / 1024 additions long (64 or more lanes, 32 numbers each, and the folds; 1024 threads
# for longer ones): `d` roundings.

def _depth(n):
    return 96 + n / 1024


def norm(x, weight, bias, eps):
    """(rows, mean, rstd, u) and how far rows, mean and rstd (of its own size) may be off."""
    x = x.double().cpu()
    n = x.shape[1]
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double().cpu()
    b = torch.zeros(n, dtype=torch.float64) if bias is None else bias.double().cpu()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    sigma = (c * c).mean(1, keepdim=True).sqrt()
    rstd = 1 / torch.sqrt(sigma ** 2 + eps)
    u = c * rstd
    d = _depth(n)
    # what is left after a mean that is itself rounded: |off| <= d U mean|x|; then c within (d + 4) U (|c| + sigma + |off|)
    off = d * U * x.abs().mean(1, keepdim=True)
    c_tol = (d + 4) * U * (c.abs() + sigma + off)
    r_tol = (2 * d + 12) * U * (sigma + off) ** 2 / (sigma ** 2 + eps) + 4 * U
    tol = w.abs() * (c_tol * rstd + u.abs() * (r_tol + 2 * U)) + 2 * U * (u * w).abs() + U * b.abs()
    return u * w + b, mean[:, 0], rstd[:, 0], u, tol, (U * mean.abs() + c_tol.max(1, keepdim=True).values)[:, 0], r_tol[:, 0]


def norm_grads(x, weight, dy, eps):
    """(dx, dweight, dbias) and how far they may be off, mean and rstd being those of 32 bits."""
    _, mean, rstd, u, _, m_tol, r_tol = norm(x, weight, None, eps)
    mean, rstd, m_tol, r_tol = (t[:, None] for t in (mean, rstd, m_tol, r_tol))
    rows, n = u.shape
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double().cpu()
    dy = dy.double().cpu()
    g = dy * w
    d = _depth(n)
    u_tol = m_tol * rstd + u.abs() * (r_tol + 3 * U)
    c1, c2 = g.mean(1, keepdim=True), (g * u).mean(1, keepdim=True)
    c1_tol = (d + 3) * U * g.abs().mean(1, keepdim=True)
    c2_tol = (d + 4) * U * (g * u).abs().mean(1, keepdim=True) + (g.abs() * u_tol).mean(1, keepdim=True)
    dx = rstd * (g - c1 - u * c2)
    dx_tol = rstd * (c1_tol + u.abs() * c2_tol + u_tol * c2.abs() + 4 * U * (g.abs() + c1.abs() + (u * c2).abs())) + dx.abs() * (r_tol + 2 * U)
    dw, db = (dy * u).sum(0), dy.sum(0)
    return dx, dw, db, dx_tol, (rows + 40) * U * (dy * u).abs().sum(0) + (dy.abs() * u_tol).sum(0), (rows + 40) * U * dy.abs().sum(0)


# ---- gated blocks

def act(z, name):
    """The activation and its slope."""
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p * (1 + z * (1 - p))
    if name == "gelu":
        p = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def gated(x, wg, wu, name):
    """(out, gate, up) and how far each may be off: k products, summed in any order, then act (slope at most 1.13; its own arithmetic 8 U of
    value and argument) and the product."""
    x, wg, wu = (t.double().cpu() for t in (x, wg, wu))
    k = x.shape[1]
    gate, up = x @ wg.T, x @ wu.T
    gate_tol, up_tol = ((k + 4) * U * (x.abs() @ w.abs().T) for w in (wg, wu))
    a, _ = act(gate, name)
    a_tol = 1.13 * gate_tol + 8 * U * (a.abs() + gate.abs())
    return a * up, gate, up, a_tol * (up.abs() + up_tol) + a.abs() * up_tol + 2 * U * (a * up).abs(), gate_tol, up_tol


def gated_grads(x, wg, wu, pre, dh, name, dtype):
    """(dx, dwg, dwu) from gate and up as they are in pre, and how far each may be off: d_gate and d_up are rounded to dtype once (float32: the last
    rounding of their arithmetic), the sums have m or 2 f products."""
    x, wg, wu, dh = (t.double().cpu() for t in (x, wg, wu, dh))
    gate, up = pre.double().cpu().unbind(1)
    a, slope = act(gate, name)
    dg, du = dh * up * slope, dh * a
    dg_tol = 16 * U * (dh * up).abs() * (1 + gate.abs()) + EPS[dtype] * dg.abs() + TINY[dtype]
    du_tol = 8 * U * dh.abs() * (a.abs() + gate.abs()) + EPS[dtype] * du.abs() + TINY[dtype]
    m, f = dg.shape
    dx_tol = dg_tol @ wg.abs() + du_tol @ wu.abs() + (2 * f + 4) * U * ((dg.abs() + dg_tol) @ wg.abs() + (du.abs() + du_tol) @ wu.abs())
    tols = [t.T @ x.abs() + (m + 4) * U * (v.abs() + t).T @ x.abs() for v, t in ((dg, dg_tol), (du, du_tol))]
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x, dx_tol, tols[0], tols[1]


# ---- AdamW

def adamw(p, g, m, v, step, lr, betas, eps, decay, scale=1.0):
    """(p, m, v) after the step and how far 32 bits may be off (p: before its rounding to fewer bits)."""
    p, g, m, v = (t.double().cpu().reshape(-1) for t in (p, g, m, v))
    g = g * scale
    b1, b2 = betas
    m_tol = 4 * U * ((b1 * m).abs() + ((1 - b1) * g).abs())
    v_tol = 6 * U * (b2 * v + (1 - b2) * g * g) + 2.0 ** -148
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    rate, spread = lr / (1 - b1 ** step), 1 / math.sqrt(1 - b2 ** step)
    low = torch.sqrt((v - v_tol).clamp(min=0)) * spread * (1 - 4 * U) + eps * (1 - 4 * U)
    bottom = torch.sqrt(v) * spread + eps
    change = rate * m / bottom
    tol = 4 * U * p.abs() + abs(rate) * (m.abs() * (1 + 8 * U) + m_tol) / low - change.abs() + 4 * U * change.abs()
    return p * (1 - lr * decay) - change, m, v, tol, m_tol, v_tol


def moments32(g, m, v, betas, scale=1.0):
    """Moments that become codes: every product and sum rounded to float32 by itself (numpy)."""
    import numpy as np
    g, m, v = (t.detach().float().cpu().reshape(-1).numpy() for t in (g, m, v))
    f = np.float32
    with np.errstate(all="ignore"):
        g = (g * f(scale)).astype(f)
        m = (m * f(betas[0])).astype(f) + (g * f(1 - betas[0])).astype(f)
        v = (v * f(betas[1])).astype(f) + ((g * g).astype(f) * f(1 - betas[1])).astype(f)
    return torch.from_numpy(m.astype(f)), torch.from_numpy(v.astype(f))


def _e4m3(code):
    """The number of an e4m3 code."""
    s, e, q = -1.0 if code & 128 else 1.0, code >> 3 & 15, code & 7
    return math.nan if code & 127 == 127 else s * (q / 8 * 2.0 ** -6 if e == 0 else (1 + q / 8) * 2.0 ** (e - 7))


E4M3 = torch.tensor([_e4m3(c) for c in range(256)], dtype=torch.float64)


def decode(m, v, exponents):
    """The numbers that codes stand for, from the definition."""
    n = m.numel()
    e = exponents.cpu().long().repeat_interleave(256, 0)[:n]
    em, ev = e[:, 0].clamp(min=8), e[:, 1].clamp(min=31)
    mf = E4M3[m.cpu().reshape(-1).long()] * torch.exp2(em.double() - 134)
    upper = v.cpu().reshape(-1).long()
    full = upper + 8 * (ev - 31)                     # upper 12 bits of a float32: 8 of exponent, 3 of mantissa
    field, q = full >> 3, (full & 7).double() / 8
    vf = torch.where(field > 0, (1 + q) * torch.exp2(field.double() - 127), q * 2.0 ** -126)
    vf = torch.where(upper > 0, vf, torch.zeros_like(vf))
    return torch.where(em == 255, torch.nan, mf), torch.where(ev == 255, torch.nan, vf)


def held(m, v):
    """What is left of moments (float32) once they are held in 8 bits: nearest numbers of the two grids, even codes on ties."""
    outs = []
    for x, first in ((m, True), (v, False)):
        n = x.numel()
        y = torch.zeros((n + 255) // 256 * 256, dtype=torch.float64)
        y[:n] = x.double()
        y = y.view(-1, 256)
        bad = ~torch.isfinite(y).all(1, keepdim=True)
        y = torch.where(bad, torch.zeros_like(y), y)

        def nearest(y, least, bits=3):               # least: the exponent below which steps no longer shrink
            step = torch.exp2((torch.frexp(y.abs()).exponent.double() - 1).clamp(min=least) - bits)
            return torch.round(y / step) * step
        top = y.abs().amax(1, keepdim=True)
        if first:
            unit = torch.exp2((torch.frexp(top).exponent.double() - 1 + 127).clamp(min=8) - 134)
            z = nearest(y / unit, -6) * unit
        else:
            z = nearest(y, -126)
            big = torch.frexp(z.amax(1, keepdim=True)).exponent.double() - 1 + 127
            big = torch.where(z.amax(1, keepdim=True) > 0, big, torch.zeros_like(big))       # (frexp has exponent 0 for 0, as for 0.5)
            base = (big.clamp(min=31) - 31)
            least = torch.where(base > 0, 1.125 * torch.exp2(base - 127), torch.full_like(base, 2.0 ** -129))
            z = torch.where(y > 0, torch.maximum(z, least), torch.zeros_like(z))
        outs.append(torch.where(bad, torch.nan, z).reshape(-1)[:n])
    return outs
