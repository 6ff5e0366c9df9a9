"""The operators of hr_scores.h in 64 bits, written from their definitions, and how far 32-bit sums may lie from them."""
import numpy as np
import torch

U = 2.0 ** -24                                     # half a unit in the last place of float32
EPS = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}       # rounding to the type, relative
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}   # its smallest number


def quantize(x):
    """x [m, k]: (int8 [m, k], float32 [m]) with both quotients rounded to float32, as numpy rounds them."""
    x = x.float().cpu().numpy()
    bad = ~np.isfinite(x).all(1)
    with np.errstate(all="ignore"):
        scale = (np.abs(np.where(np.isfinite(x), x, 0)).max(1) / np.float32(127)).astype(np.float32)
        q = np.rint((x / np.where(scale > 0, scale, np.float32(1))[:, None]).astype(np.float32))
    q[bad | (scale == 0)] = 0
    scale[bad] = np.nan
    return torch.from_numpy(q.astype(np.int8)), torch.from_numpy(scale)


def product(a, a_scale, b, b_scale, bias):
    """In 64 bits, and what 32-bit scaling of the exact sum may differ by (before the output's rounding)."""
    v = (a.double() @ b.double().T) * a_scale.double()[:, None] * b_scale.double()
    tol = 4 * U * v.abs()                          # float32 of the sum, two products, the sum with the bias
    if bias is not None:
        v = v + bias.double()
        tol = tol + 4 * U * bias.double().abs()
    return v, tol


def close(got, want, tol, dtype):
    """got (rounded to dtype) within tol of want; NaN and infinities in the same places."""
    got, want = got.double().cpu(), want.double().cpu()
    beyond = torch.isinf(want.to(dtype))               # (more than the type holds)
    want = torch.where(beyond, want.sign() * np.inf, want)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fin].nan_to_num(7.0), want[~fin].nan_to_num(7.0))
    tol = torch.as_tensor(tol, dtype=torch.float64).cpu().expand_as(want)
    # (rounding what is tol away from want: eps of the larger of both)
    off = (got - want).abs() - tol * (1 + 2 * EPS[dtype]) - EPS[dtype] * want.abs() - TINY[dtype]
    off = torch.where(fin, off, torch.zeros_like(off))
    assert float(off.max()) <= 0, f"off by {float((got - want)[fin].abs().max()):.3e}, {float(off.max()):.3e} too much"


def parts(z, scale):
    """(ln p, p, m, ln sum) of rows in 64 bits; a row without candidates has p = 0."""
    z = z.double()
    m = z.max(1, keepdim=True).values
    there = m > -np.inf
    a = (z - torch.where(there, m, torch.zeros_like(m))) * scale
    total = torch.exp(a).sum(1, keepdim=True)
    logsum = torch.where(there, torch.log(total), torch.zeros_like(total))
    logp = a - logsum
    return logp, torch.exp(logp), m[:, 0], logsum[:, 0]


def entropy(logp, p):
    return -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1) + 0.0 * logp.nan_to_num(neginf=0.0).sum(1)


def at(logp, ids):
    there = (ids >= 0) & (ids < logp.shape[1])
    return torch.where(there, torch.gather(logp, 1, torch.where(there, ids, torch.zeros_like(ids))), torch.full_like(logp[:, :1], -np.inf))


def best(z, k):
    """Entries of the k best candidates, equal scores by entry; -1 where there are fewer."""
    v, i = torch.sort(z.double(), dim=1, descending=True, stable=True)
    v, i = v[:, :k], i[:, :k]
    i = torch.where(v == -np.inf, torch.full_like(i, -1), i)
    return torch.nn.functional.pad(i, (0, k - i.shape[1]), value=-1)


def sum_error(n):
    """Relative error of a sum over a row in float32: at most n / 64 + 32 additions one after the other (a wave at least
    shares a row, and merges what its lanes have), and 4 of each term's exponential."""
    return (n / 64 + 36) * U


def logp_error(logp, logsum, scale, n):
    """Of ln p = scale (z - m) - ln sum: two roundings of the first part, the sum's error in the second; every term's exponent
    is off by three roundings of its size, and |x| exp(x) summed is at most ln sum + 1 of the sum."""
    return U * (4 + 4 * logp.nan_to_num(neginf=0.0).abs() + 8 * (logsum[:, None] + 1)) + sum_error(n)


def entropy_error(logsum, n):
    """Two terms that each have the relative error of a sum, the second of which is at most ln sum."""
    return (2 * logsum + 2) * (sum_error(n) + U * (16 + 8 * logsum))


def logprobs_grad(z, scale, given, grad_logprobs, grad_entropy):
    """Gradient by the formula, and what it may be off by before its rounding to the type."""
    logp, p, m, logsum = parts(z, scale)
    h = entropy(logp, p)
    n = z.shape[1]
    rel = float(sum_error(n)) + U * (16 + 8 * float(logsum.max()))
    g = torch.zeros_like(p)
    size = torch.zeros_like(p)
    lp = at(logp, given)
    G = torch.where(lp > -np.inf, grad_logprobs.double(), torch.zeros_like(lp))
    g.scatter_add_(1, given.clamp(0, n - 1), G)
    size.scatter_add_(1, given.clamp(0, n - 1), G.abs())
    g -= p * G.sum(1, keepdim=True)
    size += p * G.abs().sum(1, keepdim=True)
    lnp = torch.where(p > 0, logp, torch.zeros_like(logp))
    he = grad_entropy.double()[:, None]
    g -= he * p * (lnp + h[:, None])
    size += he.abs() * p * (lnp.abs() + h[:, None] + 1)
    # (an exponent x is off by 4 U |x|, and so is p)
    return scale * g, scale * size * (rel + 8 * U * lnp.abs())


def distill(z, scale, ids, teacher, weights):
    """(loss, its error, gradient, its error) by the formula."""
    logp, p, m, logsum = parts(z, scale)
    n = z.shape[1]
    lp = at(logp, ids)
    t = teacher.double()
    counts = (lp > -np.inf) & (t > -np.inf)
    some = counts.any(1, keepdim=True)
    t = torch.where(counts, t * scale, torch.full_like(t, -np.inf))
    t = t - torch.where(some, t.max(1, keepdim=True).values, torch.zeros_like(t[:, :1]))
    total = torch.where(some, torch.exp(t).sum(1, keepdim=True), torch.ones_like(t[:, :1]))
    logq = t - torch.log(total)
    q = torch.where(counts, torch.exp(logq), torch.zeros_like(t))
    lq, ls = torch.where(counts, logq, torch.zeros_like(t)), torch.where(counts, lp, torch.zeros_like(t))
    loss = (q * (lq - ls)).sum(1)
    rel = float(sum_error(n)) + U * (16 + 8 * float(logsum.max()))
    loss_tol = (q * (rel + U * 16 * (1 + lq.abs() + ls.abs()) + U * ids.shape[1])).sum(1) + U * ids.shape[1] * (q * (lq - ls).abs()).sum(1)
    w = (weights.double() * scale)[:, None]
    g = p.clone()
    g.scatter_add_(1, ids.clamp(0, n - 1), -q)
    size = p.clone().scatter_add_(1, ids.clamp(0, n - 1), q)
    g = torch.where(some & (w != 0) & (z > -np.inf), g * w, torch.zeros_like(g))
    lnp = torch.where(p > 0, logp, torch.zeros_like(logp)).abs()
    # (exponents of the teacher's scores are off by their size as well)
    at_ids = torch.zeros_like(p).scatter_add_(1, ids.clamp(0, n - 1), q * (8 * U * lq.abs() + U * ids.shape[1]))
    return loss, loss_tol, g, w.abs() * (size * (rel + 8 * U * lnp) + at_ids)
