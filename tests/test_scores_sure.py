"""Rows that are sure of one entry, and gradients of entries whose probability float32 no longer holds as a normal number, on the GPU against 64 bits."""
import math

import numpy as np
import pytest
import torch

import scores_reference as ref
import test_scores as scores

pytestmark = pytest.mark.gpu


def _sure(rows, n, raise_by, scale, seed):
    """Normal scores, one of which lies raise_by (of the exponent) above the next."""
    g = scores._gen(seed)
    z = torch.randn(rows, n, generator=g, device="cuda")
    at = torch.randint(n, (rows, 1), generator=g, device="cuda")
    return (z / scale).scatter(1, at, z.amax(1, keepdim=True) / scale + raise_by / scale), at


@pytest.mark.parametrize("dtype", scores.TYPES)
@pytest.mark.parametrize("rows,n", [(2000, 64), (200, 4096), (3, 140001)])
def test_no_log_probability_is_above_zero(rows, n, dtype):
    """The best entry's term of the sum is 1 and no other is negative: ln sum is not below 0, ln p not above."""
    hr = scores._hr()
    for raise_by in (16.0, 24.0, 40.0):
        scores._say("sure", rows, n, dtype, raise_by)
        z, at = _sure(rows, n, raise_by, 1.0, n)
        z = (z + 30 * torch.randn(rows, 1, generator=scores._gen(1), device="cuda")).to(dtype)
        r = hr.logprobs(z, at, k=2)
        assert float(r.norm[:, 1].min()) >= 0 and float(r.logprobs.max()) <= 0 and float(r.top_logprobs.max()) <= 0
        assert float(r.entropy.min()) >= 0
        logp, p, m, logsum = ref.parts(z, 1.0)
        ref.close(r.logprobs, logp.gather(1, at), ref.logp_error(logp, logsum, 1.0, n).gather(1, at), torch.float32)
        loss, norm, _ = hr.distill_forward(z, at, torch.zeros(rows, 1, device="cuda"))
        assert float(norm[:, 1].min()) >= 0 and float(loss.min()) >= 0


def _entropy_gradient(z, scale, gh):
    """-s H' p (ln p + H) in 64 bits, and how far float32 may lie from it.  p is off by the sum's error and 8 units of its exponent;
    ln p + H is a difference in which ln sum cancels: each part by as many roundings, and the sum of p ln p by those of its terms' exponents.
    Nothing of it is a unit of 1: a row that is sure of an entry has ln p + H near 0 there, and that is what its gradient is."""
    logp, p, m, logsum = ref.parts(z, float(np.float32(scale)))
    h = ref.entropy(logp, p)[:, None]
    lnp = torch.where(p > 0, logp, torch.zeros_like(logp))
    rel = float(ref.sum_error(z.shape[1])) + ref.U * (16 + 8 * float(logsum.max()))
    part = scale * gh.double()[:, None].abs() * p
    tol = part * ((lnp.abs() + h) * (rel + 8 * ref.U * lnp.abs()) + 8 * ref.U * (p * lnp * lnp).sum(1, keepdim=True))
    return -scale * gh.double()[:, None] * p * (lnp + h), tol


@pytest.mark.parametrize("raise_by", [8.0, 12.0, 16.0, 20.0, 24.0])
@pytest.mark.parametrize("rows,n,scale", [(5, 64, 1.0), (7, 4096, 1.0), (3, 32003, 0.5), (1100, 2050, 2.0), (2, 140001, 1.0)])
def test_entropy_gradient_of_rows_that_are_sure(rows, n, scale, raise_by):
    hr = scores._hr()
    scores._say("sure", rows, n, scale, raise_by)
    z, at = _sure(rows, n, raise_by, scale, n)
    gh = torch.randn(rows, generator=scores._gen(rows), device="cuda")
    r = hr.logprobs(z, at, scale=scale)
    got = hr.logprobs_backward(z, None, r, None, gh, scale=scale)
    want, tol = _entropy_gradient(z, scale, gh)
    ref.close(got, want, tol, torch.float32)
    # as a share of the row's largest element, which is what a step of an optimiser sees
    off = (got.double() - want).abs().amax(1) / want.abs().amax(1)
    assert float(off.max()) < 2 * (ref.sum_error(n) + ref.U * (40 + 16 * raise_by)), float(off.max())


@pytest.mark.parametrize("dtype", scores.TYPES)
@pytest.mark.parametrize("n", [40, 3000])
def test_gradients_of_unlikely_entries(n, dtype):
    """p from 2^-120 to 2^-240 under coefficients of up to 2^125: products of both that float32 holds are not lost."""
    hr = scores._hr()
    scores._say("unlikely", n, dtype)
    g = scores._gen(n)
    ln2 = math.log(2.0)
    z = torch.zeros(9, n, device="cuda")
    z[:, 1:] = -ln2 * torch.randint(110, 241, (9, n - 1), generator=g, device="cuda").float()
    z[1, 1:] = -ln2 * 126.0                                # at the smallest normal number, and just below
    z[2, 1:] = -ln2 * 126.3
    z[3, 5:] = -math.inf
    z = z.to(dtype)
    ids = torch.zeros(9, 1, dtype=torch.int64, device="cuda")
    teacher = torch.zeros(9, 1, device="cuda")
    weights = torch.tensor([2.0 ** 100, 1.0, 1.0, 2.0 ** 125, 2.0 ** 60, -1.0, 2.0 ** -20, 2.0 ** 125, -(2.0 ** 90)], device="cuda")
    loss, loss_tol, want, tol = ref.distill(z, 1.0, ids, teacher, weights)
    # (of the listed entry, whose p rounds to 1, the difference from q is a rounding of either)
    tol[:, 0] += 4 * ref.U * weights.double().abs()
    got_loss, got = hr.distill_step(z, ids, teacher, weights)
    ref.close(got, want, tol, dtype)
    _, norm, q = hr.distill_forward(z, ids, teacher)
    ref.close(hr.distill_backward(z, ids, q, norm, weights), want, tol, dtype)
    r = hr.logprobs(z, ids)
    ref.close(hr.logprobs_backward(z, ids, r, weights[:, None], torch.zeros(9, device="cuda")),
              *ref.logprobs_grad(z, 1.0, ids, weights[:, None], torch.zeros(9, device="cuda")), dtype)
    assert not got[3, 5:].any()


def test_no_entry_depends_on_its_neighbours():
    """The same scores beside -inf, beside likely ones and at other places of a chunk of 16 bytes: the same bits of gradient."""
    hr = scores._hr()
    n = 4001
    z = torch.randn(4, n, generator=scores._gen(1), device="cuda") * 30
    ids = torch.randint(n, (4, 5), generator=scores._gen(2), device="cuda")
    teacher = torch.randn(4, 5, generator=scores._gen(3), device="cuda")
    _, norm, q = hr.distill_forward(z, ids, teacher)
    want = hr.distill_backward(z, ids, q, norm)
    for before in (1, 2, 3):
        assert torch.equal(hr.distill_backward(scores._strided(z, before, 5, -math.inf)[0], ids, q, norm), want)
    hole = z.clone()
    holes = torch.arange(n, device="cuda") % 3 == 1
    holes = holes[None, :].repeat(4, 1).scatter(1, ids, False) & (z < z.amax(1, keepdim=True))
    hole[holes] = -math.inf
    got = hr.distill_backward(hole, ids, q, norm)
    assert torch.equal(got[~holes], want[~holes]) and not got[holes].any()
