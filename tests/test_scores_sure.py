"""Rows that are sure of one entry, on the GPU against 64 bits."""
import math

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
