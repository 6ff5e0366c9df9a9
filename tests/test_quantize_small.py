"""Quantised rows so small that their scale has few bits left, or none."""
import numpy as np
import pytest
import torch

import test_scores as scores

pytestmark = pytest.mark.gpu


def _definition(x):
    """Scale and quotient rounded to float32 as numpy rounds them, the whole number limited to what 8 bits of both signs hold alike."""
    x = x.float().cpu().numpy()
    scale = (np.abs(x).max(1) / np.float32(127)).astype(np.float32)
    with np.errstate(all="ignore"):
        q = np.rint((x / np.where(scale > 0, scale, np.float32(1))[:, None]).astype(np.float32))
    q[scale == 0] = 0
    return torch.from_numpy(np.clip(q, -127, 127).astype(np.int8)), torch.from_numpy(scale)


@pytest.mark.parametrize("k", [1, 50, 64, 200, 1000, 5000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_the_smallest_numbers(k, dtype):
    """Largest magnitudes of N times the type's smallest number: 190 of float32's are 1.496 scales of one of them, 190 quotients."""
    hr = scores._hr()
    scores._say("small", k, dtype)
    unit = 2.0 ** -149 if dtype is torch.float32 else 2.0 ** -133
    largest = [1, 2, 60, 63, 64, 65, 100, 127, 128, 150, 189, 190, 191, 200, 254, 300, 317, 318, 444, 5000, 20000, 16400, 100000]
    largest = [n for n in largest if dtype is torch.float32 or n <= 127]           # (bfloat16 has seven bits there)
    x = torch.empty(len(largest), k, dtype=torch.float64)
    g = torch.Generator().manual_seed(k)
    for r, n in enumerate(largest):
        x[r] = torch.randint(-n, n + 1, (k,), generator=g).double() * unit
        x[r, k // 2] = n * unit * (1 if r % 2 else -1)
    x = x.to(dtype).cuda()
    want, scale = _definition(x)
    assert int(scale.count_nonzero()) < len(scale) or dtype is torch.bfloat16
    q, s = hr.quantize_rows(x)
    assert torch.equal(s.cpu(), scale)
    assert torch.equal(q.cpu(), want)
    assert torch.equal(torch.sign(q.float()) * torch.sign(x.float()) < 0, torch.zeros_like(q, dtype=torch.bool))
    # the launch that quantises up to 16 rows by itself, and the one that does not
    w, ws = hr.quantize_rows(torch.randn(40, k, generator=scores._gen(3), device="cuda"))
    ws = torch.exp2(torch.arange(40, device="cuda").float()) * 2.0 ** 60
    for lo in range(0, len(largest), 8):
        part = x[lo:lo + 8].contiguous()
        assert torch.equal(hr.i8_linear(part, w, ws), hr.i8_product(q[lo:lo + 8], s[lo:lo + 8], w, ws))
