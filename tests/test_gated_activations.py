"""The activations of gated blocks by themselves: x = (z, 1), w_gate = (1, 0), w_up = (0, 1) give act(z) and, of a gradient of ones, the slope and act(z) again,
with no other rounding."""
import math

import pytest
import torch

import layers_reference as ref

pytestmark = pytest.mark.gpu
U = ref.U


def _values(z, act):
    """act(z), and by the gradients (slope, act(z)); in z's type."""
    import paper_2507_09138_amd as hr
    x = torch.stack([z, torch.ones_like(z)], 1)
    wg, wu = (torch.tensor([w], dtype=z.dtype, device="cuda") for w in ((1.0, 0.0), (0.0, 1.0)))
    r = hr.gated(x, wg, wu, act, keep=True)
    assert torch.equal(r.pre[:, 0, 0], z.float()) and bool((r.pre[:, 1, 0] == 1).all())
    d = hr.gated_backward(x, wg, wu, r.pre, torch.ones_like(r.out), act).x
    return r.out[:, 0], d[:, 0], d[:, 1]


def _grid(rows, lo, hi):
    """Numbers from one end to the other, and small ones of both signs."""
    small = torch.logspace(-30, 0, rows // 4, dtype=torch.float64)
    return torch.cat([torch.linspace(lo, hi, rows - 2 * (rows // 4), dtype=torch.float64), small, -small]).float().cuda()


@pytest.mark.parametrize("rows", [30, 20000])
def test_gelu_in_32_bits(rows):
    """Relative to itself, also where it is small.  Below -1: the reciprocal and its argument 3 U, of which up to 1.84 times as much gets into the polynomial's
    value, its fit and coefficients 1.9, its sums 2, three products 3, the exponential 4: 16.4.  -1 .. 1: 2 U of what is added to 1 / 2, at most 0.35, the sum and a
    product 2 U, of 0.158 at least: 6.3.  Above 1: what 1 loses is at most 0.159 off by 16.4 U, and 2 U: 5.2.  The slope, absolute: 0.159 of 16.4 U and 1, 0.242 of
    the 6 U of exponential and products, and the sum's 1: 6.1."""
    z = _grid(rows, -12.9, 9.0)
    value, slope, again = _values(z, "gelu")
    want, want_slope = ref.act(z.double().cpu(), "gelu")
    tol = torch.where(z.cpu() < 0, 17.0, 6.0).double() * U * want.abs()
    ref.close(value, want, tol, torch.float32)
    ref.close(again, want, tol, torch.float32)
    ref.close(slope, want_slope, 7 * U, torch.float32)


@pytest.mark.parametrize("rows", [30, 20000])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_gelu_in_16_bits(dtype, rows):
    """Off by no more than its rounding, and what 32 bits are off by."""
    z = _grid(rows, -12.9, 9.0).to(dtype)
    value, slope, again = _values(z, "gelu")
    want, want_slope = ref.act(z.double().cpu(), "gelu")
    ref.close(value, want, 17 * U * want.abs(), dtype)
    # (rounded as an operand and as a result)
    twice = 17 * U * want.abs() + ref.EPS[dtype] * want.abs() + ref.TINY[dtype]
    ref.close(again, want, twice, dtype)
    ref.close(slope, want_slope, 7 * U + ref.EPS[dtype] * want_slope.abs() + ref.TINY[dtype], dtype)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_far_and_no_numbers(act):
    import paper_2507_09138_amd as hr
    z = torch.tensor([40.0, 1e4, 1e18, 1e30, 3e38, -40.0, -1e4, -1e18, -1e30, -3e38, 0.0], device="cuda")
    value, slope, _ = _values(z, act)
    far = torch.tensor([1.0] * 5 + [0.0] * 5, device="cuda")
    assert torch.equal(value[:5], z[:5]) and (value[5:].abs() < 1e-15).all() and (slope[:10] - far).abs().max() < 1e-15 and slope[10] == 0.5
    one = torch.ones(1, 1, device="cuda")
    d = hr.gated_backward(one, one, one, torch.tensor([[[math.nan], [1.0]]], device="cuda"), one, act)
    assert d.x.isnan().all() and d.w_gate.isnan().all() and d.w_up.isnan().all()
