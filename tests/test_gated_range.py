"""Gradients of gated blocks in binary16 whose steps in between lie outside of the type's range while their results lie inside it."""
import math

import pytest
import torch

import layers_reference as ref

pytestmark = pytest.mark.gpu
F16, INF, NAN = torch.float16, math.inf, math.nan


def _hr():
    import paper_2507_09138_amd as hr
    return hr


def _randn(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def _grads(x, wg, wu, pre, dh, name):
    """As layers_reference.gated_grads, with nothing but the roundings: d_gate and d_up are rounded relative to their own size (2^-11), and to no more than
    2^-39 of the largest of their row (the gradient of x) or of their column (the matrices'): 2^-25, half of the type's smallest step, of 2^14."""
    x, wg, wu, dh = (t.double().cpu() for t in (x, wg, wu, dh))
    gate, up = pre.double().cpu().unbind(1)
    a, slope = ref.act(gate, name)
    dg, du = dh * up * slope, dh * a
    m, f = dg.shape
    off = [16 * ref.U * (dh * up).abs() * (1 + gate.abs()), 8 * ref.U * dh.abs() * (a.abs() + gate.abs())]
    row = torch.maximum(dg.abs().amax(1, keepdim=True), du.abs().amax(1, keepdim=True)) * 2.0 ** -39
    own = [o + 2.0 ** -11 * d.abs() * 1.001 for o, d in zip(off, (dg, du))]
    tols = [t + row for t in own]
    dx_tol = sum(t @ w.abs() + (2 * f + 4) * ref.U * (d.abs() + t) @ w.abs() for t, d, w in zip(tols, (dg, du), (wg, wu)))
    dw_tol = []
    for t, d in zip(own, (dg, du)):
        t = t + d.abs().amax(0, keepdim=True) * 2.0 ** -39
        dw_tol.append(t.T @ x.abs() + (m + 4) * ref.U * (d.abs() + t).T @ x.abs())
    return (dg @ wg + du @ wu, dg.T @ x, du.T @ x), (dx_tol, *dw_tol), (dg, du)


SHAPES = [(1, 40, 24), (5, 64, 64), (70, 129, 97), (300, 200, 130), (40, 72, 1100)]


def _inputs(m, k, f, seed, level_dh, level_pre, level_x, level_w):
    x = (_randn(seed, m, k) * level_x).half()
    wg, wu = ((_randn(seed + i, f, k) * level_w / math.sqrt(k)).half() for i in (1, 2))
    pre = _randn(seed + 3, m, 2, f)
    pre[:, 1] *= level_pre
    return x, wg, wu, pre, (_randn(seed + 4, m, f) * level_dh).half()


def _check(x, wg, wu, pre, dh, act):
    got = _hr().gated_backward(x, wg, wu, pre, dh, act)
    want, tols, between = _grads(x, wg, wu, pre, dh, act)
    for g, w, t in zip(got, want, tols):
        ref.close(g, w, t, F16)
    return got, want, between


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("m,k,f", SHAPES)
def test_beyond_the_largest_number(m, k, f, act):
    """grad_out * up * act' of a million and more, results of hundreds."""
    ins = _inputs(m, k, f, m + k, 4000.0, 1000.0, 2.0 ** -14, 2.0 ** -13)
    _, want, between = _check(*ins, act)
    assert float(between[0].abs().max()) > 65504 and all(float(w.abs().max()) < 60000 for w in want)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("m,k,f", SHAPES)
def test_below_the_smallest_number(m, k, f, act):
    """grad_out * up * act' below 2^-25, which rounds to 0, results that are normal numbers."""
    ins = _inputs(m, k, f, m + k + 9, 2.0 ** -19, 2.0 ** -12, 2.0 ** 14, 2.0 ** 14)
    _, want, between = _check(*ins, act)
    assert float(between[0].abs().max()) < 2.0 ** -25


@pytest.mark.parametrize("m,k,f", SHAPES[1:])
def test_rows_and_columns_of_all_sizes(m, k, f):
    """Each row of grad_out and each column of up with a size of its own, from one end of the range to the other."""
    x, wg, wu, pre, dh = _inputs(m, k, f, m + k + 20, 1.0, 1.0, 2.0 ** -10, 2.0 ** -10)
    dh = (dh.float() * torch.exp2(torch.linspace(-14, 12, m, device="cuda"))[:, None]).half()
    pre = pre * torch.exp2(torch.linspace(-12, 12, f, device="cuda").roll(f // 3))
    _check(x, wg, wu, pre, dh, "silu")
    z = torch.zeros_like(dh)                                # nothing to scale
    got = _hr().gated_backward(x, wg, wu, pre, z)
    assert not any(bool(t.any()) for t in got)


@pytest.mark.parametrize("m,k,f", SHAPES[1:])
def test_what_is_no_number_stays_in_its_row(m, k, f):
    x, wg, wu, pre, dh = _inputs(m, k, f, m + k + 30, 4000.0, 1000.0, 2.0 ** -14, 2.0 ** -13)
    want = _hr().gated_backward(x, wg, wu, pre, dh)
    dh[m - 1, f - 1], dh[m // 2, 0] = NAN, INF
    got = _hr().gated_backward(x, wg, wu, pre, dh)
    fine = [i for i in range(m) if i not in (m - 1, m // 2)]
    assert torch.equal(got.x[fine], want.x[fine]) and got.x[m - 1].isnan().all() and not got.x[m // 2].isfinite().any()
    for g, w in zip(got[1:], want[1:]):
        assert torch.equal(g[1:-1], w[1:-1]) and g[-1].isnan().all() and not g[0].isfinite().any()
