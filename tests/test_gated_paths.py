"""Every kernel of the gated blocks' tiles: which shape takes which (host arithmetic, no GPU), and all numbers of those shapes against 64 bits."""
import math

import pytest
import torch

import layers_reference as ref
from test_tile_plan import _whole, plan  # noqa: F401  (a fixture)

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16

# tokens, columns, hidden
SHAPES_16 = [(40, 768, 96), (40, 2048, 96), (64, 72, 96), (40, 1100, 2100), (40, 64, 40000), (64, 72, 40000), (64, 64, 70000), (64, 72, 70000), (100, 72, 96), (300, 64, 96), (300, 72, 6152),
             (300, 64, 6152), (300, 72, 12000), (300, 64, 12000), (40, 136, 9000), (1100, 1536, 96), (777, 136, 12000), (777, 136, 40000), (4100, 768, 1333), (4100, 4160, 296), (1024, 4040, 2072), (5000, 72, 6152),
             (1500, 200, 4104), (2050, 768, 2100), (1500, 64, 40000), (2050, 2048, 4104)]
SHAPES_32 = [(40, 768, 96), (40, 200, 96), (64, 72, 96), (64, 64, 96), (64, 64, 640), (40, 136, 96), (40, 64, 40000), (64, 72, 40000), (64, 64, 70000), (64, 72, 70000), (100, 72, 96), (100, 64, 96),
             (300, 72, 6152), (300, 64, 6152), (300, 72, 12000), (300, 64, 12000), (40, 520, 2100), (2050, 1100, 2100), (1100, 200, 9000)]


def _launches(tiles, parts, products, gated, tail):
    """What a plan launches: tiles (rows, buffers, whether rows are no whole blocks, whether workgroups take more than one), joins (shares), rows left to small tiles."""
    found = set()

    def launch(bm, bn, some):
        counts = [-(-m // bm) * -(-n // (bn // 2 if gated else bn)) * n_parts for m, n, n_parts in some]
        few = sum(counts) <= 256
        buffers = {256: 2, 128: 4 if few else 2, 64: 3 if few else 2}[bm]
        places = 512 if (bm + bn) * 128 * buffers <= 80 * 1024 else 256
        found.add((bm, buffers, tail, buffers == 2 and max(counts) > places))
        most = max(n_parts for _, _, n_parts in some)
        if most > 1:
            found.add(("join", 16 if most >= 12 else 4 if most >= 4 else 1))
    first = [(large, n, n_parts) for (n_parts, _, large), (m, n, _) in zip(parts, products) if large > 0]
    rest = [(m - large, n, n_parts) for (n_parts, _, large), (m, n, _) in zip(parts, products) if large < m]
    if first:
        launch(*tiles, first)
    if rest:
        launch(128, 128, rest)
        found.add("rest" if first else "all in small tiles")
    return found


def _taken(plan, m, k, f, es):  # noqa: F811
    """Of the forward pass, and of the gradients."""
    row = _whole(k, es)
    forward = [(-(-m // 64) * 64, f, row)]
    mp = _whole(m, es) // es
    backward = [(mp, k, 2 * _whole(f, es)), (2 * f, k, mp * es)]
    tail = (k * es) % 16 == 0 and k * es < row                # (rows of no whole 16 bytes are copied to whole blocks)
    return _launches(*plan(1, es, *forward), forward, True, tail), _launches(*plan(0, es, *backward), backward, False, False)


def test_every_kernel_is_taken(plan):  # noqa: F811
    for es, shapes in ((2, SHAPES_16), (4, SHAPES_32)):
        forward, backward = (set().union(*x) for x in zip(*(_taken(plan, m, k, f, es) for m, k, f in shapes)))
        joins = {("join", n) for n in (1, 4, 16)}
        small = {(128, 4, False, False), (128, 2, False, False), (128, 2, False, True)}
        tails = {(bm, buffers, True, more) for bm, buffers, _, more in small}
        flat = {(64, 3, tail, False) for tail in (False, True)} | {(64, 2, tail, more) for tail in (False, True) for more in (False, True)}
        large = {(256, 2, False, False), (256, 2, False, True)} if es == 2 else set()
        long = {(256, 2, True, more) for _, _, _, more in large}
        left = {"rest"} if es == 2 else set()
        assert forward >= joins | small | tails | flat | large | long | left, (joins | small | tails | flat | large | long | left) - forward
        assert backward >= joins | small | large | left, (joins | small | large | left) - backward


# ---- on the GPU, 64-bit products too

def _close(got, want, tol, dtype):
    """As layers_reference.close, of finite numbers, where they are."""
    off = (got.double() - want).abs() - tol * (1 + 2 * ref.EPS[dtype]) - ref.EPS[dtype] * want.abs() - ref.TINY[dtype]
    assert bool(got.isfinite().all()) and float(off.max()) <= 0, f"{float(off.max()):.3e} too much"


def _check(m, k, f, dtype, act):
    import paper_2507_09138_amd as hr
    print("case", m, k, f, dtype, act, flush=True)
    U = ref.U
    g = torch.Generator(device="cuda")
    g.manual_seed(m + k + f)

    def some(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    x, wg, wu, dh = some(m, k).to(dtype), (some(f, k) / math.sqrt(k)).to(dtype), (some(f, k) / math.sqrt(k)).to(dtype), some(m, f).to(dtype)
    got = hr.gated(x, wg, wu, act, keep=True)
    d = hr.gated_backward(x, wg, wu, got.pre, dh, act)
    x6, wg6, wu6, dh6 = (t.double() for t in (x, wg, wu, dh))
    gate, up = x6 @ wg6.T, x6 @ wu6.T
    tols = [(k + 4) * U * (x6.abs() @ w.abs().T) for w in (wg6, wu6)]
    a, _ = ref.act(gate, act)
    a_tol = 1.13 * tols[0] + 8 * U * (a.abs() + gate.abs())
    _close(got.out, a * up, a_tol * (up.abs() + tols[1]) + a.abs() * tols[1] + 2 * U * (a * up).abs(), dtype)
    for i, (v, t) in enumerate(((gate, tols[0]), (up, tols[1]))):
        _close(got.pre[:, i], v, t, F32)
    # the gradients from gate and up as they were kept
    gate, up = got.pre.double().unbind(1)
    a, slope = ref.act(gate, act)
    dg, du = dh6 * up * slope, dh6 * a
    dg_tol = 16 * U * (dh6 * up).abs() * (1 + gate.abs()) + ref.EPS[dtype] * dg.abs() + ref.TINY[dtype]
    du_tol = 8 * U * dh6.abs() * (a.abs() + gate.abs()) + ref.EPS[dtype] * du.abs() + ref.TINY[dtype]
    tol = dg_tol @ wg6.abs() + du_tol @ wu6.abs() + (2 * f + 4) * U * ((dg.abs() + dg_tol) @ wg6.abs() + (du.abs() + du_tol) @ wu6.abs())
    _close(d.x, dg @ wg6 + du @ wu6, tol, dtype)
    for have, v, t in ((d.w_gate, dg, dg_tol), (d.w_up, du, du_tol)):
        _close(have, v.T @ x6, t.T @ x6.abs() + (m + 4) * U * (v.abs() + t).T @ x6.abs(), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("m,k,f", SHAPES_16)
def test_in_16_bits(m, k, f, dtype):
    _check(m, k, f, dtype, ["silu", "gelu", "gelu_tanh"][(m + k + f) % 3])


@pytest.mark.gpu
@pytest.mark.parametrize("m,k,f", SHAPES_32)
def test_in_32_bits(m, k, f):
    _check(m, k, f, F32, ["silu", "gelu", "gelu_tanh"][(m + k + f) % 3])
