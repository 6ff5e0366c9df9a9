"""Layer norm, gated blocks and AdamW (hr_layers.h) on the GPU against 64-bit arithmetic of the same operands: sizes at which lanes, chunks,
tiles and blocks end, strides, special values, empty batches; in streams and graphs, and together as a training step uses them."""
import math

import pytest
import torch

import layers_reference as ref

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def _hr():
    import paper_2507_09138_amd as hr
    return hr


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(seed, *shape):
    return torch.randn(*shape, generator=_gen(seed), device="cuda")


def _say(*a):
    print("case", *a, flush=True)


def _strided(t, before, behind, fill):
    """The same matrix as a slice of columns of a wider one (rows start at odd places), and the wider one."""
    wide = torch.full((t.shape[0], before + t.shape[1] + behind), fill, dtype=t.dtype, device=t.device)
    view = wide[:, before:before + t.shape[1]]
    view.copy_(t)
    return view, wide


def _around(wide, before, n, fill):
    """Whether everything beside the slice is as it was."""
    return bool((wide[:, :before] == fill).all()) and bool((wide[:, before + n:] == fill).all())


# ---- layer norm

# where 16, 64, 256, 512 and 1024 lanes end, 8 or 4 elements each, and the rows that are held or not
NORM = [(1, 1), (5, 3), (33, 16), (17, 127), (40, 128), (7, 129), (19, 256), (70, 257), (3, 511), (9, 1000), (601, 768), (5, 1025), (4, 2047), (3, 2049),
        (6, 4096), (5, 4099), (3, 8192), (2, 8200), (3, 16384), (2, 16385), (3, 32769), (2, 70001), (1, 140000)]


def _norm_inputs(rows, n, dtype, weights):
    x = _randn(rows + n, rows, n) * torch.exp(0.5 * _randn(n, n)) + 2 * _randn(rows, rows, 1)
    w = None if weights is None else (1 + 0.3 * _randn(n + 1, n)).to(weights)
    b = None if weights is None else _randn(n + 2, n).to(weights)
    return x.to(dtype), w, b, _randn(n + 3, rows, n).to(dtype)


def _check_norm(x, w, b, dy, eps, got, grads, dtype):
    y, mean, rstd, _, y_tol, m_tol, r_tol = ref.norm(x, w, b, eps)
    ref.close(got.out, y, y_tol, dtype)
    ref.close(got.stats[:, 0], mean, m_tol, F32)
    ref.close(got.stats[:, 1], rstd, rstd * r_tol, F32)
    dx, dw, db, dx_tol, dw_tol, db_tol = ref.norm_grads(x, w, dy, eps)
    kind = F32 if w is None else w.dtype
    ref.close(grads.x, dx, dx_tol, dtype)
    ref.close(grads.weight, dw, dw_tol, kind)
    ref.close(grads.bias, db, db_tol, kind)
    assert got.out.dtype == grads.x.dtype == dtype and grads.weight.dtype == grads.bias.dtype == kind


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", NORM)
def test_norm_and_gradients(rows, n, dtype):
    hr = _hr()
    for weights, eps in ((F32, 1e-5), (dtype, 1e-2), (None, 1e-6)):
        _say("norm", rows, n, dtype, weights)
        x, w, b, dy = _norm_inputs(rows, n, dtype, weights)
        got = hr.layer_norm(x, w, b, eps)
        grads = hr.layer_norm_backward(x, w, got.stats, dy)
        _check_norm(x, w, b, dy, eps, got, grads, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(37, 100), (5, 1003), (3, 5001), (2, 20003), (2, 40001), (2, 140001)])
def test_norm_of_slices_and_in_place(rows, n, dtype):
    """Rows that begin anywhere, NaN beside them; results in the place of the inputs; what lies beside a result stays as it was."""
    hr = _hr()
    _say("norm slices", rows, n, dtype)
    x, w, b, dy = _norm_inputs(rows, n, dtype, F32)
    got = hr.layer_norm(x, w, b)
    grads = hr.layer_norm_backward(x, w, got.stats, dy)
    xs, xw = _strided(x, 3, 2, NAN)
    ys, yw = _strided(x, 1, 5, 7.0)
    ds, dw = _strided(dy, 5, 1, NAN)
    gs, gw = _strided(dy, 2, 3, 7.0)
    out = hr.layer_norm(xs, w, b, out=ys)
    assert out.out is ys and torch.equal(ys, got.out) and torch.equal(out.stats, got.stats) and _around(yw, 1, n, 7.0)
    again = hr.layer_norm_backward(xs, w, got.stats, ds, out=gs)
    assert torch.equal(gs, grads.x) and torch.equal(again.weight, grads.weight) and torch.equal(again.bias, grads.bias) and _around(gw, 2, n, 7.0)
    assert torch.equal(hr.layer_norm_backward(xs, w, got.stats, gs.copy_(dy), out=gs).x, grads.x) and _around(gw, 2, n, 7.0)
    assert torch.equal(hr.layer_norm(ys.copy_(x), w, b, out=ys).out, got.out) and _around(yw, 1, n, 7.0)
    less = hr.layer_norm_backward(x, w, got.stats, dy, parameters=False)
    assert less.weight is None and less.bias is None and torch.equal(less.x, grads.x)
    assert torch.equal(hr.layer_norm(x.T.contiguous().T, w, b).out, got.out)


@pytest.mark.parametrize("n", [50, 768, 5000, 40000])
def test_norm_far_from_zero(n):
    """A mean thousands of times the spread: what is left after it counts."""
    hr = _hr()
    x = 3000.0 + _randn(n, 6, n)
    x[3] *= 1e-3
    x[4] *= 1e6
    x[5] = -1e4 + 0.5 * _randn(n + 1, n)
    dy = _randn(n + 2, 6, n)
    got = hr.layer_norm(x)
    _check_norm(x, None, None, dy, 1e-5, got, hr.layer_norm_backward(x, None, got.stats, dy), F32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [20, 700, 3000, 17000, 40000])
def test_norm_of_rows_without_spread_and_without_numbers(n, dtype):
    hr = _hr()
    x = _randn(n, 9, n).to(dtype)
    x[1] = 0
    x[2] = 2.5
    x[4, n // 2] = NAN
    x[5, n - 1] = INF
    x[6, 0] = -INF
    w, b = 1 + _randn(n + 1, n), _randn(n + 2, n)
    got = hr.layer_norm(x, w, b)
    fine = torch.tensor([0, 1, 2, 3, 7, 8], device="cuda")
    alone = hr.layer_norm(x[fine], w, b)
    assert torch.equal(got.out[fine], alone.out) and torch.equal(got.stats[fine], alone.stats)
    assert got.out[4:7].isnan().all() and got.stats[4:7, 1].isnan().all()
    ref.close(got.out[1:3], b.double().expand(2, n), 0.0, dtype)
    y = ref.norm(x[fine], w, b, 1e-5)
    ref.close(alone.out, y[0], y[4], dtype)
    dy = _randn(n + 3, 9, n).to(dtype)
    dx = hr.layer_norm_backward(x, w, got.stats, dy).x
    assert torch.equal(dx[fine], hr.layer_norm_backward(x[fine], w, alone.stats, dy[fine]).x) and dx[4:7].isnan().all()
    dy[0, 3] = INF
    dy[7, 3] = NAN
    dx = hr.layer_norm_backward(x[fine], w, alone.stats, dy[fine]).x
    assert dx[0].isnan().any() and dx[4].isnan().all() and not dx[[1, 2, 3, 5]].isnan().any()


@pytest.mark.parametrize("n", [3, 67, 300, 768, 1500, 3000, 5000, 17000, 40000, 70001, 100000])
def test_norm_of_equal_numbers_far_from_zero(n):
    """Their spread is 0, but the first mean is off by a rounding, and the squares of what is left are larger than eps."""
    c = 10.0 ** (6 + 8 * torch.rand(200, generator=_gen(n), device="cuda"))
    x = (c * torch.sign(_randn(n + 1, 200)))[:, None].expand(200, n).contiguous()
    eps = 1e-5
    r = _hr().layer_norm(x, eps=eps)
    # K additions one after the other (160 at most here: 128 of a lane and the folds): the first mean is within K u |c| of c, what is left is exact, its
    # mean within K u of itself; so what is divided by the spread is within (K u)^2 |c| of 0, and the spread is at least sqrt eps
    bound = (162 * 2.0 ** -24) ** 2 * c / math.sqrt(eps) * 1.01
    assert torch.isfinite(r.out).all()
    assert (r.out.abs() <= bound[:, None]).all()
    assert (r.stats[:, 1] > 0).all() and (r.stats[:, 1] <= 1.0001 / math.sqrt(eps)).all()
    # one of them next to the others: the spread is far below what its square is off by
    x[:, 0] = torch.nextafter(x[:, 0], torch.zeros_like(x[:, 0]))
    r = _hr().layer_norm(x, eps=eps)
    assert torch.isfinite(r.out).all() and torch.isfinite(r.stats).all()
    g = _hr().layer_norm_backward(x, None, r.stats, torch.ones(200, n, device="cuda"))
    assert torch.isfinite(g.x).all()


def test_norm_without_rows_and_many_rows():
    hr = _hr()
    for n in (5, 3000, 40000):
        x, w = torch.empty(0, n, device="cuda"), torch.ones(n, device="cuda")
        r = hr.layer_norm(x, w)
        assert r.out.shape == (0, n) and r.stats.shape == (0, 2)
        g = hr.layer_norm_backward(x, w, r.stats, x)
        assert g.x.shape == (0, n) and torch.equal(g.weight, torch.zeros(n, device="cuda")) and torch.equal(g.bias, torch.zeros(n, device="cuda"))
    for rows, n in ((70000, 20), (9000, 513)):              # more rows than workgroups, or than what they hold at once
        x, w, b, dy = _norm_inputs(rows, n, BF16, F32)
        got = hr.layer_norm(x, w, b)
        _check_norm(x, w, b, dy, 1e-5, got, hr.layer_norm_backward(x, w, got.stats, dy), BF16)


# ---- gated blocks

# (m, k, f): single tokens, few rows, where tiles and steps of k end, odd sizes
GATED = [(1, 1, 1), (1, 64, 48), (2, 100, 33), (5, 31, 7), (16, 768, 512), (17, 96, 130), (1, 1000, 777), (33, 128, 64), (64, 64, 256), (65, 200, 129), (100, 72, 1000),
         (129, 40, 257), (128, 512, 128), (256, 256, 300), (257, 136, 385), (300, 1032, 70), (520, 192, 640)]
ACTS = ["silu", "gelu", "gelu_tanh"]


def _gated_inputs(m, k, f, dtype, seed=0):
    x = (_randn(m + k + seed, m, k) * torch.exp(0.3 * _randn(k, k))).to(dtype)
    wg, wu = ((_randn(f + i + seed, f, k) / math.sqrt(k)).to(dtype) for i in (1, 2))
    return x, wg, wu, _randn(f + 3 + seed, m, f).to(dtype)


def _check_gated(x, wg, wu, dh, act, got, grads):
    h, gate, up, h_tol, g_tol, u_tol = ref.gated(x, wg, wu, act)
    ref.close(got.out, h, h_tol, x.dtype)
    ref.close(got.pre[:, 0], gate, g_tol, F32)
    ref.close(got.pre[:, 1], up, u_tol, F32)
    dx, dg, du, dx_tol, dg_tol, du_tol = ref.gated_grads(x, wg, wu, got.pre, dh, act, x.dtype)
    ref.close(grads.x, dx, dx_tol, x.dtype)
    ref.close(grads.w_gate, dg, dg_tol, x.dtype)
    ref.close(grads.w_up, du, du_tol, x.dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,f", GATED)
def test_gated_and_gradients(m, k, f, dtype):
    hr = _hr()
    for act in (ACTS if m * k * f < 10_000_000 else ACTS[(m + k) % 3:][:1]):
        _say("gated", m, k, f, dtype, act)
        x, wg, wu, dh = _gated_inputs(m, k, f, dtype)
        got = hr.gated(x, wg, wu, act, keep=True)
        assert torch.equal(hr.gated(x, wg, wu, act).out, got.out) and hr.gated(x, wg, wu, act).pre is None
        _check_gated(x, wg, wu, dh, act, got, hr.gated_backward(x, wg, wu, got.pre, dh, act))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,f", [(1, 65, 40), (7, 64, 48), (16, 200, 100), (40, 129, 66), (130, 100, 190), (260, 72, 300)])
def test_gated_of_slices(m, k, f, dtype):
    """Rows that begin anywhere or at even places, NaN beside them; halves of one matrix; what lies beside a result stays as it was."""
    hr = _hr()
    _say("gated slices", m, k, f, dtype)
    x, wg, wu, dh = _gated_inputs(m, k, f, dtype)
    want = hr.gated(x, wg, wu, keep=True)
    grads = hr.gated_backward(x, wg, wu, want.pre, dh)
    pad = -k % 64
    for before, behind in ((3, 2), (0, pad + 64), (8, pad + 120)):
        xs, gs, us, ds = (_strided(t, before, behind, NAN)[0] for t in (x, wg, wu, dh))
        hs, hw = _strided(want.out * 0, before, behind, 7.0)
        got = hr.gated(xs, gs, us, keep=True, out=hs)
        _check_gated(x, wg, wu, dh, "silu", got, hr.gated_backward(xs, gs, us, got.pre, ds))
        assert got.out is hs and _around(hw, before, f, 7.0)
    both = torch.cat([wg, wu])
    halves = hr.gated(x, both[:f], both[f:], keep=True)
    assert torch.equal(halves.out, want.out) and torch.equal(halves.pre, want.pre)
    only = hr.gated_backward(x, wg, wu, want.pre, dh, matrices=False)
    assert only.w_gate is None and only.w_up is None and torch.equal(only.x, grads.x)
    only = hr.gated_backward(x, wg, wu, want.pre, dh, rows=False)
    assert only.x is None and torch.equal(only.w_gate, grads.w_gate) and torch.equal(only.w_up, grads.w_up)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,f", [(3, 96, 50), (40, 100, 70), (150, 72, 140)])
def test_gated_keeps_what_is_no_number_where_it_is(m, k, f, dtype):
    """A NaN or an infinity in a row of x or of a matrix reaches that row, or that column, of the result and no other, also beside rows' and tiles' ends."""
    hr = _hr()
    x, wg, wu, dh = _gated_inputs(m, k, f, dtype)
    want = hr.gated(x, wg, wu, keep=True)
    grads = hr.gated_backward(x, wg, wu, want.pre, dh)
    rows, cols = [m - 1, m // 2], [f - 1, f // 3]
    x2, wg2, wu2 = x.clone(), wg.clone(), wu.clone()
    x2[rows[0], k - 1], x2[rows[1], 0] = NAN, INF
    got = hr.gated(x2, wg, wu, keep=True)
    fine = torch.tensor([i for i in range(m) if i not in rows], device="cuda")
    assert torch.equal(got.out[fine], want.out[fine]) and got.pre[rows].logical_not().sum() == 0 and not got.pre[rows].isfinite().any()
    wg2[cols[0], k - 1], wu2[cols[1], 1] = NAN, -INF
    got = hr.gated(x, wg2, wu2, keep=True)
    left = torch.tensor([j for j in range(f) if j not in cols], device="cuda")
    assert torch.equal(got.out[:, left], want.out[:, left]) and got.pre[:, 0, cols[0]].isnan().all() and not got.pre[:, 1, cols[1]].isfinite().any()
    dh2 = dh.clone()
    dh2[rows[0], f - 1] = NAN
    back = hr.gated_backward(x, wg, wu, want.pre, dh2)
    fine = torch.tensor([i for i in range(m) if i != rows[0]], device="cuda")
    assert torch.equal(back.x[fine], grads.x[fine]) and back.x[rows[0]].isnan().all()
    assert torch.equal(back.w_gate[:f - 1], grads.w_gate[:f - 1]) and torch.equal(back.w_up[:f - 1], grads.w_up[:f - 1]) and back.w_up[f - 1].isnan().all()
    back = hr.gated_backward(x2, wg, wu, want.pre, dh)
    assert torch.equal(back.x, grads.x) and back.w_gate[:, k - 1].isnan().all() and torch.equal(back.w_gate[:, 1:k - 1], grads.w_gate[:, 1:k - 1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,f", [(70, 128, 96), (40, 136, 70), (300, 200, 130), (33, 136, 40)])
def test_gated_with_some_operands_at_odd_places(m, k, f, dtype):
    """Whichever they are, or rows that lie far apart: the same bits (more than 32 rows take one way), and nothing beside the results is written."""
    hr = _hr()
    x, wg, wu, _ = _gated_inputs(m, k, f, dtype)
    want = hr.gated(x, wg, wu, keep=True)
    odd = [_strided(t, 1, 2, NAN)[0] for t in (x, wg, wu)]
    for which in ((0,), (1,), (2,), (0, 1), (1, 2), (0, 1, 2)):
        ops = [odd[i] if i in which else t for i, t in enumerate((x, wg, wu))]
        wide = torch.full((m, f + 5), 7.0, dtype=dtype, device="cuda")
        got = hr.gated(*ops, keep=True, out=wide[:, 3:3 + f])
        assert torch.equal(got.out, want.out) and torch.equal(got.pre, want.pre) and _around(wide, 3, f, 7.0)
    if m < 100:
        far = torch.zeros(m, (1 << 21) + 64, dtype=dtype, device="cuda")[:, :k]
        got = hr.gated(far.copy_(x), wg, wu, keep=True)
        assert torch.equal(got.out, want.out) and torch.equal(got.pre, want.pre)


# tiles of 256 x 256, whole blocks of k and not, with rows that are left to small ones and without
@pytest.mark.parametrize("m,k,f,dtype", [(4100, 1032, 4104, BF16), (4352, 1024, 4352, F16), (8200, 520, 5128, F16), (4100, 1033, 4104, BF16)])
def test_gated_in_large_tiles(m, k, f, dtype):
    hr = _hr()
    x, wg, wu, dh = _gated_inputs(m, k, f, dtype)
    got = hr.gated(x, wg, wu, "gelu", keep=True)
    _check_gated(x, wg, wu, dh, "gelu", got, hr.gated_backward(x, wg, wu, got.pre, dh, "gelu"))


@pytest.mark.parametrize("act", ACTS)
def test_gated_far_arguments(act):
    """Arguments at which exponentials leave their range: 0 or the argument, slope 0 or 1, no NaN."""
    hr = _hr()
    z = torch.tensor([0.0, 1e-30, -1e-30, 5.0, -5.0, 30.0, -30.0, 89.0, -89.0, 200.0, -200.0, 1e10, -1e10, 1e18, -1e18], device="cuda")
    n = len(z)
    x, wu = torch.eye(n, device="cuda"), torch.ones(1, n, device="cuda")
    got = hr.gated(x, z[None], wu, act, keep=True)
    dh = torch.ones(n, 1, device="cuda")
    _check_gated(x, z[None], wu, dh, act, got, hr.gated_backward(x, z[None], wu, got.pre, dh, act))


def test_gated_without_rows():
    hr = _hr()
    x, wg, wu, _ = _gated_inputs(1, 40, 30, F32)
    r = hr.gated(x[:0], wg, wu, keep=True)
    assert r.out.shape == (0, 30) and r.pre.shape == (0, 2, 30)
    g = hr.gated_backward(x[:0], wg, wu, r.pre, r.out)
    assert g.x.shape == (0, 40) and not g.w_gate.any() and not g.w_up.any()


# ---- AdamW

SIZES = [1, 3, 255, 256, 257, 1000, 4095, 4096, 4097, 20000]


def _adamw_inputs(sizes, ptype, gtype, bits, master, seed, odd=False):
    """Lists of tensors, some at odd places of a larger one; moments of steps that were taken."""
    hr = _hr()
    lists = dict(params=[], grads=[], m=[], v=[], exponents=[], masters=[])
    for i, n in enumerate(sizes):
        def place(t, i=i):
            if not odd:
                return t
            wide = torch.full((t.numel() + 3,), 77, dtype=t.dtype, device="cuda")
            wide[1:-2] = t
            return wide[1:-2]
        level = 1e-3 * torch.exp(_randn(seed + i, n))
        w = _randn(seed + i + 100, n) * 0.1
        m, v = 0.3 * level * _randn(seed + i + 200, n), level ** 2 * (0.01 + _randn(seed + i + 300, n).abs())
        if bits == 8:
            codes = torch.randint(0, 256, (2, n), generator=_gen(seed + i), device="cuda", dtype=torch.uint8)
            codes[0][(codes[0] & 127) > 119] &= 119
            m, v = codes[0], codes[1]
            e = torch.randint(95, 120, ((n + 255) // 256, 2), generator=_gen(seed + i), device="cuda", dtype=torch.uint8)
        else:
            e = None
        lists["params"].append(place(w.to(ptype)))
        lists["grads"].append(place((level * _randn(seed + i + 400, n)).to(gtype)))
        lists["m"].append(place(m))
        lists["v"].append(place(v))
        lists["exponents"].append(e)
        lists["masters"].append(place(w) if master else None)
    return hr, lists


def _check_adamw(before, after, step, lr, betas, eps, decay, scale=1.0):
    for i, p in enumerate(before["params"]):
        e, w = before["exponents"][i], before["masters"][i]
        if not p.numel():
            continue
        m, v = (before["m"][i], before["v"][i]) if e is None else ref.decode(before["m"][i], before["v"][i], e)
        new, m64, v64, tol, m_tol, v_tol = ref.adamw(p if w is None else w, before["grads"][i], m, v, step, lr, betas, eps, decay[i], scale)
        ref.close(after["params"][i].reshape(-1), new, tol, p.dtype)
        if w is not None:
            ref.close(after["masters"][i].reshape(-1), new, tol, F32)
            assert torch.equal(after["params"][i], after["masters"][i].to(p.dtype))
        if e is None:
            ref.close(after["m"][i].reshape(-1), m64, m_tol, F32)
            ref.close(after["v"][i].reshape(-1), v64, v_tol, F32)
        else:
            want = ref.held(*ref.moments32(before["grads"][i], m, v, betas, scale))
            got = _hr().adamw_moments(after["m"][i], after["v"][i], after["exponents"][i])
            for name, a, b in zip("mv", got, want):
                assert torch.equal(a.double().cpu().reshape(-1), b), name
            for a, b in zip(got, ref.decode(after["m"][i], after["v"][i], after["exponents"][i])):
                assert torch.equal(a.double().cpu().reshape(-1), b)


def _copy(lists):
    return {k: [None if t is None else t.clone() for t in v] for k, v in lists.items()}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype,gtype,master", [(F32, F32, False), (F32, F16, False), (F32, BF16, False), (F16, F16, False), (F16, F32, True), (BF16, BF16, False),
                                                (BF16, BF16, True), (BF16, F32, False), (F16, BF16, True)])
def test_adamw_steps(ptype, gtype, master, bits):
    for odd in (False, True):
        _say("adamw", ptype, gtype, master, bits, odd)
        hr, lists = _adamw_inputs(SIZES, ptype, gtype, bits, master, 10, odd)
        decay = [0.1 * (i % 3) for i in range(len(SIZES))]
        before = _copy(lists)
        hr.adamw(**lists, step=7, lr=1e-2, betas=(0.8, 0.99), eps=1e-7, weight_decay=decay)
        _check_adamw(before, lists, 7, 1e-2, (0.8, 0.99), 1e-7, decay)
        if odd:
            for name in ("params", "m", "v"):
                for t in lists[name]:
                    whole = torch.as_strided(t, (t.numel() + 3,), (1,), t.storage_offset() - 1)
                    assert whole[0] == 77 and (whole[-2:] == 77).all(), name


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_the_first_step_on(bits):
    """Three steps from moments of 0, scaled gradients, a parameter without a gradient, more tensors than a launch takes, some without numbers."""
    hr = _hr()
    sizes = [(i * 37) % 700 for i in range(120)]
    params = [_randn(i, n) for i, n in enumerate(sizes)]
    state = [hr.adamw_state(p, bits) for p in params]
    lists = dict(params=params, grads=None, m=[s[0] for s in state], v=[s[1] for s in state], exponents=[s[2] for s in state], masters=[None] * 120)
    scale = torch.full((1,), 0.37, device="cuda")
    for step in (1, 2, 3):
        lists["grads"] = [1e-2 * _randn(1000 * step + i, n) for i, n in enumerate(sizes)]
        before = _copy(lists)
        lists["grads"][5] = None
        versions = [p._version for p in params]
        hr.adamw(**lists, step=step, lr=1e-3, weight_decay=0.05, grad_scale=scale)
        for name in ("params", "m", "v"):
            assert torch.equal(lists[name][5], before[name][5])
        assert all((p._version > v) == (i != 5) for i, (p, v) in enumerate(zip(params, versions)))
        keep = [i for i in range(120) if i != 5]
        _check_adamw({k: [v[i] for i in keep] for k, v in before.items()}, {k: [v[i] for i in keep] for k, v in lists.items()}, step, 1e-3, (0.9, 0.999), 1e-8,
                     [0.05] * 119, float(scale))


def test_adamw_mixed_lists_equal_calls_for_each():
    hr, a = _adamw_inputs([300, 5000], F32, F32, 32, False, 1)
    for k, part in enumerate([(BF16, BF16, 8, True), (F16, F32, 8, False), (BF16, BF16, 32, True)]):
        for name, x in _adamw_inputs([257, 4100, 8], *part, seed=10 * k)[1].items():
            a[name] += x
    b = _copy(a)
    decay = [0.01 * i for i in range(len(a["params"]))]
    hr.adamw(**a, step=3, lr=1e-2, weight_decay=decay)
    for i in range(len(decay)):
        hr.adamw(**{k: [v[i]] for k, v in b.items()}, step=3, lr=1e-2, weight_decay=decay[i])
    for name in a:
        assert all(x is None or torch.equal(x, y) for x, y in zip(a[name], b[name])), name


def test_adamw_leaves_alone_what_has_no_gradient():
    hr = _hr()
    params = [_randn(1, 300), _randn(2, 0), _randn(3, 7).half()]
    state = [hr.adamw_state(p, b) for p, b in zip(params, (8, 32, 32))]
    masters = [None, None, params[2].float()]
    before = [p.clone() for p in params]
    lists = [[s[i] for s in state] for i in range(3)]

    def step(grads):
        hr.adamw(params, grads, lists[0], lists[1], 1, 1e-2, exponents=lists[2], masters=masters)

    step([None, None, None])
    assert all(torch.equal(p, b) for p, b in zip(params, before)) and not any(bool(t.any()) for s in state for t in s if t is not None)
    step([None, params[1].clone(), torch.ones_like(params[2])])
    assert torch.equal(params[0], before[0]) and not bool((params[2] == before[2]).any()) and not bool(state[0][0].any())


def test_adamw_strange_numbers():
    """Moments in 8 bits: a NaN or an infinity makes its block's NaN and no other's; gradients so small or so large that their squares leave the range."""
    hr = _hr()
    n = 256 * 8
    p, g = _randn(1, n), _randn(2, n)
    g[10], g[300], g[600] = NAN, INF, -INF
    g[768:1024] = 0
    g[1024:1280] *= 1e-19
    g[1280:1536] *= 1e-22
    g[1536:1792] *= 1e-42
    g[1800] = 1e18
    m, v, e = hr.adamw_state(p, 8)
    lists = dict(params=[p], grads=[g], m=[m], v=[v], exponents=[e], masters=[None])
    old = p.clone()
    for step in (1, 2):
        before = _copy(lists)
        hr.adamw(**lists, step=step, lr=1e-3, eps=1e-30)
        fm, fv = hr.adamw_moments(m, v, e)
        assert fm[:768].isnan().all() and fv[:768].isnan().all() and not fm[768:].isnan().any() and not fv[768:].isnan().any()
        bm, bv = ref.decode(before["m"][0], before["v"][0], before["exponents"][0])
        want = ref.held(*ref.moments32(g, bm, bv, (0.9, 0.999)))
        assert all(torch.equal(a.double().cpu().nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip((fm, fv), want))
        real = (bv * 0.999 + 0.001 * g.double().cpu() ** 2)[768:] > 2.0 ** -140
        assert bool(((fv[768:].cpu() > 0) | ~real).all())                # (never 0 where it is above 0)
        assert (p[:768].isnan() == (torch.isnan(g[:768]) | torch.isinf(g[:768]) | (step == 2))).all()
        # (where the square leaves the range, 0.001 * 1e-44 < 2^-149, v is 0 and a step is m / eps: of any size)
        assert torch.equal(p[768:1024], old[768:1024]) and (p - old)[768:].cpu()[real].abs().max() < 4e-3 * step


def test_adamw_captured_with_a_step_on_the_device():
    """Replays with other gradients, the step raised between them, equal eager steps; eager work goes on between."""
    hr, a = _adamw_inputs([1000, 77, 5000], BF16, BF16, 8, True, 5)
    f = _adamw_inputs([33, 400], F32, F32, 32, False, 6)[1]
    for name in a:
        a[name] += f[name]
    b = _copy(a)
    step, scale = torch.ones(1, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda")
    c = _copy(a)
    hr.adamw(**c, step=step, lr=1e-2, weight_decay=0.1, grad_scale=scale)          # (loads the kernels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hr.adamw(**a, step=step, lr=1e-2, weight_decay=0.1, grad_scale=scale)
        step.add_(1)
    for k in range(1, 5):
        scale.fill_(0.5 * k)
        for x, y in zip(a["grads"], b["grads"]):
            x.copy_(torch.randn_like(x))
            y.copy_(x)
        hr.adamw(**b, step=k, lr=1e-2, weight_decay=0.1, grad_scale=scale)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in a:
            for x, y in zip(a[name], b[name]):
                if x is not None and name != "params" and x.dtype == F32:
                    # (powers of beta by the device's 64-bit pow: the two factors may differ in their last place of 32 bits)
                    assert ((x - y).abs() <= 4 * 2.0 ** -23 * x.abs().clamp(min=1e-2 * 4)).all(), (name, k)
                elif x is not None and name != "params":
                    assert torch.equal(x, y), (name, k)
    assert int(step) == 5


# ---- calls

def _step(hr, x, w, b, wg, wu, dh, p):
    r = hr.layer_norm(x, w, b)
    h = hr.gated(r.out, wg, wu, keep=True)
    g = hr.gated_backward(r.out, wg, wu, h.pre, dh)
    n = hr.layer_norm_backward(x, w, r.stats, g.x)
    hr.adamw([p["wg"], p["wu"], p["w"], p["b"]], [g.w_gate, g.w_up, n.weight, n.bias], p["m"], p["v"], 3, 1e-3, exponents=p["e"])
    return h.out, n.x, g.w_gate, g.w_up, n.weight, n.bias, p["wg"].clone(), p["wu"].clone(), p["w"].clone(), p["b"].clone()


def _step_inputs(hr, m, k, f, dtype, seed):
    x, wg, wu, dh = _gated_inputs(m, k, f, dtype, seed)
    w, b = 1 + 0.1 * _randn(seed + 1, k), _randn(seed + 2, k)
    state = [hr.adamw_state(t, 8) for t in (wg, wu, w, b)]
    return (x, w, b, wg, wu, dh), dict(wg=wg.clone(), wu=wu.clone(), w=w.clone(), b=b.clone(), m=[s[0] for s in state], v=[s[1] for s in state], e=[s[2] for s in state])


@pytest.mark.parametrize("m,k,f,dtype", [(1, 256, 512, BF16), (40, 100, 70, F16), (300, 256, 640, BF16), (130, 64, 200, F32)])
def test_on_another_stream_and_captured(m, k, f, dtype):
    """The same bits from calls that follow one another on a side stream, and from replays with new contents and eager work in between."""
    hr = _hr()
    _say("step", m, k, f, dtype)
    ins, p = _step_inputs(hr, m, k, f, dtype, 0)
    keep = {n: [t.clone() for t in v] if isinstance(v, list) else v.clone() for n, v in p.items()}

    def reset():
        for n, v in keep.items():
            for a, b in zip(p[n] if isinstance(v, list) else [p[n]], v if isinstance(v, list) else [v]):
                a.copy_(b)
    want = _step(hr, *ins, p)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            reset()
            got = _step(hr, *ins, p)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _step(hr, *ins, p)
    for seed in range(1, 5):
        new, _ = _step_inputs(hr, m, k, f, dtype, seed)
        for a, b in zip(ins, new):
            a.copy_(b)
        reset()
        want = _step(hr, *new, p)
        reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_a_block_with_its_gradients_and_step_against_autograd():
    """x + gated(norm(x)) w_down', a loss on it, all gradients and one step, in float32, against the same in 64 bits by autograd."""
    hr = _hr()
    m, k, f = 96, 80, 144
    x, wg, wu, _ = _gated_inputs(m, k, f, F32)
    w, b, wd, target = 1 + 0.1 * _randn(1, k), 0.1 * _randn(2, k), _randn(3, k, f) / math.sqrt(f), _randn(4, m, k)
    r = hr.layer_norm(x, w, b)
    h = hr.gated(r.out, wg, wu, "gelu", keep=True)
    y = x + h.out @ wd.T
    dy = (y - target) / m
    dwd = dy.T @ h.out
    g = hr.gated_backward(r.out, wg, wu, h.pre, dy @ wd, "gelu")
    n = hr.layer_norm_backward(x, w, r.stats, g.x)
    dx = dy + n.x
    leaves = [t.double().cpu().requires_grad_(True) for t in (x, w, b, wg, wu, wd)]
    x6, w6, b6, wg6, wu6, wd6 = leaves
    u = torch.nn.functional.layer_norm(x6, (k,), w6, b6, 1e-5)
    y6 = x6 + (torch.nn.functional.gelu(u @ wg6.T) * (u @ wu6.T)) @ wd6.T
    (((y6 - target.double().cpu()) ** 2).sum() / (2 * m)).backward()
    # every number is a chain of five sums of at most 144 products each, of factors near 1 in size: 5 * 150 roundings, by the norm of the result
    for got, leaf in zip((dx, n.weight, n.bias, g.w_gate, g.w_up, dwd), leaves):
        assert float((got.double().cpu() - leaf.grad).norm() / leaf.grad.norm()) < 5 * 150 * ref.U
    params, grads = [wg, wu, wd, w, b], [g.w_gate, g.w_up, dwd, n.weight, n.bias]
    state = [hr.adamw_state(p) for p in params]
    before = dict(params=[p.clone() for p in params], grads=grads, m=[s[0].clone() for s in state], v=[s[1].clone() for s in state], exponents=[None] * 5, masters=[None] * 5)
    lists = dict(params=params, grads=grads, m=[s[0] for s in state], v=[s[1] for s in state], exponents=None, masters=None)
    hr.adamw(**lists, step=1, lr=1e-3, weight_decay=0.01)
    _check_adamw(before, {**lists, "exponents": [None] * 5, "masters": [None] * 5}, 1, 1e-3, (0.9, 0.999), 1e-8, [0.01] * 5)


def test_offsets_beyond_32_bits():
    """Rows, columns and numbers that lie more than 2^32 bytes and 2^31 elements from the first equal those of a call that begins with them."""
    hr = _hr()
    rows, n = 33000, 65537
    x = torch.empty(rows, n, dtype=BF16, device="cuda").normal_(generator=_gen(1))
    w = 1 + 0.1 * _randn(2, n)
    got = hr.layer_norm(x, w)
    alone = hr.layer_norm(x[-3:], w)
    assert torch.equal(got.out[-3:], alone.out) and torch.equal(got.stats[-3:], alone.stats)
    g = hr.layer_norm_backward(x, w, got.stats, got.out)
    assert torch.equal(g.x[-3:], hr.layer_norm_backward(x[-3:], w, alone.stats, alone.out).x)
    del x, got, g, alone
    f, k = 1 << 19, 4104
    wg, wu = (torch.empty(f, k, dtype=BF16, device="cuda").normal_(generator=_gen(i)) for i in (3, 4))
    for m in (1, 20, 70):                                  # (the last 256 columns begin a tile, and a workgroup of every kernel)
        x = (_randn(m, m, k) / 64).to(BF16)
        got, tail = hr.gated(x, wg, wu, keep=True), hr.gated(x, wg[-256:], wu[-256:], keep=True)
        _, gate, up, _, g_tol, u_tol = ref.gated(x, wg[-256:], wu[-256:], "silu")
        for r in (got.pre[:, :, -256:], tail.pre):
            ref.close(r[:, 0], gate, g_tol, F32)
            ref.close(r[:, 1], up, u_tol, F32)
    del wg, wu, got, tail
    n = (1 << 31) + 1000
    p, g = (torch.empty(n, dtype=BF16, device="cuda").normal_(generator=_gen(i)) for i in (5, 6))
    m, v, e = hr.adamw_state(p, 8)
    cut = (1 << 31) - 512
    small = [t[cut:].clone() for t in (p, g, m, v)] + [e[cut // 256:].clone()]
    hr.adamw([p], [g], [m], [v], 1, 1e-2, exponents=[e])
    hr.adamw(*[[t] for t in small[:4]], 1, 1e-2, exponents=[small[4]])
    assert torch.equal(p[cut:], small[0]) and torch.equal(m[cut:], small[2]) and torch.equal(v[cut:], small[3]) and torch.equal(e[cut // 256:], small[4])
    fm, fv = hr.adamw_moments(m, v, e)
    assert all(torch.equal(a[cut:], b) for a, b in zip((fm, fv), hr.adamw_moments(*small[2:])))


def test_keyword_calls_give_the_same():
    hr = _hr()
    x, wg, wu, dh = _gated_inputs(5, 40, 24, BF16)
    r, s = hr.layer_norm(x), hr.layer_norm(eps=1e-5, bias=None, weight=None, x=x)
    assert torch.equal(r.out, s.out) and torch.equal(r.stats, s.stats)
    assert torch.equal(hr.layer_norm_backward(grad_out=x, stats=r.stats, weight=None, x=x).x, hr.layer_norm_backward(x, None, r.stats, x).x)
    h = hr.gated(w_up=wu, x=x, w_gate=wg, keep=True)
    assert torch.equal(h.out, hr.gated(x, wg, wu).out)
    assert all(torch.equal(a, b) for a, b in zip(hr.gated_backward(x, wg, wu, h.pre, dh), hr.gated_backward(grad_out=dh, pre=h.pre, x=x, w_up=wu, w_gate=wg)))


def test_what_is_refused():
    hr = _hr()
    x, wg, wu, dh = _gated_inputs(5, 40, 24, F32)
    one, r, h = torch.ones(40, device="cuda"), hr.layer_norm(x), hr.gated(x, wg, wu, keep=True)
    m, v, e = hr.adamw_state(x, 8)
    f = torch.zeros_like(x)
    wide = torch.zeros(5, 80, device="cuda")
    bad = [lambda: hr.layer_norm(x.double()), lambda: hr.layer_norm(x.cpu()), lambda: hr.layer_norm(x[0]), lambda: hr.layer_norm(x[:, :0]), lambda: hr.layer_norm(x, one[:39]),
           lambda: hr.layer_norm(x, one.half()), lambda: hr.layer_norm(x.half(), one, one.half()), lambda: hr.layer_norm(x, one.cpu()), lambda: hr.layer_norm(x, eps=-1.0),
           lambda: hr.layer_norm(x, out=wg), lambda: hr.layer_norm(x, out=x.T.contiguous().T),
           lambda: hr.layer_norm_backward(x, None, r.stats[:4], x), lambda: hr.layer_norm_backward(x, None, r.stats.half(), x), lambda: hr.layer_norm_backward(x, None, r.stats, x[:4]),
           lambda: hr.layer_norm_backward(x, None, r.stats, x.half()), lambda: hr.layer_norm_backward(x, one[:3], r.stats, x),
           lambda: hr.gated(x, wg, wu, "tanh"), lambda: hr.gated(x, wg.half(), wu), lambda: hr.gated(x, wg, wu[:23]), lambda: hr.gated(x, wg[:, :39], wu), lambda: hr.gated(x, wg.cpu(), wu),
           lambda: hr.gated(x[:, :0], wg[:, :0], wu[:, :0]), lambda: hr.gated(x, wg[:0], wu[:0]), lambda: hr.gated(x, wg, wu, out=x),
           lambda: hr.gated_backward(x, wg, wu, h.pre[:4], dh), lambda: hr.gated_backward(x, wg, wu, h.pre.half(), dh), lambda: hr.gated_backward(x, wg, wu, h.pre, dh[:, :23]),
           lambda: hr.gated_backward(x, wg, wu, h.pre, dh.half()), lambda: hr.gated_backward(x, wg, wu, h.pre, dh[:4]),
           lambda: hr.adamw([x], [x], [f], [m], 1, 1e-3), lambda: hr.adamw([x], [f], [m], [v], 1, 1e-3), lambda: hr.adamw([x], [f], [m], [v], 1, 1e-3, exponents=[e[:0]]),
           lambda: hr.adamw([x], [f[:4]], [f], [f], 1, 1e-3), lambda: hr.adamw([x], [f], [f], [f[:4]], 1, 1e-3), lambda: hr.adamw([x], [f], [f], [f.clone()], 0, 1e-3),
           lambda: hr.adamw([x, x], [f, f], [f, f.clone()], [f.clone(), f.clone()], 1, 1e-3), lambda: hr.adamw([x], [f], [f], [f], 1, 1e-3),
           lambda: hr.adamw([x], [f], [f.clone()], [f.clone()], 1, 1e-3, masters=[f]), lambda: hr.adamw([x], [f], [f.clone()], [f.clone()], 1, math.nan),
           lambda: hr.adamw([wide[:, ::2]], [f], [f.clone()], [f.clone()], 1, 1e-3), lambda: hr.adamw([x], [f], [f.clone()], [f.clone()], 1, 1e-3, betas=(0.9, 1.0)),
           lambda: hr.adamw([x], [f], [f.clone()], [f.clone()], torch.ones(2, dtype=torch.int64, device="cuda"), 1e-3),
           lambda: hr.adamw([x], [f], [f.clone()], [f.clone()], 1, 1e-3, grad_scale=torch.ones(1)), lambda: hr.adamw([x], [f], [f.clone()], [f.clone()], 1, 1e-3, weight_decay=[0.1, 0.1]),
           lambda: hr.adamw([x.double()], [f], [f.clone()], [f.clone()], 1, 1e-3), lambda: hr.adamw([x], [f.double()], [f.clone()], [f.clone()], 1, 1e-3),
           lambda: hr.adamw_moments(m, v, e[:0]), lambda: hr.adamw_moments(m, v[:4], e), lambda: hr.adamw_moments(f, v, e), lambda: hr.adamw_moments(m, v, e.cpu())]
    kept = x.clone()
    for i, call in enumerate(bad):
        with pytest.raises(hr.HrError) as err:
            call()
        assert err.value.code in (-1, -5), i
    torch.cuda.synchronize()
    assert torch.equal(x, kept)                            # nothing was enqueued by the refused calls


def _example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_encoder_layers.py")
    spec = importlib.util.spec_from_file_location("train_encoder_layers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def test_the_example_runs(capsys):
    """examples/train_encoder_layers.py, small: search, layers, distillation, gradients and steps together."""
    encoder, losses = _example().main(passages=8192, d=128, hidden=200, layers=2, nlist=64, batch=128, k=16, probes=8, steps=6)
    assert len(losses) == 6 and all(math.isfinite(x) for x in losses) and encoder.steps == 6
    assert all(bool(t.isfinite().all()) for t in encoder.tensors) and "step 5" in capsys.readouterr().out


def test_the_examples_gradients():
    """Of its encoder in float32, two layers, against autograd in 64 bits."""
    e = _example().Encoder(2, 48, 80, dtype=F32, bits=32)
    x, dy = _randn(1, 60, 48), _randn(2, 60, 48)
    y, kept = e.forward(x)
    grads = e.backward(dy, kept)
    leaves = [t.double().cpu().requires_grad_(True) for t in e.tensors]
    z = x.double().cpu()
    for i in range(0, 10, 5):
        w, b, wg, wu, wd = leaves[i:i + 5]
        u = torch.nn.functional.layer_norm(z, (48,), w, b, 1e-5)
        z = z + (torch.nn.functional.silu(u @ wg.T) * (u @ wu.T)) @ wd.T
    (z * dy.double().cpu()).sum().backward()
    # chains of up to ten sums of at most 80 products, of factors near 1 in size, by the norm of the result
    assert float((y.double().cpu() - z.detach()).norm() / z.detach().norm()) < 10 * 90 * ref.U
    for got, leaf in zip(grads, leaves):
        assert float((got.double().cpu() - leaf.grad).norm() / leaf.grad.norm()) < 10 * 90 * ref.U
