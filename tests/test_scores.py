"""Products in 8 bits, log probabilities and distillation (hr_scores.h) on the GPU against 64-bit arithmetic of the same
operands: sizes at which tiles, chunks and buffers end, rows without candidates, ties, strides, special values."""
import math

import numpy as np
import pytest
import torch

import scores_reference as ref

pytestmark = pytest.mark.gpu
INF = math.inf
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def _hr():
    import paper_2507_09138_amd as hr
    return hr


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _say(*a):
    print("case", *a, flush=True)


def _strided(t, before, behind, fill):
    """The same matrix as a slice of columns of a wider one (rows start at odd places), and the wider one."""
    wide = torch.full((t.shape[0], before + t.shape[1] + behind), fill, dtype=t.dtype, device=t.device)
    view = wide[:, before:before + t.shape[1]]
    view.copy_(t)
    return view, wide


# ---- 8 bits

QUANT_SHAPES = [(1, 1), (3, 5), (7, 63), (2, 64), (5, 65), (4, 1000), (3, 8192), (300, 768), (1, 20001), (65, 128)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k", QUANT_SHAPES)
def test_quantized_rows_are_the_definitions(m, k, dtype):
    _say("quantize", m, k, dtype)
    x = torch.randn(m, k, generator=_gen(m + k), device="cuda") * torch.exp(torch.randn(m, 1, generator=_gen(k), device="cuda"))
    x = x.to(dtype)
    if m > 2:
        x[1] = 0
        x[2, k // 2] = 0.5                                 # (ties of the rounding: multiples of half a step)
    want, scale = ref.quantize(x)
    for t in (x, _strided(x, 3, 2, 1e4)[0]):
        q, s = _hr().quantize_rows(t)
        assert torch.equal(s.cpu(), scale)
        assert torch.equal(q.cpu(), want)
        assert q.stride(0) % 64 == 0
        behind = torch.as_strided(q, (m, q.stride(0) - k), (q.stride(0), 1), k) if q.stride(0) > k else q[:, :0]
        assert not behind.any()


def test_quantized_rows_ties_specials_and_a_tight_stride():
    hr = _hr()
    steps = torch.arange(-254, 255, device="cuda", dtype=torch.float32) / 2          # every half step: even on ties
    x = torch.stack([steps, steps * 2.0 ** -140, torch.zeros_like(steps), steps, steps, steps * 3e36])
    x[3, 7], x[4, 9] = INF, math.nan
    want, scale = ref.quantize(x)
    q, s = hr.quantize_rows(x)
    assert torch.equal(q.cpu(), want) and torch.equal(s.cpu().nan_to_num(-1.0), scale.nan_to_num(-1.0))
    assert torch.isnan(s[3]) and torch.isnan(s[4]) and not q[3].any() and not q[4].any()
    m, k = x.shape
    tight = torch.full((m * k + 64,), 77, dtype=torch.int8, device="cuda")
    hr.hr_i8_quantize(x, k, hr.HR_F32, m, k, tight, k, s)
    assert torch.equal(tight[:m * k].view(m, k).cpu(), want) and (tight[m * k:] == 77).all()


def _i8(rows, k, seed):
    return torch.randint(-128, 128, (rows, k), generator=_gen(seed), device="cuda", dtype=torch.int8)


def _check_product(m, n, k, dtype, bias, lay, seed=0):
    hr = _hr()
    a, b = _i8(m, k, m + 7 * k + seed), _i8(n, k, n + 5 * k + seed)
    sa = torch.rand(m, generator=_gen(m), device="cuda") * 0.01
    sb = torch.rand(n, generator=_gen(n), device="cuda") * 0.01
    bs = torch.randn(n, generator=_gen(n + 1), device="cuda") if bias else None
    want, tol = ref.product(a.cpu(), sa.cpu(), b.cpu(), sb.cpu(), None if bs is None else bs.cpu())
    if lay == "padded":                                    # 64 bytes apart, what lies behind the rows is not zero
        a, b = _strided(a, 0, -k % 64, 99)[0], _strided(b, 0, -k % 64, -128)[0]
    elif lay == "odd":                                     # rows and the first of them at odd addresses
        a, b = _strided(a, 3, 2 - (k + 1) % 2, 99)[0], _strided(b, 1, 2 + k % 2, -128)[0]
    out, wide = _strided(torch.zeros(m, n, dtype=dtype, device="cuda"), 1, 3, 5.0)
    got = hr.i8_product(a, sa, b, sb, bias=bs, dtype=dtype, out=out)
    assert got is out
    ref.close(got, want, tol, dtype)
    assert (wide[:, :1] == 5).all() and (wide[:, n + 1:] == 5).all()
    fresh = hr.i8_product(a, sa, b, sb, bias=bs, dtype=dtype)
    assert torch.equal(fresh, got)


PRODUCT_SIZES = [(1, 1, 1), (1, 17, 15), (2, 64, 16), (3, 100, 17), (15, 33, 63), (16, 128, 64), (17, 129, 65), (33, 257, 127),
                 (64, 64, 128), (65, 300, 129), (130, 131, 333), (257, 500, 768), (1, 4097, 1000), (5, 2000, 2049), (8, 8, 8192),
                 (300, 259, 4096), (1, 3, 20000), (127, 1, 256), (1000, 70, 192), (48, 3001, 768), (100, 1030, 1100), (513, 1025, 512)]


@pytest.mark.parametrize("lay", ["contiguous", "padded", "odd"])
@pytest.mark.parametrize("m,n,k", PRODUCT_SIZES)
def test_products_at_the_edges_of_tiles(m, n, k, lay):
    _say("product", m, n, k, lay)
    dtype = TYPES[(m + n + k) % 3]
    _check_product(m, n, k, dtype, (m + n) % 2 == 0, lay)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("m,n,k", [(1, 1000, 768), (12, 777, 512), (40, 2048, 256), (300, 700, 640)])
def test_products_of_every_type(m, n, k, dtype, bias):
    _say("product", m, n, k, dtype, bias)
    _check_product(m, n, k, dtype, bias, "padded", seed=1)


@pytest.mark.parametrize("k", [70, 128, 200, 256, 300, 385, 513])
@pytest.mark.parametrize("m,n", [(4101, 4099), (3001, 2999), (40, 140003), (16, 70001), (64, 66000), (129, 60000), (4352, 4096)])
def test_products_of_many_tiles(m, n, k):
    """More tiles than workgroups, of every size, whole ones and ragged ones in turn, with one block of k and with several."""
    _say("many tiles", m, n, k)
    hr = _hr()
    dtype = TYPES[(m + k) % 3]
    a, b = _i8(m, k, m + k), _i8(n, k, n + k)
    sa = torch.rand(m, generator=_gen(m), device="cuda") * 0.01
    sb = torch.rand(n, generator=_gen(n), device="cuda") * 0.01
    bs = torch.randn(n, generator=_gen(n + 1), device="cuda") if k % 2 else None
    a, b = _strided(a, 0, -k % 64, 99)[0], _strided(b, 0, -k % 64, -128)[0]
    # (whole numbers below 2^53 in 64 bits: exact; blocks of rows keep the reference small)
    got = hr.i8_product(a, sa, b, sb, bias=bs, dtype=dtype)
    for lo in range(0, m, 1024):
        v = (a[lo:lo + 1024].double() @ b.double().T.contiguous()) * sa[lo:lo + 1024].double()[:, None] * sb.double()
        tol = 4 * ref.U * v.abs()
        if bs is not None:
            v, tol = v + bs.double(), tol + 4 * ref.U * bs.double().abs()
        off = (got[lo:lo + 1024].double() - v).abs() - tol * (1 + 2 * ref.EPS[dtype]) - ref.EPS[dtype] * v.abs() - ref.TINY[dtype]
        assert float(off.max()) <= 0, (lo, float(off.max()))
    assert torch.equal(hr.i8_product(a, sa, b, sb, bias=bs, dtype=dtype), got)


@pytest.mark.parametrize("k", [128, 200, 385, 513])
@pytest.mark.parametrize("m,n", [(3001, 3800), (3329, 3585), (4001, 7777), (8195, 6401)])
def test_products_of_rounds_of_tiles(m, n, k):
    """On both sides of the choice between large and small tiles, with less than a tile for every workgroup, two and four."""
    test_products_of_many_tiles(m, n, k)


@pytest.mark.parametrize("m,n,k", [(1, 5, 131071), (3, 40, 131071), (70, 90, 131071), (300, 300, 70000)])
def test_sums_are_exact_up_to_the_longest_rows(m, n, k):
    """Whole numbers: -128 x -128 throughout reaches 2^31 - 2^14; float32 of the exact sum is what comes back."""
    _say("longest", m, n, k)
    hr = _hr()
    one = torch.ones(max(m, n), device="cuda")
    low = torch.full((max(m, n), k), -128, dtype=torch.int8, device="cuda")
    got = hr.i8_product(low[:m], one[:m], low[:n], one[:n])
    assert (got == float(np.float32(k * 16384))).all()
    a, b = _i8(m, k, 1), _i8(n, k, 2)
    got = hr.i8_product(a, one[:m], b, one[:n]).cpu()
    want = (a.cpu().double() @ b.cpu().double().T).float()             # (sums below 2^53: exact)
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 300, 768), (1, 77, 1000), (2, 500, 65), (9, 1000, 4096), (16, 64, 8192), (17, 128, 333), (64, 600, 768),
                                   (100, 129, 40), (400, 300, 1024), (1, 1, 1), (3, 3000, 20000)])
def test_linear_is_quantize_and_product(m, n, k, dtype):
    _say("linear", m, n, k, dtype)
    hr = _hr()
    x = torch.randn(m, k, generator=_gen(m * k), device="cuda").to(dtype)
    if m > 1:
        x[m // 2] = 0
    w, ws = hr.quantize_rows(torch.randn(n, k, generator=_gen(n), device="cuda"))
    bias = torch.randn(n, generator=_gen(3), device="cuda") if k % 2 else None
    q, s = hr.quantize_rows(x)
    want = hr.i8_product(q, s, w, ws, bias=bias, dtype=dtype)
    for t in (x, _strided(x, 1, 4, 1e4)[0]):
        assert torch.equal(hr.i8_linear(t, w, ws, bias=bias, dtype=dtype), want)
    q, s = ref.quantize(x)
    v, tol = ref.product(q, s, w.cpu(), ws.cpu(), None if bias is None else bias.cpu())
    ref.close(want, v, tol, dtype)


def test_rows_that_are_not_finite_stay_among_themselves():
    hr = _hr()
    for m in (3, 80):
        x = torch.randn(m, 300, generator=_gen(1), device="cuda")
        w, ws = hr.quantize_rows(torch.randn(200, 300, generator=_gen(2), device="cuda"))
        want = hr.i8_linear(x, w, ws)
        bad = x.clone()
        bad[1, 5], bad[2, 299] = math.nan, -INF
        got = hr.i8_linear(bad, w, ws)
        assert torch.isnan(got[1:3]).all()
        keep = [i for i in range(m) if i not in (1, 2)]
        assert torch.equal(got[keep], want[keep])


# ---- rows of scores

def _scores(kind, rows, n, dtype, seed):
    g = _gen(seed)
    z = torch.randn(rows, n, generator=g, device="cuda") * 3
    if kind == "ties":
        z = torch.randint(-3, 4, (rows, n), generator=g, device="cuda").float()
    elif kind == "rising":
        z = z.sort(1).values
    elif kind == "falling":
        z = z.sort(1, descending=True).values
    elif kind == "masked":                                 # from none to all of the places, all but one in row 1
        z[torch.rand(rows, n, generator=g, device="cuda") < torch.linspace(0, 1, rows, device="cuda")[:, None]] = -INF
        z[-1] = -INF
        if rows > 1:
            z[1] = -INF
            z[1, n // 2] = 1.5
    elif kind == "lowest":                                 # masks of the lowest finite value, all of a row in row 0
        z[torch.rand(rows, n, generator=g, device="cuda") < 0.7] = torch.finfo(dtype).min
        z[0] = torch.finfo(dtype).min
    elif kind == "wide":
        z = z * 40
    elif kind == "zeros":                                  # +0 and -0 are alike
        z = torch.where(torch.rand(rows, n, generator=g, device="cuda") < 0.5, 0.0, -0.0)
    return z.to(dtype)


ROW_SIZES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (3, 63), (9, 64), (2, 65), (5, 127), (3, 130), (7, 1000), (3, 1025), (4, 4096), (5, 4099),
             (3, 16385), (2, 32003), (300, 333), (2, 131072), (1, 300001), (2, 1100003), (70, 9001), (1100, 2050), (1700, 3001), (40, 20011), (260, 52001), (200, 100003)]
KINDS = ["plain", "ties", "rising", "falling", "masked", "lowest", "wide", "zeros"]


def _check_logprobs(z, k, scale, given):
    hr = _hr()
    r = hr.logprobs(z, given, k=k, scale=scale)
    logp, p, m, logsum = ref.parts(z, float(np.float32(scale)))
    n = z.shape[1]
    err = ref.logp_error(logp, logsum, scale, n)
    if given is not None:
        ids = given.to(torch.int64)
        there = (ids >= 0) & (ids < n)
        ref.close(r.logprobs, ref.at(logp, ids), torch.where(there, err.gather(1, ids.clamp(0, n - 1)), 0.0), torch.float32)
    ref.close(r.entropy, ref.entropy(logp, p), ref.entropy_error(logsum, n), torch.float32)
    assert torch.equal(r.norm[:, 0].double(), m)
    ref.close(r.norm[:, 1], logsum, ref.sum_error(n) + ref.U * 8 * (logsum + 2), torch.float32)
    if k:
        ids = ref.best(z, k)
        assert torch.equal(r.top_ids, ids)
        ref.close(r.top_logprobs, ref.at(logp, ids), torch.where(ids >= 0, err.gather(1, ids.clamp(min=0)), 0.0), torch.float32)
    return r


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,n", ROW_SIZES)
def test_logprobs_entropy_and_alternatives(rows, n, kind):
    k = [1, 5, 20, 128, 0, 64, 10][(rows + n) % 7]
    dtype = TYPES[(n + KINDS.index(kind)) % 3]
    scale = [1.0, 0.3, 7.0][(n + len(kind)) % 3]
    _say("logprobs", rows, n, kind, dtype, k, scale)
    z = _scores(kind, rows, n, dtype, n)
    given = torch.randint(-1, n + 1, (rows, 1 + n % 5), generator=_gen(5), device="cuda")
    r = _check_logprobs(z, k, scale, given)
    # rows that start elsewhere, in a wider matrix: the same alternatives, sums in another order
    s = _strided(z, 3, 2, INF)[0]
    t = _check_logprobs(s, k, scale, given)
    assert k == 0 or torch.equal(t.top_ids, r.top_ids)
    again = _hr().logprobs(z, given, k=k, scale=scale)
    assert all(torch.equal(a, b) for a, b in zip(r, again) if a is not None)


@pytest.mark.parametrize("k", [1, 2, 16, 63, 64, 65, 127, 128])
@pytest.mark.parametrize("kind", ["plain", "ties", "rising", "falling", "masked", "lowest", "zeros"])
@pytest.mark.parametrize("rows,n", [(6, 100), (4, 2000), (3, 20000), (2, 140001)])
def test_alternatives_of_every_number(rows, n, kind, k):
    _say("alternatives", rows, n, kind, k)
    z = _scores(kind, rows, n, TYPES[k % 3], n + k)
    _check_logprobs(z, k, 1.0, None)


@pytest.mark.parametrize("k", [1, 15, 32, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("kind", ["plain", "ties", "rising", "falling", "masked", "lowest", "zeros"])
@pytest.mark.parametrize("rows,n", [(1025, 130), (1100, 2003), (1030, 8192)])
def test_alternatives_of_many_rows(rows, n, kind, k):
    _say("alternatives", rows, n, kind, k)
    z = _scores(kind, rows, n, TYPES[k % 3], n + k)
    _check_logprobs(z, k, 1.0, None)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_with_nan_or_infinity(dtype):
    hr = _hr()
    for n in (5, 700, 70001):
        _say("specials", dtype, n)
        z = _scores("plain", 6, n, dtype, n)
        clean = hr.logprobs(z, torch.zeros(6, 1, dtype=torch.int64, device="cuda"), k=3)
        z[1, n // 2], z[3, n - 1], z[4, 0] = math.nan, INF, math.nan
        z[4, 1:] = -INF
        z[5] = -INF
        given = torch.tensor([[0, -1], [1, -1], [0, 5], [0, -1], [0, -1], [0, n]], device="cuda")
        r = hr.logprobs(z, given, k=3)
        for row in (1, 3, 4):
            assert torch.isnan(r.logprobs[row, 0]) and r.logprobs[row, 1] == -INF
            assert torch.isnan(r.entropy[row]) and torch.isnan(r.norm[row, 1])
            assert (r.top_ids[row] == -1).all() and torch.isnan(r.top_logprobs[row]).all()
        assert (r.logprobs[5] == -INF).all() and r.entropy[5] == 0 and r.norm[5, 0] == -INF and r.norm[5, 1] == 0
        assert (r.top_ids[5] == -1).all() and (r.top_logprobs[5] == -INF).all()
        for row in (0, 2):
            assert torch.equal(r.entropy[row], clean.entropy[row]) and torch.equal(r.top_ids[row], clean.top_ids[row])
        g = hr.logprobs_backward(z, given, r, torch.ones(6, 2, device="cuda"), torch.ones(6, device="cuda"))
        assert torch.isnan(g[[1, 3]]).all() and not g[5].any() and torch.isfinite(g[[0, 2]]).all()


def test_a_lowest_value_row_is_uniform():
    hr = _hr()
    for dtype in TYPES:
        for scale in (1.0, 5.0):
            z = torch.full((2, 777), torch.finfo(dtype).min, dtype=dtype, device="cuda")
            r = hr.logprobs(z, torch.zeros(2, 1, dtype=torch.int64, device="cuda"), k=2, scale=scale)
            assert torch.allclose(r.logprobs, torch.full_like(r.logprobs, -math.log(777)), rtol=1e-6)
            assert torch.allclose(r.entropy, torch.full_like(r.entropy, math.log(777)), rtol=1e-6)
            assert r.top_ids.tolist() == [[0, 1], [0, 1]]
            g = hr.logprobs_backward(z, torch.zeros(2, 1, dtype=torch.int64, device="cuda"), r, torch.ones(2, 1, device="cuda"), scale=scale)
            want = scale * ((torch.arange(777, device="cuda") == 0).double() - 1 / 777)
            ref.close(g, want.expand(2, -1), 1e-6 * scale, dtype)


@pytest.mark.parametrize("rows,n", [(3, 300), (2000, 3001), (2, 140001)])
def test_an_offset_changes_nothing(rows, n):
    hr = _hr()
    _say("offsets", rows, n)
    g = torch.Generator(device="cuda").manual_seed(n)
    z = torch.randint(-40, 1, (rows, n), generator=g, device="cuda").float()
    given = torch.randint(n, (rows, 3), generator=g, device="cuda")
    want = hr.logprobs(z, given, k=4)
    logp, p, _, _ = ref.parts(z, 1.0)
    ref.close(want.entropy, ref.entropy(logp, p), 1e-5, torch.float32)
    # whole numbers that float32 holds, and their products with log2(e) on both sides of 2^23 and 2^24
    for offset in (4096, 2**22, 5814500, 5814540, 2**23, 11629060, 11629100, 2**24 - 40):
        for sign in (1, -1):
            r = hr.logprobs(z + sign * offset, given, k=4)
            ref.close(r.logprobs, want.logprobs, 2e-5, torch.float32)
            ref.close(r.entropy, want.entropy, 2e-5, torch.float32)
            assert torch.equal(r.norm[:, 0] - sign * offset, want.norm[:, 0]) and torch.equal(r.top_ids, want.top_ids)
    # a row with scores of both kinds: what lies below adds nothing
    for low in (-(2.0**25), -(2.0**23), -(2.0**22), torch.finfo(torch.float32).min):
        for top in (0.0, -(2.0**21), -5814520.0, -(2.0**22)):
            mixed = torch.cat([torch.full((rows, n), low, device="cuda"), z + top, torch.full((rows, 77), low, device="cuda")], 1)
            r = hr.logprobs(mixed, given + n, k=4)
            if low < top - 200:
                ref.close(r.logprobs, want.logprobs, 2e-5, torch.float32)
                ref.close(r.entropy, want.entropy, 2e-5, torch.float32)
                assert torch.equal(r.top_ids, want.top_ids + n)


@pytest.mark.parametrize("rows,n", [(3, 300), (2000, 3001), (2, 140001)])
def test_scores_whose_products_with_the_scale_do_not_fit(rows, n):
    hr = _hr()
    _say("large", rows, n)
    g = torch.Generator(device="cuda").manual_seed(n)
    step = torch.randint(-1000, 1000, (rows, n), generator=g, device="cuda").float()
    best = torch.randint(n, (rows, 2), generator=g, device="cuda")
    # two entries share all of p; whole numbers of 2^100 and a scale of 2^30, and the same below 0, beyond the other way
    for offset in (1001.0, 1001.0 - 2**14):
        z = step
        z = z.scatter(1, best, 1000.0) + offset
        z *= 2.0 ** 100
        r = hr.logprobs(z, best, k=1, scale=2.0 ** 30)
        twins = (best[:, :1] != best[:, 1:]).double()                  # (ln 2 where they are two)
        ref.close(r.entropy, math.log(2) * twins[:, 0], 1e-6, torch.float32)
        ref.close(r.logprobs, (-math.log(2) * twins).expand(-1, 2), 1e-6, torch.float32)
        assert torch.equal(r.norm[:, 0], z.amax(1)) and torch.equal(r.top_ids[:, 0], best.amin(1))
    # the largest scale that there is: two entries 2^-99 apart are a factor exp(-1e30 / 2^99) = exp(-1.577) apart
    z = (step - 2000.0).scatter(1, best[:, :1], 0.0)
    other = (best[:, :1] + 1) % n
    z = z.scatter(1, other, -(2.0 ** -99))
    r = hr.logprobs(z, torch.cat([best[:, :1], other], 1), scale=1e30)
    d = float(torch.tensor(1e30, dtype=torch.float32)) * 2.0 ** -99
    want = torch.tensor([0.0, -d], dtype=torch.float64) - math.log1p(math.exp(-d))
    ref.close(r.logprobs, want.expand(rows, 2), 4e-6, torch.float32)
    ref.close(r.entropy, -(want.exp() * want).sum().expand(rows), 4e-6, torch.float32)
    with pytest.raises(hr.HrError):
        hr.logprobs(z, scale=1.1e30)


@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "lowest", "wide"])
@pytest.mark.parametrize("rows,n", [(1, 1), (2, 7), (5, 64), (3, 65), (7, 1000), (4, 4099), (2, 32003), (300, 333), (2, 131073), (1100, 2050), (1, 600001)])
def test_gradient_of_logprobs_and_entropy(rows, n, kind):
    hr = _hr()
    dtype = TYPES[(rows + n + len(kind)) % 3]
    scale = [1.0, 0.5, 3.0][n % 3]
    _say("gradient", rows, n, kind, dtype, scale)
    z = _scores(kind, rows, n, dtype, n + 1)
    g = _gen(rows)
    given = torch.randint(-1, n + 1, (rows, 3), generator=g, device="cuda")
    given[:, 1] = given[:, 0]                              # given twice: counts twice
    up, uh = torch.randn(rows, 3, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    uh[0] = 0
    r = hr.logprobs(z, given, scale=scale)
    want, tol = ref.logprobs_grad(z, scale, given, up, uh)
    got = hr.logprobs_backward(z, given, r, up, uh, scale=scale)
    ref.close(got, want, tol, dtype)
    zero = torch.zeros_like(uh)
    ref.close(hr.logprobs_backward(z, given, r, up, None, scale=scale), *ref.logprobs_grad(z, scale, given, up, zero), dtype)
    ref.close(hr.logprobs_backward(z, None, r, None, uh, scale=scale), *ref.logprobs_grad(z, scale, given, up * 0, uh), dtype)
    out, wide = _strided(torch.zeros_like(z), 1, 2, 5.0)   # rows of the gradient that lie otherwise than those of the scores
    assert torch.equal(hr.logprobs_backward(z, given, r, up, uh, scale=scale, out=out), got)
    assert (wide[:, :1] == 5).all() and (wide[:, n + 1:] == 5).all()
    own = z.clone()                                        # in the place of the scores
    assert torch.equal(hr.logprobs_backward(own, given, r, up, uh, scale=scale, out=own), got)


def test_gradient_against_differences():
    """Central differences of the forward call in float32: h = 2^-6 leaves h^2 / 6 times a third derivative (below 4 scale^3
    of these losses' weights) and the forward's rounding over h."""
    hr = _hr()
    n, scale = 40, 1.5
    z = _scores("plain", 1, n, torch.float32, 3) / 2
    z[0, 7] = -INF
    given = torch.tensor([[3, 3, 11, -1, 7]], device="cuda")
    up, uh = torch.tensor([[0.5, -1.0, 0.7, 9.0, 9.0]], device="cuda"), torch.tensor([0.8], device="cuda")
    h = 2.0 ** -6
    batch = z.repeat(2 * n, 1)
    i = torch.arange(n, device="cuda")
    batch[i, i] += h
    batch[n + i, i] -= h
    r = hr.logprobs(batch, given.repeat(2 * n, 1), scale=scale)
    f = (torch.where(r.logprobs > -INF, r.logprobs, 0.0).double() * up.double()).sum(1) + (r.entropy * uh).double()
    diff = (f[:n] - f[n:]) / (2 * h)
    got = hr.logprobs_backward(z, given, hr.logprobs(z, given, scale=scale), up, uh, scale=scale)[0].double()
    tol = h * h / 6 * 4 * scale ** 3 * 3.0 + 3 * 8 * 40 * ref.U / h
    assert float((got - diff).abs().max()) < tol
    ids, teacher = torch.tensor([[5, 2, -1, 30, 7]], device="cuda"), torch.tensor([[1.0, 0.3, 8.0, -0.5, 4.0]], device="cuda")
    loss, _, _ = hr.distill_forward(batch, ids.repeat(2 * n, 1), teacher.repeat(2 * n, 1), scale=scale)
    diff = (loss[:n] - loss[n:]).double() / (2 * h)
    _, g = hr.distill_step(z, ids, teacher, scale=scale)
    assert float((g[0].double() - diff).abs().max()) < tol


def _teacher(z, k, seed):
    rows, n = z.shape
    g = _gen(seed)
    ids = torch.randint(-1, n + 1, (rows, k), generator=g, device="cuda")
    teacher = torch.randn(rows, k, generator=g, device="cuda") * 2
    teacher[torch.rand(rows, k, generator=g, device="cuda") < 0.1] = -INF
    weights = torch.randn(rows, generator=g, device="cuda")
    if rows > 2:
        ids[1] = -1                                        # nobody taught this row
        weights[2] = 0
    if k > 2:
        ids[0, 2] = ids[0, 0]                              # listed twice
    return ids, teacher, weights


@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "lowest", "wide"])
@pytest.mark.parametrize("rows,n,k", [(1, 1, 1), (2, 7, 3), (5, 64, 8), (3, 65, 100), (7, 1000, 16), (4, 4099, 512), (2, 32003, 64), (300, 333, 10),
                                      (2, 131073, 128), (1100, 2050, 20), (1, 600001, 511)])
def test_distillation(rows, n, k, kind):
    hr = _hr()
    dtype = TYPES[(rows + n + len(kind)) % 3]
    scale = [1.0, 0.5, 3.0][k % 3]
    _say("distill", rows, n, k, kind, dtype, scale)
    z = _scores(kind, rows, n, dtype, n + 2)
    ids, teacher, weights = _teacher(z, k, n + k)
    want, loss_tol, grad, grad_tol = ref.distill(z, scale, ids, teacher, weights)
    loss, norm, q = hr.distill_forward(z, ids, teacher, scale=scale)
    ref.close(loss, want, loss_tol, torch.float32)
    got = hr.distill_backward(z, ids, q, norm, weights, scale=scale)
    ref.close(got, grad, grad_tol, dtype)
    loss1, step = hr.distill_step(z, ids, teacher, weights, scale=scale)
    ref.close(loss1, want, loss_tol, torch.float32)
    ref.close(step, grad, grad_tol, dtype)
    ref.close(hr.distill_step(z, ids, teacher, scale=scale)[1], *ref.distill(z, scale, ids, teacher, torch.ones_like(weights))[2:], dtype)
    again = hr.distill_step(z, ids, teacher, weights, scale=scale)
    assert torch.equal(again[0], loss1) and torch.equal(again[1], step)
    out, wide = _strided(torch.zeros_like(z), 1, 2, 5.0)
    s = _strided(z, 3, 1, INF)[0]
    ref.close(hr.distill_step(s, ids, teacher, weights, scale=scale, out=out)[1], grad, grad_tol, dtype)
    assert (wide[:, :1] == 5).all() and (wide[:, n + 1:] == 5).all()
    own = z.clone()
    loss2, g2 = hr.distill_step(own, ids, teacher, weights, scale=scale, out=own)
    assert g2 is own and torch.equal(loss2, loss1) and torch.equal(own, step)
    own = z.clone()
    assert torch.equal(hr.distill_backward(own, ids, q, norm, weights, scale=scale, out=own), got)


def test_distillation_of_rows_that_take_no_part():
    hr = _hr()
    for n in (50, 40000):
        z = _scores("plain", 5, n, torch.float32, n)
        ids = torch.randint(n, (5, 4), generator=_gen(1), device="cuda")
        teacher = torch.randn(5, 4, generator=_gen(2), device="cuda")
        z[1, 3] = math.nan                                 # weight 0: the gradient is 0 all the same
        z[2, ids[2]] = -INF                                # the student cannot take any of the teacher's entries
        teacher[3] = -INF
        teacher[4, 1] = math.nan
        weights = torch.tensor([1.0, 0.0, 1.0, 1.0, 1.0], device="cuda")
        loss, g = hr.distill_step(z, ids, teacher, weights)
        assert torch.isnan(loss[1]) and not g[1].any()
        assert loss[2] == 0 and not g[2].any() and loss[3] == 0 and not g[3].any()
        assert torch.isnan(loss[4]) and torch.isnan(g[4, ids[4, 0]])
        assert torch.isfinite(loss[0]) and torch.isfinite(g[0]).all()


# ---- where the calls run

def test_nothing_is_written_behind_a_workspace():
    """Exactly the bytes asked for, between guards: what lies around them stays, and the results are those of any workspace."""
    hr = _hr()
    guard = 4096

    def room(need):
        t = torch.full((need + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda")
        assert t.data_ptr() % 256 == 0
        return t, t[guard:]

    def check(t, need):
        torch.cuda.synchronize()
        assert (t[:guard] == 0xA5).all() and (t[guard + need:] == 0xA5).all()

    for m, n, k in ((1, 1000, 768), (17, 300, 4096), (64, 256, 8192), (100, 200, 3333), (300, 100, 1000)):
        x = torch.randn(m, k, generator=_gen(1), device="cuda")
        w, ws = hr.quantize_rows(torch.randn(n, k, generator=_gen(2), device="cuda"))
        need = hr.hr_i8_workspace_bytes(m, n, k)
        t, at = room(need)
        out = torch.empty(m, n, device="cuda")
        hr.hr_i8_linear(x, k, hr.HR_F32, w, w.stride(0), ws, None, m, n, k, out, n, hr.HR_F32, at, need)
        check(t, need)
        assert torch.equal(out, hr.i8_linear(x, w, ws))
        q, s = hr.quantize_rows(x)
        hr.hr_i8_product(q, q.stride(0), s, w, w.stride(0), ws, None, m, n, k, out, n, hr.HR_F32, at, need)
        check(t, need)
        assert torch.equal(out, hr.i8_linear(x, w, ws))
    for rows, n, k in ((1, 100, 5), (1, 200001, 20), (60, 60000, 3), (64, 131072, 128), (255, 50000, 10), (300, 50000, 0)):
        z = _scores("plain", rows, n, torch.float32, n)
        need = hr.hr_logprobs_workspace_bytes(rows, n, k)
        t, at = room(need)
        entropy, norm = torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda")
        ids, top = torch.empty(rows, k, dtype=torch.int64, device="cuda"), torch.empty(rows, k, device="cuda")
        hr.hr_logprobs(z, n, hr.HR_F32, rows, n, 1.0, None, 0, k, None, entropy, norm, ids, top, at, need)
        check(t, need)
        r = hr.logprobs(z, k=k)
        assert torch.equal(entropy, r.entropy) and (k == 0 or torch.equal(ids, r.top_ids))
        kk = max(k, 1)
        want, teacher, weights = _teacher(z, kk, 3)
        need = hr.hr_distill_workspace_bytes(rows, n, kk)
        t, at = room(need)
        loss, g = torch.empty(rows, device="cuda"), torch.empty_like(z)
        hr.hr_distill_step(z, n, hr.HR_F32, rows, n, 1.0, want, teacher, kk, weights, loss, None, None, g, n, at, need)
        check(t, need)
        a, b = hr.distill_step(z, want, teacher, weights)
        assert torch.equal(a, loss) and torch.equal(b, g)


def test_rows_beyond_32_bits():
    """Rows more than 2^31 elements apart: offsets of rows are 64-bit numbers."""
    hr = _hr()
    far = 2 ** 31 + 24
    big = torch.empty(2 * far + 4096, dtype=torch.float16, device="cuda")
    z = big.as_strided((3, 1500), (far, 1), 5)
    z.copy_(_scores("plain", 3, 1500, torch.float16, 1))
    r = _check_logprobs(z, 9, 1.0, torch.tensor([[3], [7], [1499]], device="cuda"))
    want, tol = ref.logprobs_grad(z, 1.0, torch.tensor([[3], [7], [1499]], device="cuda"), torch.ones(3, 1, device="cuda"), torch.ones(3, device="cuda"))
    got = hr.logprobs_backward(z, torch.tensor([[3], [7], [1499]], device="cuda"), r, torch.ones(3, 1, device="cuda"), torch.ones(3, device="cuda"), out=z)
    ref.close(got, want, tol, torch.float16)
    b8 = big.view(torch.int8)
    for m in (2, 70):
        a, b = _i8(m, 256, 3), _i8(4, 256, 4)
        wide = b8.as_strided((4, 256), (far // 16 * 16, 1), 16)
        wide.copy_(b)
        one = torch.ones(m, device="cuda")
        want = (a.cpu().double() @ b.cpu().double().T).float()
        assert torch.equal(hr.i8_product(a, one, wide, torch.ones(4, device="cuda")).cpu(), want)
        assert torch.equal(hr.i8_product(wide, torch.ones(4, device="cuda"), a, one).cpu(), want.T)
        q, s = ref.quantize(big.as_strided((2, 300), (far, 1), 1).copy_(torch.randn(2, 300, generator=_gen(1), device="cuda")))
        got = hr.quantize_rows(big.as_strided((2, 300), (far, 1), 1))
        assert torch.equal(got[0].cpu(), q) and torch.equal(got[1].cpu(), s)


def _chain(hr, x, w, ws, ids, teacher, given):
    z = hr.i8_linear(x, w, ws)
    r = hr.logprobs(z, given, k=5)
    loss, g = hr.distill_step(z, ids, teacher)
    return z, r.logprobs, r.entropy, r.top_ids, loss, g, hr.logprobs_backward(z, given, r, r.logprobs.exp(), r.entropy)


def _chain_inputs(hr, m, n, k, seed):
    g = _gen(seed)
    w, ws = hr.quantize_rows(torch.randn(n, k, generator=_gen(9), device="cuda"))
    return (torch.randn(m, k, generator=g, device="cuda"), w, ws, torch.randint(n, (m, 6), generator=g, device="cuda"),
            torch.randn(m, 6, generator=g, device="cuda"), torch.randint(n, (m, 2), generator=g, device="cuda"))


@pytest.mark.parametrize("m,n,k", [(3, 5000, 256), (200, 3000, 768), (2, 200000, 64)])
def test_another_stream(m, n, k):
    hr = _hr()
    ins = _chain_inputs(hr, m, n, k, 1)
    want = _chain(hr, *ins)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(5):
            got = _chain(hr, *ins)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("m,n,k", [(1, 4000, 768), (100, 2000, 320), (2, 150000, 64)])
def test_captured_in_a_graph(m, n, k):
    """Replayed with new contents, with eager work between the replays: every one equals the eager result."""
    hr = _hr()
    ins = _chain_inputs(hr, m, n, k, 1)
    _chain(hr, *ins)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _chain(hr, *ins)
    for seed in range(2, 6):
        new = _chain_inputs(hr, m, n, k, seed)
        for a, b in zip(ins, new):
            a.copy_(b)
        want = _chain(hr, *new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_empty_batches():
    hr = _hr()
    z = torch.empty(0, 10, device="cuda")
    none = torch.empty(0, 2, dtype=torch.int64, device="cuda")
    r = hr.logprobs(z, none, k=3)
    assert r.top_ids.shape == (0, 3) and r.logprobs.shape == (0, 2)
    assert hr.logprobs_backward(z, none, r, torch.empty(0, 2, device="cuda")).shape == (0, 10)
    loss, g = hr.distill_step(z, none, torch.empty(0, 2, device="cuda"))
    assert loss.shape == (0,) and g.shape == (0, 10)
    w, ws = hr.quantize_rows(torch.randn(4, 10, device="cuda"))
    assert hr.i8_linear(z, w, ws).shape == (0, 4)
    assert hr.i8_product(w, ws, w[:0], ws[:0]).shape == (4, 0)
    assert hr.quantize_rows(z)[0].shape == (0, 10)


def test_what_is_refused():
    hr = _hr()
    z = torch.randn(3, 10, device="cuda")
    ids = torch.zeros(3, 2, dtype=torch.int64, device="cuda")
    t = torch.zeros(3, 2, device="cuda")
    w, ws = hr.quantize_rows(z)
    r = hr.logprobs(z, ids)
    bad = [lambda: hr.logprobs(z.double()), lambda: hr.logprobs(z.cpu()), lambda: hr.logprobs(z[0]), lambda: hr.logprobs(z, k=129),
           lambda: hr.logprobs(z, k=-1), lambda: hr.logprobs(z, scale=0.0), lambda: hr.logprobs(z, scale=math.nan),
           lambda: hr.logprobs(z, scale=INF), lambda: hr.logprobs(z, ids.float()), lambda: hr.logprobs(z, ids[:2]), lambda: hr.logprobs(z, ids.cpu()),
           lambda: hr.logprobs(z, torch.zeros(3, 513, dtype=torch.int64, device="cuda")), lambda: hr.logprobs(z[:, :0]),
           lambda: hr.logprobs_backward(z, None, r, t), lambda: hr.logprobs_backward(z, ids, r, t[:, :1]),
           lambda: hr.logprobs_backward(z, ids, r, t, out=z.T.contiguous().T), lambda: hr.logprobs_backward(z, ids, r, t, out=z.half()),
           lambda: hr.distill_step(z, ids, t.half()), lambda: hr.distill_step(z, ids, t[:, :1]), lambda: hr.distill_step(z, ids[:, :0], t[:, :0]),
           lambda: hr.distill_step(z, ids, t, weights=t), lambda: hr.distill_forward(z, ids, t, scale=-1.0),
           lambda: hr.distill_backward(z, ids, t, r.norm[:2]),
           lambda: hr.i8_linear(z, w.float(), ws), lambda: hr.i8_linear(z, w[:, :9], ws), lambda: hr.i8_linear(z, w, ws[:2]),
           lambda: hr.i8_linear(z, w, ws, dtype=torch.int8), lambda: hr.i8_linear(z, w, ws, bias=ws.half()), lambda: hr.i8_linear(z, w, ws, out=z),
           lambda: hr.i8_product(w, ws, w, ws.cpu()), lambda: hr.quantize_rows(w), lambda: hr.quantize_rows(z[:, :0])]
    for i, call in enumerate(bad):
        with pytest.raises(hr.HrError) as e:
            call()
        assert e.value.code in (-1, -5), i
    ws_small = torch.empty(16, dtype=torch.uint8, device="cuda")
    with pytest.raises(hr.HrError) as e:
        hr.hr_logprobs(z, 10, hr.HR_F32, 3, 10, 1.0, None, 0, 0, None, r.entropy, None, None, None, ws_small, 16)
    assert e.value.code == -3


def test_the_example_teaches_its_encoder(capsys):
    """examples/teach_query_encoder.py, small: search, product in 8 bits, distillation and log probabilities together."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "teach_query_encoder.py")
    spec = importlib.util.spec_from_file_location("teach_query_encoder", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    before, after, losses = example.main(passages=8192, d=128, nlist=64, batch=128, k=16, probes=8, steps=30)
    assert losses[-1] < 0.8 * losses[0] and after > before
