"""The C entry points of hr_layers.h by themselves, where the tensor functions always ask for the same: gradients at distances and odd places of their own, one of two
vector gradients, workspaces of layer norm between guards, with one for all batches."""
import pytest
import torch

from test_gated_workspaces import CODE, Room, _hr, _inputs

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def _wide(rows, cols, before, behind, dtype):
    """A slice of columns of a matrix full of sevens, and the matrix."""
    whole = torch.full((rows, before + cols + behind), 7.0, dtype=dtype, device="cuda")
    return whole[:, before:before + cols], whole


def _kept(whole, before, cols):
    return bool((whole[:, :before] == 7).all()) and bool((whole[:, before + cols:] == 7).all())


# few rows, small tiles, parts of k, many tiles, large tiles with rows left to small ones
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("m,k,f", [(0, 33, 20), (3, 100, 70), (40, 2048, 96), (300, 200, 131), (2050, 1100, 2100), (1024, 4040, 2072)])
def test_gradients_of_gated_blocks_at_odd_places(m, k, f, dtype):
    """Those of both matrices as halves of one, side by side, and all three at distances of their own; nothing beside them is written."""
    hr = _hr()
    print("case", m, k, f, dtype, flush=True)
    x, wg, wu, dh = _inputs(m, k, f, dtype)
    kind = CODE[dtype]
    if m:
        r = hr.gated(x, wg, wu, keep=True)
        want, pre = hr.gated_backward(x, wg, wu, r.pre, dh), r.pre
    else:
        want, pre = (torch.zeros(s, k, dtype=dtype, device="cuda") for s in (0, f, f)), torch.empty(0, 2, f, device="cuda")
    room = Room(hr.hr_gated_backward_workspace_bytes(m, k, f, kind))
    dx, dx_all = _wide(m, k, 3, 2, dtype)
    both = torch.full((f, 2 * k + 6), 7.0, dtype=dtype, device="cuda")                  # gate's, one number, up's, between others
    dg, du = both[:, 2:2 + k], both[:, 3 + k:3 + 2 * k]
    hr.hr_gated_backward(x, k, wg, k, wu, k, kind, m, k, f, hr.HR_SILU, pre, dh, f, dx, dx_all.stride(0), dg, both.stride(0), du, both.stride(0), room.at, room.need)
    room.check()
    assert all(torch.equal(a, b) for a, b in zip((dx, dg, du), want))
    assert _kept(dx_all, 3, k) and bool((both[:, :2] == 7).all()) and bool((both[:, 2 + k] == 7).all()) and bool((both[:, 3 + 2 * k:] == 7).all())
    # the gradient of x or those of the matrices alone
    dx_all.fill_(7.0)
    kept = both.clone()
    hr.hr_gated_backward(x, k, wg, k, wu, k, kind, m, k, f, hr.HR_SILU, pre, dh, f, dx, dx_all.stride(0), None, 0, None, 0, room.at, room.need)
    room.check()
    assert _kept(dx_all, 3, k) and torch.equal(both, kept)
    both.fill_(7.0)
    hr.hr_gated_backward(x, k, wg, k, wu, k, kind, m, k, f, hr.HR_SILU, pre, dh, f, None, 0, dg, both.stride(0), du, both.stride(0), room.at, room.need)
    room.check()
    assert torch.equal(both, kept)


# rows that 16 lanes hold, a wave, workgroups; longer ones in stripes; one row and more than there are workgroups
NORMS = [(1, 3), (5, 100), (700, 33), (9, 1000), (33, 4096), (1300, 768), (3, 8200), (5, 16384), (2, 16385), (4, 50021), (1, 300000)]


def _norm_inputs(rows, n, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + n)
    return [torch.randn(*s, generator=g, device="cuda") for s in ((rows, n), (n,), (rows, n))], dtype


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rows,n", NORMS)
def test_layer_norm_asks_for_what_it_uses(rows, n, dtype):
    """A workspace of exactly its size, one of both vector gradients, none, and neither rows nor vectors' neighbours written."""
    hr = _hr()
    print("case", rows, n, dtype, flush=True)
    (x, w, dy), _ = _norm_inputs(rows, n, dtype)
    x, dy = x.to(dtype), dy.to(dtype)
    stats = hr.layer_norm(x, w).stats
    want = hr.layer_norm_backward(x, w, stats, dy)
    room = Room(hr.hr_layer_norm_workspace_bytes(rows, n))
    for weight, bias, out in ((True, True, True), (True, False, True), (False, True, True), (False, False, True), (True, True, False), (False, True, False)):
        dx, dx_all = _wide(rows, n, 1, 2, dtype)
        vectors = torch.full((2, n + 2), 7.0, device="cuda")
        dw, db = vectors[0, 1:-1], vectors[1, 1:-1]
        hr.hr_layer_norm_backward(x, n, CODE[dtype], rows, n, w, CODE[F32], stats, dy, n, dx if out else None, dx_all.stride(0), dw if weight else None, db if bias else None,
                                  room.at, room.need)
        room.check()
        assert _kept(dx_all, 1, n) and bool((vectors[:, 0] == 7).all()) and bool((vectors[:, -1] == 7).all())
        for asked, got, should in ((out, dx, want.x), (weight, dw, want.weight), (bias, db, want.bias)):
            assert torch.equal(got, should) if asked else bool((got == 7).all())


@pytest.mark.parametrize("n", [100, 4096, 16384, 20000])
def test_one_workspace_of_layer_norm_for_all_batches(n):
    hr = _hr()
    (x, w, dy), _ = _norm_inputs(1030, n, F32)
    room = Room(hr.hr_layer_norm_workspace_bytes(1030, n))
    for rows in (0, 1, 2, 100, 511, 513, 1030):
        stats = hr.layer_norm(x[:rows], w).stats
        want = hr.layer_norm_backward(x[:rows], w, stats, dy[:rows])
        dx, dw, db = torch.empty(rows, n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        hr.hr_layer_norm_backward(x, n, 0, rows, n, w, 0, stats, dy, n, dx, n, dw, db, room.at, room.need)
        room.check()
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), want))
