"""Workspaces of gated blocks: what is enough for a batch is enough for every smaller one (no GPU), and the calls on the GPU use no more than they ask for."""
import os

import pytest
import torch


def _hr():
    import paper_2507_09138_amd as hr
    from paper_2507_09138_amd import build
    if not os.path.exists(build.LIB):
        build.build()
    return hr


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("k,f", [(1, 1), (64, 64), (100, 333), (768, 2048), (1000, 1333), (4096, 10752), (8192, 74), (132, 8278), (2048, 6152), (72, 70000)])
def test_enough_for_fewer_rows(k, f, dtype):
    hr = _hr()
    rows = [*range(0, 700), *range(700, 2600, 61), 4095, 4096, 4097, 8192, 8193, 20000]
    for of in (hr.hr_gated_workspace_bytes, hr.hr_gated_backward_workspace_bytes):
        sizes = [of(m, k, f, dtype) for m in rows]
        assert all(s > 0 and s % 256 == 0 for s in sizes)
        worse = [(rows[i], rows[i + 1]) for i in range(len(rows) - 1) if sizes[i] > sizes[i + 1]]
        assert not worse, worse[:5]


F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
CODE = {F32: 0, F16: 1, BF16: 2}
GUARD = 4096


class Room:
    """A workspace of exactly so many bytes between guards."""

    def __init__(self, need):
        self.all, self.need = torch.full((need + 2 * GUARD,), 0xA5, dtype=torch.uint8, device="cuda"), need
        assert self.all.data_ptr() % 256 == 0
        self.at = self.all[GUARD:]

    def check(self):
        torch.cuda.synchronize()
        assert bool((self.all[:GUARD] == 0xA5).all()) and bool((self.all[GUARD + self.need:] == 0xA5).all())


def _inputs(m, k, f, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(m + k + f)

    def some(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    return some(m, k).to(dtype), (some(f, k) / k ** 0.5).to(dtype), (some(f, k) / k ** 0.5).to(dtype), some(m, f).to(dtype)


def _both_ways(hr, x, wg, wu, dh, dtype, forward, backward):
    """Forward and backward in these two workspaces."""
    (m, k), f = x.shape, wg.shape[0]
    kind = CODE[dtype]
    out, pre = torch.empty(m, f, dtype=dtype, device="cuda"), torch.empty(m, 2, f, device="cuda")
    hr.hr_gated(x, x.stride(0), wg, wg.stride(0), wu, wu.stride(0), kind, m, k, f, hr.HR_SILU, out, f, pre, forward.at, forward.need)
    dx, dg, du = torch.empty_like(x, memory_format=torch.contiguous_format), torch.empty(f, k, dtype=dtype, device="cuda"), torch.empty(f, k, dtype=dtype, device="cuda")
    hr.hr_gated_backward(x, x.stride(0), wg, wg.stride(0), wu, wu.stride(0), kind, m, k, f, hr.HR_SILU, pre, dh, dh.stride(0), dx, k, dg, k, du, k,
                         backward.at, backward.need)
    forward.check()
    backward.check()
    return out, pre, dx, dg, du


def _binding(hr, x, wg, wu, dh):
    r = hr.gated(x, wg, wu, keep=True)
    return (*r, *hr.gated_backward(x, wg, wu, r.pre, dh))


# single rows and few, tiles of each size, in parts of k and not, one workgroup a tile and many tiles a workgroup
SIZES = [(1, 100, 70), (20, 768, 512), (40, 1000, 333), (64, 2048, 300), (100, 4096, 130), (300, 200, 130), (777, 1000, 1333), (2050, 1100, 2100), (4100, 1032, 4104)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("m,k,f", SIZES)
def test_nothing_is_written_behind_a_workspace(m, k, f, dtype):
    """Exactly the bytes asked for, operands as they are and (all but the largest) at odd places, which are copied: the results are those of any workspace."""
    hr = _hr()
    print("case", m, k, f, dtype, flush=True)
    ops = _inputs(m, k, f, dtype)
    odd = [torch.zeros(t.shape[0], t.shape[1] + 3, dtype=dtype, device="cuda")[:, 1:-2].copy_(t) for t in ops]
    for x, wg, wu, dh in [ops, odd] if m < 2000 else [ops]:
        rooms = Room(hr.hr_gated_workspace_bytes(m, k, f, CODE[dtype])), Room(hr.hr_gated_backward_workspace_bytes(m, k, f, CODE[dtype]))
        got = _both_ways(hr, x, wg, wu, dh, dtype, *rooms)
        assert all(torch.equal(a, b) for a, b in zip(got, _binding(hr, x, wg, wu, dh)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("most,k,f", [(300, 1000, 777), (129, 4096, 200), (1100, 64, 96)])
def test_one_workspace_for_all_batches(most, k, f, dtype):
    """Asked for once, for the largest batch, and used for smaller ones, which may be in more parts."""
    hr = _hr()
    print("case", most, k, f, dtype, flush=True)
    x, wg, wu, dh = _inputs(most, k, f, dtype)
    rooms = Room(hr.hr_gated_workspace_bytes(most, k, f, CODE[dtype])), Room(hr.hr_gated_backward_workspace_bytes(most, k, f, CODE[dtype]))
    for m in sorted({0, 1, 17, 32, 33, 64, 65, 96, 97, 128, 200, 256, 257, 640, most}):
        if m <= most:
            got = _both_ways(hr, x[:m], wg, wu, dh[:m], dtype, *rooms)
            assert all(torch.equal(a, b) for a, b in zip(got, _binding(hr, x[:m], wg, wu, dh[:m]))), m
