"""Products of up to 16 rows a: whether a shape fits the LDS of a workgroup (host arithmetic, no GPU), and products on both sides of that."""
import ctypes
import os
import re
import subprocess

import pytest

import test_scores as scores

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIMIT = 160 * 1024                     # LDS of a workgroup on gfx950


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("few")
    (tmp / "few.cpp").write_text('#include "i8_few.h"\nextern "C" void few(long m, long n, long k, int* out)\n'
                                 '{ using namespace hr; const int s = few_share(n, (int)k); out[0] = few_rows(m, n, k); out[1] = s; out[2] = few_lds((int)m, (int)k, s);\n'
                                 '  out[3] = kRingBytes; out[4] = few_zeros((int)m, (int)k); out[5] = few_scales((int)m, (int)k); out[6] = few_sums((int)m, (int)k); }\n')
    so = str(tmp / "few.so")
    subprocess.run(["hipcc", "-x", "hip", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2507_09138_amd", "csrc"), str(tmp / "few.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.few.argtypes = [ctypes.c_long] * 3 + [ctypes.POINTER(ctypes.c_int)]

    def ask(m, n, k):
        out = (ctypes.c_int * 7)()
        lib.few(m, n, k, out)
        return tuple(out)
    return ask


def test_every_launch_fits(rule):
    """What the parts take, added up here once more: of every shape that is let through, with one wave and with eight for rows of b."""
    shares, refused = set(), set()
    for m in range(1, 17):
        for k in sorted({*range(128, 131072, 128), *range(129, 131072, 1280), 1, 127, 131071}):
            for n in (1, 64, 4096, 16384, 32753, 65520, 65521, 1 << 20):
                takes, share, lds, rings, zeros, scales, sums = rule(m, n, k)
                row = -(-k // 128) * 128 + 16
                assert share in (1, 2, 4, 8) and (share == 1 or -(-k // 128) >= 2 * share)
                want = 8 * 4 * 2048 + m * row + 16 + 16 * 4 + 16 * 4 + (7 * 64 * 16 if share > 1 else 0)
                assert lds == want and rings == 65536 and zeros == rings + m * row and scales == zeros + 16 and sums == scales + 128
                assert all(at % 16 == 0 for at in (zeros, scales, sums))
                if takes:
                    assert want <= LIMIT, (m, n, k)
                    shares.add(share)
                else:
                    refused.add(m)
    assert shares == {1, 2, 4, 8} and refused == set(range(1, 17))
    assert not any(rule(17, n, 128)[0] for n in (1, 1 << 20))


def test_the_kernel_has_no_other_lds():
    """Where something static is declared in the kernel, it has to be counted."""
    text = open(os.path.join(ROOT, "paper_2507_09138_amd", "csrc", "i8.hip")).read()
    body = text[text.index("void k_i8_few("):text.index("static hipError_t launch_quantize")]
    assert [ln for ln in body.splitlines() if "__shared__" in ln and "extern __shared__" not in ln] == []


def test_the_limit_that_a_launch_sets_is_the_same_for_all():
    """The attribute belongs to the process: a launch that set its own size would take room from one of another thread."""
    text = open(os.path.join(ROOT, "paper_2507_09138_amd", "csrc", "i8.hip")).read()
    body = text[text.index("static hipError_t launch_few("):text.index("struct Tiling")]
    assert re.findall(r"MaxDynamicSharedMemorySize, ([^)]*)\)", body) == ["kWorkgroupLds"]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(16, 64, 5504), (16, 64, 5632), (16, 300, 5633), (16, 70000, 5632), (15, 100, 6016), (13, 100, 7040), (11, 300, 8192), (8, 200, 11392),
                                   (8, 100, 11008), (4, 50, 22400), (2, 40, 45000), (1, 33, 90000), (1, 33, 92032)])
@pytest.mark.parametrize("lay", ["padded", "odd"])
def test_products_where_rows_no_longer_fit(m, n, k, lay):
    scores._say("few", m, n, k, lay)
    scores._check_product(m, n, k, scores.TYPES[(m + n) % 3], True, lay)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", [(16, 64, 5632), (11, 300, 8192), (8, 200, 11392), (1, 33, 92032)])
@pytest.mark.parametrize("dtype", scores.TYPES)
def test_linear_where_rows_no_longer_fit(m, n, k, dtype):
    scores._say("few linear", m, n, k, dtype)
    hr = scores._hr()
    x = scores.torch.randn(m, k, generator=scores._gen(m), device="cuda").to(dtype)
    w, ws = hr.quantize_rows(scores.torch.randn(n, k, generator=scores._gen(n), device="cuda"))
    q, s = hr.quantize_rows(x)
    got = hr.i8_linear(x, w, ws, dtype=dtype)
    assert scores.torch.equal(got, hr.i8_product(q, s, w, ws, dtype=dtype))
    rq, rs = scores.ref.quantize(x)
    scores.ref.close(got, *scores.ref.product(rq, rs, w.cpu(), ws.cpu(), None), dtype)


@pytest.mark.gpu
def test_threads_with_launches_of_different_sizes():
    """Two threads whose launches of the same kernel want little and much of LDS: neither's takes room from the other's."""
    import threading
    hr, torch = scores._hr(), scores.torch
    ins, want, failed = [], [], []
    for m, k in ((1, 256), (16, 5504)):
        x = torch.randn(m, k, generator=scores._gen(m), device="cuda").half()
        w, ws = hr.quantize_rows(torch.randn(100, k, generator=scores._gen(k), device="cuda"))
        q, s = hr.quantize_rows(x)
        ins.append((q, s, w, ws))
        want.append(hr.i8_product(*ins[-1]))
    torch.cuda.synchronize()

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                got = [hr.i8_product(*ins[i]) for _ in range(500)]
            torch.cuda.synchronize()
            if not all(torch.equal(g, want[i]) for g in got):
                failed.append((i, "other values"))
        except Exception as e:                             # (said below, not in the thread)
            failed.append((i, e))

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
