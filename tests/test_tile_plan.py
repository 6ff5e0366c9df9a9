"""Which tiles and parts of k the products of gated blocks take (host arithmetic, no GPU)."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r'''
#include "tile_plan.h"
namespace hr { int fail(int code, const char*, ...) { return code; } }
using namespace hr;
// products of [m, n, bytes of k], 1 or 2: bm, bn, then of each parts, part_k, large
extern "C" void plan(int gated, long es, int count, const long* shapes, long* out)
{
    TileArgs p[2] = {};
    for (int i = 0; i < count; ++i) {
        p[i].m = shapes[3 * i];
        p[i].n = shapes[3 * i + 1];
        p[i].k = (int)shapes[3 * i + 2];
    }
    const Tiling t = plan_tiles(gated, es, p, count);
    out[0] = t.bm;
    out[1] = t.bn;
    for (int i = 0; i < count; ++i) {
        out[2 + 3 * i] = p[i].parts;
        out[3 + 3 * i] = p[i].part_k;
        out[4 + 3 * i] = p[i].large;
    }
}
'''


def _whole(n, es):
    return -(-n * es // 128) * 128


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("plan")
    (tmp / "plan.cpp").write_text(SOURCE)
    so = str(tmp / "plan.so")
    subprocess.run(["hipcc", "-x", "hip", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2507_09138_amd", "csrc"), str(tmp / "plan.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.plan.argtypes = [ctypes.c_int, ctypes.c_long, ctypes.c_int, ctypes.POINTER(ctypes.c_long), ctypes.POINTER(ctypes.c_long)]

    def ask(gated, es, *shapes):
        """(bm, bn), [(parts, part_k, large)] of products [m, n, bytes of k]."""
        out = (ctypes.c_long * 8)()
        lib.plan(gated, es, len(shapes), (ctypes.c_long * 6)(*[x for s in shapes for x in s]), out)
        return (out[0], out[1]), [tuple(out[2 + 3 * i:5 + 3 * i]) for i in range(len(shapes))]
    return ask


def _forward(plan, m, k, f, es):
    return plan(1, es, (m, f, _whole(k, es)))


def _backward(plan, m, k, f, es):
    return plan(0, es, (m, k, 2 * _whole(f, es)), (2 * f, k, _whole(m, es)))


SHAPES = [(m, k, f) for m in (33, 64, 65, 300, 777, 1100, 2050, 2100, 4100, 8192) for k in (64, 200, 768, 1032, 2048, 4096) for f in (100, 1333, 5128, 6152, 9000, 10752)]


@pytest.mark.parametrize("es", [2, 4])
def test_rows_are_left_to_small_tiles_only_where_that_was_counted(plan, es):
    """The count of large tiles for whole rounds and small ones for the other rows is that of products in one part: none of a launch in parts is cut."""
    cut = split = 0
    for m, k, f in SHAPES:
        for (bm, bn), parts in (_forward(plan, m, k, f, es), _backward(plan, m, k, f, es)):
            rows = (m, 2 * f)
            left = [large < r for (_, _, large), r in zip(parts, rows)]
            assert all(0 <= large <= r for (_, _, large), r in zip(parts, rows))
            assert not any(left) or (bm == 256 and all(n == 1 for n, _, _ in parts)), (m, k, f, es)
            cut += any(left)
            split += any(n > 1 for n, _, _ in parts)
    assert split > 20 and (cut > 20 or es == 4)
