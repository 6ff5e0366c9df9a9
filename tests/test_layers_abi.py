"""hr_layers.h: every declared symbol is exported, constants agree, arguments are refused on the host before anything is enqueued (no GPU
needed); the 64-bit forms that the GPU tests compare with, pinned to examples and to differences."""
import ctypes
import math
import os
import re

import pytest
import torch

import layers_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
A, B, C, D = P(4096), P(8192), P(12288), P(16384)      # never dereferenced: validation fails first
BIG = 1 << 40


@pytest.fixture(scope="module")
def hr():
    import paper_2507_09138_amd as hr
    if not os.path.exists(os.path.join(ROOT, "paper_2507_09138_amd", "libhr_ivf.so")):
        from paper_2507_09138_amd import build
        build.build()
    hr.layer_norm                                      # (resolves the binding, which declares the argument types)
    return hr


def test_every_declared_symbol_is_exported(hr):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hr_layers.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(hr_[a-z0-9_]+)\s*\(", text))
    assert names == {"hr_layer_norm", "hr_layer_norm_workspace_bytes", "hr_layer_norm_backward", "hr_gated_workspace_bytes", "hr_gated",
                     "hr_gated_backward_workspace_bytes", "hr_gated_backward", "hr_adamw", "hr_adamw_moments"}
    for n in names:
        assert hasattr(hr.lib, n) and callable(getattr(hr, n)), n
    for name in ("HR_SILU", "HR_GELU", "HR_GELU_TANH", "HR_ADAMW_BLOCK"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(hr, name)
    assert "#define HR_GATED_MAX (1 << 19)" in text and hr.HR_GATED_MAX == 1 << 19
    assert ctypes.sizeof(hr.hr_adamw_tensor) == 72 and hr.hr_adamw_tensor.weight_decay.offset == 56 and hr.hr_adamw_tensor.grad_dtype.offset == 64


def test_workspaces(hr):
    rows = (0, 1, 2, 3, 15, 16, 17, 64, 100, 511, 512, 513, 4096, 100000)
    for n in (1, 768, 16384, 16385, 50021, 1 << 22, 1 << 30):
        sizes = [hr.hr_layer_norm_workspace_bytes(r, n) for r in rows]
        assert all(s > 0 and s % 256 == 0 for s in sizes) and sizes == sorted(sizes)
        assert sizes[-1] < 100_000 * 8 + max(8 * n, 64 << 20) + 4096
    assert hr.hr_layer_norm_workspace_bytes(-1, 5) == 0 and hr.hr_layer_norm_workspace_bytes(1, 0) == 0 and hr.hr_layer_norm_workspace_bytes(1, (1 << 30) + 1) == 0
    assert hr.hr_layer_norm_workspace_bytes(1 << 31, 5) == 0
    for f in (hr.hr_gated_workspace_bytes, hr.hr_gated_backward_workspace_bytes):
        for k, h in ((1, 1), (100, 333), (768, 2048), (4096, 10752), (999, 40001)):
            for dtype in (0, 1, 2):
                sizes = [f(m, k, h, dtype) for m in (0, 1, 2, 15, 16, 17, 33, 63, 64, 65, 100, 128, 129, 200, 256, 257, 300, 512, 777, 1000, 2048, 4100, 8192, 20000)]
                assert all(s > 0 and s % 256 == 0 for s in sizes), (k, h, dtype)
        for bad in ((-1, 1, 1, 0), (1, 0, 1, 0), (1, 1, 0, 0), (1, 1, 1, 3), ((1 << 19) + 1, 1, 1, 0), (1, (1 << 19) + 1, 1, 0), (1, 1, (1 << 19) + 1, 0)):
            assert f(*bad) == 0, bad
        assert f(1 << 19, 1 << 12, 1 << 15, 0) > 0 and f(1 << 19, 1 << 19, 1 << 19, 0) == 0


def test_norm_arguments(hr):
    L = hr.lib
    base = dict(x=A, ldx=10, dt=0, rows=3, n=10, w=B, b=C, wdt=0, eps=1e-5, out=D, ldo=10, stats=C, dy=B, ldg=10, dx=D, ldgx=10, dw=C, db=C, ws=A, bytes=BIG)

    def forward(**kw):
        v = {**base, **kw}
        return L.hr_layer_norm(v["x"], v["ldx"], v["dt"], v["rows"], v["n"], v["w"], v["b"], v["wdt"], v["eps"], v["out"], v["ldo"], v["stats"], None)

    def backward(**kw):
        v = {**base, **kw}
        return L.hr_layer_norm_backward(v["x"], v["ldx"], v["dt"], v["rows"], v["n"], v["w"], v["wdt"], v["stats"], v["dy"], v["ldg"], v["dx"], v["ldgx"],
                                        v["dw"], v["db"], v["ws"], v["bytes"], None)

    for f in (forward, backward):
        for kw in (dict(x=None), dict(ldx=9), dict(dt=3), dict(wdt=1), dict(dt=1, wdt=2), dict(rows=-1), dict(rows=1 << 31), dict(n=0), dict(n=(1 << 30) + 1, ldx=BIG),
                   dict(x=P(4098)), dict(w=P(4098)), dict(stats=P(4098)), dict(dt=2, x=P(4097))):
            assert f(**kw) == -1, (f, kw)
    for kw in (dict(out=None), dict(ldo=9), dict(out=P(4098)), dict(b=P(4098)), dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf), dict(out=A, ldo=11)):
        assert forward(**kw) == -1, kw
    assert forward(rows=0) == 0 and forward(rows=0, x=None, out=None) == 0
    for kw in (dict(dy=None), dict(ldg=9), dict(ldgx=9), dict(dx=P(4098)), dict(dx=B, ldgx=11), dict(dw=P(4098)), dict(db=P(4098)), dict(stats=None)):
        assert backward(**kw) == -1, kw
    assert backward(ws=None) == -3 and backward(ws=P(4100)) == -3 and backward(bytes=255) == -3


def test_gated_arguments(hr):
    L = hr.lib
    base = dict(x=A, ldx=8, g=B, ldg=8, u=C, ldu=8, dt=0, m=3, k=8, f=6, act=0, out=D, ldo=6, pre=C, ws=A, bytes=BIG, dh=D, ldh=6, dx=D, lddx=8, dg=D, lddg=8, du=D, lddu=8)

    def forward(**kw):
        v = {**base, **kw}
        return L.hr_gated(v["x"], v["ldx"], v["g"], v["ldg"], v["u"], v["ldu"], v["dt"], v["m"], v["k"], v["f"], v["act"], v["out"], v["ldo"], v["pre"], v["ws"], v["bytes"], None)

    def backward(**kw):
        v = {**base, **kw}
        return L.hr_gated_backward(v["x"], v["ldx"], v["g"], v["ldg"], v["u"], v["ldu"], v["dt"], v["m"], v["k"], v["f"], v["act"], v["pre"], v["dh"], v["ldh"],
                                   v["dx"], v["lddx"], v["dg"], v["lddg"], v["du"], v["lddu"], v["ws"], v["bytes"], None)

    for f in (forward, backward):
        for kw in (dict(x=None), dict(g=None), dict(u=None), dict(ldx=7), dict(ldg=7), dict(ldu=7), dict(dt=3), dict(dt=-1), dict(m=-1), dict(k=0), dict(f=0), dict(act=3),
                   dict(act=-1), dict(m=(1 << 19) + 1), dict(k=(1 << 19) + 1, ldx=BIG, ldg=BIG, ldu=BIG), dict(f=(1 << 19) + 1, ldo=BIG, ldh=BIG), dict(x=P(4098)), dict(g=P(4098)),
                   dict(dt=1, u=P(4097)), dict(pre=P(4098))):
            assert f(**kw) == -1, (f, kw)
        assert f(ws=None) == -3 and f(ws=P(4100)) == -3 and f(bytes=255) == -3
        assert f(m=1 << 19, k=1 << 19, f=1 << 19, ldx=BIG, ldg=BIG, ldu=BIG, ldo=BIG, ldh=BIG) == -5
    for kw in (dict(out=None), dict(ldo=5), dict(out=P(4098))):
        assert forward(**kw) == -1, kw
    assert forward(m=0) == 0
    for kw in (dict(pre=None), dict(dh=None), dict(ldh=5), dict(dx=P(4098)), dict(lddx=7), dict(dg=None), dict(du=None), dict(lddg=7), dict(lddu=7), dict(dg=P(4098)), dict(du=P(4098))):
        assert backward(**kw) == -1, kw


def test_adamw_arguments(hr):
    T = hr.hr_adamw_tensor
    fine = dict(param=4096, grad=8192, master=None, m=12288, v=16384, exponents=None, n=5, weight_decay=0.1, param_dtype=0, grad_dtype=0)
    rule = dict(lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, step=1)

    def call(tensors, **kw):
        v = {**rule, **kw}
        t = (T * max(1, len(tensors)))(*[T(**{**fine, **x}) for x in tensors])
        return hr.lib.hr_adamw(ctypes.cast(t, P), len(tensors), v["lr"], v["b1"], v["b2"], v["eps"], v["step"], v.get("dev"), v.get("scale"), None)

    for x in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(n=-1), dict(n=(1 << 36) + 1), dict(weight_decay=math.nan), dict(weight_decay=math.inf),
              dict(param_dtype=3), dict(grad_dtype=-1), dict(master=4096), dict(param=4098), dict(grad=4097, grad_dtype=1), dict(m=12290), dict(v=16385),
              dict(param_dtype=2, master=4098)):
        assert call([{}, x]) == -1, x
        assert "tensor 1" in hr.hr_last_error()
    for kw in (dict(lr=math.nan), dict(lr=math.inf), dict(b1=-0.1), dict(b1=1.0), dict(b2=1.0), dict(b2=math.nan), dict(eps=-1.0), dict(eps=math.inf), dict(step=0),
               dict(dev=P(4100)), dict(scale=P(4098))):
        assert call([{}], **kw) == -1, kw
    assert call([]) == 0 and call([dict(n=0, param=None, grad=None, m=None, v=None)]) == 0
    assert hr.lib.hr_adamw(None, 1, 1e-3, 0.9, 0.9, 0.0, 1, None, None, None) == -1 and hr.lib.hr_adamw(None, -1, 1e-3, 0.9, 0.9, 0.0, 1, None, None, None) == -1
    M = hr.lib.hr_adamw_moments
    assert M(None, B, C, 5, A, D, None) == -1 and M(A, None, C, 5, A, D, None) == -1 and M(A, B, None, 5, A, D, None) == -1 and M(A, B, C, -1, A, D, None) == -1
    assert M(A, B, C, 5, P(4098), D, None) == -1 and M(A, B, C, 0, A, D, None) == 0 and M(A, B, C, 5, None, None, None) == 0


def test_binding_refuses_host_tensors(hr):
    x, w = torch.zeros(3, 8), torch.zeros(5, 8)
    for call in (lambda: hr.layer_norm(x), lambda: hr.layer_norm_backward(x, None, x, x), lambda: hr.gated(x, w, w), lambda: hr.gated_backward(x, w, w, x, x),
                 lambda: hr.adamw([x], [x], [x], [x], 1, 1e-3), lambda: hr.adamw_moments(x, x, x), lambda: hr.adamw([x], [], [x], [x], 1, 1e-3), lambda: hr.adamw_state(x, 16)):
        with pytest.raises(hr.HrError) as e:
            call()
        assert e.value.code == -1
    hr.adamw([], [], [], [], 1, 1e-3)


# ---- the 64-bit forms

def _differences(f, x, h=1e-6):
    g = torch.zeros_like(x)
    for i in range(x.numel()):
        e = torch.zeros_like(x).view(-1)
        e[i] = h
        g.view(-1)[i] = (f(x + e.view_as(x)) - f(x - e.view_as(x))) / (2 * h)
    return g


def test_norm_example_and_differences():
    y = ref.norm(torch.tensor([[1.0, 2.0, 3.0, 6.0]]), None, None, 0.0)[0]
    assert torch.allclose(y, torch.tensor([[-2.0, -1.0, 0.0, 3.0]], dtype=torch.float64) / math.sqrt(3.5))
    g = torch.Generator().manual_seed(1)
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 7), (7,), (7,), (3, 7)))
    dx, dw, db = ref.norm_grads(x, w, dy, 1e-3)[:3]
    assert torch.allclose(dx, _differences(lambda x: float((ref.norm(x, w, b, 1e-3)[0] * dy).sum()), x), atol=1e-8)
    assert torch.allclose(dw, _differences(lambda w: float((ref.norm(x, w, b, 1e-3)[0] * dy).sum()), w), atol=1e-8)
    assert torch.allclose(db, _differences(lambda b: float((ref.norm(x, w, b, 1e-3)[0] * dy).sum()), b), atol=1e-8)


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
def test_gated_examples_and_differences(name):
    z = torch.tensor([0.0, 1.0, -1.0, 40.0, -40.0], dtype=torch.float64)
    at_one = {"silu": 0.7310585786300049, "gelu": 0.8413447460685429, "gelu_tanh": 0.8411919906082768}[name]
    assert torch.allclose(ref.act(z, name)[0], torch.tensor([0.0, at_one, at_one - 1, 40.0, 0.0], dtype=torch.float64), atol=1e-12)
    g = torch.Generator().manual_seed(2)
    x, wg, wu, dh = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 4), (5, 4), (5, 4), (3, 5)))
    pre = torch.stack([x @ wg.T, x @ wu.T], 1)
    got = ref.gated_grads(x, wg, wu, pre, dh, name, torch.float32)[:3]
    for i, t in enumerate((x, wg, wu)):
        args = [x, wg, wu]

        def f(t, i=i, args=args):
            return float((ref.gated(*(t if j == i else a for j, a in enumerate(args)), name)[0] * dh).sum())
        assert torch.allclose(got[i], _differences(f, t), atol=1e-7)


def test_adamw_example():
    """One number, two steps by hand; a first step is lr in size whatever the gradient."""
    p, g = torch.tensor([2.0]), torch.tensor([0.25])
    new, m, v, *_ = ref.adamw(p, g, torch.zeros(1), torch.zeros(1), 1, 0.1, (0.9, 0.99), 0.0, 0.5)
    assert torch.allclose(new, torch.tensor([2 * (1 - 0.05) - 0.1], dtype=torch.float64)) and torch.allclose(m, torch.tensor([0.025], dtype=torch.float64))
    new, m, v, *_ = ref.adamw(new, g, m, v, 2, 0.1, (0.9, 0.99), 0.0, 0.5)
    assert torch.allclose(new, torch.tensor([1.8 * 0.95 - 0.1], dtype=torch.float64))


def test_codes_of_moments():
    """The table of e4m3 is torch's; every number that codes stand for is held as itself; halves go to the even code; nothing becomes 0."""
    table = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(table.nan_to_num(500.0), ref.E4M3.nan_to_num(500.0))
    codes = torch.arange(256, dtype=torch.uint8)
    for ev in (31, 32, 100, 127, 254):
        m, v = ref.decode(torch.where((codes & 127) > 119, codes & 119, codes), codes, torch.tensor([[max(ev - 1, 8), ev]], dtype=torch.uint8))
        if ev < 254 and ev != 31:                                    # (the largest code has to be there for the exponent to be this one; v's is 31 or the top code's)
            assert torch.equal(ref.held(torch.zeros(256), v.float())[1], v)
    assert torch.equal(ref.decode(codes, codes, torch.tensor([[255, 255]], dtype=torch.uint8))[0].isnan(), torch.ones(256, dtype=torch.bool))
    x = torch.zeros(256)
    x[:5] = torch.tensor([1.0, 1.0625, 1.1875, 2.0 ** -40, 1.9])
    m, v = ref.held(x, x)
    assert v[:3].tolist() == [1.0, 1.0, 1.25] and v[3] == 1.125 * 2.0 ** -31 and v[4] == 1.875 and v[5] == 0
    assert m[:3].tolist() == [1.0, 1.0, 1.25] and m[3] == 0
