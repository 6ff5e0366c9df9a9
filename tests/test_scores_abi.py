"""hr_scores.h: every declared symbol is exported, constants agree, and arguments are refused on the host before anything
is enqueued (no GPU needed); the 64-bit forms that the GPU tests compare with, pinned to examples and to differences."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import scores_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
A, B, C, D = P(4096), P(8192), P(12288), P(16384)      # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def hr():
    import paper_2507_09138_amd as hr
    if not os.path.exists(os.path.join(ROOT, "paper_2507_09138_amd", "libhr_ivf.so")):
        from paper_2507_09138_amd import build
        build.build()
    hr.logprobs                                        # (resolves the binding, which declares the argument types)
    return hr


def test_every_declared_symbol_is_exported(hr):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hr_scores.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(hr_[a-z0-9_]+)\s*\(", text))
    assert {"hr_i8_quantize", "hr_i8_product", "hr_i8_linear", "hr_logprobs", "hr_logprobs_backward", "hr_distill_forward", "hr_distill_backward",
            "hr_distill_step"} <= names
    for n in names:
        assert hasattr(hr.lib, n) and callable(getattr(hr, n)), n
    assert int(re.search(r"#define HR_I8_K_MAX (\d+)", text).group(1)) == hr.HR_I8_K_MAX
    assert int(re.search(r"#define HR_LIST_MAX (\d+)", text).group(1)) == hr.HR_LIST_MAX


def test_workspace_of_fewer_rows_is_enough(hr):
    for f in (lambda r: hr.hr_i8_workspace_bytes(r, 5000, 768), lambda r: hr.hr_logprobs_workspace_bytes(r, 131072, 20),
              lambda r: hr.hr_distill_workspace_bytes(r, 131072, 20)):
        sizes = [f(r) for r in (1, 2, 3, 7, 16, 17, 60, 64, 65, 200, 256, 300, 511, 512, 1000, 2000, 5000)]
        assert all(s > 0 and s % 256 == 0 for s in sizes) and sizes == sorted(sizes)
    sizes = [hr.hr_logprobs_workspace_bytes(8, 131072, k) for k in range(0, 129)]
    assert sizes == sorted(sizes)
    assert hr.hr_i8_workspace_bytes(5, 0, 700) > 0 and hr.hr_i8_workspace_bytes(0, 5, 700) > 0          # (nothing to do, but no error)
    assert hr.hr_i8_workspace_bytes(1, 1, 0) == 0 and hr.hr_i8_workspace_bytes(-1, 1, 1) == 0 and hr.hr_i8_workspace_bytes(1, 1, 131072) == 0
    assert hr.hr_logprobs_workspace_bytes(1, 0, 1) == 0 and hr.hr_logprobs_workspace_bytes(1, 10, 129) == 0
    assert hr.hr_distill_workspace_bytes(1, 10, 0) == 0 and hr.hr_distill_workspace_bytes(1, 10, 513) == 0


def test_product_arguments(hr):
    L = hr.lib
    big = 1 << 40
    q = dict(x=A, ldx=64, dtype=0, m=4, k=64, q=B, ldq=64, scale=C)

    def quantize(**kw):
        v = {**q, **kw}
        return L.hr_i8_quantize(v["x"], v["ldx"], v["dtype"], v["m"], v["k"], v["q"], v["ldq"], v["scale"], None)

    for kw in (dict(x=None), dict(q=None), dict(scale=None), dict(ldx=63), dict(ldq=63), dict(dtype=3), dict(dtype=-1), dict(m=-1), dict(k=0),
               dict(x=P(4098)), dict(dtype=1, x=P(4097)), dict(k=(1 << 30) + 1, ldx=big, ldq=big)):
        assert quantize(**kw) == -1, kw
    assert quantize(m=0) == 0

    p = dict(a=A, lda=64, sa=B, b=C, ldb=64, sb=D, bias=None, m=4, n=4, k=64, out=A, ldo=4, dt=0, ws=B, bytes=big)

    def product(**kw):
        v = {**p, **kw}
        return L.hr_i8_product(v["a"], v["lda"], v["sa"], v["b"], v["ldb"], v["sb"], v["bias"], v["m"], v["n"], v["k"], v["out"], v["ldo"], v["dt"],
                               v["ws"], v["bytes"], None)

    def linear(**kw):
        v = {**p, "dt_x": 0, **kw}
        return L.hr_i8_linear(v["a"], v["lda"], v["dt_x"], v["b"], v["ldb"], v["sb"], v["bias"], v["m"], v["n"], v["k"], v["out"], v["ldo"], v["dt"],
                              v["ws"], v["bytes"], None)

    for f in (product, linear):
        for kw in (dict(a=None), dict(b=None), dict(sb=None), dict(out=None), dict(lda=63), dict(ldb=63), dict(ldo=3), dict(dt=9), dict(m=-1), dict(n=-1),
                   dict(k=0), dict(k=131072, lda=131072, ldb=131072), dict(out=P(4098)), dict(dt=2, out=P(4097))):
            assert f(**kw) == -1, (f, kw)
        assert f(ws=None) == -3 and f(ws=P(4100)) == -3 and f(bytes=255) == -3
        assert f(m=1 << 24, n=(1 << 31) - 1, ldo=1 << 31) == -5
        assert f(m=0) == 0 and f(n=0) == 0
    assert product(sa=None) == -1 and linear(dt_x=5) == -1 and linear(a=P(4098)) == -1
    assert "x is not aligned" in hr.hr_last_error()


def test_row_arguments(hr):
    L = hr.lib
    big = 1 << 40
    base = dict(z=A, ld=10, dt=0, rows=3, n=10, scale=1.0, ids=B, k=2, vals=C, ws=D, bytes=big, given=B, ng=2, lp=C, out=D, ldg=10, norm=C, loss=C, entropy=C,
                gl=C, ge=C, top_ids=B, top=C, q=C)

    def call(which, **kw):
        v = {**base, **kw}
        z = (v["z"], v["ld"], v["dt"], v["rows"], v["n"], v["scale"])
        if which == "logprobs":
            return L.hr_logprobs(*z, v["given"], v["ng"], v["k"], v["lp"], v["entropy"], v["norm"], v["top_ids"], v["top"], v["ws"], v["bytes"], None)
        if which == "logprobs_backward":
            return L.hr_logprobs_backward(*z, v["given"], v["ng"], v["entropy"], v["norm"], v["gl"], v["ge"], v["out"], v["ldg"], None)
        if which == "forward":
            return L.hr_distill_forward(*z, v["ids"], v["vals"], v["k"], v["loss"], v["norm"], v["q"], v["ws"], v["bytes"], None)
        if which == "backward":
            return L.hr_distill_backward(*z, v["ids"], v["q"], v["k"], v["norm"], None, v["out"], v["ldg"], None)
        return L.hr_distill_step(*z, v["ids"], v["vals"], v["k"], None, v["loss"], None, None, v["out"], v["ldg"], v["ws"], v["bytes"], None)

    for which in ("logprobs", "logprobs_backward", "forward", "backward", "step"):
        for kw in (dict(z=None), dict(ld=9), dict(dt=3), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(n=0), dict(n=(1 << 30) + 1, ld=1 << 31, ldg=1 << 31),
                   dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(z=P(4098)), dict(dt=1, z=P(4097))):
            assert call(which, **kw) == -1, (which, kw)
        assert call(which, rows=0) == 0
    for which in ("logprobs_backward", "backward", "step"):
        for kw in (dict(out=None), dict(ldg=9), dict(out=P(4098)), dict(out=A, ldg=11)):
            assert call(which, **kw) == -1, (which, kw)
    for which in ("logprobs", "forward", "step"):
        assert call(which, ws=None) == -3 and call(which, ws=P(4100)) == -3 and call(which, bytes=10) == -3, which
    for kw in (dict(ng=-1), dict(ng=513), dict(k=-1), dict(k=129), dict(given=None), dict(lp=None), dict(top_ids=None), dict(top=None)):
        assert call("logprobs", **kw) == -1, kw
    for kw in (dict(ng=513), dict(norm=None), dict(given=None), dict(entropy=None)):
        assert call("logprobs_backward", **kw) == -1, kw
    for which in ("forward", "backward", "step"):
        for kw in (dict(k=0), dict(k=513), dict(ids=None)):
            assert call(which, **kw) == -1, (which, kw)
    assert call("forward", vals=None) == -1 and call("forward", loss=None) == -1 and call("step", vals=None) == -1 and call("backward", q=None) == -1
    assert call("backward", norm=None) == -1


def test_binding_refuses_host_tensors(hr):
    z, ids, t = torch.zeros(3, 8), torch.zeros(3, 2, dtype=torch.int64), torch.zeros(3, 2)
    q = torch.zeros(3, 8, dtype=torch.int8)
    for call in (lambda: hr.logprobs(z), lambda: hr.distill_forward(z, ids, t), lambda: hr.distill_step(z, ids, t), lambda: hr.quantize_rows(z),
                 lambda: hr.i8_linear(z, q, t[:, 0]), lambda: hr.i8_product(q, t[:, 0], q, t[:, 0]),
                 lambda: hr.distill_backward(z, ids, t, t), lambda: hr.logprobs_backward(z, ids, None)):
        with pytest.raises(hr.HrError) as e:
            call()
        assert e.value.code == -1


# ---- the 64-bit forms

def test_quantize_example():
    q, s = ref.quantize(torch.tensor([[127.0, -63.5, 0.5, 1.5], [0.0, 0.0, 0.0, 0.0], [math.inf, 1.0, 0.0, 0.0]]))
    assert q.tolist() == [[127, -64, 0, 2], [0] * 4, [0] * 4]
    assert s[0] == 1 and s[1] == 0 and torch.isnan(s[2])


def test_rows_example():
    z = torch.tensor([[0.0, math.log(3.0), -math.inf, 0.0]])
    logp, p, m, logsum = ref.parts(z, 1.0)
    assert np.allclose(p.numpy(), [[0.2, 0.6, 0.0, 0.2]])
    assert np.isclose(float(ref.entropy(logp, p)), -(0.4 * math.log(0.2) + 0.6 * math.log(0.6)))
    assert ref.best(z, 4).tolist() == [[1, 0, 3, -1]] and ref.best(z, 6).tolist() == [[1, 0, 3, -1, -1, -1]]
    assert ref.at(logp, torch.tensor([[-1, 2, 4, 1]])).tolist()[0][:3] == [-math.inf] * 3
    # teacher on entries 0 and 1 alike: loss = ln(1/2) - (ln 0.2 + ln 0.6) / 2
    loss, _, g, _ = ref.distill(z, 1.0, torch.tensor([[0, 1, 2, -1]]), torch.tensor([[4.0, 4.0, 9.0, 9.0]]), torch.ones(1))
    assert np.isclose(float(loss), math.log(0.5) - (math.log(0.2) + math.log(0.6)) / 2)
    assert np.allclose(g.numpy(), [[0.2 - 0.5, 0.6 - 0.5, 0.0, 0.2]])


def test_gradients_of_the_formulas_are_differences():
    g = torch.Generator().manual_seed(3)
    n, scale, h = 12, 1.7, 1e-5
    z = torch.randn(1, n, generator=g, dtype=torch.float64)
    given, up, uh = torch.tensor([[2, 2, 9, -1]]), torch.tensor([[1.0, -0.3, 0.4, 5.0]]), torch.tensor([0.9])
    ids, t = torch.tensor([[3, 7, 3, -1]]), torch.tensor([[0.5, 1.0, -1.0, 3.0]])

    def policy(z):
        logp, p, _, _ = ref.parts(z, scale)
        lp = ref.at(logp, given)
        return (torch.where(lp > -math.inf, lp, torch.zeros_like(lp)) * up).sum(1) + ref.entropy(logp, p) * uh

    def teach(z):
        return ref.distill(z, scale, ids, t, torch.ones(1))[0]

    for f, grad in ((policy, ref.logprobs_grad(z, scale, given, up, uh)[0]), (teach, ref.distill(z, scale, ids, t, torch.ones(1))[2])):
        for i in range(n):
            e = torch.zeros_like(z)
            e[0, i] = h
            assert abs(float((f(z + e) - f(z - e)) / (2 * h)) - float(grad[0, i])) < 1e-8, i
