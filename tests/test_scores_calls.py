"""How the functions of scores.py are called: by keyword, wrongly more than once, on tensors that autograd follows."""
import inspect

import pytest
import torch

import test_scores as scores

FUNCTIONS = ["quantize_rows", "i8_product", "i8_linear", "logprobs", "logprobs_backward", "distill_forward", "distill_backward", "distill_step"]


@pytest.mark.parametrize("name", FUNCTIONS)
def test_arguments_go_by_their_names(name):
    """Every argument by keyword reaches the function's own checks (host tensors are refused); what is missing is named."""
    hr = scores._hr()
    f = getattr(hr, name)
    names = [p.name for p in inspect.signature(f).parameters.values() if p.default is p.empty]
    with pytest.raises(hr.HrError) as e:
        f(**{n: torch.zeros(3, 8) for n in names})
    assert f"{names[0]} must be a device tensor" in str(e.value)
    with pytest.raises(TypeError, match=repr(names[0])):
        f()


@pytest.mark.gpu
def test_keyword_calls_give_the_same():
    hr = scores._hr()
    z = torch.randn(3, 50, device="cuda")
    ids, t = torch.zeros(3, 2, dtype=torch.int64, device="cuda"), torch.zeros(3, 2, device="cuda")
    r = hr.logprobs(given=ids, logits=z, k=2)
    assert all(torch.equal(a, b) for a, b in zip(r, hr.logprobs(z, ids, 2)))
    assert torch.equal(hr.logprobs_backward(grad_logprobs=t + 1, result=r, given=ids, logits=z), hr.logprobs_backward(z, ids, r, t + 1))
    assert torch.equal(hr.distill_step(teacher=t, ids=ids, logits=z)[1], hr.distill_step(z, ids, t)[1])
    w, ws = hr.quantize_rows(x=z)
    assert torch.equal(hr.i8_linear(x=z, b=w, b_scale=ws), hr.i8_product(b_scale=ws, b=w, a_scale=ws, a=w))


def test_a_refusal_says_why_every_time():
    """Sizes of workspaces are kept from call to call, refusals are not: the same wrong call has the same message after another's."""
    hr = scores._hr()
    from paper_2507_09138_amd import scores as layer
    for need, bad, other, text in ((layer._i8_bytes, (3, 4, 0), (3, 4, 131072), "k=0 "), (layer._logprobs_bytes, (3, 10, 129), (3, 10, -1), "k=129 "),
                                   (layer._distill_bytes, (3, 10, 513), (3, 0, 5), "k=513 ")):
        for _ in range(2):
            with pytest.raises(hr.HrError, match=text):
                need(*bad)
            with pytest.raises(hr.HrError) as e:
                need(*other)
            assert text not in str(e.value)
        assert need(3, 10, 5) == need(3, 10, 5) > 0


@pytest.mark.gpu
def test_a_refused_call_says_why_every_time():
    hr = scores._hr()
    z = torch.randn(3, 10, device="cuda")
    for _ in range(2):
        with pytest.raises(hr.HrError, match="k=129 "):
            hr.logprobs(z, k=129)
        with pytest.raises(hr.HrError, match="scale="):
            hr.logprobs(z, scale=-1.0)


@pytest.mark.gpu
def test_what_is_written_over_is_known_to_autograd():
    """Results are not recorded; a result in the place of a tensor that a backward pass needs is an error there, not a wrong gradient."""
    hr = scores._hr()
    ids, t = torch.zeros(3, 2, dtype=torch.int64, device="cuda"), torch.zeros(3, 2, device="cuda")
    w, ws = hr.quantize_rows(torch.randn(10, 64, device="cuda"))

    def written(call):
        x = torch.randn(3, 10, device="cuda", requires_grad=True)
        y = torch.exp(x)                                   # (its backward pass needs y)
        before = y._version
        call(y)
        assert y._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()

    def norm_q(y):
        return hr.distill_forward(y, ids, t)[:0:-1]

    written(lambda y: hr.distill_step(y, ids, t, out=y.detach()))
    written(lambda y: hr.distill_step(y, ids, t, out=y))
    written(lambda y: hr.distill_backward(y, ids, *norm_q(y), out=y))
    written(lambda y: hr.logprobs_backward(y, ids, hr.logprobs(y, ids), t, out=y))
    written(lambda y: hr.i8_linear(torch.randn(3, 64, device="cuda"), w, ws, out=y))
    written(lambda y: hr.i8_product(w[:3], ws[:3], w, ws, out=y))
    # scores that a model made, their gradient in their place: what a training step does with it
    x = torch.randn(3, 10, device="cuda", requires_grad=True)
    y = 2 * x
    want = hr.distill_step(y, ids, t)[1]
    assert not want.requires_grad and not hr.logprobs(y, ids).logprobs.requires_grad
    grad = hr.distill_step(y, ids, t, out=y)[1].detach()
    y.backward(grad)
    assert torch.equal(x.grad, 2 * want)
    with torch.inference_mode():
        z = torch.randn(3, 10, device="cuda")
        assert hr.distill_step(z, ids, t, out=z)[1] is z
