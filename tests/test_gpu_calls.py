"""The native argument marshalling of the short calls: it takes their ordinary forms,
with the bits of the checked path, and leaves every other form to that path."""
import pytest
import torch

from gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu


def _api():
    require_gpu()
    from paper_2604_21290_amd import api
    return api


class Sub(torch.Tensor):
    pass


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(7, 40), (2, 3, 33), (40,), (1, 1)])
def test_ordinary_forms(dtype, shape):
    api = _api()
    n = api._calls()
    torch.manual_seed(0)
    C = shape[-1]
    x, dy = torch.randn(shape, device="cuda").to(dtype), torch.randn(shape, device="cuda").to(dtype)
    gamma, beta = torch.randn(C, device="cuda").to(dtype), torch.randn(C, device="cuda").to(dtype)
    cur = torch.cuda.current_stream()  # named, it goes through the checked path
    for g, b in ((gamma, beta), (None, None), (gamma, None)):
        y, mean, rstd = n.layer_norm(x, g, b, 1e-5, True)
        for got, want in zip((y, mean, rstd), api.layer_norm(x, g, b, stats=True, stream=cur)):
            assert got.shape == want.shape and got.dtype == want.dtype and torch.equal(got, want)
        assert torch.equal(n.layer_norm(x, g, b, 1e-5, False), y)
        for got, want in zip(n.layer_norm_backward(dy, x, mean, rstd, g),
                             api.layer_norm_backward(dy, x, mean, rstd, g, stream=cur)):
            assert got.shape == want.shape and got.dtype == want.dtype and torch.equal(got, want)
        q, s = n.layer_norm_q8(x, g, b, 1e-5)
        want = api.layer_norm_q8(x, g, b, stream=cur)
        assert torch.equal(q, want.q) and torch.equal(s, want.scale)
    q, s = n.quantize_rows(x)
    xq = api.quantize_rows(x, stream=cur)
    assert torch.equal(q, xq.q) and torch.equal(s, xq.scale) and s.shape == shape[:-1]
    W = api.quantize_rows(torch.randn(5, C, device="cuda"))
    bias, res = torch.randn(5, device="cuda").to(dtype), torch.randn(shape[:-1] + (5,), device="cuda").to(dtype)
    for bi, r, act in ((bias, res, 1), (None, None, 0)):
        got = n.linear_q8(xq.q, xq.scale, C, W.q, W.scale, C, bi, act, r, dtype == torch.bfloat16)
        want = api.linear_q8(xq, W, bi, act, r, dtype, stream=cur)
        assert got.shape == want.shape and got.dtype == want.dtype and torch.equal(got, want)
    torch.cuda.synchronize()


def test_strided_rows_are_an_ordinary_form():
    api = _api()
    x = torch.randn(9, 100, device="cuda")[:, 3:70]
    assert torch.equal(api._calls().layer_norm(x, None, None, 1e-5, False), api.layer_norm(x.contiguous()))


def test_other_forms_are_left():
    api = _api()
    n = api._calls()
    x = torch.randn(6, 40, device="cuda")
    v = torch.randn(40, device="cuda")
    left = [
        lambda: n.layer_norm(x.cpu(), None, None, 1e-5, False),
        lambda: n.layer_norm(x.half(), None, None, 1e-5, False),
        lambda: n.layer_norm(x.t(), None, None, 1e-5, False),
        lambda: n.layer_norm(x[:0], None, None, 1e-5, False),
        lambda: n.layer_norm(x, v[:39], None, 1e-5, False),
        lambda: n.layer_norm(x, v.bfloat16(), None, 1e-5, False),
        lambda: n.layer_norm(x, v.cpu(), None, 1e-5, False),
        lambda: n.layer_norm(x, v.reshape(1, 40), None, 1e-5, False),
        lambda: n.layer_norm(x, None, None, -1.0, False),
        lambda: n.layer_norm("x", None, None, 1e-5, False),
        lambda: n.layer_norm(x.as_subclass(Sub), None, None, 1e-5, False),
        lambda: n.layer_norm_backward(x, x.bfloat16(), v[:6], v[:6], None),
        lambda: n.layer_norm_backward(x[:5], x, v[:6], v[:6], None),
        lambda: n.layer_norm_backward(x, x, v[:5], v[:6], None),
        lambda: n.layer_norm_backward(x, x, None, v[:6], None),
        lambda: n.quantize_rows(x.long()),
        lambda: n.layer_norm_q8(x, None, v[::2], 1e-5),
    ]
    for i, f in enumerate(left):
        assert f() is None, i
    q, s = n.quantize_rows(x)
    ok = [q, s, 40, q, s, 40, None, 0, None, False]
    assert n.linear_q8(*ok) is not None
    for at, bad in ((0, q[:, :32]), (0, q[:0]), (0, q.cpu()), (0, q.float()), (1, s[:5]), (1, s.double()), (1, None),
                    (2, 56), (2, 0), (3, q.reshape(6, 1, 48)), (4, None), (4, s[:5]), (5, 41), (6, s[:5]),
                    (6, s.bfloat16()), (7, 9), (8, x), (8, torch.zeros(6, 6, device="cuda").t()[:, :5])):
        args = list(ok)
        args[at] = bad
        assert n.linear_q8(*args) is None, (at, bad)
    with pytest.raises(TypeError):
        n.layer_norm(x, None, None, "eps", False)
    torch.cuda.synchronize()


def test_calls_without_the_shortcut_have_the_same_bits(monkeypatch):
    """Where _calls.so cannot be loaded, the Python path takes the ordinary forms too."""
    api = _api()
    x, dy = torch.randn(9, 72, device="cuda"), torch.randn(9, 72, device="cuda")
    gamma, beta = torch.randn(72, device="cuda"), torch.randn(72, device="cuda")

    def every():
        y, mean, rstd = api.layer_norm(x, gamma, beta, stats=True)
        q, n = api.quantize_rows(x), api.layer_norm_q8(x, gamma, beta)
        out = api.linear_q8(n, q, act_out=api.GL_ACT_GELU, dtype=torch.float32)
        return [y, mean, rstd, *api.layer_norm_backward(dy, x, mean, rstd, gamma), q.q, q.scale, n.q, n.scale, out]

    api._calls()
    want = every()
    monkeypatch.setattr(api, "_native", api._NoCalls)
    got = every()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_negated_views_are_refused():
    """A view that torch holds as the negative of its memory is not read without its sign."""
    api = _api()
    x = torch.randn(6, 64, device="cuda")
    neg, v = torch._neg_view(x), torch.randn(64, device="cuda")
    _, mean, rstd = api.layer_norm(x, stats=True)
    q = api.quantize_rows(x)
    for call in (lambda: api.layer_norm(neg), lambda: api.quantize_rows(neg), lambda: api.layer_norm_q8(neg),
                 lambda: api.layer_norm(x, torch._neg_view(v)), lambda: api.layer_norm_backward(neg, x, mean, rstd),
                 lambda: api.layer_norm_backward(x, x, torch._neg_view(mean), rstd),
                 lambda: api.linear_q8(q, q, bias=torch._neg_view(v[:6]), dtype=torch.float32)):
        with pytest.raises(ValueError, match="negat"):
            call()
    assert torch.equal(api.layer_norm(neg.resolve_neg()), api.layer_norm(-x))


def test_outputs_are_detached():
    """No call is recorded by autograd, by the shortcut or by the Python path."""
    api = _api()
    x = torch.randn(6, 64, device="cuda", requires_grad=True)
    w = torch.nn.Parameter(torch.randn(64, device="cuda"))
    cur = torch.cuda.current_stream()
    for stream in (None, cur):
        for t in (*api.layer_norm(x, w, stats=True, stream=stream), api.quantize_rows(x, stream=stream).scale,
                  api.layer_norm_q8(x, w, stream=stream).scale,
                  api.linear_q8(api.quantize_rows(x), api.quantize_rows(x), stream=stream)):
            assert not t.requires_grad
    torch.cuda.synchronize()
