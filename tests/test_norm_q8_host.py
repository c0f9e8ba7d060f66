"""Argument checks of layer norm and the 8-bit layers at the C ABI, on the host
(fake, never-dereferenced addresses stand in for device pointers)."""
import ctypes
import os

import pytest
import torch

from paper_2604_21290_amd import api

pytestmark = [pytest.mark.skipif(not os.path.exists(api.LIB_PATH), reason="libgraphleap.so not built"),
              pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-only checks (fake pointers)")]

A = 1 << 24
P = lambda i, off=0: ctypes.c_void_p(A * (i + 1) + off)  # noqa: E731


def _st(s):
    return api.STATUS[s]


def _norm(x=P(0), R=64, C=100, ld=100, gamma=P(1), beta=P(2), eps=1e-5, dt=1, out=P(3), mean=None, rstd=None):
    return _st(api.lib().gl_layer_norm(x, R, C, ld, gamma, beta, eps, dt, out, mean, rstd, None))


def test_layer_norm_refusals():
    assert _norm(x=None) == _norm(out=None) == "GL_ERR_NULL_PTR"
    assert _norm(dt=2) == "GL_ERR_UNSUPPORTED"
    for bad in (dict(R=0), dict(C=0), dict(R=-1), dict(ld=99), dict(ld=-100), dict(ld=1 << 40), dict(eps=-1e-9),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(R=1 << 30, C=1 << 20, ld=1 << 20),
                dict(R=(1 << 30) + 1, C=1, ld=1), dict(R=1, C=(1 << 29) + 1, ld=(1 << 29) + 1)):
        assert _norm(**bad) == "GL_ERR_BAD_SHAPE", bad
    assert _norm(x=P(0, 1)) == _norm(out=P(3, 1)) == _norm(gamma=P(1, 1)) == "GL_ERR_ALIGNMENT"
    assert _norm(x=P(0, 2), dt=0) == _norm(mean=P(5, 2)) == "GL_ERR_ALIGNMENT"
    assert _norm(out=P(0, 64)) == "GL_ERR_ALIAS"
    assert _norm(mean=P(4), rstd=P(4, 64)) == "GL_ERR_ALIAS"
    assert _norm(mean=P(0, 128)) == _norm(out=P(1, 64)) == "GL_ERR_ALIAS"
    # a strided x reaches to the end of its last row
    assert _norm(ld=1000, out=P(0, 63 * 2000 + 198)) == "GL_ERR_ALIAS"
    assert "layer_norm" in api.lib().gl_last_error().decode()


def _grad(dy=P(0), lddy=100, x=P(1), ldx=100, R=64, C=100, mean=P(2), rstd=P(3), gamma=P(4), dt=1, dx=P(5),
          dg=P(6), db=P(7), ws=P(8), n=1 << 23):
    return _st(api.lib().gl_layer_norm_backward(dy, lddy, x, ldx, R, C, mean, rstd, gamma, dt, dx, dg, db, ws, n,
                                                None))


def test_layer_norm_backward_refusals():
    for bad in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None, dg=None, db=None)):
        assert _grad(**bad) == "GL_ERR_NULL_PTR", bad
    assert _grad(dt=3) == "GL_ERR_UNSUPPORTED"
    for bad in (dict(R=0), dict(C=0), dict(ldx=99), dict(lddy=99)):
        assert _grad(**bad) == "GL_ERR_BAD_SHAPE", bad
    for bad in (dict(dy=P(0, 1)), dict(mean=P(2, 2)), dict(dg=P(6, 2)), dict(dx=P(5, 1))):
        assert _grad(**bad) == "GL_ERR_ALIGNMENT", bad
    for bad in (dict(dx=P(0, 16)), dict(dx=P(1, 16)), dict(dg=P(5, 64)), dict(db=P(6, 64)), dict(dg=P(2, 64)),
                dict(R=5000, ws=P(1, 64)), dict(R=5000, ws=P(6, 64))):
        assert _grad(**bad) == "GL_ERR_ALIAS", bad
    many = dict(R=5000)
    need = api.lib().gl_layer_norm_backward_workspace_bytes(5000, 100, 1)
    assert need >= 800
    assert _grad(ws=None, **many) == _grad(n=need - 1, **many) == _grad(ws=P(8, 8), **many) == "GL_ERR_WORKSPACE"
    assert api.lib().gl_layer_norm_backward_workspace_bytes(0, 100, 1) == 0
    assert api.lib().gl_layer_norm_backward_workspace_bytes(64, 100, 5) == 0
    assert api.lib().gl_layer_norm_backward_workspace_bytes(1, (1 << 29) + 1, 1) == 0


def _q8(x=P(0), R=64, K=100, ld=100, dt=1, q=P(1), s=P(2)):
    return _st(api.lib().gl_quantize_rows(x, R, K, ld, dt, q, s, None))


def _nq8(x=P(0), R=64, K=100, ld=100, gamma=None, beta=None, eps=1e-5, dt=1, q=P(1), s=P(2)):
    return _st(api.lib().gl_layer_norm_q8(x, R, K, ld, gamma, beta, eps, dt, q, s, None))


@pytest.mark.parametrize("call", [_q8, _nq8])
def test_rows_to_8_bits_refusals(call):
    assert call(x=None) == call(q=None) == call(s=None) == "GL_ERR_NULL_PTR"
    assert call(dt=-1) == "GL_ERR_UNSUPPORTED"
    for bad in (dict(R=0), dict(K=0), dict(K=131072, ld=131072), dict(ld=5)):
        assert call(**bad) == "GL_ERR_BAD_SHAPE", bad
    assert call(q=P(1, 8)) == call(s=P(2, 2)) == call(x=P(0, 1)) == "GL_ERR_ALIGNMENT"
    assert call(q=P(0, 16)) == call(s=P(1, 64 * 112 - 4)) == "GL_ERR_ALIAS"


def test_layer_norm_q8_eps():
    assert _nq8(eps=-1.0) == "GL_ERR_BAD_SHAPE"


def test_q8_row_bytes():
    f = api.lib().gl_q8_row_bytes
    assert [f(k) for k in (1, 16, 17, 80, 131071)] == [16, 16, 32, 80, 131072]
    assert [f(k) for k in (0, -5, 131072)] == [0, 0, 0]
    with pytest.raises(api.GraphLeapError):
        api.q8_row_bytes(0)


def _lin(q=P(0), s=P(1), R=64, K=100, W=P(2), ws=P(3), bias=P(4), Cout=50, act=0, res=None, dt=1, out=P(5)):
    return _st(api.lib().gl_linear_q8(q, s, R, K, W, ws, bias, Cout, act, res, dt, out, None))


def test_linear_q8_refusals():
    for bad in (dict(q=None), dict(s=None), dict(W=None), dict(ws=None), dict(out=None)):
        assert _lin(**bad) == "GL_ERR_NULL_PTR", bad
    assert _lin(dt=4) == _lin(act=2) == "GL_ERR_UNSUPPORTED"
    for bad in (dict(R=0), dict(Cout=0), dict(K=0), dict(K=131072), dict(R=1 << 30, Cout=1 << 20),
                dict(R=(1 << 30) + 1, K=1, Cout=1), dict(R=1, K=1, Cout=(1 << 30) + 1)):
        assert _lin(**bad) == "GL_ERR_BAD_SHAPE", bad
    for bad in (dict(q=P(0, 8)), dict(W=P(2, 4)), dict(s=P(1, 2)), dict(ws=P(3, 1)), dict(out=P(5, 1)),
                dict(bias=P(4, 1)), dict(res=P(6, 1)), dict(dt=0, out=P(5, 2))):
        assert _lin(**bad) == "GL_ERR_ALIGNMENT", bad
    for bad in (dict(out=P(0, 16)), dict(out=P(1, 16)), dict(out=P(2, 16)), dict(out=P(3, 16)), dict(out=P(4, 16)),
                dict(res=P(5, 16))):
        assert _lin(**bad) == "GL_ERR_ALIAS", bad


def test_layer_norm_backward_workspace_stays_small():
    """32 MiB, or an eighth of dy and x (as bf16) where rows are wider than 2048 vectors."""
    f = api.lib().gl_layer_norm_backward_workspace_bytes
    widths = sorted({w + d for e in range(27) for w in (1 << e,) for d in (-1, 0, 1) if w + d > 0} | {80, 1001, 2560, 20000})
    for dt, wide in ((0, 2048 * 4), (1, 2048 * 8)):
        for C in widths:
            for R in (1, 2, 31, 32, 33, 63, 64, 100, 256, 1000, 5000, 100352, 1 << 20, 1 << 30):
                if R * C > 1 << 40:
                    continue
                n = f(R, C, dt)
                assert 0 <= n <= max(32 << 20, R * C // 4 if C > wide else 0), (R, C, dt, n)
                if C > wide and R < 64:
                    assert n == 0, (R, C, dt, n)


class _Big:
    """Stands in for a contiguous device tensor of any size; its address is never read."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, shape, dtype, at):
        self.shape, self.dtype, self.at = torch.Size(shape), dtype, at

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def is_neg(self):
        return False

    def data_ptr(self):
        return self.at

    def record_stream(self, s):
        pass


def test_counts_past_32_bits_are_refused(monkeypatch):
    """2^32 + 5 rows are not taken for 5: ctypes cuts a count to 32 bits without a word."""
    class Stream:
        cuda_stream = 0
    monkeypatch.setattr(api, "_native", type("No", (), {}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    n, bf, far = (1 << 32) + 5, torch.bfloat16, 1 << 45
    x, out = _Big((n, 1), bf, far), _Big((n, 1), bf, 2 * far)
    q = api.Q8Rows(_Big((n, 16), torch.int8, 3 * far), _Big((n,), torch.float32, 4 * far), 1)
    few = api.Q8Rows(_Big((3, 16), torch.int8, 5 * far), _Big((3,), torch.float32, 6 * far), 1)
    calls = [lambda: api.layer_norm(x, out=out, stream=Stream),
             lambda: api.layer_norm_backward_workspace(x),
             lambda: api.layer_norm_backward(x, x, q.scale, q.scale, need=(False, True, True),
                                             ws=api.Workspace(0, "cpu"), stream=Stream),
             lambda: api.quantize_rows(x, out=q, stream=Stream),
             lambda: api.layer_norm_q8(x, out=q, stream=Stream),
             lambda: api.linear_q8(q, few, out=_Big((n, 3), bf, 7 * far), stream=Stream),
             lambda: api.linear_q8(few, q, out=_Big((3, n), bf, 7 * far), stream=Stream)]
    for i, call in enumerate(calls):
        with pytest.raises(api.GraphLeapError) as e:
            call()
        assert e.value.status == 2, i
