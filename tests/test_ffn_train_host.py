"""Argument checks of the gated layer, the layers' backward passes and a block's end at the
C ABI, on the host (fake, never-dereferenced addresses stand in for device pointers)."""
import ctypes
import os

import pytest
import torch

from paper_2604_21290_amd import api

pytestmark = [pytest.mark.skipif(not os.path.exists(api.LIB_PATH), reason="libgraphleap.so not built"),
              pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-only checks (fake pointers)")]

A = 1 << 32
P = lambda i, off=0: ctypes.c_void_p(A * (i + 1) + off)  # noqa: E731


def _st(s):
    return api.STATUS[s]


def _gated(x=P(0), R=64, K=96, W=P(1), bias=P(2), F=40, act=2, dt=1, h=P(3), pre=P(4), ws=None, n=0):
    return _st(api.lib().gl_gated_linear(x, R, K, W, bias, F, act, dt, h, pre, ws, n, None))


SIZES = (dict(R=0), dict(K=0), dict(R=-1), dict(R=(1 << 28) + 1, K=8), dict(K=(1 << 20) + 1), dict(R=1 << 28, K=512))


def test_gated_linear_refusals():
    assert _gated(x=None) == _gated(W=None) == _gated(h=None) == "GL_ERR_NULL_PTR"
    assert _gated(dt=2) == _gated(act=3) == _gated(act=-1) == "GL_ERR_UNSUPPORTED"
    for bad in SIZES + (dict(F=0), dict(F=-3), dict(F=(1 << 19) + 1), dict(K=1 << 20, F=1 << 19)):
        assert _gated(**bad) == "GL_ERR_BAD_SHAPE", bad
    for bad in (dict(x=P(0, 8)), dict(W=P(1, 2)), dict(bias=P(2, 1)), dict(h=P(3, 1)), dict(pre=P(4, 1)), dict(dt=0, h=P(3, 2))):
        assert _gated(**bad) == "GL_ERR_ALIGNMENT", bad
    for bad in (dict(h=P(0, 64)), dict(pre=P(1, 64)), dict(h=P(2, 16)), dict(pre=P(3, 64)), dict(h=P(0, 64 * 96 * 2 - 2))):
        assert _gated(**bad) == "GL_ERR_ALIAS", bad
    f = api.lib().gl_gated_linear_workspace_bytes
    assert f(64, 96, 40, 1) == f(32, 97, 40, 1) == f(0, 96, 40, 1) == f(64, 96, 40, 7) == f(64, 96, 0, 1) == 0
    need = f(64, 97, 40, 1)
    assert need >= (64 + 80) * 104 * 2
    odd = dict(K=97)
    assert _gated(**odd) == _gated(ws=P(5), n=need - 1, **odd) == _gated(ws=P(5, 8), n=need, **odd) == "GL_ERR_WORKSPACE"
    assert _gated(ws=P(0), n=need, **odd) == _gated(ws=P(4, 256), n=need, **odd) == "GL_ERR_ALIAS"
    assert "gated_linear" in api.lib().gl_last_error().decode()


def _back(dy=P(0), x=P(1), R=64, K=96, W=P(2), N=40, dt=1, dx=P(3), dW=P(4), db=P(5), ws=P(6), n=1 << 30):
    return _st(api.lib().gl_linear_backward(dy, x, R, K, W, N, dt, dx, dW, db, ws, n, None))


def _gback(dy=P(0), x=P(1), R=64, K=96, W=P(2), N=40, dt=1, dx=P(3), dW=P(4), db=P(5), ws=P(6), n=1 << 30, pre=P(7), act=1):
    return _st(api.lib().gl_gated_linear_backward(dy, x, R, K, W, pre, N // 2, act, dt, dx, dW, db, ws, n, None))


@pytest.mark.parametrize("call", [_back, _gback])
def test_backward_refusals(call):
    for bad in (dict(dy=None), dict(x=None), dict(W=None), dict(dx=None, dW=None, db=None)):
        assert call(**bad) == "GL_ERR_NULL_PTR", bad
    assert call(dt=5) == "GL_ERR_UNSUPPORTED"
    for bad in SIZES + (dict(N=0), dict(N=-4), dict(N=(1 << 20) + 2)):
        assert call(**bad) == "GL_ERR_BAD_SHAPE", bad
    for bad in (dict(dy=P(0, 8)), dict(x=P(1, 4)), dict(W=P(2, 2)), dict(dx=P(3, 1)), dict(dW=P(4, 1)), dict(db=P(5, 2))):
        assert call(**bad) == "GL_ERR_ALIGNMENT", bad
    for bad in (dict(dx=P(1, 64)), dict(dx=P(0, 64)), dict(dW=P(2, 64)), dict(db=P(3, 64)), dict(dW=P(3, 64)), dict(ws=P(3)),
                dict(ws=P(2)), dict(ws=P(5))):
        # (a workspace of nothing overlaps nothing)
        many = dict(R=5000, K=97) if "ws" in bad else {}
        assert call(**bad, **many) == "GL_ERR_ALIAS", bad
    many = dict(R=5000)
    f = api.lib().gl_linear_backward_workspace_bytes if call is _back else \
        lambda R, K, N, dt: api.lib().gl_gated_linear_backward_workspace_bytes(R, K, N // 2, dt)
    need = f(5000, 96, 40, 1)
    assert need > 0
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=P(6, 8))):
        assert call(**bad, **many) == "GL_ERR_WORKSPACE", bad
    assert f(0, 96, 40, 1) == f(64, 96, 40, 3) == f(64, 0, 40, 1) == 0
    # what is read for a gradient that is not asked for is not required: past every check the
    # launch itself fails without a GPU
    assert call(x=None, dW=None) == call(W=None, dx=None) == call(x=None, W=None, dx=None, dW=None) == "GL_ERR_HIP"


def test_gated_backward_has_more_to_refuse():
    assert _gback(pre=None) == "GL_ERR_NULL_PTR"
    assert _gback(act=4) == "GL_ERR_UNSUPPORTED"
    assert _gback(pre=P(7, 8)) == "GL_ERR_ALIGNMENT"
    assert _gback(dx=P(7, 64)) == "GL_ERR_ALIAS"


@pytest.mark.parametrize("dt", [0, 1])
def test_backward_workspace_stays_small(dt):
    """Copies of what has odd rows, the gated layer's gradient of pre, 256 rows of sums, and
    parts of at most 256 MiB for each product."""
    es = (4, 2)[dt]
    up = lambda n: (n * es + 15) // 16 * 16  # noqa: E731
    for R in (1, 7, 64, 1000, 12544, 100352, 1 << 20):
        for K in (1, 8, 80, 333, 640, 4096, 20000):
            for N in (2, 16, 320, 1002, 5120, 65536):
                if max(R * K, R * N, K * N) > 1 << 32:
                    continue
                copies = (R + N) * up(K) if K % (16 // es) else 0
                rest = 256 * N * 4 + (2 << 28) + 8 * 256
                n = api.lib().gl_linear_backward_workspace_bytes(R, K, N, dt)
                assert 0 <= n <= copies + (R * up(N) if N % (16 // es) else 0) + rest, (R, K, N, n)
                n = api.lib().gl_gated_linear_backward_workspace_bytes(R, K, N // 2, dt)
                assert R * N * es <= n <= copies + R * up(N) + rest, (R, K, N, n)


def _res(x=P(0), ldx=100, b=P(1), ldb=100, R=64, C=100, norm=0, eps=1e-5, post=1, pg=P(2), pb=P(3), scale=P(4), gate=P(5), per=1,
         g=P(6), be=P(7), dt=1, s=P(8), y=P(9), st=(P(10), P(11), P(12), P(13))):
    return _st(api.lib().gl_residual_norm(x, ldx, b, ldb, R, C, norm, eps, post, pg, pb, scale, gate, per, g, be, dt, s, y, *st, None))


def test_residual_norm_refusals():
    assert _res(x=None) == _res(b=None) == _res(s=None) == "GL_ERR_NULL_PTR"
    assert _res(dt=2) == _res(norm=2) == _res(norm=-1) == "GL_ERR_UNSUPPORTED"
    for bad in (dict(R=0), dict(C=0), dict(ldx=99), dict(ldb=99), dict(per=0), dict(per=-2), dict(eps=-1e-9), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(R=1 << 30, C=1 << 20, ldx=1 << 20, ldb=1 << 20), dict(ldb=1 << 40)):
        assert _res(**bad) == "GL_ERR_BAD_SHAPE", bad
    for bad in (dict(x=P(0, 1)), dict(b=P(1, 1)), dict(s=P(8, 1)), dict(y=P(9, 1)), dict(gate=P(5, 2)), dict(pg=P(2, 1)),
                dict(scale=P(4, 1)), dict(be=P(7, 1)), dict(st=(P(10, 2), P(11), P(12), P(13)))):
        assert _res(**bad) == "GL_ERR_ALIGNMENT", bad
    for bad in (dict(s=P(0)), dict(s=P(1, 64)), dict(y=P(8, 64)), dict(y=P(5, 16)), dict(s=P(4, 16)),
                dict(st=(P(10), P(10, 16), P(12), P(13))), dict(st=(P(8, 64), P(11), P(12), P(13)))):
        assert _res(**bad) == "GL_ERR_ALIAS", bad
    # a strided x reaches to the end of its last row; a gate of 8 rows has 8 values
    assert _res(ldx=1000, s=P(0, 63 * 2000 + 198)) == "GL_ERR_ALIAS"
    assert _res(per=8, s=P(5, 8 * 4 - 2)) == "GL_ERR_ALIAS" and _res(per=8, s=P(5, 8 * 4)) == "GL_ERR_HIP"


def _rback(ds=P(0), dy=P(1), b=P(2), s=P(3), ld=100, R=64, C=100, norm=0, post=1, st=(P(4), P(5), P(6), P(7)), pg=P(8), pb=P(9),
           scale=P(10), gate=P(11), per=1, g=P(12), dt=1, dx=P(13), db=P(14), f=(P(15), P(16), P(17), P(18), P(19), P(20)),
           ws=P(21), n=1 << 30):
    return _st(api.lib().gl_residual_norm_backward(ds, ld, dy, ld, b, ld, s, ld, R, C, norm, post, *st, pg, pb, scale, gate, per,
                                                   g, dt, dx, db, *f, ws, n, None))


def test_residual_norm_backward_refusals():
    none = (None,) * 6
    for bad in (dict(ds=None, dy=None), dict(b=None), dict(s=None), dict(dx=None, db=None, f=none), dict(st=(None, P(5), P(6), P(7))),
                dict(st=(P(4), None, P(6), P(7))), dict(st=(P(4), P(5), None, P(7))), dict(st=(P(4), P(5), P(6), None))):
        assert _rback(**bad) == "GL_ERR_NULL_PTR", bad
    assert _rback(dt=3) == _rback(norm=5) == "GL_ERR_UNSUPPORTED"
    assert _rback(post=0) == _rback(dy=None) == "GL_ERR_UNSUPPORTED"  # the gradient of a norm that is not there
    for bad in (dict(R=0), dict(C=0), dict(ld=99), dict(per=0)):
        assert _rback(**bad) == "GL_ERR_BAD_SHAPE", bad
    for bad in (dict(ds=P(0, 1)), dict(dy=P(1, 1)), dict(b=P(2, 1)), dict(s=P(3, 1)), dict(st=(P(4, 2), P(5), P(6), P(7))),
                dict(dx=P(13, 1)), dict(f=(P(15, 2),) + none[1:]), dict(gate=P(11, 1))):
        assert _rback(**bad) == "GL_ERR_ALIGNMENT", bad
    for bad in (dict(dx=P(0)), dict(db=P(2, 64)), dict(dx=P(3, 64)), dict(db=P(13, 64)), dict(f=(P(13, 64),) + none[1:]),
                dict(ws=P(0)), dict(ws=P(14)), dict(ws=P(20))):
        assert _rback(**bad) == "GL_ERR_ALIAS", bad
    need = api.lib().gl_residual_norm_backward_workspace_bytes(64, 100, 1)
    assert need > 0
    for bad in (dict(ws=None), dict(n=need - 1), dict(ws=P(21, 8))):
        assert _rback(**bad) == "GL_ERR_WORKSPACE", bad
    # no sums asked for, none needed; root mean squares have no means
    assert _rback(f=none, ws=None, n=0) == "GL_ERR_HIP"
    assert _rback(norm=1, st=(None, P(5), None, P(7))) == "GL_ERR_HIP"
    f = api.lib().gl_residual_norm_backward_workspace_bytes
    assert f(0, 100, 1) == f(64, 0, 1) == f(64, 100, 9) == f(1, (1 << 29) + 1, 1) == 0


def test_residual_norm_backward_workspace_stays_small():
    """Twelve bytes a row, and 64 MiB or (rows wider than the widest tile) half of b as bf16."""
    f = api.lib().gl_residual_norm_backward_workspace_bytes
    for dt, wide in ((0, 8192), (1, 8192)):
        for C in (1, 7, 8, 80, 1001, 2560, 8192, 8193, 20000, 1 << 20):
            for R in (1, 31, 33, 64, 1000, 100352, 1 << 20):
                if R * C <= 1 << 36:
                    n = f(R, C, dt)
                    assert 0 < n <= 12 * R + 1024 + max(64 << 20, 16 * C * max(1, R // 32) if C > wide else 0), (R, C, dt, n)


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
    x, W = _Big((n, 8), bf, far), _Big((6, 8), bf, 2 * far)
    few, many = _Big((3, 8), bf, 3 * far), _Big((2 * n, 8), bf, 4 * far)
    calls = [lambda: api.gated_linear(x, W, stream=Stream), lambda: api.gated_linear(few, many, stream=Stream),
             lambda: api.linear_backward(few, x, W, stream=Stream), lambda: api.linear_backward(few, few, many, stream=Stream),
             lambda: api.gated_linear_backward(few, x, W, few, stream=Stream), lambda: api.gated_linear_workspace(x, W),
             lambda: api.linear_backward_workspace(x, W), lambda: api.gated_linear_backward_workspace(few, many),
             lambda: api.residual_norm(x, x, stream=Stream), lambda: api.residual_norm_backward(x, None, x, None, (None,) * 4, stream=Stream),
             lambda: api.residual_norm_backward_workspace(x)]
    for i, call in enumerate(calls):
        with pytest.raises(api.GraphLeapError) as e:
            call()
        assert e.value.status == 2, i


def test_constants_are_the_headers():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "graphleap.h")).read()
    for name in ("GL_ACT_SILU", "GL_ACT_GELU", "GL_NORM_LAYER", "GL_NORM_RMS"):
        assert f"{name} = {getattr(api, name)}" in text, name
