"""What the operators that train a gated FFN refuse or ask for before anything is launched, on
the host (stand-ins for device tensors, whose addresses are never read)."""
import os

import pytest
import torch

from paper_2604_21290_amd import api
from test_ffn_train_host import _Big

pytestmark = [pytest.mark.skipif(not os.path.exists(api.LIB_PATH), reason="libgraphleap.so not built"),
              pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-only checks (fake pointers)")]

BF, FAR = torch.bfloat16, 1 << 45


class Stream:
    cuda_stream = 0


@pytest.fixture(autouse=True)
def _python_path(monkeypatch):
    monkeypatch.setattr(api, "_native", type("No", (), {}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(api, "_new", lambda shape, dtype, x, stream: _Big(shape, dtype, 9 * FAR))
    monkeypatch.setattr(api, "_scratch", lambda *a: (None, 0, None))


@pytest.mark.parametrize("off", [1 << 32, -(1 << 32), 1 << 40])
def test_choices_past_32_bits_are_refused(off):
    """2^32 + 1 is not taken for the GELU, nor 2^32 for layer norm: ctypes cuts a value short."""
    x, W, h = _Big((40, 8), BF, FAR), _Big((8, 8), BF, 2 * FAR), _Big((40, 4), BF, 3 * FAR)
    pre, b = _Big((40, 8), BF, 4 * FAR), _Big((40, 8), BF, 5 * FAR)
    calls = [lambda: api.gated_linear(x, W, act=off + api.GL_ACT_GELU, stream=Stream),
             lambda: api.gated_linear_backward(h, x, W, pre, act=off + api.GL_ACT_SILU, stream=Stream),
             lambda: api.residual_norm(x, b, kind=off + api.GL_NORM_RMS, stream=Stream),
             lambda: api.residual_norm_backward(x, None, b, None, (None,) * 4, kind=off, stream=Stream)]
    for i, call in enumerate(calls):
        with pytest.raises(api.GraphLeapError) as e:
            call()
        assert api.STATUS[e.value.status] == "GL_ERR_UNSUPPORTED", i


@pytest.mark.parametrize("R,K,F,dt", [(278, 2912, 112, 0), (40, 8192, 16, 1), (33, 4096, 4, 0)])
def test_a_parted_contraction_needs_a_workspace(R, K, F, dt):
    """Though its rows are whole vectors, which the header promises nothing about."""
    L, P = api.lib(), lambda i: i * FAR  # noqa: E731
    need = L.gl_gated_linear_workspace_bytes(R, K, F, dt)
    assert need >= 2 * R * 2 * F * 4
    call = lambda ws, n: api.STATUS[L.gl_gated_linear(P(1), R, K, P(2), None, F, 1, dt, P(3), None, ws, n, None)]  # noqa: E731
    assert call(None, 0) == call(P(4), need - 1) == "GL_ERR_WORKSPACE"
    assert L.gl_gated_linear_workspace_bytes(32, K, F, dt) == 0
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "graphleap.h")).read()
    assert "ask for every layer" in text and "many of whole vectors" not in text
