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
