"""The gated layer, the layers' backward passes and a block's end with its gradients, on the
GPU, against float64 (ffn_train_ref.py, where the tolerances are derived)."""
import pytest
import torch

import ffn_train_ref as ref
from paper_2604_21290_amd import api

pytestmark = pytest.mark.gpu

ACTS = {"none": api.GL_ACT_NONE, "gelu": api.GL_ACT_GELU, "silu": api.GL_ACT_SILU}
TYPES = [torch.float32, torch.bfloat16]


def _rand(seed, *shape, dtype=torch.float32, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


def within(name, got, want, bound):
    assert got.shape == want.shape, (name, got.shape, want.shape)
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), (name, float(off.max()), float((off > 0).double().mean()))


def _weight(seed, N, K, dtype):
    return _rand(seed, N, K, dtype=dtype, size=K ** -0.5)


# one row to the largest tiles; whole vectors and odd sizes; contractions shorter than a
# stage, of whole stages and past them
GATED = [(1, 8, 8), (1, 640, 2560), (1, 37, 5), (3, 1, 1), (16, 200, 24), (17, 100, 33), (64, 129, 40), (65, 129, 40),
         (65, 8, 3), (100, 192, 96), (196, 192, 768), (300, 64, 700), (777, 501, 333), (1500, 72, 1100), (2600, 648, 2560),
         (278, 2912, 112), (70, 4001, 33), (40, 3000, 7), (32, 1030, 50)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K,F", GATED)
def test_gated_linear(R, K, F, dtype):
    x, W = _rand(1, R, K, dtype=dtype), _weight(2, 2 * F, K, dtype)
    bias = _rand(3, 2 * F, dtype=dtype, size=0.3)
    for name, b in (("silu", bias), ("gelu", None), ("none", bias)):
        h, pre = api.gated_linear(x, W, b, act=ACTS[name], keep=True)
        eh, ep, bh, bp = ref.gated(x, W, b, name)
        within("pre", pre, ep, bp)
        within(name, h, eh, bh)
        assert torch.equal(api.gated_linear(x, W, b, act=ACTS[name]), h)


# (R, K, N): as above, and few outputs of long sums over rows (parts of the contraction)
BACK = [(1, 8, 8), (1, 1, 1), (2, 3, 6), (5, 16, 24), (33, 37, 10), (65, 129, 40), (300, 64, 700), (1000, 192, 768),
        (3001, 101, 34), (6272, 192, 64), (20000, 40, 16), (2600, 640, 2560), (70, 2000, 4104), (8200, 1032, 2056)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K,N", BACK)
def test_linear_backward(R, K, N, dtype):
    dy, x, W = _rand(1, R, N, dtype=dtype), _rand(2, R, K, dtype=dtype), _weight(3, N, K, dtype)
    got = api.linear_backward(dy, x, W)
    want, bound = ref.products(dy.double(), x, W)
    for name, g, w, b in zip(("dx", "dW", "dbias"), got, want, bound):
        within(name, g, w, b)
    for i in range(3):
        one = api.linear_backward(dy, x, W, need=[i == j for j in range(3)])
        assert torch.equal(one[i], got[i]) and all(one[j] is None for j in range(3) if j != i)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K,N", BACK)
def test_gated_linear_backward(R, K, N, dtype):
    F = max(1, N // 2)
    dh, x, W = _rand(1, R, F, dtype=dtype), _rand(2, R, K, dtype=dtype), _weight(3, 2 * F, K, dtype)
    for name in ("gelu", "silu", "none"):
        pre = api.gated_linear(x, W, None, act=ACTS[name], keep=True)[1]
        got = api.gated_linear_backward(dh, x, W, pre, act=ACTS[name])
        want, bound = ref.gated_backward(dh, x, W, pre, name)
        for n, g, w, b in zip(("dx", "dW", "dbias"), got, want, bound):
            within((name, n), g, w, b)
