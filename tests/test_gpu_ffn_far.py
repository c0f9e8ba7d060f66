"""Gradients of the layers and of a block's end where a matrix has more than 2^30 elements
of either type (4 GiB in fp32), on the GPU against float64 (ffn_train_ref.py): the first and
the last rows hold values of their own, all between them count for nothing."""
import pytest
import torch

import ffn_train_ref as ref
from gpu_helpers import require_gpu
from paper_2604_21290_amd import api

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
R, ENDS = (1 << 20) + 5, 70


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def _rand(seed, *shape, dtype=torch.float32, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


def _rows(seed, C, dtype):
    t = torch.zeros(R, C, dtype=dtype, device="cuda")
    t[:ENDS], t[-ENDS:] = _rand(seed, ENDS, C, dtype=dtype), _rand(seed + 100, ENDS, C, dtype=dtype)
    return t


def ends(t):
    return torch.cat([t[:ENDS], t[-ENDS:]])


def within(name, got, want, bound):
    assert got.shape == want.shape, (name, got.shape, want.shape)
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), (name, float(off.max()), float((off > 0).double().mean()))


def layer_within(got, want, bound):
    """Sums over rows add zeros to those of the ends, which is exact."""
    for name, g, w, b in zip(("dx", "dW", "dbias"), got, want, bound):
        within(name, ends(g) if name == "dx" else g, w, b)
    assert not got[0][ENDS:-ENDS].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_layer(dtype):
    K, F = 8, 1024
    x, dh, W = _rows(1, K, dtype), _rows(2, F, dtype), _rand(3, 2 * F, K, dtype=dtype, size=K ** -0.5)
    h, pre = api.gated_linear(x, W, keep=True)
    eh, ep, bh, bp = ref.gated(ends(x), W, None, "silu")
    within("h", ends(h), eh, bh)
    within("pre", ends(pre), ep, bp)
    got = api.gated_linear_backward(dh, x, W, pre)
    layer_within(got, *ref.gated_backward(ends(dh), ends(x), W, ends(pre), "silu"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [1032, 1025])  # whole vectors, and rows that are copied first
def test_layer(N, dtype):
    K = 8
    x, dy, W = _rows(1, K, dtype), _rows(2, N, dtype), _rand(3, N, K, dtype=dtype, size=K ** -0.5)
    layer_within(api.linear_backward(dy, x, W), *ref.products(ends(dy).double(), ends(x), W))


@pytest.mark.parametrize("dtype", TYPES)
def test_block_end(dtype):
    C = 1032
    x, b, dy = (_rows(i, C, dtype) for i in (1, 2, 3))
    how = dict(post=(_rand(4, C, dtype=dtype), None), norm=(_rand(5, C, dtype=dtype), None))
    s, _, st = api.residual_norm(x, b, stats=True, **how)
    got = api.residual_norm_backward(None, dy, b, s, st, **how)
    want = ref.residual_backward(None, ends(dy), ends(b), ends(s), [ends(t) for t in st], how["post"], None, None, how["norm"],
                                 False)
    for name, g in (("dx", ends(got.dx)), ("db", ends(got.db)), ("dpost", got.dpost[0]), ("dnorm", got.dnorm[0])):
        within(name, g, *want[name])
    assert not got.dx[ENDS:-ENDS].any() and not got.db[ENDS:-ENDS].any()
