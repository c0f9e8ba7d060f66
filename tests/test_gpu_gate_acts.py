"""GELU and SiLU of the gated layer and their derivatives, value by value over their range, on
the GPU against float64.  Phi is taken from erfc, which keeps its bits in the tail."""
import math

import pytest
import torch

import ffn_train_ref as ref
from gpu_helpers import require_gpu
from paper_2604_21290_amd import api

pytestmark = pytest.mark.gpu

ACTS = {"gelu": api.GL_ACT_GELU, "silu": api.GL_ACT_SILU}


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def _gates(name, dtype):
    """Gates over the whole range in which the result is a normal number of fp32."""
    low = -12.8 if name == "gelu" else -87.0
    g = torch.cat([torch.linspace(low, 8.0, 20000, dtype=torch.float64), torch.linspace(-2.0, 2.0, 4001, dtype=torch.float64),
                   torch.logspace(-20, 4, 1001, dtype=torch.float64)])
    return g.to(dtype).cuda()


def _act(name, g):
    g = g.double()
    if name == "silu":
        return ref.act("silu", g)
    p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def test_the_reference_keeps_its_bits():
    """erfc of float64 in the tail against the asymptotic series of Phi(-a) a sqrt(2 pi) e^(a^2 / 2),
    1 - 1 / a^2 + 3 / a^4 - 15 / a^6 + ..., whose error is below its first term left out."""
    a = torch.linspace(8.0, 12.8, 500, dtype=torch.float64, device="cuda")
    series, term, left = torch.ones_like(a), torch.ones_like(a), None
    for k in range(1, 16):
        term = -term * (2 * k - 1) / (a * a)
        left = term.abs() * (2 * k + 1) / (a * a)
        series = series + term
    want = series * torch.exp(-a * a / 2) / (a * math.sqrt(2 * math.pi))
    got = 0.5 * torch.special.erfc(a / math.sqrt(2))
    # (e^(-a^2 / 2) moves by a^2 half steps of its argument)
    assert bool(((got - want).abs() <= want * (left * 2 + 4 * a * a * 2.0 ** -53 + 1e-14)).all())


@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("R", [1, 70, 300])  # few rows, and tiles
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_forward(name, R, dtype):
    """h = act(g) with u = 1: the products are the biases alone, exactly."""
    g = _gates(name, dtype)
    F = g.numel()
    x, W = torch.ones(R, 8, dtype=dtype, device="cuda"), torch.zeros(2 * F, 8, dtype=dtype, device="cuda")
    h = api.gated_linear(x, W, torch.cat([g, torch.ones_like(g)]), act=ACTS[name])
    a, _ = _act(name, g)
    bound = (ref.act_error(name, g.double(), dtype == torch.float32) + ref.U) * a.abs()
    r = ref.half(dtype)
    bound = bound * (1 + r) + (r * a.abs() if dtype == torch.bfloat16 else 0.0)
    for row in (0, R - 1):
        off = (h[row].double() - a).abs() - bound
        assert bool((off <= 0).all()), (float(g[off.argmax()]), float(h[row][off.argmax()]), float(a[off.argmax()]))


@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients(name, dtype):
    """dbias of one row with dh = u = 1 is [act'(g) | act(g)], not rounded."""
    g = _gates(name, dtype)
    F = g.numel()
    one = torch.ones_like(g)
    x, W = torch.ones(1, 8, dtype=dtype, device="cuda"), torch.zeros(2 * F, 8, dtype=dtype, device="cuda")
    db = api.gated_linear_backward(one[None], x, W, torch.cat([g, one])[None], act=ACTS[name])[2].double()
    a, da = _act(name, g)
    assert bool(((db[F:] - a).abs() <= (ref.act_error(name, g.double(), True) + ref.U) * a.abs()).all())
    assert bool(((db[:F] - da).abs() <= ref.grad_error(name, g.double()) + ref.U).all())


def test_silu_below_its_range():
    """What is under 2^-119 may be 0, and is of silu's sign and no larger."""
    g = torch.linspace(-87.0, -120.0, 4000, device="cuda")
    F = g.numel()
    x, W = torch.ones(1, 8, device="cuda"), torch.zeros(2 * F, 8, device="cuda")
    h = api.gated_linear(x, W, torch.cat([g, torch.ones_like(g)]), act=api.GL_ACT_SILU)[0].double()
    a = ref.act("silu", g.double())[0]
    assert bool((h <= 0).all()) and bool(((h - a).abs() <= 2.0 ** -119).all())
    kept = a.abs() > 2.0 ** -119
    assert bool(((h - a).abs()[kept] <= (ref.act_error("silu", g.double(), True) * a.abs())[kept]).all())
