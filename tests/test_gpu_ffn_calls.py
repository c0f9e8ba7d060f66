"""The operators that train a gated FFN, called as their documentation allows and rarely
done: where the statistics come from, what the outputs share, values past 32 bits."""
import importlib.util
import os

import pytest
import torch

from gpu_helpers import require_gpu
from paper_2604_21290_amd import api

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def _rand(seed, *shape, dtype=torch.float32, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "ffn_gated.py")
    spec = importlib.util.spec_from_file_location("ffn_gated", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _end(R, C, dtype=torch.float32):
    """(b, its block's end's keywords, s, statistics, ds, dy)"""
    vec = [_rand(10 + i, C, dtype=dtype) for i in range(5)]
    how = dict(post=(vec[0], vec[1]), scale=vec[2], gate=_rand(20, R), norm=(vec[3], vec[4]))
    x, b, ds, dy = (_rand(i, R, C, dtype=dtype) for i in range(4))
    s, _, st = api.residual_norm(x, b, stats=True, **how)
    return b, how, s, st, ds, dy


def flat(grads):
    return [t for g in grads for t in (g if isinstance(g, tuple) else (g,))]


@pytest.mark.parametrize("R,C", [(300, 72), (196, 1), (4096, 4)])
def test_statistics_from_an_iterator(R, C):
    """Whose tensors nobody else holds: they live until the kernel has read them."""
    b, how, s, st, ds, dy = _end(R, C)
    want = flat(api.residual_norm_backward(ds, dy, b, s, st, **how))
    for kept in (list(st), (t.clone() for t in st), map(torch.clone, st), iter(st)):
        got = flat(api.residual_norm_backward(ds, dy, b, s, kept, **how))
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    with pytest.raises(ValueError, match="mean_b"):
        api.residual_norm_backward(ds, dy, b, s, (t[:-1].clone() for t in st), **how)


def test_choices_past_32_bits_are_refused():
    """By the native marshalling too, which would cast 2^32 + 1 to the GELU."""
    x, W = _rand(1, 40, 8), _rand(2, 8, 8)
    h, pre = api.gated_linear(x, W, keep=True)
    b, how, s, st, ds, dy = _end(40, 8)
    for off in (1 << 32, -(1 << 32)):
        for call in (lambda: api.gated_linear(x, W, act=off + api.GL_ACT_GELU),
                     lambda: api.gated_linear_backward(h, x, W, pre, act=off + api.GL_ACT_GELU),
                     lambda: api.residual_norm(x, b, kind=off, **how),
                     lambda: api.residual_norm_backward(ds, dy, b, s, st, kind=off + api.GL_NORM_RMS, **how)):
            with pytest.raises(api.GraphLeapError) as e:
                call()
            assert api.STATUS[e.value.status] == "GL_ERR_UNSUPPORTED"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", [(17001, 24), (101, 40), (5001, 80), (99, 250), (37, 500), (5, 5)])
def test_an_infinity_in_the_last_row_counts_once(R, C, dtype):
    """The last row's infinities (in b, then in its gate) are terms of the sums over rows once:
    a workgroup's rows past the last, which repeat it, add no 0 x infinity."""
    inf = float("inf")
    b, dy = _rand(1, R, C, dtype=dtype), (1 + _rand(2, R, C).abs()).to(dtype)
    scale, gate = (1 + _rand(3, C).abs()).to(dtype), 1 + _rand(4, R).abs()
    b[-1, 1::2], b[-1, 0::4] = inf, -inf
    g = api.residual_norm_backward(dy, None, b, None, (None,) * 4, scale=scale, gate=gate)
    want = (dy.double() * gate.double()[:, None] * b.double()).sum(0)
    special = ~b[-1].isfinite()
    assert torch.equal(g.dscale[special].double(), want[special]) and want[special].isinf().all()
    assert g.dscale[~special].isfinite().all()
    b[-1], gate[-1] = 1.0, inf
    g = api.residual_norm_backward(dy, None, b, None, (None,) * 4, scale=scale, gate=gate)
    assert bool((g.dscale == inf).all())
    st = api.residual_norm(b, b, post=(None, None), stats=True)[2]
    g = api.residual_norm_backward(dy, None, b, None, st, post=(scale, scale), gate=gate)
    assert bool((g.dpost[1] == inf).all())


@pytest.mark.parametrize("C", [8, 72])
def test_gradients_do_not_share_a_storage(C):
    """Keeping or saving one keeps no other, and one that grows leaves the others alone."""
    b, how, s, st, ds, dy = _end(300, C)
    got = flat(api.residual_norm_backward(ds, dy, b, s, st, **how))
    assert len({t.untyped_storage().data_ptr() for t in got}) == len(got) == 8
    assert all(t.storage_offset() == 0 and t.untyped_storage().nbytes() == t.nbytes for t in got)
    for i, t in enumerate(got):
        others = [o.clone() for o in got]
        t.resize_(t.numel() + 512)[-512:] = 9.0
        assert all(torch.equal(o, g) for k, (o, g) in enumerate(zip(others, got)) if k != i)


def test_the_example_has_first_derivatives_alone():
    """Its gradients are detached: a penalty on them is refused, not left out of the slope."""
    m = _example()
    w = m.make_weights(12, 8, torch.float32)
    x, gate = _rand(1, 2, 5, 12).requires_grad_(), torch.ones(2, device="cuda")
    s, y = m.GatedFfn.apply(x, gate, *(w[k] for k in m.NAMES))
    dx, = torch.autograd.grad((s * s).sum() + (y * y).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        ((dx * dx).sum() + (x * x).sum()).backward()


def test_gradients_of_memory_that_torch_did_not_allocate():
    """Such a tensor has no allocator of its own to make the small outputs by."""
    b, how, s, st, ds, dy = _end(300, 72)
    want = flat(api.residual_norm_backward(ds, dy, b, s, st, **how))
    args = [torch.from_dlpack(t) for t in (ds, dy, b, s)]
    assert args[2].data_ptr() == b.data_ptr()
    got = flat(api.residual_norm_backward(*args, st, **how))
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    got[3].resize_(1000).zero_()
    with torch.inference_mode():
        got = flat(api.residual_norm_backward(ds, dy, b, s, st, **how))
    assert all(torch.equal(g, w) for g, w in zip(got, want))
