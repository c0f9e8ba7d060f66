"""A block's end and its gradients (residual_norm) on the GPU against float64
(ffn_train_ref.py, where the tolerances are derived)."""
import pytest
import torch

import ffn_train_ref as ref
from paper_2604_21290_amd import api

pytestmark = pytest.mark.gpu

EPS = 1e-5
TYPES = [torch.float32, torch.bfloat16]
# rows shorter than a vector, one lane group after the other, ragged ends, whole workgroups
# a row, and past the widest of them
SHAPES = [(1, 1), (5, 3), (1, 8), (33, 40), (17, 100), (196, 192), (20000, 24), (17000, 61), (5000, 250), (300, 512),
          (130, 1001), (40, 2560), (9, 4100), (700, 5000), (6, 8192), (40, 20000)]
# post, betas, scale, gate (rows to one; 0: none), norm, rms
WAYS = [(True, True, True, 1, True, False), (False, False, True, 0, True, False), (True, False, False, 4, True, True),
        (True, True, True, 0, False, False), (False, True, False, 3, True, False), (False, False, False, 0, False, True)]


def _rand(seed, *shape, dtype=torch.float32, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


def within(name, got, want, bound):
    assert got.shape == want.shape, (name, got.shape, want.shape)
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), (name, float(off.max()), float((off > 0).double().mean()))


def _case(R, C, dtype, way):
    post, betas, scale, gate, norm, rms = way
    gate = gate if gate < 2 or R % gate == 0 else 1
    w = {}
    w["post"] = ((1 + _rand(11, C, size=0.2)).to(dtype), _rand(12, C, dtype=dtype, size=0.2) if betas else None) if post else None
    w["norm"] = ((1 + _rand(13, C, size=0.2)).to(dtype), _rand(14, C, dtype=dtype, size=0.2) if betas else None) if norm else None
    w["scale"] = _rand(15, C, dtype=dtype, size=0.5) if scale else None
    w["gate"] = _rand(16, R // gate) if gate else None
    x, b = _rand(1, R, C, dtype=dtype) + 0.5, _rand(2, R, C, dtype=dtype) * 2 - 0.3
    rows = None if not gate else w["gate"].repeat_interleave(gate)
    return x, b, w, gate, rows, rms


def _shaped(t, gate):
    """Rows [R, C] as [images, rows, C] where a gate has several rows."""
    return t.unflatten(0, (-1, gate)) if gate > 1 else t


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,C", SHAPES)
def test_residual_norm(R, C, dtype):
    for way in WAYS:
        x, b, w, gate, rows, rms = _case(R, C, dtype, way)
        kind = api.GL_NORM_RMS if rms else api.GL_NORM_LAYER
        s, y, stats = api.residual_norm(_shaped(x, gate), _shaped(b, gate), kind=kind, eps=EPS, stats=True, **w)
        want = ref.residual(x, b, w["post"], w["scale"], rows, w["norm"], rms, EPS)
        bound = ref.residual_bounds(x, b, w["post"], w["scale"], rows, w["norm"], rms, EPS, want)
        names = ("s", "y", "mean_b", "rstd_b", "mean_s", "rstd_s")
        for name, g, e, o in zip(names, (s, y) + tuple(stats), want, bound):
            if e is None or (rms and name.startswith("mean")):
                assert g is None, name
                continue
            within((way, name), g.reshape(e.shape), e, o)
        s2, y2 = api.residual_norm(_shaped(x, gate), _shaped(b, gate), kind=kind, eps=EPS, **w)
        assert torch.equal(s, s2) and (y is None or torch.equal(y, y2))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,C", SHAPES)
def test_residual_norm_backward(R, C, dtype):
    for i, way in enumerate(WAYS):
        x, b, w, gate, rows, rms = _case(R, C, dtype, way)
        kind = api.GL_NORM_RMS if rms else api.GL_NORM_LAYER
        s, _, stats = api.residual_norm(_shaped(x, gate), _shaped(b, gate), kind=kind, eps=EPS, stats=True, **w)
        dy = _rand(3, R, C, dtype=dtype) if w["norm"] else None
        ds = None if i == 1 else _rand(4, R, C, dtype=dtype)
        up = lambda t: None if t is None else _shaped(t, gate)  # noqa: E731
        got = api.residual_norm_backward(up(ds), up(dy), up(b), s, stats, kind=kind, **w)
        flat = [None if t is None else t.reshape(-1) for t in stats]
        want = ref.residual_backward(ds, dy, b, s.reshape(R, C), flat, w["post"], w["scale"], rows, w["norm"], rms)
        vals = dict(dx=got.dx.reshape(R, C), db=got.db.reshape(R, C), dscale=got.dscale, dgate=got.dgate)
        vals["dpost"], vals["dpost_bias"] = got.dpost or (None, None)
        vals["dnorm"], vals["dnorm_bias"] = got.dnorm or (None, None)
        assert (got.dpost is None) == (w["post"] is None) and (got.dnorm is None) == (w["norm"] is None)
        for name, g in vals.items():
            if g is None:
                continue
            e, o = want[name]
            if name == "dgate" and gate > 1:
                e, o = (t.view(-1, gate) for t in (e, o))
                # (the sum over the gate's rows)
                e, o = e.sum(1), o.sum(1) + gate * ref.U * (e.abs() + o).sum(1)
            within((way, name), g, e, o)
