"""A block's end with gates of many rows and rows of three axes, on the GPU against float64
(ffn_train_ref.py, where the tolerances are derived)."""
import pytest
import torch

import ffn_train_ref as ref
from gpu_helpers import require_gpu
from paper_2604_21290_amd import api

pytestmark = pytest.mark.gpu

EPS = 1e-5
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def _rand(seed, *shape, dtype=torch.float32, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


def within(name, got, want, bound):
    assert got.shape == want.shape, (name, got.shape, want.shape)
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), (name, float(off.max()), float((off > 0).double().mean()))


def _vectors(C, dtype):
    return dict(post=((1 + _rand(11, C, size=0.2)).to(dtype), _rand(12, C, dtype=dtype, size=0.2)),
                norm=((1 + _rand(13, C, size=0.2)).to(dtype), _rand(14, C, dtype=dtype, size=0.2)),
                scale=_rand(15, C, dtype=dtype, size=0.5))


def check(x, b, ds, dy, s_of, how, rows_per_gate):
    """A call's results on rows of any axes and strides, against its rows one after the other."""
    flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
    gate = how["gate"].reshape(-1).repeat_interleave(rows_per_gate)
    s, y, st = api.residual_norm(x, b, eps=EPS, stats=True, **how)
    args = (flat(x), flat(b), how["post"], how["scale"], gate, how["norm"], False, EPS)
    want = ref.residual(*args)
    for name, g, e, o in zip(("s", "y", "mean_b", "rstd_b", "mean_s", "rstd_s"), (s, y, *st), want, ref.residual_bounds(*args, want)):
        assert g.is_contiguous() and g.shape[:-1 if g.dim() == x.dim() else None] == x.shape[:-1], name
        within(name, g.reshape(e.shape), e, o)
    g = api.residual_norm_backward(ds, dy, b, s_of(s), st, **how)
    want = ref.residual_backward(flat(ds), flat(dy), flat(b), flat(s), [t.reshape(-1) for t in st], how["post"], how["scale"],
                                 gate, how["norm"], False)
    assert g.dgate.shape == how["gate"].shape
    per = lambda t: t.view(-1, rows_per_gate)  # noqa: E731
    e, o = want["dgate"]
    # (the sum over a gate's rows)
    want["dgate"] = per(e).sum(1), per(o).sum(1) + rows_per_gate * ref.U * per(e.abs() + o).sum(1)
    for name, v in (("dx", flat(g.dx)), ("db", flat(g.db)), ("dscale", g.dscale), ("dgate", g.dgate.reshape(-1)), ("dpost", g.dpost[0]),
                    ("dpost_bias", g.dpost[1]), ("dnorm", g.dnorm[0]), ("dnorm_bias", g.dnorm[1])):
        within(name, v, *want[name])


# gates of more rows than a wave sums, and of as many or one more than the limit; rows by
# values, by lane groups, by a workgroup, and past the widest of them
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gates,per,C", [(3, 512, 40), (3, 513, 40), (1, 3136, 80), (5, 1025, 6), (2, 700, 2560), (2, 600, 16500),
                                         (130, 520, 3), (2, 20000, 24)])
def test_gates_of_many_rows(gates, per, C, dtype):
    x, b, ds, dy = (_rand(i, gates, per, C, dtype=dtype) for i in range(4))
    check(x, b, ds, dy, lambda s: s, dict(_vectors(C, dtype), gate=_rand(20, gates)), per)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", [3, 24, 61, 640])
def test_rows_of_three_axes(C, dtype):
    """Slices of wider rows, axes of one, and axes that lie the other way round in memory."""
    B, N = 6, 35

    def wide(seed, *lead):
        t = torch.full((*lead, C + 9), float("nan"), dtype=dtype, device="cuda")
        t[..., 2:C + 2] = _rand(seed, *lead, C, dtype=dtype)
        return t[..., 2:C + 2]
    vectors = _vectors(C, dtype)

    def as_wide(s):
        t = wide(0, *s.shape[:-1])
        t.copy_(s)
        return t
    for lead, gate in (((B, N), B), ((B, 1, N), B), ((1, B, N), 1), ((B, N, 1), B)):
        x, b, ds, dy = (wide(i, *lead) for i in range(4))
        shape = lead[:1]
        check(x, b, ds, dy, as_wide, dict(vectors, gate=_rand(20, *shape)), B * N // gate)
        check(x, b, ds, dy, as_wide, dict(vectors, gate=_rand(21, *lead)), 1)
    # images whose rows do not follow on each other are no rows a uniform stride apart
    bad = wide(5, B, N + 1)[:, :N]
    turned = wide(6, N, B).transpose(0, 1)
    for t in (bad, turned):
        for call in (lambda: api.residual_norm(t, t.contiguous()), lambda: api.residual_norm(t.contiguous(), t),
                     lambda: api.residual_norm_backward(t, None, t.contiguous(), None, (None,) * 4),
                     lambda: api.residual_norm_backward(t.contiguous(), None, t, None, (None,) * 4)):
            with pytest.raises(ValueError, match="uniform stride"):
                call()
