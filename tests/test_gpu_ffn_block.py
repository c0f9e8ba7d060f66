"""The operators that train a gated FFN together, as they are used: a block's forward and
backward pass against float64 autograd, examples/ffn_gated.py, other streams, replayed
graphs, strided and unaligned rows, offsets past 32 bits, what is not finite, refusals."""
import importlib.util
import math
import os

import pytest
import torch

import ffn_train_ref as ref
from gpu_helpers import require_gpu
from paper_2604_21290_amd import api

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()


def _rand(seed, *shape, dtype=torch.float32, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


def _example():
    spec = importlib.util.spec_from_file_location("ffn_gated", os.path.join(ROOT, "examples", "ffn_gated.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _norm64(t, g, b, eps=1e-5):
    mean = t.mean(-1, keepdim=True)
    var = (t - mean).square().mean(-1, keepdim=True)
    return (t - mean) * (var + eps).rsqrt() * g + b


def _block64(x, gate, w):
    F = w["W"].shape[0] // 2
    pre = _norm64(x, w["gamma"], w["beta"]) @ w["W"].t() + w["bias"]
    z = torch.nn.functional.silu(pre[..., :F]) * pre[..., F:]
    o = z @ w["Wd"].t() + w["bd"]
    s = x + gate[:, None, None] * w["scale"] * _norm64(o, w["post_gamma"], w["post_beta"])
    return s, _norm64(s, w["next_gamma"], w["next_beta"])


@pytest.mark.parametrize("B,N,C,F", [(2, 5, 12, 8), (3, 49, 40, 96), (4, 196, 192, 384)])
def test_block_against_autograd(B, N, C, F):
    """In fp32 (gl_linear takes whole vectors: F a multiple of 4).  A chain of sums of n = C, F, 2 F and rows: to first order a result's 2-norm is
    off by at most 2^-24 times the lengths of the sums on its way, each times what a norm
    makes of a relative error (the 2-norm of its derivative's terms, below 4 here): 4 x 4 n."""
    m = _example()
    w = {k: t.float() + 0.1 * _rand(i, *t.shape) for i, (k, t) in enumerate(m.make_weights(C, F, torch.float32).items())}
    x, gate = _rand(50, B, N, C), torch.linspace(0.0, 1.5, B, device="cuda")
    cs, cy = _rand(51, B, N, C), _rand(52, B, N, C)
    leaves = [x.clone().requires_grad_(), gate.clone().requires_grad_(), *(w[k].clone().requires_grad_() for k in m.NAMES)]
    s, y = m.GatedFfn.apply(*leaves)
    got = [s, y, *torch.autograd.grad((s * cs).sum() + (y * cy).sum(), leaves)]
    x64, gate64, *w64 = [t.detach().double().requires_grad_() for t in leaves]
    s64, y64 = _block64(x64, gate64, dict(zip(m.NAMES, w64)))
    want = [s64, y64, *torch.autograd.grad((s64 * cs.double()).sum() + (y64 * cy.double()).sum(), [x64, gate64, *w64])]
    bound = 16 * (3 * C + 3 * F + B * N) * ref.U
    for name, g, e in zip(("s", "y", "x", "gate") + m.NAMES, got, want):
        off = float((g.double() - e).norm() / e.norm().clamp_min(1e-30))
        assert off <= bound, (name, off, bound)


def test_example_runs():
    sizes = _example().main("vig_ti", 3)["sizes"]
    assert len(sizes) == 3 and all(math.isfinite(v) for v in sizes)


@pytest.mark.parametrize("act", [api.GL_ACT_GELU, api.GL_ACT_SILU])
def test_gated_gradient_against_differences(act):
    """The loss sum(h c) along a direction: its slope from two fp32 forward passes h apart in
    the input by +-e is off by e^2 / 6 of the third derivative (act's, below 3, times the
    direction's three factors) and by the passes' own rounding over e."""
    R, K, F = 40, 24, 33
    x, W, b = _rand(1, R, K), _rand(2, 2 * F, K, size=K ** -0.5), _rand(3, 2 * F, size=0.3)
    c, e = _rand(4, R, F), 2.0 ** -6
    h, pre = api.gated_linear(x, W, b, act=act, keep=True)
    dx, dW, db = api.gated_linear_backward(c, x, W, pre, act=act)
    for i, (t, d) in enumerate(((x, dx), (W, dW), (b, db))):
        v = _rand(10 + i, *t.shape)
        v = v / v.norm()
        args = [[x, W, b] for _ in range(2)]
        args[0][i], args[1][i] = t + e * v, t - e * v
        up, down = ((api.gated_linear(*a, act=act).double() * c.double()).sum() for a in args)
        slope = float((up - down) / (args[0][i].double() - args[1][i].double()).norm())
        want = float((d.double() * v.double()).sum())
        # third derivative along v: at most 3 sum |c| (|dg| + |du|)^3 with dg, du the change of pre
        pu = api.gated_linear(*args[0], act=act, keep=True)[1] - api.gated_linear(*args[1], act=act, keep=True)[1]
        rate = (pu[:, :F].abs() + pu[:, F:].abs()).double() / (2 * e)
        third = float((3 * (1 + pre[:, F:].abs().double()) * c.abs().double() * rate ** 3).sum())
        rounding = float((h.abs().double() * c.abs().double()).sum()) * (2 * K + 40) * ref.U / e
        assert abs(slope - want) <= e * e / 6 * third + rounding + 1e-4 * abs(want), (i, slope, want)


def test_residual_gradient_against_differences():
    """As above; the norms' third derivatives are taken from the slopes at e and 2 e, whose
    difference is 3 times the error of the first."""
    R, C = 30, 20
    w = dict(post=(1 + 0.2 * _rand(1, C), 0.2 * _rand(2, C)), scale=_rand(3, C), gate=1 + 0.3 * _rand(4, R),
             norm=(1 + 0.2 * _rand(5, C), 0.2 * _rand(6, C)))
    x, b, cs, cy = _rand(7, R, C), _rand(8, R, C), _rand(9, R, C), _rand(10, R, C)

    def loss(x, b, scale, gate, pg, pb, ng, nb):
        s, y = api.residual_norm(x, b, post=(pg, pb), scale=scale, gate=gate, norm=(ng, nb))
        return float((s.double() * cs.double()).sum() + (y.double() * cy.double()).sum())
    s, _, st = api.residual_norm(x, b, stats=True, **w)
    g = api.residual_norm_backward(cs, cy, b, s, st, **w)
    args = [x, b, w["scale"], w["gate"], *w["post"], *w["norm"]]
    size = float((cs.abs().double() * s.abs().double()).sum() + cy.abs().double().sum() * 3)
    for i, d in enumerate((g.dx, g.db, g.dscale, g.dgate, *g.dpost, *g.dnorm)):
        v = _rand(20 + i, *d.shape)
        v = v / v.norm()

        def slope(e):
            a, c = list(args), list(args)
            a[i], c[i] = args[i] + e * v, args[i] - e * v
            return (loss(*a) - loss(*c)) / float((a[i].double() - c[i].double()).norm())
        e = 2.0 ** -7
        one, two = slope(e), slope(2 * e)
        want = float((d.double() * v.double()).sum())
        rounding = size * (4 * C + 60) * ref.U / e
        assert abs(one - want) <= abs(two - one) + rounding + 1e-4 * abs(want), (i, one, two, want)


def _calls(seed, R=300, C=72, F=50, dtype=torch.bfloat16):
    """Every operator once, as (call, inputs)."""
    x, W = _rand(seed, R, C, dtype=dtype), _rand(seed + 1, 2 * F, C, dtype=dtype, size=C ** -0.5)
    dh, dy, b = _rand(seed + 2, R, F, dtype=dtype), _rand(seed + 3, R, 2 * F, dtype=dtype), _rand(seed + 4, R, C, dtype=dtype)
    bias, vec, gate = _rand(seed + 5, 2 * F, dtype=dtype), _rand(seed + 6, C, dtype=dtype), _rand(seed + 7, R)
    how = dict(post=(vec, vec), scale=vec, gate=gate, norm=(vec, vec))
    pre = api.gated_linear(x, W, bias, keep=True)[1]
    s, _, st = api.residual_norm(x, b, stats=True, **how)

    def run(**k):
        out = list(api.gated_linear(x, W, bias, keep=True, **k))
        out += api.gated_linear_backward(dh, x, W, pre, **k)
        out += api.linear_backward(dy, x, W, **k)
        r = api.residual_norm(x, b, stats=True, **how, **k)
        out += [*r[:2], *r[2]]
        g = api.residual_norm_backward(x, b, b, s, st, **how, **k)
        return out + [g.dx, g.db, g.dgate, g.dscale, *g.dpost, *g.dnorm]
    return run, [x, W, dh, dy, b, bias, vec, gate, pre]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_other_stream_and_python_path(dtype, monkeypatch):
    run, _ = _calls(1, dtype=dtype)
    want = [t.clone() for t in run()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = run(stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(s):
        got = run()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    monkeypatch.setattr(api, "_native", api._NoCalls)
    assert all(torch.equal(a, b) for a, b in zip(run(), want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_graph_replays(dtype):
    """Captured once and replayed on new inputs, with eager work between the replays; two
    graphs of the same call do not share their workspaces."""
    run, ins = _calls(3, R=700, dtype=dtype)
    run()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run())
        graphs.append(g)
    for turn in range(4):
        for i, t in enumerate(ins):
            t.copy_(_rand(100 * turn + i, *t.shape, dtype=t.dtype, size=0.5))
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_workspace_of_the_caller():
    x, W, dy = _rand(1, 500, 41), _rand(2, 30, 41), _rand(3, 500, 30)
    want = api.linear_backward(dy, x, W)
    ws = api.linear_backward_workspace(x, W)
    assert ws.nbytes and all(torch.equal(a, b) for a, b in zip(api.linear_backward(dy, x, W, ws=ws), want))
    with pytest.raises(api.GraphLeapError):
        api.linear_backward(dy, x, W, ws=api.Workspace(ws.nbytes - 256, x.device))
    dh, pre = _rand(4, 500, 15), _rand(5, 500, 30)
    ws = api.gated_linear_backward_workspace(x, W)
    assert all(torch.equal(a, b) for a, b in zip(api.gated_linear_backward(dh, x, W, pre, ws=ws),
                                                 api.gated_linear_backward(dh, x, W, pre)))
    ws = api.gated_linear_workspace(x, W)
    assert torch.equal(api.gated_linear(x, W, ws=ws), api.gated_linear(x, W))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,C,gap,shift", [(50, 33, 7, 1), (300, 640, 3, 5), (20000, 20, 1, 3), (7, 1, 3, 1), (40, 5000, 24, 1)])
def test_strided_and_unaligned_rows(R, C, gap, shift, dtype):
    """Rows out of wider ones, from any element on; what lies between them is NaN and stays."""
    def rows(seed):
        buf = torch.full((shift + R * (C + gap),), float("nan"), dtype=dtype, device="cuda")
        t = buf[shift:].view(R, C + gap)[:, :C]
        t.copy_(_rand(seed, R, C, dtype=dtype))
        return t
    x, b, ds, dy = (rows(i) for i in range(4))
    vec = lambda i: _rand(10 + i, C + 1, dtype=dtype)[1:]  # noqa: E731  (at any element too)
    how = dict(post=(vec(0), vec(1)), scale=vec(2), gate=_rand(20, R + 1)[1:], norm=(vec(3), vec(4)))
    s, y, st = api.residual_norm(x, b, stats=True, **how)
    flat = {k: (tuple(t.clone() for t in v) if isinstance(v, tuple) else v.clone()) for k, v in how.items()}
    want = api.residual_norm(x.clone().contiguous(), b.clone().contiguous(), stats=True, **flat)
    assert torch.equal(s, want[0]) and torch.equal(y, want[1]) and all(torch.equal(a, e) for a, e in zip(st, want[2]))
    sv = rows(30)
    sv.copy_(s)
    got = api.residual_norm_backward(ds, dy, b, sv, st, **how)
    want = api.residual_norm_backward(*(t.clone().contiguous() for t in (ds, dy, b)), s, st, **flat)
    for a, e in zip(got, want):
        for p, q in zip(a, e) if isinstance(a, tuple) else ((a, e),):
            assert torch.equal(p, q)


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_gate_at_its_limits(name):
    """GELU and SiLU of the infinities are their limits, a NaN is a NaN, and neither reaches
    other rows or columns; their derivatives likewise."""
    act = api.GL_ACT_GELU if name == "gelu" else api.GL_ACT_SILU
    inf = float("inf")
    g = torch.tensor([inf, -inf, float("nan"), 3.4e38, -3.4e38, 0.0, -0.0, 1e-40, -100.0, 100.0], device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        gate = g.to(dtype)
        F = gate.numel()
        x = torch.ones(1, 8, dtype=dtype, device="cuda") / 8
        for R in (1, 70):  # both kernels
            W = torch.zeros(2 * F, 8, dtype=dtype, device="cuda")
            bias = torch.cat([gate, torch.full((F,), 2.0, dtype=dtype, device="cuda")])
            h = api.gated_linear(x.expand(R, 8).contiguous(), W, bias, act=act)
            for r in (0, R - 1):
                v = h[r].tolist()
                assert v[0] == inf and v[1] == 0 and math.isnan(v[2]) and v[4] == 0 and v[5] == 0 and v[6] == 0
                assert abs(v[8]) < 1e-30 and v[9] == 200
        pre = torch.cat([gate, torch.full((F,), 2.0, dtype=dtype, device="cuda")])[None]
        dh = torch.ones(1, F, dtype=dtype, device="cuda")
        db = api.gated_linear_backward(dh, x, W, pre, act=act, need=(False, False, True))[2].tolist()
        assert db[0] == 2 and db[1] == 0 and math.isnan(db[2]) and db[3] == 2 and db[4] == 0
        assert db[5] == 1 and db[6] == 1 and abs(db[8]) < 1e-30 and db[9] == 2
        assert db[F] == inf and db[F + 1] == 0 and math.isnan(db[F + 2]) and db[F + 9] == 100


def test_what_is_not_finite_stays_in_its_row():
    """A NaN in a row of x (and past the rows' ends, which odd sizes pad with zeros) reaches
    that row's results and the sums over rows alone."""
    for dtype in (torch.float32, torch.bfloat16):
        for R, K, F in ((70, 31, 9), (200, 64, 40)):
            x, W = _rand(1, R, K, dtype=dtype), _rand(2, 2 * F, K, dtype=dtype)
            x[5, 3] = float("nan")
            h, pre = api.gated_linear(x, W, keep=True)
            assert h[5].isnan().all() and not h[:5].isnan().any() and not h[6:].isnan().any()
            dy = _rand(3, R, 2 * F, dtype=dtype)
            dy[7, 2] = float("inf")
            dx, dW, db = api.linear_backward(dy, x, W)
            bad = torch.zeros(R, dtype=torch.bool, device="cuda")
            bad[7] = True
            assert torch.equal(~dx.isfinite().all(1), bad)
            col = torch.zeros(K, dtype=torch.bool, device="cuda")
            col[3] = True
            row = torch.zeros(2 * F, dtype=torch.bool, device="cuda")
            row[2] = True
            assert torch.equal(~dW.isfinite(), row[:, None] | col[None]) and torch.equal(~db.isfinite(), row)
    x, b = _rand(4, 40, 24), _rand(5, 40, 24)
    b[3, 0], x[9, 1] = float("nan"), float("inf")
    s, y = api.residual_norm(x, b, post=(None, None), norm=(None, None))
    assert s[3].isnan().all() and y[3].isnan().all() and s[9, 1] == float("inf") and y[9].isnan().all()
    rest = torch.ones(40, dtype=torch.bool, device="cuda")
    rest[3] = rest[9] = False
    assert s[rest].isfinite().all() and y[rest].isfinite().all()


@pytest.mark.parametrize("C", [5, 24, 100, 1000, 2560, 20000])
def test_rows_of_one_value(C):
    """A row of equal values has them as its mean: its norm is beta, with eps of any size."""
    for v in (1e5, -3.0, 1e-20, 0.0):
        x = torch.full((40, C), v, device="cuda")
        beta = _rand(1, C)
        s, y = api.residual_norm(x, torch.zeros_like(x), post=(None, None), norm=(None, beta), eps=1e-12)
        assert torch.equal(s, x) and float((y - beta).abs().max()) <= 1e-3, (C, v)


def test_a_shut_gate():
    """A gate of 0: s is x, b's gradient and the row's part of the vectors' are zero."""
    for dtype in (torch.float32, torch.bfloat16):
        x, b = _rand(1, 6, 9, 40, dtype=dtype), _rand(2, 6, 9, 40, dtype=dtype)
        gate = torch.tensor([0.0, 1.25, 0.0, 1.25, 1.25, 0.0], device="cuda")
        shut = gate == 0
        how = dict(post=(None, None), gate=gate, norm=(None, None))
        s, _, st = api.residual_norm(x, b, stats=True, **how)
        assert torch.equal(s[shut], x[shut]) and not torch.equal(s, x)
        g = api.residual_norm_backward(x, b, b, s, st, **how)
        assert not g.db[shut].any() and g.db[~shut].any() and g.dgate.shape == gate.shape and g.dgate.all()


def test_offsets_past_32_bits():
    """More than 2^31 elements, and 2^32 bytes, in every tensor of rows."""
    R, C = (1 << 21) + 5, 1032
    x = torch.zeros(R, C, dtype=torch.bfloat16, device="cuda")
    b = torch.zeros_like(x)
    x[-70:], b[-70:] = _rand(1, 70, C, dtype=torch.bfloat16), _rand(2, 70, C, dtype=torch.bfloat16)
    one = (torch.ones(C, dtype=torch.bfloat16, device="cuda"), None)
    s, y, st = api.residual_norm(x, b, post=one, norm=one, stats=True)
    st70 = api.residual_norm(x[-70:].clone(), b[-70:].clone(), post=one, norm=one, stats=True)
    assert torch.equal(s[-70:], st70[0]) and torch.equal(y[-70:], st70[1]) and not s[:-70].any()
    g = api.residual_norm_backward(None, x, b, s, st, post=one, norm=one)
    e = api.residual_norm_backward(None, x[-70:].clone(), b[-70:].clone(), st70[0], st70[2], post=one, norm=one)
    assert torch.equal(g.dx[-70:], e.dx) and torch.equal(g.db[-70:], e.db)
    assert float((g.dnorm[0] - e.dnorm[0]).norm() / e.dnorm[0].norm()) < R * ref.U
    del s, y, st, g, b
    F = 1024
    W = _rand(3, 2 * F, 8, dtype=torch.bfloat16)
    x = x[:, :8].contiguous()
    h, pre = api.gated_linear(x, W, keep=True)
    h70, pre70 = api.gated_linear(x[-70:].clone(), W, keep=True)
    # (other tiles, the same products: sums of eight in one instruction)
    assert float((h[-70:].double() - h70.double()).abs().max()) <= 2.0 ** -7 * float(h70.abs().max())
    dh = torch.zeros(R, F, dtype=torch.bfloat16, device="cuda")
    dh[-70:] = _rand(4, 70, F, dtype=torch.bfloat16)
    got = api.gated_linear_backward(dh, x, W, pre)
    want, bound = ref.gated_backward(dh[-70:], x[-70:], W, pre[-70:], "silu")
    for i, (a, e, o) in enumerate(zip(got, want, bound)):
        assert bool(((a[-70:] if i == 0 else a).double() - e).abs().le(o).all()), i
    assert not got[0][:-70].any()


def test_refusals():
    x, W = _rand(1, 10, 16), _rand(2, 8, 16)
    dy, pre, dh = _rand(3, 10, 8), _rand(4, 10, 8), _rand(5, 10, 4)
    bad = [lambda: api.gated_linear(x, W[:7]), lambda: api.gated_linear(x, W[:, :15]), lambda: api.gated_linear(x.t(), W),
           lambda: api.gated_linear(x, W.bfloat16()), lambda: api.gated_linear(x.cpu(), W), lambda: api.gated_linear(x, W, dy),
           lambda: api.linear_backward(dh, x, W), lambda: api.linear_backward(dy.bfloat16(), x, W),
           lambda: api.linear_backward(dy, x, W, need=(False, False, False)), lambda: api.linear_backward(dy.t(), x, W),
           lambda: api.gated_linear_backward(dy, x, W, pre), lambda: api.gated_linear_backward(dh, x, W, dh),
           lambda: api.gated_linear_backward(dh, x, W, pre.t().contiguous().t()),
           lambda: api.residual_norm(x, x[:5]), lambda: api.residual_norm(x, x.bfloat16()), lambda: api.residual_norm(x.t(), x.t()),
           lambda: api.residual_norm(x, x, gate=_rand(6, 5)), lambda: api.residual_norm(x, x, gate=_rand(6, 10, 16)),
           lambda: api.residual_norm(x, x, gate=_rand(6, 10).double()), lambda: api.residual_norm(x, x, scale=_rand(6, 15)),
           lambda: api.residual_norm(x, x, norm=(x[0, :15].clone(), None)),
           lambda: api.residual_norm_backward(None, None, x, x, (None,) * 4),
           lambda: api.residual_norm_backward(x, x, x, x, (None,) * 4, norm=(None, None)),
           lambda: api.residual_norm_backward(x, x, x, x, (None,) * 4),
           lambda: api.residual_norm_backward(x, None, x, None, (None,) * 4, post=(None, None)),
           lambda: api.residual_norm_backward(x, None, x[:9], None, (None,) * 4)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} is not refused")
    half = x.half()
    for call in (lambda: api.gated_linear(half, W.half()), lambda: api.residual_norm(half, half),
                 lambda: api.linear_backward(dy.half(), half, W.half())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: api.gated_linear(x, W, act=3), lambda: api.residual_norm(x, x, kind=2),
                 lambda: api.residual_norm(x, x, eps=-1.0), lambda: api.gated_linear(x[:0], W),
                 lambda: api.gated_linear(_rand(7, 161)[1:].view(10, 16), W)):
        with pytest.raises(api.GraphLeapError):
            call()
    # gl_linear and gl_linear_q8 have no SiLU
    with pytest.raises(api.GraphLeapError):
        api.linear(x, W, act_out=api.GL_ACT_SILU)
