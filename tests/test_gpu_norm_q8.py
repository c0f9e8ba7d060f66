"""GPU parity of layer norm, its gradient and the 8-bit layers against the float64
oracle: widths around every tile's edge, rows shorter than a vector, strided and
unaligned rows, a single row, zero and constant rows, rows that are not finite,
offsets past 32 bits, other streams, replayed graphs.

Bounds (u = 2^-8 bf16, 2^-24 fp32 for one rounding to the stored type; e = 2^-24;
D = 80 + C / 256 fp32 additions at most between a term and its row's sum):
  mean    D e avg|x|
  rstd    (D + 8) e rstd: squares, their sum, the product with 1/C, eps, the root
  y       |gamma| rstd (mean's + |d| (D + 12) e) + 3 e (|y| + |beta|), then u |y|
  dx      rstd (4 e |h| + (D + 4) e (avg|h| + |xh| avg|h xh|) + 4 e |xh| avg|h xh|), u |dx|
  dgamma  (R / 16 + 256) e sum|dy xh| + 3 e sum|dy xh|; dbeta alike: a lane adds at
          most R / 16 rows, then the workgroups' sums are added
  8 bits  of stored rows: equal.  Of a norm: half a step, and y's bound in steps
  layer   3 e |sum| + e |y|, through the GELU 1.13 times that and 3e-7 |y|; u |out|"""
import numpy as np
import pytest
import torch

from gpu_helpers import from_dev, require_gpu
from oracle import norm_q8_ref as Q

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _api():
    require_gpu()
    from paper_2604_21290_amd import api
    return api


def _say(*a):
    print("[gpu-test]", *a, flush=True)


def _f64(t):
    return t.detach().cpu().double().numpy()


def _rows(g, R, C, dtype, gap=0, shift=0):
    """R rows of C channels, C + gap elements apart, the first one `shift` in."""
    spread = np.exp(0.5 * g.standard_normal(C))
    x = (g.standard_normal((R, C)) * spread + 0.5 * g.standard_normal(C)) * np.exp(0.3 * g.standard_normal((R, 1)))
    buf = torch.full((shift + R * (C + gap),), float("nan"), dtype=dtype, device="cuda")
    t = buf[shift:].view(R, C + gap)[:, :C]
    t.copy_(torch.from_numpy(x).to(dtype))
    return t


def _vec(g, n, dtype, about=0.0):
    return torch.from_numpy(about + 0.3 * g.standard_normal(n)).to(dtype).cuda()


def _y_bound(x, y, mean, rstd, gamma, beta):
    C = x.shape[-1]
    D = 80 + C / 256
    gam = 1.0 if gamma is None else np.abs(gamma)
    bet = 0.0 if beta is None else np.abs(beta)
    dm = D * E32 * np.abs(x).mean(-1, keepdims=True)
    d = np.abs(x - mean[:, None])
    return gam * rstd[:, None] * (dm + d * (D + 12) * E32) + 3 * E32 * (np.abs(y) + bet)


def _within(name, got, ref, bound):
    assert np.isfinite(got).all(), name
    over = np.abs(got - ref) > bound
    assert not over.any(), (name, np.argwhere(over)[:4], float((np.abs(got - ref) / np.maximum(bound, 1e-300)).max()))


def _edges(dt):
    E = 8 if dt == "bf16" else 4
    out = {1, 2, 3, E - 1, E, E + 1, 80, 192}
    for n in (16, 32, 64, 128, 256, 512, 1024, 2048):
        out |= {n * E, n * E + 1} if n > 64 else {n * E - 1, n * E, n * E + 1}
    return sorted(out)


NORM_CASES = [(dt, C, (1, 3, 37)[i % 3], (0, 0, 5)[i % 3], i % 2, i % 4 != 3)
              for dt in ("bf16", "f32") for i, C in enumerate(_edges(dt))]
NORM_CASES += [("bf16", 80, 4099, 0, 0, True), ("f32", 192, 1000, 0, 0, True), ("bf16", 640, 2051, 3, 1, True),
               ("bf16", 33, 20001, 0, 1, True), ("bf16", 64, 16384, 0, 0, True), ("bf16", 65, 16390, 0, 0, True),
               ("bf16", 123, 16385, 2, 1, False), ("bf16", 192, 20000, 0, 0, True), ("bf16", 13, 16400, 5, 1, True),
               ("f32", 31, 17001, 1, 0, True), ("f32", 90, 16385, 0, 0, True), ("f32", 16, 65537, 0, 0, False), ("bf16", 2560, 700, 0, 0, True)]
# one launch of more than one trip over the rows, and wide rows' sums through the workspace
NORM_CASES += [("bf16", 100, 799, 0, 1, True), ("f32", 37, 513, 3, 0, False), ("bf16", 1003, 640, 0, 0, True),
               ("bf16", 3001, 1024, 1, 0, True), ("f32", 1999, 1030, 0, 0, True), ("bf16", 2561, 1100, 0, 1, True),
               ("bf16", 5423, 1027, 0, 0, True), ("bf16", 7000, 1029, 8, 0, False), ("f32", 5001, 1040, 0, 1, True)]
# rows of 257 to 512 chunks: more than one turn, and more rows than one chunk a lane takes
NORM_CASES += [("bf16", 4093, 1037, 0, 1, True), ("bf16", 2051, 4101, 3, 0, True), ("f32", 1025, 12289, 0, 0, True)]


@pytest.mark.parametrize("dt,C,R,gap,shift,affine", NORM_CASES)
def test_layer_norm_and_gradient(dt, C, R, gap, shift, affine):
    api = _api()
    _say("norm", dt, C, R, gap, shift, affine)
    dtype = DT[dt]
    g = np.random.default_rng(C * 7 + R)
    x, dy = _rows(g, R, C, dtype, gap, shift), _rows(g, R, C, dtype, gap, shift)
    gamma = _vec(g, C, dtype, 1.0) if affine else None
    beta = _vec(g, C, dtype) if affine else None
    y, mean, rstd = api.layer_norm(x, gamma, beta, 1e-5, stats=True)
    y2 = api.layer_norm(x, gamma, beta, 1e-5)
    dx, dg, db = api.layer_norm_backward(dy, x, mean, rstd, gamma)
    dx2, none, db2 = api.layer_norm_backward(dy, x, mean, rstd, gamma, need=(True, False, True))
    dx3 = api.layer_norm_backward(dy, x, mean, rstd, gamma, need=(True, False, False))[0]
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dx, dx3)
    assert none is None and torch.equal(db, db2)
    xf, dyf = _f64(x), _f64(dy)
    gam, bet = (None, None) if not affine else (_f64(gamma), _f64(beta))
    ry, rm, rr = Q.layer_norm_ref(xf, gam, bet, float(np.float32(1e-5)))
    D = 80 + C / 256
    _within("mean", _f64(mean), rm, D * E32 * np.abs(xf).mean(-1) + E32 * np.abs(rm))
    _within("rstd", _f64(rstd), rr, (D + 8) * E32 * rr
            + rr ** 3 * (D * E32 * np.abs(xf).mean(-1)) ** 2)
    _within("y", _f64(y), ry, _y_bound(xf, ry, rm, rr, gam, bet) + U[dtype] * np.abs(ry))
    # the gradient is that of the statistics it is given
    m, s = _f64(mean), _f64(rstd)
    rdx, rdg, rdb = Q.layer_norm_backward_ref(dyf, xf, m, s, gam)
    xh = (xf - m[:, None]) * s[:, None]
    h = dyf if gam is None else dyf * gam
    ah, ahx = np.abs(h).mean(-1, keepdims=True), np.abs(h * xh).mean(-1, keepdims=True)
    b = s[:, None] * (4 * E32 * np.abs(h) + (D + 4) * E32 * (ah + np.abs(xh) * ahx) + 4 * E32 * np.abs(xh) * ahx)
    _within("dx", _f64(dx), rdx, b + U[dtype] * np.abs(rdx))
    n = R / 16 + 259
    _within("dgamma", _f64(dg), rdg, n * E32 * np.abs(dyf * xh).sum(0))
    _within("dbeta", _f64(db), rdb, n * E32 * np.abs(dyf).sum(0))


@pytest.mark.parametrize("dt,C,R,gap,shift,affine", NORM_CASES)
def test_rows_to_8_bits(dt, C, R, gap, shift, affine):
    api = _api()
    _say("q8", dt, C, R, gap, shift)
    dtype = DT[dt]
    g = np.random.default_rng(C * 11 + R)
    x = _rows(g, R, C, dtype, gap, shift)
    if R > 2:
        x[1] = 0
        x[2] = x[2] * 2.0 ** -60
    gamma = _vec(g, C, dtype, 1.0) if affine else None
    beta = _vec(g, C, dtype) if affine else None
    a = api.quantize_rows(x)
    b = api.layer_norm_q8(x, gamma, beta, 1e-5)
    torch.cuda.synchronize()
    Kp = api.q8_row_bytes(C)
    for r in (a, b):
        assert r.q.shape == (R, Kp) and r.scale.shape == (R,) and r.K == C
        assert not r.q[:, C:].any(), "the bytes after a row are zero"
    xf = _f64(x)
    rq, rs = Q.quantize_rows_ref(xf)
    if dt == "f32":  # the definition's fp32 quotient
        x32 = xf.astype(np.float32)
        top = np.abs(x32).max(-1, keepdims=True)
        rq = np.rint(x32 * np.float32(127) / np.where(top > 0, top, np.float32(1))).astype(np.int64)
    assert (a.q[:, :C].cpu().numpy() == rq).all()
    assert (np.abs(_f64(a.scale) - rs) <= 2 * E32 * rs).all()
    gam, bet = (None, None) if not affine else (_f64(gamma), _f64(beta))
    ry, rm, rr = Q.layer_norm_ref(xf, gam, bet, float(np.float32(1e-5)))
    by = _y_bound(xf, ry, rm, rr, gam, bet)
    top, btop = np.abs(ry).max(-1, keepdims=True), by.max(-1, keepdims=True)
    some = top[:, 0] > 4 * btop[:, 0]  # a row whose norm is zero has rounding alone
    steps = 127 / np.where(top > 0, top, 1)
    lim = 0.5 + steps * (by + btop) * 1.01 + 127 * 4 * E32
    off = np.abs(b.q[:, :C].cpu().numpy() - ry * steps)
    assert (off <= lim)[some].all(), float((off - lim)[some].max())
    assert (np.abs(_f64(b.scale) - top[:, 0] / 127) <= (btop[:, 0] + 2 * E32 * top[:, 0]) / 127)[some].all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_8_bit_ties_and_all_values(dt):
    """Every bf16 magnitude of two binades against several tops: ties go to even."""
    api = _api()
    m = torch.arange(128, 256, dtype=torch.float64)
    for top in (1.0, 254.0, 129.0, 255.0, 2.0 ** -100, 3 * 2.0 ** 120):
        row = torch.cat([m / 256, m / 512, -m / 256, torch.tensor([1.0], dtype=torch.float64)]) * top
        x = row.to(DT[dt]).cuda().reshape(1, -1)
        a = api.quantize_rows(x)
        torch.cuda.synchronize()
        xf = _f64(x)
        q = np.rint(xf * 127 / np.abs(xf).max())
        assert (a.q[:, : x.shape[1]].cpu().numpy() == q).all(), top


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("C", [3, 80, 640, 5000])
def test_rows_that_are_not_finite(dt, C):
    api = _api()
    dtype = DT[dt]
    g = np.random.default_rng(C)
    x = _rows(g, 6, C, dtype)
    clean = x.clone()
    x[1, C - 1] = float("nan")
    x[3, 0] = float("inf")
    x[4, C // 2] = float("-inf")
    bad = [1, 3, 4]
    good = [0, 2, 5]
    for t in (api.layer_norm(x), api.quantize_rows(x), api.layer_norm_q8(x)):
        torch.cuda.synchronize()
        if isinstance(t, torch.Tensor):
            assert torch.isnan(t[bad]).all()
            assert torch.equal(t[good], api.layer_norm(clean)[good])
        else:
            assert torch.isnan(t.scale[bad]).all() and not t.q[bad].any()
            assert torch.isfinite(t.scale[good]).all()
    # what is computed from such rows is NaN, and nothing else is
    W = api.quantize_rows(_rows(g, 5, C, dtype))
    out = api.linear_q8(api.quantize_rows(x), W, dtype=dtype)
    ref = api.linear_q8(api.quantize_rows(clean), W, dtype=dtype)
    torch.cuda.synchronize()
    assert torch.isnan(out[bad]).all() and torch.equal(out[good], ref[good])


def test_constant_and_zero_rows():
    api = _api()
    x = torch.zeros((4, 192), device="cuda")
    x[1] = 3.0
    x[2] = -1e-30
    x[3] = 2.0 ** -119
    y, mean, rstd = api.layer_norm(x, None, None, 1e-5, stats=True)
    a = api.quantize_rows(x)
    torch.cuda.synchronize()
    assert (y[0] == 0).all() and rstd[0].item() == pytest.approx(1e-5 ** -0.5, rel=1e-6)
    # a constant row: the deviations are the mean's rounding
    assert y[1].abs().max().item() <= 3.0 * 80 * E32 * 320
    assert (a.q[0] == 0).all() and a.scale[0] == 0
    assert (a.q[1] == 127).all() and (a.q[2] == -127).all()
    assert (a.q[3] == 0).all() and a.scale[3] == 0


LAYER_CASES = [
    # R, K, Cout, gelu, residual, bias
    (1, 1, 1, False, False, True), (1, 16, 8, False, True, True), (1, 640, 2560, True, False, True),
    (2, 15, 7, False, True, False), (3, 17, 33, True, True, True), (7, 130, 250, False, False, True),
    (16, 64, 64, False, True, True), (17, 128, 16, True, False, True), (31, 4665, 72, False, True, True),
    (33, 257, 129, False, True, True), (64, 2560, 640, False, True, True), (65, 63, 65, False, False, False),
    (128, 1024, 128, False, True, True), (129, 129, 129, True, True, True), (196, 192, 768, True, False, True),
    (777, 1001, 333, False, False, True), (1000, 80, 320, True, False, True), (1025, 1040, 1025, False, True, True),
    (4100, 320, 80, False, True, True), (6272, 192, 768, True, False, True), (12544, 72, 641, False, True, True),
    (20000, 96, 24, False, True, True), (2049, 4096, 515, False, False, True), (5, 131071, 9, False, False, True),
    (8192, 640, 2048, True, True, True), (3000, 16, 4000, False, True, True),
    # tiles of 256 x 256 with ragged edges, of 128 x 128, and of 64 x 64 in two rounds
    (16380, 1000, 1010, True, True, True), (20000, 200, 300, False, True, True),
    (33000, 48, 40, False, True, True), (33000, 130, 40, True, False, True),
    # on both sides of the rule for few rows
    (16, 300, 5000, False, True, True), (17, 300, 5000, False, True, True), (256, 4096, 256, False, True, True),
    (257, 4096, 257, True, True, True), (196, 2560, 640, False, True, True), (1, 131071, 33, False, False, True),
]


def _layer(g, api, R, K, Cout, dtype, gelu, residual, bias):
    q = torch.zeros((R, api.q8_row_bytes(K)), dtype=torch.int8, device="cuda")
    q[:, :K] = torch.from_numpy(g.integers(-127, 128, (R, K), dtype=np.int8))
    w = torch.zeros((Cout, api.q8_row_bytes(K)), dtype=torch.int8, device="cuda")
    w[:, :K] = torch.from_numpy(g.integers(-128, 128, (Cout, K), dtype=np.int8))
    # scales of one dense layer: outputs of order one
    xs = torch.from_numpy(np.exp(0.4 * g.standard_normal(R)) / 73).float().cuda()
    ws = torch.from_numpy(np.exp(0.4 * g.standard_normal(Cout)) / (73 * K ** 0.5)).float().cuda()
    b = _vec(g, Cout, dtype) if bias else None
    res = _rows(g, R, Cout, dtype) if residual else None
    return api.Q8Rows(q, xs, K), api.Q8Rows(w, ws, K), b, res


def _check_layer(x, W, b, res, gelu, out, rows=None):
    q, s = x.q[:, : x.K].cpu().numpy(), _f64(x.scale)
    o, r = out, res
    if rows is not None:
        q, s, o, r = q[rows], s[rows], out[rows], None if res is None else res[rows]
    wq, ws = W.q[:, : W.K].cpu().numpy(), _f64(W.scale)
    bf, rf = None if b is None else _f64(b), None if r is None else _f64(r)
    lin = Q.linear_q8_ref(q, s, wq, ws)
    y = lin if bf is None else lin + bf
    ref = Q.linear_q8_ref(q, s, wq, ws, bf, gelu, rf)
    bound = 3 * E32 * np.abs(lin) + E32 * np.abs(y)
    if gelu:
        bound = 1.13 * bound + 3e-7 * np.abs(y)
    if rf is not None:
        bound = bound + E32 * (np.abs(ref) + np.abs(rf))
    _within("layer", _f64(o), ref, bound + U[out.dtype] * np.abs(ref) + 1e-37)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("R,K,Cout,gelu,residual,bias", LAYER_CASES)
def test_linear_q8(dt, R, K, Cout, gelu, residual, bias):
    api = _api()
    _say("linear_q8", dt, R, K, Cout, gelu, residual, bias)
    g = np.random.default_rng(R + 3 * K + 5 * Cout)
    x, W, b, res = _layer(g, api, R, K, Cout, DT[dt], gelu, residual, bias)
    act = api.GL_ACT_GELU if gelu else api.GL_ACT_NONE
    out = api.linear_q8(x, W, b, act, res, DT[dt])
    again = api.linear_q8(x, W, b, act, res, DT[dt])
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    _check_layer(x, W, b, res, gelu, out)
    if res is not None:  # the residual updated in place
        api.linear_q8(x, W, b, act, res, DT[dt], out=res)
        torch.cuda.synchronize()
        assert torch.equal(res, out)


# short rows: every number of 64-byte steps of K and its edges, column tiles of 64 and 96
# with and without a rest, one and more strips a wave, and the sizes next to those taken
SHORT_CASES = [
    (5000, 1, 80, False, False, True), (5121, 16, 77, True, True, True), (7000, 63, 65, False, True, False),
    (3333, 64, 96, True, False, True), (2500, 65, 97, False, True, True), (1111, 129, 500, True, False, False),
    (4099, 192, 192, True, True, True), (999, 200, 771, False, True, True), (2047, 241, 129, False, False, True),
    (2047, 250, 129, True, True, True), (2047, 257, 129, False, True, True), (1501, 320, 320, True, True, True),
    (1501, 321, 320, False, True, True), (513, 100, 2048, False, False, True), (513, 100, 2049, False, False, True),
    (40009, 80, 320, True, True, True), (60001, 320, 80, False, True, True), (30011, 300, 8, False, True, True),
    (41000, 80, 7, True, True, True), (131089, 48, 1, False, True, True), (26216, 40, 640, False, False, False),
]


# few outputs of long rows, more rows than columns and the other way round
SHORT_CASES += [(1910, 2993, 57, True, True, True), (1885, 2699, 81, False, False, True), (300, 6000, 300, False, True, True),
                (1200, 2560, 96, True, False, False), (33, 4100, 1000, False, True, True), (5000, 1000, 3, True, True, True)]
# K split between groups of waves: fewer stages than groups, a rest of them, several tiles
# a workgroup
SHORT_CASES += [(500, 3000, 500, True, True, True), (871, 4336, 320, False, True, True), (100, 1000, 2000, True, False, True),
                (64, 4096, 4096, False, True, False), (129, 3969, 4033, True, True, True), (130, 400, 2050, False, True, True),
                (783, 4097, 201, False, False, True), (1100, 5000, 333, True, True, True), (40, 513, 3001, False, True, True)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("R,K,Cout,gelu,residual,bias", SHORT_CASES)
def test_linear_q8_short_rows(dt, R, K, Cout, gelu, residual, bias):
    api = _api()
    _say("linear_q8, short rows", dt, R, K, Cout, gelu, residual, bias)
    g = np.random.default_rng(R + 3 * K + 5 * Cout)
    x, W, b, res = _layer(g, api, R, K, Cout, DT[dt], gelu, residual, bias)
    act = api.GL_ACT_GELU if gelu else api.GL_ACT_NONE
    buf = torch.full((R * Cout + 128,), 7.0, dtype=DT[dt], device="cuda")
    out = buf[64: 64 + R * Cout].view(R, Cout)
    api.linear_q8(x, W, b, act, res, DT[dt], out=out)
    torch.cuda.synchronize()
    assert (buf[:64] == 7).all() and (buf[64 + R * Cout:] == 7).all(), "outside the output"
    _check_layer(x, W, b, res, gelu, out)
    if res is not None:  # the residual updated in place
        api.linear_q8(x, W, b, act, res, DT[dt], out=res)
        torch.cuda.synchronize()
        assert torch.equal(res, out)


@pytest.mark.parametrize("R,Cout,shift", [(5, 64, 1), (300, 257, 3), (5000, 640, 5), (20000, 81, 7)])
def test_linear_q8_unaligned_output(R, Cout, shift):
    api = _api()
    g = np.random.default_rng(R)
    x, W, b, _ = _layer(g, api, R, 200, Cout, torch.bfloat16, False, False, True)
    buf = torch.full((shift + R * Cout + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[shift: shift + R * Cout].view(R, Cout)
    api.linear_q8(x, W, b, out=out)
    torch.cuda.synchronize()
    assert (buf[:shift] == 7).all() and (buf[shift + R * Cout:] == 7).all(), "outside the output"
    _check_layer(x, W, b, None, False, out)


def test_gradient_of_very_many_columns():
    """More columns than one launch of the sums' kernel has threads for."""
    api = _api()
    C = 2 ** 26 + 9
    _say("gradient of", C, "columns")
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(2, C, generator=g, device="cuda", dtype=torch.float32) for _ in range(2))
    y, mean, rstd = api.layer_norm(x, stats=True)
    _, dgamma, dbeta = api.layer_norm_backward(dy, x, mean, rstd, need=(False, True, True))
    torch.cuda.synchronize()
    assert torch.equal(dbeta, dy[0] + dy[1])
    terms = dy * ((x - mean[:, None]) * rstd[:, None])
    # a term rounds three times, the sum once
    assert ((dgamma - terms[0] - terms[1]).abs() <= 4 * E32 * terms.abs().sum(0) + 1e-37).all()


def test_linear_q8_one_row_of_very_many_columns():
    """More 16-column units than one launch has workgroups of 512 threads for."""
    api = _api()
    N = 2 ** 26 + 40
    _say("one row to", N, "columns")
    w = torch.randint(-127, 128, (N, 16), dtype=torch.int8, device="cuda")
    w[:, 5:] = 0
    W = api.Q8Rows(w, torch.ones(N, device="cuda"), 5)
    q = torch.zeros((1, 16), dtype=torch.int8, device="cuda")
    q[0, :5] = torch.tensor([3, -7, 127, 0, -127])
    out = api.linear_q8(api.Q8Rows(q, torch.ones(1, device="cuda"), 5), W, dtype=torch.float32)
    torch.cuda.synchronize()
    # whole numbers below 2^24: exact
    assert torch.equal(out[0], sum(float(q[0, k]) * w[:, k].float() for k in range(5)))


def test_linear_q8_extremes_are_exact():
    """The longest rows of the largest products: the sum is near 2^31 and exact."""
    api = _api()
    K = api.GL_MAX_Q8_K
    q = torch.zeros((3, api.q8_row_bytes(K)), dtype=torch.int8, device="cuda")
    w = torch.zeros((2, api.q8_row_bytes(K)), dtype=torch.int8, device="cuda")
    q[:, :K], w[0, :K], w[1, :K] = -128, -128, 127
    q[1, 5], q[2, :K] = 127, 1
    one = torch.ones(3, device="cuda")
    out = api.linear_q8(api.Q8Rows(q, one, K), api.Q8Rows(w, one[:2].clone(), K), dtype=torch.float32)
    torch.cuda.synchronize()
    ref = _f64(q[:, :K]) @ _f64(w[:, :K]).T
    assert ref.max() == 16384 * K
    assert (np.abs(_f64(out) - ref) <= E32 * np.abs(ref)).all()


@pytest.mark.parametrize("R,Cout", [(3, 24), (1000, 1000)])
def test_linear_q8_overflow_and_gelu_limits(R, Cout):
    """Outputs past fp32: infinities, which the GELU takes to infinity and 0."""
    api = _api()
    g = np.random.default_rng(R)
    x, W, _, _ = _layer(g, api, R, 100, Cout, torch.float32, False, False, False)
    x.scale.fill_(3e38)
    W.scale.fill_(1e6)
    lin = api.linear_q8(x, W, dtype=torch.float32)
    gelu = api.linear_q8(x, W, act_out=api.GL_ACT_GELU, dtype=torch.float32)
    torch.cuda.synchronize()
    ref = x.q[:, :100].double() @ W.q[:, :100].double().t()
    inf = torch.tensor(float("inf"), device="cuda")
    assert torch.equal(lin[ref != 0], torch.where(ref > 0, inf, -inf)[ref != 0])
    assert torch.equal(gelu[ref != 0], torch.where(ref > 0, inf, 0 * ref.float())[ref != 0])


def test_offsets_past_32_bits():
    api = _api()
    g = np.random.default_rng(9)
    # rows 2^31 elements apart
    C, ld = 200, 2 ** 31 + 8
    buf = torch.empty(2 * ld + C, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, C), (ld, 1))
    x.copy_(_rows(g, 3, C, torch.bfloat16))
    xc = x.contiguous()
    _say("strided rows past 2^31")
    y, mean, rstd = api.layer_norm(x, stats=True)
    assert torch.equal(y, api.layer_norm(xc))
    a, b = api.quantize_rows(x), api.quantize_rows(xc)
    assert torch.equal(a.q, b.q)
    r1 = api.layer_norm_backward(x, x, mean, rstd)
    r2 = api.layer_norm_backward(xc, xc, mean, rstd)
    assert all(torch.equal(s, t) for s, t in zip(r1, r2))
    # many rows that lie far apart, and narrow ones (a wave holds four of the latter)
    for R, C, ld in ((600, 64, 1 << 25), (5, 40, 1 << 31), (5000, 24, 1 << 22)):
        buf = torch.empty((R - 1) * ld + C, dtype=torch.bfloat16, device="cuda")
        s = buf.as_strided((R, C), (ld, 1))
        s.copy_(_rows(g, R, C, torch.bfloat16))
        c = s.contiguous()
        _say("rows", R, C, "of stride", ld)
        y, mean, rstd = api.layer_norm(s, stats=True)
        ref = Q.layer_norm_ref(_f64(c), None, None, float(np.float32(1e-5)))
        _within("y", _f64(y), ref[0], _y_bound(_f64(c), *ref, None, None) + U[torch.bfloat16] * np.abs(ref[0]))
        assert torch.equal(api.quantize_rows(s).q, api.quantize_rows(c).q)
        dx, dg, _ = api.layer_norm_backward(s, s, mean, rstd)
        cx, cg, _ = api.layer_norm_backward(c, c, mean, rstd)
        # sums in another order: as near as each is to the exact ones
        assert ((dx.float() - cx.float()).abs() <= 2.0 ** -7 * cx.float().abs() + 2.0 ** -14 * rstd[:, None]
                * c.float().abs().amax()).all()
        assert ((dg - cg).abs() <= 2.0 ** -12 * (c.float() * ((c.float() - mean[:, None]) * rstd[:, None])).abs().sum(0)).all()
        torch.cuda.synchronize()
        del buf, s
    del x
    torch.cuda.synchronize()
    # an output of more than 2^31 elements
    R, K, Cout = 540000, 32, 4000
    _say("output past 2^31")
    x, W, b, _ = _layer(g, api, R, K, Cout, torch.bfloat16, False, False, True)
    out = api.linear_q8(x, W, b)
    torch.cuda.synchronize()
    rows = torch.tensor([0, 1, 268435, 536870, 536871, 539998, R - 1])
    _check_layer(x, W, b, None, False, out, rows=rows)
    y = api.layer_norm(out)
    torch.cuda.synchronize()
    assert torch.equal(y[rows], api.layer_norm(out[rows].contiguous()))


def test_leading_axes_and_empty_dimensions():
    api = _api()
    g = np.random.default_rng(1)
    x = _rows(g, 24, 64, torch.bfloat16).reshape(2, 3, 4, 64)
    y, mean, rstd = api.layer_norm(x, stats=True)
    assert y.shape == x.shape and mean.shape == (2, 3, 4)
    assert torch.equal(y.reshape(24, 64), api.layer_norm(x.reshape(24, 64)))
    wide = _rows(g, 24, 128, torch.bfloat16).reshape(2, 12, 128)[:, :, 32:96]
    assert torch.equal(api.layer_norm(wide), api.layer_norm(wide.contiguous()))
    q = api.quantize_rows(wide)
    assert q.q.shape == (2, 12, 64) and q.scale.shape == (2, 12)
    W = api.quantize_rows(_rows(g, 10, 64, torch.bfloat16))
    assert api.linear_q8(q, W).shape == (2, 12, 10)
    torch.cuda.synchronize()


def test_refusals():
    api = _api()
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        api.layer_norm(x, v[:63])
    with pytest.raises(ValueError):
        api.layer_norm(x, v.float())
    with pytest.raises(ValueError):
        api.layer_norm(x.cpu())
    with pytest.raises(ValueError):
        api.layer_norm(x.t())
    with pytest.raises(ValueError):
        api.layer_norm(torch.zeros((4, 6, 64), dtype=torch.bfloat16, device="cuda")[:, ::2][:, :, :32][::3, 1:])
    with pytest.raises(TypeError):
        api.layer_norm(x.half())
    with pytest.raises(api.GraphLeapError):
        api.layer_norm(x, eps=-1.0)
    with pytest.raises(api.GraphLeapError):
        api.layer_norm(x, eps=float("nan"))
    with pytest.raises(api.GraphLeapError):
        api.layer_norm(x[:0])
    with pytest.raises(api.GraphLeapError):
        api.layer_norm(x, out=x)
    m = torch.zeros(4, device="cuda")
    with pytest.raises(ValueError):
        api.layer_norm_backward(x[:3], x, m, m)
    with pytest.raises(ValueError):
        api.layer_norm_backward(x, x, m[:3], m)
    with pytest.raises(api.GraphLeapError):
        api.layer_norm_backward(x, x, m, m, need=(False, False, False))
    with pytest.raises(api.GraphLeapError) as e:
        y = torch.zeros((5000, 64), dtype=torch.bfloat16, device="cuda")
        api.layer_norm_backward(y, y, *2 * [torch.zeros(5000, device="cuda")], ws=api.Workspace(16, x.device))
    assert e.value.status == 9
    q = api.quantize_rows(x)
    with pytest.raises(ValueError):
        api.linear_q8(q, api.quantize_rows(x[:, :32]))
    with pytest.raises(ValueError):
        api.linear_q8(q, q, bias=v)
    with pytest.raises(ValueError):
        api.linear_q8(q, q, residual=x)
    with pytest.raises(ValueError):
        api.quantize_rows(x, out=api.quantize_rows(x[:, :32]))
    with pytest.raises(TypeError):
        api.linear_q8(q, q, dtype=torch.float16)


def test_other_stream_and_graph_replay():
    """The calls run where they are told to; recorded, they replay to the same bits."""
    api = _api()
    g = np.random.default_rng(4)
    R, C, H = 777, 192, 768
    x = _rows(g, R, C, torch.bfloat16)
    dy = _rows(g, R, C, torch.bfloat16)
    gamma, beta = _vec(g, C, torch.bfloat16, 1.0), _vec(g, C, torch.bfloat16)
    W = api.quantize_rows(_rows(g, H, C, torch.bfloat16))
    y, mean, rstd = api.layer_norm(x, gamma, beta, stats=True)

    def step(stream=None):
        n = api.layer_norm_q8(x, gamma, beta, stream=stream)
        h = api.linear_q8(n, W, act_out=api.GL_ACT_GELU, stream=stream)
        q = api.quantize_rows(h, stream=stream)
        grads = api.layer_norm_backward(dy, x, mean, rstd, gamma, stream=stream)
        return (n.q, n.scale, h, q.q, q.scale) + grads

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rec = step()
    for i in range(4):
        for t in rec:
            t.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(rec, want)), i
        assert all(torch.equal(a, b) for a, b in zip(step(), want)), i


def test_gradient_against_differences():
    """Differences of the forward pass in fp32, along random directions."""
    api = _api()
    g = np.random.default_rng(8)
    R, C = 5, 96
    x, dy = _rows(g, R, C, torch.float32), _rows(g, R, C, torch.float32)
    gamma, beta = _vec(g, C, torch.float32, 1.0), _vec(g, C, torch.float32)
    _, mean, rstd = api.layer_norm(x, gamma, beta, stats=True)
    dx, dg, db = api.layer_norm_backward(dy, x, mean, rstd, gamma)

    def loss(x, gamma, beta):
        return float((api.layer_norm(x, gamma, beta).double() * dy.double()).sum())

    for which, grad in enumerate((dx, dg, db)):
        args = [x.contiguous(), gamma, beta]
        v = torch.from_numpy(g.standard_normal(tuple(grad.shape))).float().cuda()
        step = 2.0 ** -9
        up, dn = list(args), list(args)
        up[which], dn[which] = args[which] + step * v, args[which] - step * v
        want = float((grad.double() * v.double()).sum())
        # the step's own rounding, fp32 of the outputs, and the third derivative
        near = float(dy.abs().double().sum())
        assert abs((loss(*up) - loss(*dn)) / (2 * step) - want) <= near * (16 * E32 / step + 4 * step ** 2), which


# one size for each of the layer's kernels: few rows, strips, tiles
@pytest.mark.parametrize("R,K,Cout", [(3, 100, 24), (1000, 100, 1000), (1000, 1000, 1000)])
def test_linear_q8_scales_whose_product_leaves_fp32(R, K, Cout):
    """The sum meets the row's scale first: a zero sum stays zero where the scales' product
    would overflow, and none of its bits are lost where that product would be subnormal."""
    api = _api()
    _say("linear_q8, scales", R, K, Cout)
    g = np.random.default_rng(R)
    x, W, b, _ = _layer(g, api, R, K, Cout, torch.float32, False, False, True)
    x.q[:, :K:2] = 0
    W.q[1::2, 1:K:2] = 0  # every other column's sums are zero
    x.scale.fill_(3e38)
    W.scale.fill_(1e6)
    out = api.linear_q8(x, W, b, dtype=torch.float32)
    gelu = api.linear_q8(x, W, act_out=api.GL_ACT_GELU, dtype=torch.float32)
    torch.cuda.synchronize()
    ref = x.q[:, :K].double() @ W.q[:, :K].double().t()
    assert (ref == 0).sum() >= R * (Cout // 2)
    assert torch.equal(out[ref == 0], b.expand(R, Cout)[ref == 0])
    assert not gelu[ref == 0].any()
    # scales of a product near 2^-140, sums of 2^19 and more: three roundings, as of any other scales
    x, W, _, _ = _layer(g, api, R, K, Cout, torch.float32, False, False, False)
    for t in (x.q, W.q):
        t[:, :K] = t[:, :K].clamp(min=-127).abs() | 64
    x.scale.mul_(2.0 ** -64)
    W.scale.mul_(2.0 ** -62)
    out = api.linear_q8(x, W, dtype=torch.float32)
    torch.cuda.synchronize()
    assert float(x.scale.max()) * float(W.scale.max()) < 2.0 ** -126
    ref = Q.linear_q8_ref(x.q[:, :K].cpu().numpy(), _f64(x.scale), W.q[:, :K].cpu().numpy(), _f64(W.scale))
    some = np.abs(ref) >= 2.0 ** -125
    assert some.mean() > 0.9
    assert (np.abs(_f64(out) - ref) <= 3 * E32 * np.abs(ref) + 2.0 ** -149)[some].all()


def _gelu_sweep(api, R, n, dtype):
    """The GELU of n arguments of -12.5 .. 12.5 and of some of either end, in R rows: sums
    and rows' scales of one, so that an argument is its channel's scale."""
    v = torch.linspace(-12.5, 12.5, n - 8, dtype=torch.float64).float()
    ends = torch.tensor([0.0, -0.0, 1e-30, -1e-30, -14.0, -40.0, 1e30, -1e30])
    v = torch.cat([v, ends]).cuda()
    one = torch.zeros((max(R, n), 16), dtype=torch.int8, device="cuda")
    one[:, 0] = 1
    x, W = api.Q8Rows(one[:R], torch.ones(R, device="cuda"), 1), api.Q8Rows(one[:n], v, 1)
    return v.double().cpu(), api.linear_q8(x, W, act_out=api.GL_ACT_GELU, dtype=dtype)


# few rows, strips, tiles
@pytest.mark.parametrize("R,n", [(3, 20011), (500, 2048), (600, 20011)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_gelu_over_its_range(dt, R, n):
    """Relative to x Phi(x), tail and all.  fp32: t 3 e, its polynomial 4 e and a fit of
    0.64 (1 + |x|) e, two products 2 e, the exponential 2 e, the sum e, and the exponent's
    rounding of 4 e relative to x^2 / 2; bf16: a fit within min(5.7e-7 e^(1.5 |x|), 2.8e-3)."""
    api = _api()
    _say("gelu", dt, R, n)
    v, out = _gelu_sweep(api, R, n, DT[dt])
    torch.cuda.synchronize()
    assert all(torch.equal(out[0], out[r]) for r in range(1, R))
    got = out[0].double().cpu()
    ref = 0.5 * v * torch.special.erfc(-v * 0.5 ** 0.5)
    a = v.abs()
    bound = (13 + a + 2 * a * a) * E32
    if dt == "bf16":
        bound = bound + torch.clamp(5.7e-7 * torch.exp(1.5 * a), max=2.8e-3) + U[DT[dt]]
    off = (got - ref).abs() / ref.abs().clamp(min=1e-300)
    mid = slice(0, n - 8)
    assert (off <= bound)[mid].all(), (v[mid][(off > bound)[mid]][:4], float((off / bound)[mid].max()))
    assert got[-8:].tolist()[:2] == [0.0, 0.0] and (got[-8:] - ref[-8:]).abs()[:4].max() <= 2e-32
    assert got[-4:-2].abs().max() <= 1e-36 and got[-1] == 0
    assert got[-2] == v[-2].to(DT[dt]).double()


# rows wider than the tiles: one group of rows, several with and without a rest, and more
# columns than one launch of the sums' kernel has threads for
@pytest.mark.parametrize("dt,R,C", [("bf16", 33, 16385), ("f32", 63, 8193), ("bf16", 64, 16391), ("f32", 300, 9001),
                                    ("bf16", 1001, 17000), ("bf16", 64, 2 ** 24 + 9)])
def test_gradient_of_wide_rows_in_groups(dt, R, C):
    api = _api()
    _say("gradient, wide rows", dt, R, C)
    g = torch.Generator(device="cuda").manual_seed(R)
    x, dy = (torch.randn(R, C, generator=g, device="cuda").to(DT[dt]) for _ in range(2))
    gamma = (1 + 0.3 * torch.randn(C, generator=g, device="cuda")).to(DT[dt])
    _, mean, rstd = api.layer_norm(x, gamma, stats=True)
    dx, dg, db = api.layer_norm_backward(dy, x, mean, rstd, gamma)
    only_g = api.layer_norm_backward(dy, x, mean, rstd, gamma, need=(False, True, False))[1]
    only_b = api.layer_norm_backward(dy, x, mean, rstd, gamma, need=(False, False, True))[2]
    torch.cuda.synchronize()
    assert torch.equal(dg, only_g) and torch.equal(db, only_b)
    n = (R / 16 + 259) * E32
    step = 2 ** 20
    for c in range(0, C, step):
        cols = slice(c, c + step)
        d = dy[:, cols].double()
        xh = (x[:, cols].double() - mean.double()[:, None]) * rstd.double()[:, None]
        assert ((dg[cols].double() - (d * xh).sum(0)).abs() <= n * (d * xh).abs().sum(0)).all(), c
        assert ((db[cols].double() - d.sum(0)).abs() <= n * d.abs().sum(0)).all(), c
    assert torch.isfinite(dx).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("C", [5, 77, 192, 1000, 1001, 2561, 6000, 20000, 65535])
def test_rows_of_one_value_are_beta(dt, C):
    """Values of eight bits: up to 2^16 of them add up exactly in fp32, the mean is their
    value, and nothing is left of the row but beta."""
    api = _api()
    _say("rows of one value", dt, C)
    vals = torch.tensor([3.0, -1000.0, 99840.0, 2.0 ** 60 * 1.9921875, 1.5 * 2.0 ** -60, 0.0], device="cuda")
    x = vals[:, None].expand(6, C).to(DT[dt]).contiguous()
    g = np.random.default_rng(C)
    gamma, beta = _vec(g, C, DT[dt], 1.0), _vec(g, C, DT[dt])
    y, mean, rstd = api.layer_norm(x, gamma, beta, stats=True)
    n, b = api.layer_norm_q8(x, gamma, beta), api.quantize_rows(beta)
    torch.cuda.synchronize()
    assert torch.equal(mean, vals)
    assert ((rstd - 1e-5 ** -0.5).abs() <= 4 * E32 * 1e-5 ** -0.5).all()
    assert torch.equal(y, beta.expand(6, C))
    assert (n.scale == b.scale).all() and (n.q[:, :C] - b.q[:C]).abs().max() <= 1
    # the mean of a row with an infinity is that infinity
    x[1, C // 2], x[2, 0] = float("inf"), float("-inf")
    y, mean, rstd = api.layer_norm(x, gamma, beta, stats=True)
    torch.cuda.synchronize()
    assert torch.isposinf(mean[1]) and torch.isneginf(mean[2]) and torch.isnan(y[1:3]).all()


@pytest.mark.parametrize("eps", [0.0, 1e-40])
@pytest.mark.parametrize("C,R", [(3, 4), (80, 4), (192, 4), (2560, 4), (20000, 4), (20, 16400), (120, 5000), (1001, 1000)])
def test_variances_below_the_normal_range(C, R, eps):
    """A subnormal variance with an eps as small has a root: squares and their sum are then
    off by 2^-150 each, 2^-148 of the variance altogether at most."""
    api = _api()
    _say("subnormal variances", C, R, eps)
    g = np.random.default_rng(C)
    size = np.resize([1e-17, 1e-18, 1e-19, 1e-20], (R, 1))
    x = torch.from_numpy(g.standard_normal((R, C)) * size).float().cuda()
    y, mean, rstd = api.layer_norm(x, eps=eps, stats=True)
    q = api.layer_norm_q8(x, eps=eps)
    torch.cuda.synchronize()
    xf = _f64(x)
    ry, rm, rr = Q.layer_norm_ref(xf, None, None, float(np.float32(eps)))
    low = 2.0 ** -148 * rr ** 2
    _within("rstd", _f64(rstd), rr, (80 + C / 256 + 8) * E32 * rr + low * rr
            + rr ** 3 * ((80 + C / 256) * E32 * np.abs(xf).mean(-1)) ** 2)
    _within("y", _f64(y), ry, _y_bound(xf, ry, rm, rr, None, None) + (low[:, None] + E32) * np.abs(ry))
    assert (q.q[:, :C].abs().amax(1) == 127).all() and torch.isfinite(q.scale).all()
