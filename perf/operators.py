"""The normalisation and 8-bit operators of this package, as they are timed and checked.

norm        layer norm over the channels, with or without the rows' statistics
norm_grad   its backward pass: the input's gradient, and the weight's and the
            bias's, summed over all rows
linear_q8   a fully connected layer on rows that are already 8-bit integers with
            a scale each, against weights with a scale for each output channel
layer_q8    the same layer as a block runs it, from the features: each row is
            normalised (or not), brought to 8 bits and multiplied

`run` computes them with elementary torch operations in 32 bits where `own` is
false, and calls `paper_2604_21290_amd.api` where it is true.

listed()          the fixed cases
draw(rng)         one more case of the same ranges
prepare(case, s)  inputs, statistics and 8-bit weights of a case
run(state)        one pass; returns the outputs
work(case)        bytes and operations one pass cannot do without
exact(case, s)    the same outputs in float64, from the definitions
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
# the most that a drawn case of each kind costs: elements of a row operator,
# multiplications of a matrix product
MOST_ROWS = 32768 * 2560
MOST_PRODUCT = 16384 * 4096 * 4096


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _rows(kind, R, C, dtype="bf16", gap=0, stats=True):
    """R rows of C channels, `gap` elements apart in memory (a slice of wider rows)."""
    return dict(kind=kind, R=R, C=C, dtype=dtype, gap=gap, stats=stats)


def _layer(kind, R, K, Cout, dtype="bf16", gelu=False, residual=False, norm=False):
    """R rows, K -> Cout channels; `dtype` is that of bias, residual and output.
    Features that are normalised come in `dtype` too, and then the output is bf16:
    it has what 8 bits of a norm leave."""
    return dict(kind=kind, R=R, K=K, Cout=Cout, dtype=dtype, gelu=gelu, residual=residual, norm=norm)


def listed():
    return [
        # one image of ViG-Ti being served in fp32: all launch and latency
        dict(_rows("norm", 196, 192, "fp32", stats=False), name="norm_one_image_fp32"),
        # the first pyramid stage's batch: very many rows, narrower than a wave's load
        dict(_rows("norm", 100352, 80), name="norm_pyr_s1"),
        # wide rows of a large batch: the largest norm, all memory
        dict(_rows("norm", 32768, 2560, stats=False), name="norm_wide"),
        # the gradients of one image's norm in fp32, as in a calibration step
        dict(_rows("norm_grad", 196, 192, "fp32"), name="norm_grad_one_image_fp32"),
        # the first pyramid stage's batch: a sum over 100352 rows for each weight
        dict(_rows("norm_grad", 100352, 80), name="norm_grad_pyr_s1"),
        # odd rows out of wider ones, which no vector load fits
        dict(_rows("norm_grad", 8193, 1001, gap=7), name="norm_grad_odd_slice"),
        # a single row through the FFN's first layer of ViG-B: the weights' bytes
        dict(_layer("linear_q8", 1, 640, 2560, gelu=True), name="linear_q8_one_row"),
        # the FFN's second layer of ViG-B on its batch of 64, with the residual
        dict(_layer("linear_q8", 12544, 2560, 640, residual=True), name="linear_q8_vig_b_ffn2"),
        # a large generic product: the matrix cores
        dict(_layer("linear_q8", 16384, 4096, 4096), name="linear_q8_large"),
        # the norm and the FFN's first layer of ViG-Ti on its batch of 32
        dict(_layer("layer_q8", 6272, 192, 768, gelu=True, norm=True), name="layer_q8_vig_ti_ffn1"),
        # the FFN's second layer of the first pyramid stage: many rows, few columns
        dict(_layer("layer_q8", 100352, 320, 80, residual=True), name="layer_q8_pyr_s1_ffn2"),
        # an odd layer in fp32, without a norm
        dict(_layer("layer_q8", 777, 1001, 333, "fp32"), name="layer_q8_odd_fp32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "linear_q8", "layer_q8"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    while True:
        if kind in ("norm", "norm_grad"):
            R, C = _log_int(rng, 1, 131072), _log_int(rng, 8, 8192)
            if rng.random() < 0.5:  # whole vectors, as most widths are
                C = max(8, C // 8 * 8)
            gap = rng.choice([0, 0, 0, rng.randrange(1, 65)])
            if R * C <= MOST_ROWS:
                return _rows(kind, R, C, dtype, gap, kind == "norm_grad" or rng.random() < 0.5)
            continue
        big = kind == "linear_q8"
        R, K, Cout = _log_int(rng, 1, 16384 if big else 100352), _log_int(rng, 16, 8192 if big else 4096), \
            _log_int(rng, 8, 8192 if big else 4096)
        if rng.random() < 0.5:
            K, Cout = K // 16 * 16, Cout // 8 * 8
        norm = not big and rng.random() < 0.5
        if R * max(K, Cout) <= MOST_ROWS and R * K * Cout <= MOST_PRODUCT:
            return _layer(kind, R, K, Cout, dtype, rng.random() < 0.4, rng.random() < 0.4, norm)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _features(g, R, C, dtype, gap=0):
    """Rows as a block's norm meets them: every channel has its own spread and
    offset (a few much larger than the rest), every row its own size."""
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    spread = torch.exp(0.5 * n(C))
    x = (n(R, C) * spread + 0.5 * n(C)) * torch.exp(0.3 * n(R, 1))
    wide = torch.zeros(R, C + gap, dtype=DTYPE[dtype], device="cuda")
    wide[:, :C] = x.to(DTYPE[dtype])
    return wide[:, :C]


def _vector(g, n, dtype, about=0.0, spread=0.1):
    return (about + spread * torch.randn(n, generator=g, device="cuda")).to(DTYPE[dtype])


def _stored_q8(x):
    """x [R, K] as 8-bit rows of whole 16 bytes (zeros at their ends), and the scales."""
    R, K = x.shape
    top = x.abs().amax(1, keepdim=True)
    q = torch.zeros(R, (K + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    q[:, :K] = torch.where(top > 0, torch.round(x * 127 / top), torch.zeros_like(x)).to(torch.int8)
    return q, (top / 127).flatten()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, dtype = case, case["dtype"]
    s = dict(case=case)
    if c["kind"] in ("norm", "norm_grad"):
        s["x"] = _features(g, c["R"], c["C"], dtype, c["gap"])
        s["gamma"], s["beta"] = _vector(g, c["C"], dtype, 1.0, 0.2), _vector(g, c["C"], dtype)
        if c["kind"] == "norm_grad":
            s["dy"] = _features(g, c["R"], c["C"], dtype, c["gap"])
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
        return s
    R, K, Cout = c["R"], c["K"], c["Cout"]
    # weights: Kaiming-uniform, brought to 8 bits once
    W = (2 * torch.rand(Cout, K, generator=g, device="cuda") - 1) * math.sqrt(6.0 / K)
    s["Wq"], s["Ws"] = _stored_q8(W)
    s["bias"] = _vector(g, Cout, dtype if not c["norm"] else "bf16")
    out = "bf16" if c["norm"] else dtype
    s["residual"] = _features(g, R, Cout, out) if c["residual"] else None
    x = _features(g, R, K, dtype)
    if c["kind"] == "layer_q8" and not c["norm"]:  # the hidden layer of an FFN: after its GELU
        x = (0.5 * x.float() * (1 + torch.erf(x.float() * 0.5 ** 0.5))).to(DTYPE[dtype])
    if c["norm"]:
        s["gamma"], s["beta"] = _vector(g, K, dtype, 1.0, 0.2), _vector(g, K, dtype)
    if c["kind"] == "linear_q8":
        s["xq"], s["xs"] = _stored_q8(x.float())
    else:
        s["x"] = x
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _plain_norm(x, gamma, beta):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    return d * rstd * gamma.float() + beta.float(), mean.flatten(), rstd.flatten()


def _plain_layer(q, xs, s):
    c = s["case"]
    y = q @ s["Wq"][:, :c["K"]].float().t()
    y = y * (xs[:, None] * s["Ws"]) + s["bias"].float()
    if c["gelu"]:
        y = 0.5 * y * (1 + torch.erf(y * 0.5 ** 0.5))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["bias"].dtype)


def _plain(s):
    c = s["case"]
    if c["kind"] == "norm":
        y, mean, rstd = _plain_norm(s["x"], s["gamma"], s["beta"])
        y = y.to(s["x"].dtype)
        return {"y": y, "mean": mean, "rstd": rstd} if c["stats"] else {"y": y}
    if c["kind"] == "norm_grad":
        dy = s["dy"].float()
        xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        h = dy * s["gamma"].float()
        dx = s["rstd"][:, None] * (h - h.mean(1, keepdim=True) - xhat * (h * xhat).mean(1, keepdim=True))
        return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}
    if c["kind"] == "linear_q8":
        return _plain_layer(s["xq"][:, :c["K"]].float(), s["xs"], s)
    h = _plain_norm(s["x"], s["gamma"], s["beta"])[0] if c["norm"] else s["x"].float()
    top = h.abs().amax(1, keepdim=True)
    q = torch.where(top > 0, torch.round(h * 127 / top), torch.zeros_like(h))
    return _plain_layer(q, (top / 127).flatten(), s)


def _own(s):
    from paper_2604_21290_amd import api
    c = s["case"]
    if c["kind"] == "norm":
        if not c["stats"]:
            return {"y": api.layer_norm(s["x"], s["gamma"], s["beta"], EPS)}
        y, mean, rstd = api.layer_norm(s["x"], s["gamma"], s["beta"], EPS, stats=True)
        return {"y": y, "mean": mean, "rstd": rstd}
    if c["kind"] == "norm_grad":
        dx, dgamma, dbeta = api.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    W = api.Q8Rows(s["Wq"], s["Ws"], c["K"])
    if c["kind"] == "linear_q8":
        x = api.Q8Rows(s["xq"], s["xs"], c["K"])
    elif c["norm"]:
        x = api.layer_norm_q8(s["x"], s["gamma"], s["beta"], EPS)
    else:
        x = api.quantize_rows(s["x"])
    return api.linear_q8(x, W, s["bias"], act_out=api.GL_ACT_GELU if c["gelu"] else api.GL_ACT_NONE,
                         residual=s["residual"], dtype=s["bias"].dtype)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    R = c["R"]
    if c["kind"] == "norm":
        C = c["C"]
        return {"bytes": 2 * R * C * es + 2 * C * es + (8 * R if c["stats"] else 0), "flops": 8 * R * C}
    if c["kind"] == "norm_grad":
        C = c["C"]
        return {"bytes": 3 * R * C * es + 8 * R + C * es + 8 * C, "flops": 14 * R * C}
    K, Cout = c["K"], c["Cout"]
    os = 2 if c["norm"] else es
    b = Cout * K + 4 * Cout + os * Cout + (2 if c["residual"] else 1) * R * Cout * os
    b += R * (K + 4) if c["kind"] == "linear_q8" else R * K * es + (2 * K * es if c["norm"] else 0)
    return {"bytes": b, "flops": 2 * R * K * Cout}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s, c = prepare(case, seed), case
    d = lambda t: t.to(torch.float64)  # noqa: E731
    norm = c["kind"] in ("norm", "norm_grad") or c["norm"]
    if norm:
        x, gamma, beta = d(s["x"]), d(s["gamma"]), d(s["beta"])
        n = x.shape[1]
        mu = x.sum(1) / n
        var = ((x - mu.unsqueeze(1)) ** 2).sum(1) / n
        inv = (var + EPS) ** -0.5
    if c["kind"] == "norm_grad":
        # with the statistics that the call is given
        mu, inv = d(s["mean"]), d(s["rstd"])
        dy = d(s["dy"])
        z = torch.addcmul((-mu * inv).unsqueeze(1), x, inv.unsqueeze(1))
        u = dy * gamma
        a, b = u.sum(1) / n, (u * z).sum(1) / n
        return {"dx": (u - a.unsqueeze(1) - z * b.unsqueeze(1)) * inv.unsqueeze(1),
                "dgamma": (dy * z).sum(0), "dbeta": dy.sum(0)}
    if norm:
        y = gamma * ((x - mu.unsqueeze(1)) * inv.unsqueeze(1)) + beta
        if c["kind"] == "norm":
            return {"y": y, "mean": mu, "rstd": inv} if c["stats"] else {"y": y}
    elif c["kind"] == "layer_q8":
        y = d(s["x"])
    if c["kind"] == "linear_q8":
        q, scale = d(s["xq"][:, :c["K"]]), d(s["xs"])
    else:
        scale = y.abs().max(1).values / 127
        q = torch.round(y / torch.where(scale > 0, scale, torch.ones_like(scale)).unsqueeze(1))
    # one row block at a time: sums of products of whole numbers, exact in 64 bits
    W, parts = d(s["Wq"][:, :c["K"]]).t().contiguous(), []
    for r in range(0, c["R"], 8192):
        parts.append(torch.mm(q[r:r + 8192].contiguous(), W))
    y = torch.cat(parts) * scale.unsqueeze(1) * d(s["Ws"]).unsqueeze(0) + d(s["bias"])
    if c["gelu"]:
        y = y * torch.special.ndtr(y)
    return y + d(s["residual"]) if s["residual"] is not None else y
