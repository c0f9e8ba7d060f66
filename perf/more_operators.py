"""The operators that train a gated FFN, as they are timed and checked.

gated          a gated fully connected layer, act(x Wg^T + bg) (x Wu^T + bu), with or
               without the products that its backward pass takes
gated_grad     its backward pass: the input's, the weight's and the bias's gradients
linear_grad    the backward pass of a plain fully connected layer
residual       the end of a block: its output is normalised (or not), scaled by channel
               and by a gate for each image or row, added to the features that went by
               it, and the sum normalised for the next block
residual_grad  its backward pass: the gradients of both streams, of the gates, of the
               scale and of both norms' weights

`run` computes them with elementary torch operations in 32 bits where `own` is
false, and calls `paper_2604_21290_amd.api` where it is true.

listed()          the fixed cases
draw(rng)         one more case of the same ranges
prepare(case, s)  inputs, weights and what a forward pass has kept
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
# the most that a drawn case of each kind costs: multiplications of one of the products
# (a backward pass has two), elements of a row operator
MOST_PRODUCT = {"bf16": 16384 * 2048 * 4096, "fp32": 16384 * 512 * 2048}
MOST_ROWS = 32768 * 2560


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _gated(kind, R, K, F, dtype="bf16", act="silu", bias=True, keep=True):
    """R rows, K -> F channels through 2 F products; keep: return those too (training)."""
    return dict(kind=kind, R=R, K=K, F=F, dtype=dtype, act=act, bias=bias, keep=keep)


def _linear(R, K, Cout, dtype="bf16"):
    return dict(kind="linear_grad", R=R, K=K, Cout=Cout, dtype=dtype)


def _residual(kind, R, C, dtype="bf16", post=True, rms=False, scale=True, gate=0, gap=0, keep=True):
    """R rows of C channels, `gap` elements apart in memory.  post: the block's output is
    normalised first; rms: by its mean square alone; gate: rows to a gate (0: none);
    keep: return the rows' statistics too (training)."""
    return dict(kind=kind, R=R, C=C, dtype=dtype, post=post, rms=rms, scale=scale, gate=gate, gap=gap, keep=keep)


def listed():
    return [
        # a single row through the gated FFN of ViG-B being served: the weights' bytes
        dict(_gated("gated", 1, 640, 2560, keep=False), name="gated_one_row"),
        # the FFN of ViG-B on its batch of 64, in training: the matrix cores
        dict(_gated("gated", 12544, 640, 2560, act="gelu"), name="gated_vig_b"),
        # an odd layer in fp32, whose rows are no whole vectors
        dict(_gated("gated", 777, 501, 333, "fp32", act="gelu", keep=False), name="gated_odd_fp32"),
        # the FFN of ViG-Ti on its batch of 32: short products, many launches' worth of latency
        dict(_gated("gated_grad", 6272, 192, 768, act="gelu"), name="gated_grad_vig_ti"),
        # a large generic layer: the most work of all
        dict(_gated("gated_grad", 16384, 2048, 4096, bias=False), name="gated_grad_large"),
        # the FFN's second layer of ViG-B: its weight's gradient sums 12544 rows for few outputs
        dict(_linear(12544, 2560, 640), name="linear_grad_vig_b_ffn2"),
        # odd sizes throughout, as a classifier's head has them
        dict(_linear(3001, 1001, 333), name="linear_grad_odd"),
        # one image of ViG-Ti in fp32 being served: all launch and latency
        dict(_residual("residual", 196, 192, "fp32", post=False, keep=False), name="residual_one_image_fp32"),
        # wide rows of a large batch, both norms and a gate for each image: all memory
        dict(_residual("residual", 32768, 2560, gate=256), name="residual_wide"),
        # one image's gradients in fp32, a gate for each row
        dict(_residual("residual_grad", 196, 192, "fp32", gate=1), name="residual_grad_one_image_fp32"),
        # the first pyramid stage's batch with stochastic depth: sums over 100352 narrow rows
        dict(_residual("residual_grad", 100352, 80, post=False, gate=3136), name="residual_grad_pyr_s1"),
        # wide rows between two norms by the mean square
        dict(_residual("residual_grad", 32768, 2560, rms=True), name="residual_grad_wide_rms"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["gated", "gated_grad", "linear_grad", "residual", "residual_grad"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    while True:
        if kind.startswith("residual"):
            R, C = _log_int(rng, 1, 131072), _log_int(rng, 8, 8192)
            if rng.random() < 0.5:  # whole vectors, as most widths are
                C = max(8, C // 8 * 8)
            if R * C > MOST_ROWS:
                continue
            images = _log_int(rng, 1, 64)
            gate = rng.choice([0, 1, images])
            R = R if gate < 2 else max(1, R // gate) * gate
            return _residual(kind, R, C, dtype, rng.random() < 0.6, rng.random() < 0.5, rng.random() < 0.6, gate,
                             rng.choice([0, 0, 0, rng.randrange(1, 65)]), kind == "residual_grad" or rng.random() < 0.5)
        R, K, F = _log_int(rng, 1, 32768), _log_int(rng, 16, 4096), _log_int(rng, 8, 8192)
        if rng.random() < 0.6:
            K, F = K // 16 * 16, max(8, F // 8 * 8)
        if R * K * F > MOST_PRODUCT[dtype]:
            continue
        if kind == "linear_grad":
            return _linear(R, K, F, dtype)
        return _gated(kind, R, K, F, dtype, rng.choice(["silu", "gelu"]), rng.random() < 0.5,
                      kind == "gated_grad" or rng.random() < 0.5)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _features(g, R, C, dtype, gap=0, size=1.0):
    """Rows as a block meets them: every channel has its own spread and offset (a few
    much larger than the rest), every row its own size."""
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    spread = torch.exp(0.5 * n(C))
    x = (n(R, C) * spread + 0.5 * n(C)) * torch.exp(0.3 * n(R, 1)) * size
    wide = torch.zeros(R, C + gap, dtype=DTYPE[dtype], device="cuda")
    wide[:, :C] = x.to(DTYPE[dtype])
    return wide[:, :C]


def _vector(g, n, dtype, about=0.0, spread=0.1):
    return (about + spread * torch.randn(n, generator=g, device="cuda")).to(DTYPE[dtype])


def _weight(g, Cout, K, dtype):
    """Uniform, of the size that keeps the features' size through a layer."""
    return ((2 * torch.rand(Cout, K, generator=g, device="cuda") - 1) * math.sqrt(3.0 / K)).to(DTYPE[dtype])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, R, dtype = case, case["R"], case["dtype"]
    s = dict(case=case)
    if c["kind"] == "linear_grad":
        s["x"], s["W"] = _features(g, R, c["K"], dtype), _weight(g, c["Cout"], c["K"], dtype)
        s["dy"] = _features(g, R, c["Cout"], dtype, size=0.1)
        return s
    if c["kind"].startswith("gated"):
        K, F = c["K"], c["F"]
        # normalised features, the gate's weight rows before the other product's
        s["x"], s["W"] = _features(g, R, K, dtype, size=0.7), _weight(g, 2 * F, K, dtype)
        s["bias"] = _vector(g, 2 * F, dtype) if c["bias"] else None
        if c["kind"] == "gated_grad":  # as the forward pass kept them
            pre = s["x"].float() @ s["W"].float().t()
            s["pre"] = (pre if s["bias"] is None else pre + s["bias"].float()).to(DTYPE[dtype])
            s["dh"] = _features(g, R, F, dtype, size=0.1)
        return s
    C = c["C"]
    s["b"] = _features(g, R, C, dtype, c["gap"])
    s["post"] = None
    if c["post"]:
        s["post"] = (_vector(g, C, dtype, 1.0, 0.2), None if c["rms"] else _vector(g, C, dtype))
    s["norm"] = (_vector(g, C, dtype, 1.0, 0.2), None if c["rms"] else _vector(g, C, dtype))
    s["scale"] = _vector(g, C, dtype, 0.3, 0.1) if c["scale"] else None
    # of a gate for each image some are shut (stochastic depth); one for each row is a router's
    s["gate"] = None
    if c["gate"]:
        u = torch.rand(R // c["gate"], generator=g, device="cuda")
        s["gate"] = u.clamp_min(0.01) if c["gate"] == 1 else (u < 0.8).float() / 0.8
    x = _features(g, R, C, dtype, c["gap"])
    if c["kind"] == "residual":
        s["x"] = x
        return s
    # as the forward pass kept them
    v, _, s["mean_b"], s["rstd_b"], s["mean_s"], s["rstd_s"] = _plain_join(dict(s, x=x))
    s["s"] = v.to(DTYPE[dtype])
    s["ds"], s["dy"] = (_features(g, R, C, dtype, size=0.1) for _ in range(2))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _plain_norm(x, w, rms):
    mean = None if rms else x.mean(1)
    d = x if rms else x - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).mean(1) + EPS)
    y = d * rstd[:, None] * w[0].float()
    return y if w[1] is None else y + w[1].float(), mean, rstd


def _plain_factor(s, R):
    """Gate times scale, and the gate alone, by row."""
    c = s["case"]
    gate = torch.ones(R, 1, device="cuda") if s["gate"] is None else s["gate"].repeat_interleave(c["gate"])[:, None]
    return gate * s["scale"].float() if s["scale"] is not None else gate, gate


def _plain_join(s):
    """The sum, its norm and the statistics, in 32 bits."""
    c = s["case"]
    b, mb, rb = s["b"].float(), None, None
    if s["post"] is not None:
        b, mb, rb = _plain_norm(b, s["post"], c["rms"])
    v = s["x"].float() + _plain_factor(s, b.shape[0])[0] * b
    y, ms, rs = _plain_norm(v, s["norm"], c["rms"])
    return v, y, mb, rb, ms, rs


def _plain_norm_grad(dy, x, mean, rstd, w):
    xhat = (x if mean is None else x - mean[:, None]) * rstd[:, None]
    h = dy * w.float()
    d = h - xhat * (h * xhat).mean(1, keepdim=True)
    return (d if mean is None else d - h.mean(1, keepdim=True)) * rstd[:, None], xhat


def _plain_residual_grad(s):
    c, out = s["case"], {}
    dy, b = s["dy"].float(), s["b"].float()
    dv, xs = _plain_norm_grad(dy, s["s"].float(), s["mean_s"], s["rstd_s"], s["norm"][0])
    dv = dv + s["ds"].float()
    out["dx"] = dv
    factor, gate = _plain_factor(s, b.shape[0])
    dn, n = dv * factor, b
    if s["post"] is not None:
        db, xb = _plain_norm_grad(dn, b, s["mean_b"], s["rstd_b"], s["post"][0])
        n = xb * s["post"][0].float()
        n = n if s["post"][1] is None else n + s["post"][1].float()
        out["dpost"] = (dn * xb).sum(0)
        if s["post"][1] is not None:
            out["dpost_bias"] = dn.sum(0)
    else:
        db = dn
    out["db"] = db
    if s["scale"] is not None:
        out["dscale"] = (dv * gate * n).sum(0)
    if s["gate"] is not None:
        rows = (dv * n * s["scale"].float() if s["scale"] is not None else dv * n).sum(1)
        out["dgate"] = rows.view(-1, c["gate"]).sum(1)
    out["dnorm"] = (dy * xs).sum(0)
    if s["norm"][1] is not None:
        out["dnorm_bias"] = dy.sum(0)
    return {k: v.to(s["b"].dtype) if k in ("dx", "db") else v for k, v in out.items()}


def _plain(s):
    c = s["case"]
    dt = DTYPE[c["dtype"]]
    if c["kind"] == "residual_grad":
        return _plain_residual_grad(s)
    if c["kind"] == "residual":
        v, y, mb, rb, ms, rs = _plain_join(s)
        out = {"s": v.to(dt), "y": y.to(dt)}
        if c["keep"]:
            out |= {k: t for k, t in (("mean_b", mb), ("rstd_b", rb), ("mean_s", ms), ("rstd_s", rs)) if t is not None}
        return out
    if c["kind"] == "linear_grad":
        dy, x, W = s["dy"].float(), s["x"].float(), s["W"].float()
        return {"dx": (dy @ W).to(dt), "dW": (dy.t() @ x).to(dt), "dbias": dy.sum(0)}
    x, W = s["x"].float(), s["W"].float()
    if c["kind"] == "gated":
        pre = x @ W.t()
        pre = pre if s["bias"] is None else pre + s["bias"].float()
    else:
        pre = s["pre"].float()
    p, u = pre[:, :c["F"]], pre[:, c["F"]:]
    if c["act"] == "silu":
        sig = 1 / (1 + torch.exp(-p))
        a, da = p * sig, sig * (1 + p * (1 - sig))
    else:
        cdf = 0.5 * torch.special.erfc(p * -0.5 ** 0.5)
        a, da = p * cdf, cdf + p * torch.exp(-0.5 * p * p) * (2 * math.pi) ** -0.5
    if c["kind"] == "gated":
        h = (a * u).to(dt)
        return {"h": h, "pre": pre.to(dt)} if c["keep"] else {"h": h}
    dh = s["dh"].float()
    dpre = torch.cat([dh * u * da, dh * a], 1)
    out = {"dx": (dpre @ W).to(dt), "dW": (dpre.t() @ x).to(dt)}
    return out | {"dbias": dpre.sum(0)} if c["bias"] else out


def _own(s):
    from paper_2604_21290_amd import api
    c = s["case"]
    if c["kind"] == "linear_grad":
        dx, dW, dbias = api.linear_backward(s["dy"], s["x"], s["W"])
        return {"dx": dx, "dW": dW, "dbias": dbias}
    if c["kind"].startswith("gated"):
        act = api.GL_ACT_SILU if c["act"] == "silu" else api.GL_ACT_GELU
        if c["kind"] == "gated":
            if not c["keep"]:
                return {"h": api.gated_linear(s["x"], s["W"], s["bias"], act=act)}
            h, pre = api.gated_linear(s["x"], s["W"], s["bias"], act=act, keep=True)
            return {"h": h, "pre": pre}
        dx, dW, dbias = api.gated_linear_backward(s["dh"], s["x"], s["W"], s["pre"], act=act, need=(True, True, c["bias"]))
        return {"dx": dx, "dW": dW, "dbias": dbias} if c["bias"] else {"dx": dx, "dW": dW}
    # a gate for each image: the rows as [images, rows, C]
    rows = (lambda t: t) if c["gate"] < 2 else lambda t: t.unflatten(0, (-1, c["gate"]))
    flat = (lambda t: t) if c["gate"] < 2 else lambda t: t.flatten(0, 1)
    how = dict(post=s["post"], scale=s["scale"], gate=s["gate"], norm=s["norm"],
               kind=api.GL_NORM_RMS if c["rms"] else api.GL_NORM_LAYER)
    if c["kind"] == "residual":
        if not c["keep"]:
            v, y = api.residual_norm(rows(s["x"]), rows(s["b"]), eps=EPS, **how)
            return {"s": flat(v), "y": flat(y)}
        v, y, kept = api.residual_norm(rows(s["x"]), rows(s["b"]), eps=EPS, stats=True, **how)
        out = {"s": flat(v), "y": flat(y)}
        return out | {k: flat(t) for k, t in zip(("mean_b", "rstd_b", "mean_s", "rstd_s"), kept) if t is not None}
    kept = [None if s[k] is None else rows(s[k]) for k in ("mean_b", "rstd_b", "mean_s", "rstd_s")]
    d = api.residual_norm_backward(rows(s["ds"]), rows(s["dy"]), rows(s["b"]), rows(s["s"]), kept, **how)
    out = {"dx": flat(d.dx), "db": flat(d.db), "dscale": d.dscale, "dgate": d.dgate, "dnorm": d.dnorm[0],
           "dnorm_bias": d.dnorm[1]}
    if d.dpost is not None:
        out |= {"dpost": d.dpost[0], "dpost_bias": d.dpost[1]}
    return {k: t for k, t in out.items() if t is not None}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c, R = case, case["R"]
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "linear_grad":
        K, N = c["K"], c["Cout"]
        return {"bytes": es * (R * N + 2 * R * K + 2 * N * K) + 4 * N, "flops": 4 * R * N * K}
    if c["kind"].startswith("gated"):
        K, F = c["K"], c["F"]
        if c["kind"] == "gated":
            b = es * (R * K + 2 * F * K + R * F + (2 * F if c["bias"] else 0) + (2 * R * F if c["keep"] else 0))
            return {"bytes": b, "flops": 4 * R * F * K}
        return {"bytes": es * (3 * R * F + 2 * R * K + 4 * F * K) + (8 * F if c["bias"] else 0), "flops": 8 * R * F * K}
    C, gates = c["C"], 4 * (R // c["gate"]) if c["gate"] else 0
    stats = 4 * R * (1 if c["rms"] else 2) * (2 if c["post"] else 1)
    vectors = C * ((1 if c["rms"] else 2) * (2 if c["post"] else 1) + (1 if c["scale"] else 0))
    if c["kind"] == "residual":
        return {"bytes": es * (4 * R * C + vectors) + gates + (stats if c["keep"] else 0), "flops": (16 if c["post"] else 9) * R * C}
    return {"bytes": es * (6 * R * C + vectors) + 2 * gates + stats + 4 * vectors, "flops": (30 if c["post"] else 18) * R * C}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _exact_act(name, p):
    """An activation and its derivative."""
    if name == "silu":
        sig = torch.sigmoid(p)
        return p * sig, sig + p * sig * torch.sigmoid(-p)
    cdf = torch.special.ndtr(p)
    return p * cdf, cdf + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    s, c = prepare(case, seed), case
    d = lambda t: None if t is None else t.to(torch.float64)  # noqa: E731
    if c["kind"] == "linear_grad":
        dy = d(s["dy"])
        return {"dx": torch.mm(dy, d(s["W"])), "dW": torch.mm(dy.t().contiguous(), d(s["x"])), "dbias": dy.sum(0)}
    if c["kind"].startswith("gated"):
        x, W, F = d(s["x"]), d(s["W"]), c["F"]
        if c["kind"] == "gated":
            pre = torch.mm(x, W.t().contiguous())
            if c["bias"]:
                pre += d(s["bias"])
            h = _exact_act(c["act"], pre[:, :F])[0] * pre[:, F:]
            return {"h": h, "pre": pre} if c["keep"] else {"h": h}
        g, u = d(s["pre"]).split(F, dim=1)
        a, da = _exact_act(c["act"], g)
        dh = d(s["dh"])
        dg, du = dh * u * da, dh * a
        out = {"dx": torch.mm(dg, W[:F]) + torch.mm(du, W[F:]),
               "dW": torch.cat([torch.mm(t.t().contiguous(), x) for t in (dg, du)])}
        return out | {"dbias": torch.cat([dg.sum(0), du.sum(0)])} if c["bias"] else out
    n, R = c["C"], c["R"]
    post, norm = s["post"], s["norm"]
    b = d(s["b"])
    gate = torch.ones(R, dtype=torch.float64, device="cuda")
    if c["gate"]:
        gate = d(s["gate"]).unsqueeze(1).expand(-1, c["gate"]).reshape(-1)
    scale = d(s["scale"]) if c["scale"] else torch.ones(n, dtype=torch.float64, device="cuda")
    shift = lambda w: 0.0 if w[1] is None else d(w[1])  # noqa: E731

    def stats(t):
        mu = torch.zeros(R, dtype=torch.float64, device="cuda") if c["rms"] else t.sum(1) / n
        return mu, (((t - mu.unsqueeze(1)) ** 2).sum(1) / n + EPS) ** -0.5

    if c["kind"] == "residual":
        out = {}
        if post is not None:
            mu, inv = stats(b)
            out |= {"rstd_b": inv} if c["rms"] else {"mean_b": mu, "rstd_b": inv}
            b = (b - mu.unsqueeze(1)) * inv.unsqueeze(1) * d(post[0]) + shift(post)
        v = torch.addcmul(d(s["x"]), b * scale, gate.unsqueeze(1))
        mu, inv = stats(v)
        out |= {"rstd_s": inv} if c["rms"] else {"mean_s": mu, "rstd_s": inv}
        y = (v - mu.unsqueeze(1)) * inv.unsqueeze(1) * d(norm[0]) + shift(norm)
        return {"s": v, "y": y} | (out if c["keep"] else {})

    # with the statistics that the call is given
    def back(dy, t, mean, rstd, w):
        r = d(rstd).unsqueeze(1)
        z = t * r if mean is None else (t - d(mean).unsqueeze(1)) * r
        u = dy * d(w)
        du = u - z * ((u * z).sum(1) / n).unsqueeze(1)
        if mean is not None:
            du -= (u.sum(1) / n).unsqueeze(1)
        return du * r, z

    dy = d(s["dy"])
    dv, z = back(dy, d(s["s"]), s["mean_s"], s["rstd_s"], norm[0])
    dv += d(s["ds"])
    out = {"dx": dv, "dnorm": (dy * z).sum(0)}
    if norm[1] is not None:
        out["dnorm_bias"] = dy.sum(0)
    dn, v = dv * gate.unsqueeze(1) * scale, b
    out["db"] = dn
    if post is not None:
        out["db"], z = back(dn, b, s["mean_b"], s["rstd_b"], post[0])
        out["dpost"] = (dn * z).sum(0)
        if post[1] is not None:
            out["dpost_bias"] = dn.sum(0)
        v = z * d(post[0]) + shift(post)
    if c["scale"]:
        out["dscale"] = (dv * v * gate.unsqueeze(1)).sum(0)
    if c["gate"]:
        out["dgate"] = (dv * v * scale).sum(1).view(-1, c["gate"]).sum(1)
    return out
