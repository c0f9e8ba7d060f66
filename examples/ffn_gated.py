"""A gated FFN between two norms, trained in place of a ViG block's FFN.

    python examples/ffn_gated.py [workload] [steps]

    N = norm(X);  Z = act(N Wg^T + bg) * (N Wu^T + bu);  O = Z Wd^T + bd
    S = X + gate scale norm(O);  Y = norm(S)

The block's forward pass is four calls (layer_norm, gated_linear, linear, residual_norm)
and its backward pass four more; `GatedFfn` is one torch.autograd.Function around them, so
that the rest of a program is plain torch.  It is fitted to what the block's own FFN
(GELU, inputs.make_vig_params) gives on the same features, with stochastic depth: each
image's gate is shut in one step of ten.
Weights and features are random (paper_2604_21290_amd.inputs); needs a GPU.
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_21290_amd import api, inputs  # noqa: E402

NAMES = ("gamma", "beta", "W", "bias", "Wd", "bd", "post_gamma", "post_beta", "scale", "next_gamma", "next_beta")


def to_gpu(s: inputs.Stored) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(s.value)).float().cuda()


class GatedFfn(torch.autograd.Function):
    """(S, Y) of x [images, N, C], gate [images] (float32) and the weights in the order of
    NAMES, W [2F, C] the gate's rows before the other product's."""

    @staticmethod
    def forward(ctx, x, gate, *w):
        gamma, beta, W, bias, Wd, bd, pg, pb, scale, ng, nb = w
        n, mean, rstd = api.layer_norm(x, gamma, beta, stats=True)
        z, pre = api.gated_linear(n, W, bias, act=api.GL_ACT_SILU, keep=True)
        o = api.linear(z, Wd, bd)
        s, y, kept = api.residual_norm(x, o, post=(pg, pb), scale=scale, gate=gate, norm=(ng, nb), stats=True)
        ctx.save_for_backward(x, gate, n, mean, rstd, z, pre, o, s, *kept, *w)
        return s, y

    @staticmethod
    @once_differentiable  # the calls' results are detached
    def backward(ctx, ds, dy):
        x, gate, n, mean, rstd, z, pre, o, s, *rest = ctx.saved_tensors
        kept, (gamma, beta, W, bias, Wd, bd, pg, pb, scale, ng, nb) = rest[:4], rest[4:]
        g = api.residual_norm_backward(ds.contiguous(), dy.contiguous(), o, s, kept, post=(pg, pb), scale=scale, gate=gate,
                                       norm=(ng, nb))
        dz, dWd, dbd = api.linear_backward(g.db, z, Wd)
        dn, dW, dbias = api.gated_linear_backward(dz, n, W, pre, act=api.GL_ACT_SILU)
        dx, dgamma, dbeta = api.layer_norm_backward(dn, x, mean, rstd, gamma)
        grads = (dgamma, dbeta, dW, dbias, dWd, dbd, *g.dpost, g.dscale, *g.dnorm)
        return dx + g.dx, g.dgate, *(d.to(x.dtype) for d in grads)


def make_weights(C: int, F: int, dtype=torch.bfloat16, seed: int = 0) -> dict:
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    w = dict(gamma=torch.ones(C), beta=torch.zeros(C), W=n(2 * F, C) * C ** -0.5, bias=torch.zeros(2 * F),
             Wd=n(C, F) * F ** -0.5, bd=torch.zeros(C), post_gamma=torch.ones(C), post_beta=torch.zeros(C),
             scale=torch.full((C,), 0.5), next_gamma=torch.ones(C), next_beta=torch.zeros(C))
    return {k: t.to(dtype).cuda() for k, t in w.items()}


def main(name: str = "vig_ti", steps: int = 60) -> dict:
    wl = inputs.WORKLOADS[name]
    p = inputs.make_vig_params(wl, 0)
    W1, b1, W2, b2 = (to_gpu(p[k]).bfloat16() for k in ("W_1", "b_1", "W_2", "b_2"))
    x = to_gpu(inputs.make_features(wl)).bfloat16() * wl.C ** 0.5  # rows of unit variance
    target = api.linear(api.linear(x, W1, b1, act_out=api.GL_ACT_GELU), W2, b2, residual=x).float()
    # float32 copies that the steps are added to; the layers run in bf16
    weights = make_weights(wl.C, 2 * wl.C)
    master = {k: t.float().requires_grad_() for k, t in weights.items()}
    opt = torch.optim.Adam(master.values(), lr=2e-3)
    g = torch.Generator(device="cuda").manual_seed(1)
    sizes = []
    for _ in range(steps):
        shut = torch.rand(wl.B, generator=g, device="cuda") < 0.1
        gate = torch.where(shut, 0.0, 1.0)
        s, _ = GatedFfn.apply(x, gate, *(master[k].bfloat16() for k in NAMES))
        open_ = ~shut
        diff = (s.float() - target)[open_]
        loss = diff.square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        sizes.append(float(diff.detach().norm() / (target - x.float())[open_].norm()))
    print(f"{name}: [{wl.B}, {wl.N}, {wl.C}], the gated FFN is {sizes[0]:.3f} of the FFN's output away from it, "
          f"{sizes[-1]:.3f} after {steps} steps")
    return {"sizes": sizes}


if __name__ == "__main__":
    main(*(sys.argv[1:2] or ["vig_ti"]), *[int(a) for a in sys.argv[2:3]])
