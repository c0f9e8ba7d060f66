"""A ViG block's FFN behind a layer norm, on 8-bit integers, and the tuning of its norm.

    python examples/ffn_q8.py [workload] [steps]

The block's FFN (Y = GELU(N W_1^T + b_1) W_2^T + b_2 + X, N the layer norm of X) runs in
bf16 and on 8-bit rows, where each activation row and each output channel of a weight
has a scale of its own:

    layer_norm_q8 -> linear_q8 (GELU) -> quantize_rows -> linear_q8 (+ X)

Then the norm alone, 2 C numbers, is tuned behind 8-bit weights that stay as they are:
starting from ones and zeros, its weight and bias are fitted to what the first bf16 layer
gives with a norm of its own.  The difference's gradient goes back through the layer as
if it had not been rounded, and through layer_norm_backward.
Weights and features are random (paper_2604_21290_amd.inputs); needs a GPU.
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_21290_amd import api, inputs  # noqa: E402


def to_gpu(s: inputs.Stored) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(s.value)).float().cuda()


class FfnQ8:
    """The FFN's weights in bf16 and in 8 bits, and its norm."""

    def __init__(self, params: dict):
        self.W1, self.b1, self.W2, self.b2 = (to_gpu(params[n]).bfloat16() for n in ("W_1", "b_1", "W_2", "b_2"))
        C = self.W1.shape[1]
        g = torch.Generator().manual_seed(C)
        self.gamma = (1 + 0.3 * torch.randn(C, generator=g)).cuda().bfloat16()
        self.beta = (0.2 * torch.randn(C, generator=g)).cuda().bfloat16()
        self.W1q, self.W2q = api.quantize_rows(self.W1), api.quantize_rows(self.W2)

    def bf16(self, x):
        h = api.linear(api.layer_norm(x, self.gamma, self.beta), self.W1, self.b1, act_out=api.GL_ACT_GELU)
        return api.linear(h, self.W2, self.b2, residual=x)

    def q8(self, x):
        n = api.layer_norm_q8(x, self.gamma, self.beta)
        h = api.linear_q8(n, self.W1q, self.b1, act_out=api.GL_ACT_GELU)
        return api.linear_q8(api.quantize_rows(h), self.W2q, self.b2, residual=x)


def tune_norm(x, target, Wq: api.Q8Rows, b, steps: int, rate: float = 0.05):
    """Fit a norm's weight and bias so that the 8-bit layer Wq, b on x [R, C] gives
    `target` (all float32): Adam's steps on the mean square of the difference.
    Returns (gamma, beta, the difference's size before each step and after the last)."""
    p = [torch.ones(x.shape[1], device=x.device), torch.zeros(x.shape[1], device=x.device)]
    m, v = [torch.zeros_like(t) for t in p], [torch.zeros_like(t) for t in p]
    back = Wq.dequantize().t().contiguous()  # the gradient's weights: [C, Cout]
    _, mean, rstd = api.layer_norm(x, stats=True)
    ws = api.layer_norm_backward_workspace(x)
    sizes = []
    for t in range(steps + 1):
        diff = api.linear_q8(api.layer_norm_q8(x, *p), Wq, b, dtype=torch.float32) - target
        sizes.append(float(diff.norm() / target.norm()))
        if t == steps:
            return p[0], p[1], sizes
        dy = api.linear(diff * (2.0 / diff.numel()), back)
        _, *grads = api.layer_norm_backward(dy, x, mean, rstd, p[0], need=(False, True, True), ws=ws)
        step = rate * (1 - t / steps)
        for i, g in enumerate(grads):
            m[i] = 0.9 * m[i] + 0.1 * g
            v[i] = 0.99 * v[i] + 0.01 * g * g
            p[i] = p[i] - step * (m[i] / (1 - 0.9 ** (t + 1))) / ((v[i] / (1 - 0.99 ** (t + 1))).sqrt() + 1e-20)


def main(name: str = "vig_ti", steps: int = 100) -> dict:
    w = inputs.WORKLOADS[name]
    ffn = FfnQ8(inputs.make_vig_params(w, 0))
    x = to_gpu(inputs.make_features(w)).bfloat16() * w.C ** 0.5  # rows of unit variance
    y, yq = ffn.bf16(x), ffn.q8(x)
    rel = float((yq.float() - y.float()).norm() / (y.float() - x.float()).norm())
    print(f"{name}: [{w.B}, {w.N}, {w.C}], the 8-bit FFN is {rel:.4f} of its output away from bf16's")
    rows = x.reshape(-1, w.C)
    target = api.linear(api.layer_norm(rows, ffn.gamma, ffn.beta), ffn.W1, ffn.b1).float()
    *_, sizes = tune_norm(rows.float(), target, ffn.W1q, ffn.b1.float(), steps)
    print(f"first layer with a plain norm: {sizes[0]:.4f} away, after {steps} steps on its weight and bias "
          f"{sizes[-1]:.4f}")
    return {"ffn": rel, "sizes": sizes}


if __name__ == "__main__":
    main(*(sys.argv[1:2] or ["vig_ti"]), *[int(a) for a in sys.argv[2:3]])
