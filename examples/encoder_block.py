"""One training step of a transformer encoder block in a 1/e/m format: the quantized layers and products of this library with the
operators between them.

  x -> QKV layer -> attention -> output layer -> dropout, + x, norm -> feed-forward (two layers, ReLU) -> dropout, + , norm -> y

Every tensor that enters or leaves a layer is rounded to the format, sums inside are fp32; master weights and their gradients are fp32.

    python examples/encoder_block.py [--tokens 512 --batch 8 --hidden 1024 --inner 4096 --heads 16 --window 0 --sinks 0 --format 6 9]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2103_15940_amd as fmt  # noqa: E402


class EncoderBlock:
    """Weights of a block ([out, in], as torch's Linear has them) and its forward and backward pass."""

    def __init__(self, hidden, inner, heads, kv_heads=None, seed=0, device="cuda"):
        self.heads, self.kv_heads, self.dim = heads, kv_heads or heads, hidden // heads
        g = torch.Generator().manual_seed(seed)
        wide = (heads + 2 * self.kv_heads) * self.dim

        def matrix(out, inputs):
            return (torch.randn(out, inputs, generator=g) * inputs ** -0.5).to(device)

        def vector(n, value=0.0):
            return (value + 0.05 * torch.randn(n, generator=g)).to(device)

        self.weights = {"qkv": matrix(wide, hidden), "qkv_bias": vector(wide), "out": matrix(hidden, hidden), "out_bias": vector(hidden),
                        "up": matrix(inner, hidden), "up_bias": vector(inner), "down": matrix(hidden, inner), "down_bias": vector(hidden),
                        "gamma1": vector(hidden, 1.0), "beta1": vector(hidden), "gamma2": vector(hidden, 1.0), "beta2": vector(hidden)}

    def forward(self, x, f, rng, p=0.1, causal=False, window=0, sinks=0, k_lens=None):
        """x: [batch, tokens, hidden] fp32.  Returns y and what the backward pass needs."""
        w, (b, n, hidden) = self.weights, x.shape
        h, hk, d = self.heads, self.kv_heads, self.dim
        x2 = x.reshape(b * n, hidden)
        qkv = fmt.fmt_linear(x2, w["qkv"], w["qkv_bias"], f)
        parts = qkv.view(b, n, h + 2 * hk, d)
        how = dict(causal=causal, window=window, sinks=sinks, k_lens=k_lens)
        o, lse = fmt.fmt_attention_fwd(parts[:, :, :h], parts[:, :, h:h + hk], parts[:, :, h + hk:], f, **how)
        a = fmt.fmt_linear(o.view(b * n, h * d), w["out"], w["out_bias"], f)
        y1, z1, mean1, rstd1 = fmt.fmt_layernorm_fwd(a, w["gamma1"], w["beta1"], f, residual=x2, p=p, rng=rng, site=0)
        u = torch.relu(fmt.fmt_linear(y1, w["up"], w["up_bias"], f))
        m = fmt.fmt_linear(u, w["down"], w["down_bias"], f)
        y2, z2, mean2, rstd2 = fmt.fmt_layernorm_fwd(m, w["gamma2"], w["beta2"], f, residual=y1, p=p, rng=rng, site=1)
        kept = dict(x2=x2, parts=parts, o=o, lse=lse, how=how, y1=y1, z1=z1, mean1=mean1, rstd1=rstd1, u=u, z2=z2, mean2=mean2, rstd2=rstd2,
                    rng=rng, p=p, shape=x.shape)
        return y2.view(b, n, hidden), kept

    def backward(self, dy, kept, f):
        """Gradients of the input and of every weight."""
        w, k, (b, n, hidden) = self.weights, kept, kept["shape"]
        h, hk, d = self.heads, self.kv_heads, self.dim
        g = {}

        def layer(name, gradient, inputs):            # of a fully connected layer: dX, and dW and db into g
            g[name] = fmt.fmt_gemm(gradient, inputs, f, transA=True)
            g[name + "_bias"] = gradient.sum(0)
            return fmt.fmt_quantize(fmt.fmt_gemm(gradient, w[name], f), f)

        dz2, dm, g["gamma2"], g["beta2"] = fmt.fmt_layernorm_bwd(dy.reshape(b * n, hidden), k["z2"], k["mean2"], k["rstd2"], w["gamma2"], f,
                                                                 p=k["p"], rng=k["rng"], site=1)
        du = layer("down", dm, k["u"]) * (k["u"] > 0)
        dy1 = dz2 + layer("up", du, k["y1"])
        dz1, da, g["gamma1"], g["beta1"] = fmt.fmt_layernorm_bwd(dy1, k["z1"], k["mean1"], k["rstd1"], w["gamma1"], f, p=k["p"], rng=k["rng"], site=0)
        do = layer("out", da, k["o"].view(b * n, h * d)).view(b, n, h, d)
        parts = k["parts"]
        grads = fmt.fmt_attention_bwd(do, parts[:, :, :h], parts[:, :, h:h + hk], parts[:, :, h + hk:], k["o"], k["lse"], f, **k["how"])
        dqkv = torch.cat(grads, 2).view(b * n, (h + 2 * hk) * d)
        dx = dz1 + layer("qkv", dqkv, k["x2"])
        return dx.view(b, n, hidden), g


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 512), ("batch", 8), ("hidden", 1024), ("inner", 4096), ("heads", 16), ("window", 0), ("sinks", 0), ("steps", 5)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--format", type=int, nargs=2, default=(6, 9))
    a = ap.parse_args()
    f = (*a.format, True)
    block, rng = EncoderBlock(a.hidden, a.inner, a.heads), fmt.new_rng(1)
    x, target = (torch.randn(a.batch, a.tokens, a.hidden, device="cuda") for _ in range(2))
    for step in range(a.steps):
        torch.cuda.synchronize()
        began = time.perf_counter()
        y, kept = block.forward(x, f, rng, causal=a.window > 0, window=a.window, sinks=a.sinks)
        dy = (y - target) * (2.0 / y.numel()) * 1024.0                      # loss scale 1024
        _, grads = block.backward(dy, kept, f)
        for name, grad in grads.items():
            block.weights[name] -= 2.0 / 1024.0 * grad
        rng[1] += 1
        torch.cuda.synchronize()
        print("step %d: loss %.4f, %.2f ms" % (step, float((y - target).square().mean()), (time.perf_counter() - began) * 1e3), flush=True)


if __name__ == "__main__":
    main()
