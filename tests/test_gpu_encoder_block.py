"""The encoder block of examples/encoder_block.py: its gradients against automatic differentiation of the same block in 64 bits.

In 1/7/15 every rounding is within 2^-16 of its value; the chain from any weight to its gradient passes at most 24 of them
(forward and backward), and products average them.  32 * 2^-16 of a gradient's norm leaves room for their correlations."""
import os
import sys

import pytest

import layerdef as L

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import encoder_block
    finally:
        sys.path.pop(0)
    return encoder_block


def reference(block, x, dy, rng, p, seen):
    w = {k: v.detach().cpu().double().requires_grad_() for k, v in block.weights.items()}
    x = x.cpu().double().requires_grad_()
    b, n, hidden = x.shape
    h, hk, d = block.heads, block.kv_heads, block.dim
    seed, step = (int(v) for v in rng.tolist())
    masks = []
    for site in (0, 1):
        kept, factor = L.drop_mask(b * n, hidden, p, seed, step, site)
        masks.append(torch.from_numpy(kept).double().view(b, n, hidden) * float(factor))
    norm = lambda z, g, c: torch.nn.functional.layer_norm(z, (hidden,), g, c, 1e-5)  # noqa: E731
    q, k, v = torch.split((x @ w["qkv"].t() + w["qkv_bias"]).view(b, n, h + 2 * hk, d).transpose(1, 2), (h, hk, hk), 1)
    k, v = (t.repeat_interleave(h // hk, 1) for t in (k, v))
    s = (q @ k.transpose(2, 3) * d ** -0.5).masked_fill(~seen, -float("inf"))
    o = (torch.softmax(s, 3) @ v).transpose(1, 2).reshape(b, n, h * d)
    y1 = norm(x + masks[0] * (o @ w["out"].t() + w["out_bias"]), w["gamma1"], w["beta1"])
    y2 = norm(y1 + masks[1] * (torch.relu(y1 @ w["up"].t() + w["up_bias"]) @ w["down"].t() + w["down_bias"]), w["gamma2"], w["beta2"])
    y2.backward(dy.cpu().double())
    return y2.detach(), x.grad, {k: t.grad for k, t in w.items()}


@pytest.mark.parametrize("causal,window,sinks,kv_heads", [(False, 0, 0, 4), (True, 9, 2, 2)])
def test_step_against_automatic_differentiation(example, causal, window, sinks, kv_heads):
    fmt = example.fmt
    f = (7, 15, True)
    block = example.EncoderBlock(96, 160, 4, kv_heads)
    rng = fmt.new_rng(77, 3)
    x, dy = torch.randn(2, 37, 96, device="cuda"), torch.randn(2, 37, 96, device="cuda")
    y, kept = block.forward(x, f, rng, p=0.2, causal=causal, window=window, sinks=sinks)
    dx, grads = block.backward(dy, kept, f)
    seen = torch.from_numpy(L.visible(37, 37, 37, 0, causal, window, sinks))
    want_y, want_dx, want = reference(block, x, dy, rng, 0.2, seen)
    got = {"y": (y, want_y), "dx": (dx, want_dx)} | {k: (grads[k], want[k]) for k in want}
    for name, (a, b) in got.items():
        assert float((a.cpu().double() - b).norm() / b.norm()) <= 32 * 2.0 ** -16, name


def test_training_lowers_the_loss(example):
    fmt = example.fmt
    f = (6, 9, True)
    block, rng = example.EncoderBlock(128, 256, 2), fmt.new_rng(1)
    x, target = torch.randn(4, 64, 128, device="cuda"), torch.randn(4, 64, 128, device="cuda")
    losses = []
    for _ in range(8):
        y, kept = block.forward(x, f, rng, p=0.0)
        losses.append(float((y - target).square().mean()))
        _, grads = block.backward((y - target) * (2.0 / y.numel()) * 1024.0, kept, f)
        for name, grad in grads.items():
            block.weights[name] -= 4.0 / 1024.0 * grad            # 20 diverges in 64 bits too
    assert losses[-1] < 0.98 * losses[0], losses
