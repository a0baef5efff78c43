"""Tunes the norms and biases of feed-forward blocks whose linears are frozen in MXFP4, so that they follow their 16-bit originals.

A block is  x + W2 gelu(W1 norm(x) + b1) + b2.  Its weights become 4-bit codes once; what is left to learn is a few vectors.  Forward: the layer norm
writes MXFP4 directly, the linear reads it and has the activation in its epilogue, the second linear quantises in the call and adds the skip connection.
Backward: gradients pass through the frozen codes, the activation and the norms down to the first block.  The output is also kept in 4 bits, as a skip connection of a UNet might be.

    python examples/tune_norms.py [--rows 4096] [--width 1280] [--hidden 5120] [--blocks 2] [--steps 100]
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2405_17873_amd as mq  # noqa: E402

EPS = 1e-5


class Block:
    def __init__(self, w1, b1, w2, b2, gain, shift):
        self.w1, self.w2 = mq.mx_quantize_weights(w1), mq.mx_quantize_weights(w2)
        self.learned = [t.float().clone() for t in (b1, b2, gain, shift)]  # masters in 32 bits

    def forward(self, x):
        b1, b2, gain, shift = self.learned
        n, mean, rstd = mq.layer_norm_mx(x, gain, shift, EPS, want_stats=True)
        h, a = mq.mx_linear(n, self.w1, b1.to(x.dtype), dtype=x.dtype, act="gelu", want_pre=True)
        y = mq.mx_linear(h, self.w2, b2.to(x.dtype), residual=x)
        self.saved = x, mean, rstd, a
        return y

    def backward(self, dy):
        """Gradient of the input; gradients of `learned` in their order."""
        x, mean, rstd, a = self.saved
        da, db1 = mq.act_grad(mq.mx_linear_grad(dy, self.w2), a, "gelu")
        dn = mq.mx_linear_grad(da, self.w1)
        dx, dgain, dshift = mq.layer_norm_grad(dn, x, self.learned[2], mean, rstd, residual=dy)
        return dx, [db1, dy.float().sum(0), dgain, dshift]


def original(x, w1, b1, w2, b2, gain, shift):
    n = F.layer_norm(x, x.shape[1:], gain, shift, EPS)
    return x + F.linear(F.gelu(F.linear(n, w1, b1)), w2, b2)


@torch.no_grad()
def tune(rows=4096, width=1280, hidden=5120, blocks=2, steps=100, rate=3e-3, seed=0, say=print):
    """Returns the losses: mean squared error against the originals, relative to what the originals add to the input."""
    g = torch.Generator().manual_seed(seed)

    def rand(*shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=g) * std + mean).to(torch.bfloat16).cuda()

    params = [(rand(hidden, width, std=width ** -0.5), rand(hidden, std=0.1), rand(width, hidden, std=hidden ** -0.5), rand(width, std=0.1),
               rand(width, std=0.2, mean=1.0), rand(width, std=0.1)) for _ in range(blocks)]
    model = [Block(*p) for p in params]
    learned = [t for b in model for t in b.learned]
    adam = torch.optim.Adam(learned, lr=rate)
    losses = []
    for step in range(steps):
        x = rand(rows, width)
        want = x
        for p in params:
            want = original(want, *p)
        y = x
        for b in model:
            y = b.forward(y)
        err, unit = y.float() - want.float(), (want - x).float().pow(2).mean()
        losses.append(float(err.pow(2).mean() / unit))
        dy = (err / (rows * unit)).to(x.dtype)
        for b in reversed(model):
            dy, grads = b.backward(dy)
            for t, d in zip(b.learned, grads):
                t.grad = d
        adam.step()
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step:4d}: error {losses[-1]:.4f} of what the blocks add", flush=True)
    kept = mq.mx_quantize(y)
    back = mq.mx_dequantize(kept, y.dtype)
    say(f"output kept in {kept.data.numel()} bytes, {y.numel() * 2} in 16 bits; relative error {float((back - y).float().norm() / y.float().norm()):.3f}", flush=True)
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("rows", 4096), ("width", 1280), ("hidden", 5120), ("blocks", 2), ("steps", 100)):
        ap.add_argument("--" + name, type=int, default=value)
    tune(**vars(ap.parse_args()))
