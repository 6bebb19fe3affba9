"""Trains a small normalised convolution pipeline on a synthetic task: the
target is a fixed random convolution of the input, so the loss can fall.

    python examples/train_norm_stack.py [--steps 30] [--fp32] [--micro-batches 4]

Every forward, backward, norm and update runs in libtgp.so; see
paper_2004_09910_amd/training.py for how they are put together.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2004_09910_amd.training import NormPipeline  # noqa: E402
from workloads.specs import (BF16, CKPT_EXCEPT_LAST, CONV1X1, CONV3X3, DWCONV3X3, FP32, Layer,  # noqa: E402
                             Net)


def network(c=64, hw=32):
    """Three partitions: 3x3 stem, a depthwise / pointwise cell, a linear 3x3 head."""
    layers = (Layer(CONV3X3, 16, c), Layer(CONV3X3, c, c),
              Layer(DWCONV3X3, c, c, relu=False, bias=False), Layer(CONV1X1, c, 2 * c),
              Layer(CONV1X1, 2 * c, c), Layer(CONV3X3, c, 16, relu=False))
    return Net("norm-stack", layers, 16, hw, hw)


def train(steps=30, dtype=BF16, batch=16, m=4, log=print):
    net = network()
    sess = NormPipeline(net, dtype, n=3, balance=[2, 2, 2])
    sess.plan(batch, m, CKPT_EXCEPT_LAST)
    g = torch.Generator(device="cuda").manual_seed(0)
    kernel = torch.randn(16, 16, 3, 3, device="cuda", generator=g) / 12
    losses = []
    for k in range(steps):
        x = torch.randn(batch, 16, 32, 32, device="cuda", generator=g)
        t = torch.nn.functional.conv2d(x, kernel, padding=1)
        dt = torch.bfloat16 if dtype == BF16 else torch.float32
        x, t = (v.permute(0, 2, 3, 1).to(dt).contiguous() for v in (x, t))
        losses.append(sess.train_step(x, t).item())
        if log and (k % 5 == 0 or k + 1 == steps):
            log(f"step {k:3d}  loss {losses[-1]:.4f}")
    sess.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--micro-batches", type=int, default=4)
    ap.add_argument("--fp32", action="store_true")
    a = ap.parse_args()
    train(a.steps, FP32 if a.fp32 else BF16, m=a.micro_batches)
