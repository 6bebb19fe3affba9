"""Gated blocks whose gates lie far below zero, where the activation is a small
part of its argument: accuracy relative to what comes out.

All gates of a block lie within a half of one bias.  A gate g is off by the
roundings of its sum of nine terms, 2^-24 of |g| + 1 each: D = 10 x 2^-24 (|g| + 1).
Both act and act' change there by a relative (|g| + 1) for one of g (GELU; SiLU by
1), so h, dg and du are off by (|g| + 1) D of themselves.  The activation's own
arithmetic: 2^-20 in float32; of bfloat16 networks, whose factors keep 16 bits, one
more 2^-16 of the exponential.  FP32 and the roundings are those of
test_gpu_gated.py, as 2-norms relative to the result's."""
import pytest
import torch

import block_ops_ref as ref
from test_gpu_gated import FP32, NAMES, TOL, Block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [4, 90, 600])      # few pixels; narrow ones; the backward's large tiles
@pytest.mark.parametrize("cin,hidden", [(8, 72), (8, 300)])
@pytest.mark.parametrize("act,far", [(1, -2.0), (1, -3.0), (1, -5.0), (1, -8.0), (1, -11.0), (0, -10.0), (0, -40.0)])
def test_far_below_zero(act, far, cin, hidden, rows, dt):
    b = Block(rows, cin, hidden, 24, dt, act)
    b.w[0].mul_(0.1)
    b.w[3].copy_(far + 0.05 * b.w[3])
    b.w[5].zero_()                       # y is what the hidden channels give
    D = 10 * 2.0 ** -24 * (abs(far) + 1.5)
    own = 2.0 ** -20 + (2.0 ** -16 if dt == "bf16" else 0.0) + D * (abs(far) + 1.5 if act else 1.0)
    x, dy, w = b.x.cpu(), b.dy.cpu(), b.host()
    e = ref.rel(b.forward(), ref.gated(x, w, act))
    assert e <= TOL[dt]["y"] + own, ("y", e, own)
    got, want = b.backward(), ref.gated(x, w, act, dy)
    for name, p, q in zip(("dx",) + NAMES, got, want):
        e = ref.rel(p, q)
        assert e <= TOL[dt]["dx" if name == "dx" else "b" if name.startswith("b_") else "w"] + own, (name, e, own)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("act", [0, 1])
def test_largest_gates(act, dt):
    """Gates whose square or exponential passes the largest float32 leave nothing (below zero) or themselves."""
    b = Block(70, 8, 72, 24, dt, act, bias=True)
    b.w[0].zero_()
    b.w[3].copy_(torch.where(torch.arange(72, device="cuda") % 2 == 0, -3e19, 3.0))
    x, w = b.x.cpu(), b.host()
    want, got = ref.gated(x, w, act), b.forward()
    assert bool(torch.isfinite(got).all()) and ref.rel(got, want) <= TOL[dt]["y"] + FP32
    assert all(bool(torch.isfinite(t).all()) for t in b.backward())
