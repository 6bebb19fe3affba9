"""Results of a bfloat16 gated block value by value: each is the definition's value
rounded once, but for what its terms are off by.

A float32 sum of K terms is off by at most 7 sqrt(K) 2^-24 of the terms' 2-norm
(roundings of either sign: a chance of 10^-10 a value), and so are errors of the
terms themselves, of which each has its bound:
  dg, du, dh   sums of cin and cout products of bfloat16s
  h = act(g) u       |act'(g) u| of g's, |act(g)| of u's, 2^-16 of itself for its two
                     bfloat16 parts, 2^-18 for the activation's arithmetic
  dg = dh u act'(g)  the same of its three factors, |act''| at most 1, and act' off by
                     2^-22 (1 + |g|)
The result's own rounding: 2^-8 of it."""
import pytest
import torch

import block_ops_ref as ref
from gpu_util import say
from test_gpu_gated import NAMES, Block

pytestmark = pytest.mark.gpu
U, SURE = 2.0 ** -24, 7.0


def _sum(a, b, off=None):
    """Terms' 2-norm of a @ b."""
    return ((a * a) @ (b * b)).sqrt()


def _bounds(b):
    """y, dx and how far float32 sums and factors of two bfloat16 parts may be from them before the last rounding."""
    x, dy = b.x.cpu().double(), b.dy.cpu().double()
    wg, wu, wd, bg, bu, bd = (None if t is None else t.double() for t in b.host())
    zero = torch.zeros((), dtype=torch.float64)
    bg, bu, bd = (zero if t is None else t for t in (bg, bu, bd))
    g, u, dh = x @ wg.T + bg, x @ wu.T + bu, dy @ wd
    a, slope = ref.act(g, b.act)
    eg, eu = (SURE * U * (b.cin + 1) ** 0.5 * (_sum(x, w.T) + v.abs()) for w, v in ((wg, bg), (wu, bu)))
    ed = SURE * U * b.cout ** 0.5 * _sum(dy, wd)
    own = 2.0 ** -16 + 2.0 ** -18
    h = a * u
    eh = (slope * u).abs() * eg + a.abs() * eu + own * h.abs()
    y, ey = h @ wd.T + bd, SURE * (_sum(eh, wd.T) + U * (b.hidden + 1) ** 0.5 * (_sum(h, wd.T) + bd.abs()))
    dg, du = dh * u * slope, dh * a
    eg = (u * slope).abs() * ed + (dh * slope).abs() * eu + (dh * u).abs() * (eg + 4 * U * (1 + g.abs())) + own * dg.abs()
    eu = a.abs() * ed + (dh * slope).abs() * (SURE * U * (b.cin + 1) ** 0.5 * (_sum(x, wg.T) + bg.abs())) + own * du.abs()
    dx, ex = dg @ wg + du @ wu, SURE * ((_sum(eg, wg) ** 2 + _sum(eu, wu) ** 2).sqrt() +
                                        U * (2 * b.hidden) ** 0.5 * (_sum(dg, wg) ** 2 + _sum(du, wu) ** 2).sqrt())
    return y, ey, dx, ex


def _once(got, want, off, what):
    d = (got.cpu().double() - want).abs()
    worst = float((d / (2.0 ** -8 * want.abs() + 1.01 * off + 1e-30)).max())
    assert worst <= 1, (what, worst)


def _check(rows, cin, hidden, cout, forward=True, backward=False, **kw):
    say("gated, one rounding", rows, cin, hidden, cout)
    b = Block(rows, cin, hidden, cout, "bf16", kw.pop("act", (rows + cin + hidden) % 2), **kw)
    y, ey, dx, ex = _bounds(b)
    if forward:
        _once(b.forward(), y, ey, "y")
    if backward:
        _once(b.backward()[0], dx, ex, "dx")
        _once(b.backward(want=(False,) * 6)[0], dx, ex, "dx alone")


@pytest.mark.parametrize("rows,cin,hidden,cout", [(1, 300, 40, 64), (1, 260, 1000, 512), (3, 64, 300, 64), (32, 257, 65, 33),
                                                  (33, 64, 1031, 300), (64, 320, 72, 24)])
def test_few_pixels(rows, cin, hidden, cout):
    _check(rows, cin, hidden, cout)


# every pair of widths that one launch of few channels is made for, hidden channels of several tiles and an odd end
@pytest.mark.parametrize("cout", [40, 64, 72, 128, 136, 250, 256])
@pytest.mark.parametrize("cin", [24, 64, 72, 128, 129, 192, 200, 256])
def test_narrow(cin, cout):
    _check(70, cin, 520, cout)
    _check(203, cin, 1031 - 2 * cin, cout)


@pytest.mark.parametrize("cout", [24, 64, 65, 128])
@pytest.mark.parametrize("cin", [24, 64, 65, 128])
@pytest.mark.parametrize("hidden", [256, 270, 520])
def test_narrow_float32(cin, cout, hidden):
    """The same of a float32 network, by test_gpu_gated.py's bounds."""
    Block(131, cin, hidden, cout, "fp32", (cin + hidden) % 2).check()


# small tiles, a split sum, large tiles with one and with several a compute unit
@pytest.mark.parametrize("rows,cin,hidden,cout", [(65, 257, 40, 24), (300, 264, 200, 72), (150, 300, 1500, 264), (2100, 264, 520, 2048),
                                                  (4200, 264, 1100, 1100)])
def test_wide(rows, cin, hidden, cout):
    _check(rows, cin, hidden, cout)


# on both sides of where one launch takes it
@pytest.mark.parametrize("rows", [1, 33, 64, 100, 3000])
@pytest.mark.parametrize("cin,hidden,cout", [(64, 256, 64), (24, 72, 40), (33, 250, 61), (64, 129, 1), (1, 65, 64),
                                             (64, 64, 64), (64, 257, 64), (65, 256, 64), (64, 256, 65)])
def test_narrow_backward(rows, cin, hidden, cout):
    _check(rows, cin, hidden, cout, forward=False, backward=True)


@pytest.mark.parametrize("rows,cin,hidden,cout", [(3, 8, 16, 8), (65, 257, 40, 24), (300, 264, 200, 72), (150, 300, 1500, 264),
                                                  (1100, 2048, 264, 264), (2100, 2048, 264, 40), (4200, 1100, 520, 136)])
def test_backward(rows, cin, hidden, cout):
    _check(rows, cin, hidden, cout, forward=False, backward=True)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("rows,cin,hidden,cout", [(16, 16, 72, 16), (40, 8, 200, 24), (70, 12, 256, 9),       # one launch
                                                  (16, 16, 300, 16), (33, 8, 24, 8), (300, 16, 300, 8)])     # tile products
def test_weights_gradients(rows, cin, hidden, cout, act):
    """Float32 sums of factors with 24 bits: off by sqrt(K) 2^-24 of their norm for the sum over the pixels, for g and
    u and for dh, and by 8 x 2^-24 for the activation's arithmetic."""
    say("gated, weights' gradients", rows, cin, hidden, cout, act)
    b = Block(rows, cin, hidden, cout, "bf16", act)
    tol = U * (rows ** 0.5 + 2 * cin ** 0.5 + cout ** 0.5 + 8)
    want = ref.gated(b.x.cpu(), b.host(), act, b.dy.cpu())
    for name, p, q in zip(NAMES, b.backward()[1:], want[1:]):
        assert ref.rel(p, q) <= tol, (name, ref.rel(p, q), tol)
