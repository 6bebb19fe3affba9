"""The norms around a residual block at widths that no kernel of the largest number
of vectors holds in registers, read a value or two at a time: against the 64-bit
definition, with guard values around every tensor, to the tolerances of
test_gpu_residual_norm.py (a row's sums are chains of 32 additions in float64 or
float32 and a tree)."""
import pytest

from test_gpu_residual_norm import Run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("c,ld,off", [(4095, 0, 0), (4096, 4097, 1), (4097, 0, 0), (4098, 0, 0), (5000, 5001, 0),
                                      (5001, 0, 0), (6144, 6145, 1), (8190, 8190, 1), (8191, 0, 0), (8192, 8193, 1),
                                      (8193, 0, 0)])
def test_widths_read_a_value_at_a_time(c, ld, off, post, dt):
    Run(6, c, dt, (0, 1, 3)[c % 3], post, ld=ld, off=off).check()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("rows,c,group", [(300, 4104, 100), (260, 9000, 130), (90, 4097, 1), (90, 5001, 0), (1100, 4104, 2),
                                          (1026, 4101, 513)])
def test_wide_rows_of_shared_gates(rows, c, group, post, dt):
    """Gates whose pixels several blocks take, and more gates than blocks."""
    Run(rows, c, dt, group, post).check()


@pytest.mark.parametrize("rows,group", [(6000, 6000), (9000, 4500), (7000, 0)])
def test_sums_of_one_sign_over_many_wide_rows(rows, group):
    """Gradients of a gate and a scale over thousands of pixels whose terms are alike, so that what a sum leaves out
    adds up: chains of 64 additions at most, 64 x 2^-24 of the terms' magnitudes, and three roundings of a term."""
    c = 4097
    a = Run(rows, c, "fp32", group, post=False)
    a.dout.fill_(0.1)
    a.f.fill_(0.3)
    out, _, st = a.forward(z=None)
    got = a.backward(out, st, dz=False)
    term = a.dout[0].double() * a.f[0].double()
    sc = a.vec["scale"].double()
    q = rows if a.gate is None else group * a.gate.double().sum(0)
    assert float((got["scale"].double() - term * q).abs().max()) <= 67 * 2.0 ** -24 * float((term * q).abs().max())
    if group:
        want = group * sc * term
        assert float(((got["dgate"].double() - want).abs() / want).max()) <= 67 * 2.0 ** -24
