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
