"""What the gated block's workspace is for: copies, and what lies between launches."""
import pytest

import paper_2004_09910_amd as tgp


def _up(v, m):
    return -(-v // m) * m


@pytest.mark.parametrize("dtype,parts", [(tgp.BF16, 1), (tgp.FP32, 3)])
@pytest.mark.parametrize("rows,cin,hidden,cout", [(147456, 64, 256, 64), (5000, 100, 1000, 72), (12544, 128, 512, 33)])
def test_one_launch_keeps_copies_alone(rows, cin, hidden, cout, dtype, parts):
    s = tgp.gated_shape(cin, hidden, cout, dtype, 0)
    w = 2 * hidden * _up(cin, 8) + cout * _up(hidden, 8)
    assert tgp.gated_workspace(s, rows, False) <= 2 * parts * (w + rows * _up(cin, 8)) + 8 * 256


@pytest.mark.parametrize("dtype", [tgp.BF16, tgp.FP32])
@pytest.mark.parametrize("rows", [1, 32, 33, 64])
def test_few_pixels_keep_their_hidden_channels_alone(rows, dtype):
    s = tgp.gated_shape(1024, 4097, 1024, dtype, 0)
    assert tgp.gated_workspace(s, rows, False) <= 4 * (32 if rows <= 32 else 64) * 4112 + 256


def test_narrow_backward_keeps_copies_and_ranges():
    """Of 4194374 pixels: copies of x and dy at most, and 256 ranges of the gradients' sums."""
    s = tgp.gated_shape(64, 256, 64, tgp.BF16, 0)
    sums = 3 * 64 * 256 + 2 * 256 + 64
    assert tgp.gated_workspace(s, 1 << 22, True) <= 2 * (1 << 22) * 128 + 2 * 3 * 64 * 256 + 4 * 256 * sums + 12 * 256
