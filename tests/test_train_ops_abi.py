"""Refusals of the layer norm, update and step calls: every check runs on the
host, so these need no GPU (addresses are never read)."""
import ctypes

import pytest

import paper_2004_09910_amd as tgp

P = 1 << 20          # an aligned address that nothing reads


def _fwd(**kw):
    a = dict(rows=4, C=8, dtype=tgp.BF16, x=P, ldx=8, gain=P, bias=P, eps=1e-5, y=P, ldy=8, stats=P)
    a.update(kw)
    return tgp.call_status("tgp_layer_norm_forward", a["rows"], a["C"], a["dtype"], a["x"], a["ldx"],
                           a["gain"], a["bias"], a["eps"], a["y"], a["ldy"], a["stats"], None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(C=0), dict(dtype=2), dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7),
    dict(x=P + 1), dict(y=P + 1), dict(gain=P + 2), dict(bias=P + 1), dict(stats=P + 4),
    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(rows=1 << 41),
    dict(dtype=tgp.FP32, x=P + 2), dict(ldx=1 << 60), dict(rows=1 << 62, C=1 << 30)])
def test_forward_refusals(kw):
    assert _fwd(**kw) == tgp.EINVAL
    assert "layer_norm_forward" in tgp.last_error()


def test_forward_of_no_rows_needs_no_tensors():
    assert _fwd(rows=0, x=None, y=None, gain=None, bias=None, stats=None) == tgp.OK


def _bwd(**kw):
    a = dict(rows=4, C=8, dtype=tgp.BF16, dy=P, lddy=8, x=P, ldx=8, gain=P, stats=P, dx=P, lddx=8, dgain=P,
             dbias=P, overwrite=1, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return tgp.call_status("tgp_layer_norm_backward", a["rows"], a["C"], a["dtype"], a["dy"], a["lddy"],
                           a["x"], a["ldx"], a["gain"], a["stats"], a["dx"], a["lddx"], a["dgain"],
                           a["dbias"], a["overwrite"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), tgp.EINVAL), (dict(C=0), tgp.EINVAL), (dict(dtype=7), tgp.EINVAL),
    (dict(dy=None), tgp.EINVAL), (dict(x=None), tgp.EINVAL), (dict(stats=None), tgp.EINVAL),
    (dict(lddy=7), tgp.EINVAL), (dict(ldx=0), tgp.EINVAL), (dict(lddx=7), tgp.EINVAL),
    (dict(dgain=None), tgp.EINVAL), (dict(dbias=None), tgp.EINVAL),
    (dict(dx=None, dgain=None, dbias=None), tgp.EINVAL), (dict(overwrite=2), tgp.EINVAL),
    (dict(ws=None), tgp.EINVAL), (dict(ws=P + 4), tgp.EINVAL), (dict(ws_bytes=4), tgp.ENOSPACE),
    (dict(dx=P + 1), tgp.EINVAL), (dict(dgain=P + 2), tgp.EINVAL), (dict(stats=P + 4), tgp.EINVAL)])
def test_backward_refusals(kw, want):
    assert _bwd(**kw) == want
    assert "layer_norm_backward" in tgp.last_error()


def test_backward_workspace():
    with pytest.raises(tgp.TgpError):
        tgp.layer_norm_backward_workspace(4, 0, tgp.BF16)
    assert tgp.call_status("tgp_layer_norm_backward_workspace", 4, 8, tgp.BF16, None) == tgp.EINVAL
    assert tgp.layer_norm_backward_workspace(0, 8, tgp.BF16) == 0
    assert tgp.layer_norm_backward_workspace(1 << 20, 64, tgp.BF16) > 0


def _mu(tensors=((16, 32, P, P, P),), n=None, mu=0.9, nesterov=1, steps=5, eps=1e-7, ws=P, ws_bytes=1 << 40):
    t = tgp.muon_tensors(tensors) if tensors is not None else None
    return tgp.call_status("tgp_muon_update", len(t) if n is None else n, t, mu, nesterov, steps, eps, ws,
                           ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), tgp.EINVAL), (dict(tensors=None, n=1), tgp.EINVAL), (dict(tensors=[(0, 4, P, P, P)]), tgp.EINVAL),
    (dict(tensors=[(4, -1, P, P, P)]), tgp.EINVAL), (dict(tensors=[(4, 4, None, P, P)]), tgp.EINVAL),
    (dict(tensors=[(4, 4, P, P, None)]), tgp.EINVAL), (dict(tensors=[(4, 4, P + 8, P, P)]), tgp.EINVAL),
    (dict(tensors=[(4, 4, P, P + 4, P)]), tgp.EINVAL), (dict(tensors=[(4, 4, P, P, P + 2)]), tgp.EINVAL),
    (dict(tensors=[(4, 4, P, P, P), (1 << 16, 1 << 16, P, P, P)]), tgp.EUNSUPPORTED),
    (dict(mu=float("nan")), tgp.EINVAL), (dict(nesterov=2), tgp.EINVAL), (dict(steps=0), tgp.EINVAL),
    (dict(eps=-1e-3), tgp.EINVAL), (dict(ws=None), tgp.EINVAL), (dict(ws=P + 128), tgp.EINVAL),
    (dict(ws_bytes=100), tgp.ENOSPACE)])
def test_muon_refusals(kw, want):
    assert _mu(**kw) == want
    assert "muon_update" in tgp.last_error()


def test_muon_of_nothing_and_workspaces():
    assert _mu(tensors=[], ws=None, ws_bytes=0) == tgp.OK
    assert tgp.muon_workspace(tgp.muon_tensors([])) == 0
    one = tgp.muon_workspace(tgp.muon_tensors([(64, 576, None, None, None)]))
    two = tgp.muon_workspace(tgp.muon_tensors([(64, 576, None, None, None)] * 2))
    assert 0 < one < two
    assert tgp.call_status("tgp_muon_workspace", 1, tgp.muon_tensors([(4, 4, P, P, P)]), None) == tgp.EINVAL
    v = ctypes.c_size_t()
    assert tgp.call_status("tgp_muon_workspace", 1, tgp.muon_tensors([(4, 0, P, P, P)]), ctypes.byref(v)) == tgp.EINVAL


@pytest.mark.parametrize("t", [(-1, P, P, P, 0.1), (4, None, P, P, 0.1), (4, P, P, None, 0.1), (4, P + 4, P, P, 0.1),
                               (4, P, P + 2, P, 0.1), (4, P, P, P + 8, 0.1), (4, P, P, P, float("nan")),
                               (1 << 50, P, P, P, 0.1)])
def test_weight_step_refusals(t):
    assert tgp.call_status("tgp_weight_step", 1, tgp.step_tensors([t]), 0.1, None) == tgp.EINVAL
    assert "weight_step" in tgp.last_error()


def test_step_lists():
    assert tgp.call_status("tgp_weight_step", 0, None, 0.1, None) == tgp.OK
    assert tgp.call_status("tgp_weight_step", 1, None, 0.1, None) == tgp.EINVAL
    assert tgp.call_status("tgp_weight_step", -1, None, 0.1, None) == tgp.EINVAL
    assert tgp.call_status("tgp_weight_step", 0, None, float("inf"), None) == tgp.EINVAL
    assert tgp.call_status("tgp_weight_step", 1, tgp.step_tensors([(0, None, None, None, 0.1)]), 0.1, None) == tgp.OK
    assert tgp.call_status("tgp_adamw_step", 0, None, 0.1, 0.9, 0.9, 1e-8, 0.0, 1, None) == tgp.OK


@pytest.mark.parametrize("kw", [dict(rate=float("nan")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.5),
                                dict(eps=-1.0), dict(decay=float("inf")), dict(step=0),
                                dict(t=(4, P, P, None, P, P)), dict(t=(4, P, P, P, None, P)),
                                dict(t=(4, P, P, P, P, P + 4)), dict(t=(-4, P, P, P, P, P))])
def test_adamw_refusals(kw):
    a = dict(t=(4, P, None, P, P, P), rate=0.1, beta1=0.9, beta2=0.9, eps=1e-8, decay=0.0, step=1)
    a.update(kw)
    assert tgp.call_status("tgp_adamw_step", 1, tgp.adamw_tensors([a["t"]]), a["rate"], a["beta1"], a["beta2"],
                           a["eps"], a["decay"], a["step"], None) == tgp.EINVAL
    assert "adamw_step" in tgp.last_error()


@pytest.fixture
def no_launch():
    """Every launch is skipped (and fails), so that calls whose checks pass end without touching a device."""
    tgp.debug_fail_launch(1)
    yield
    tgp.debug_fail_launch(0)


@pytest.mark.parametrize("c", [(1 << 30) + 1, (1 << 31) - 256, (1 << 31) - 1])
def test_rows_longer_than_the_kernels_count(no_launch, c):
    """The kernels step through a row's channels by a block's threads in 32 bits."""
    for dtype in (tgp.BF16, tgp.FP32):
        assert _fwd(rows=1, C=c, dtype=dtype, ldx=c, ldy=c) == tgp.EUNSUPPORTED
        assert _bwd(rows=1, C=c, dtype=dtype, lddy=c, ldx=c, lddx=c, ws_bytes=1 << 60) == tgp.EUNSUPPORTED
        v = ctypes.c_size_t()
        assert tgp.call_status("tgp_layer_norm_backward_workspace", 1, c, dtype, ctypes.byref(v)) == tgp.EUNSUPPORTED
    assert _fwd(rows=1, C=1 << 30, ldx=1 << 30, ldy=1 << 30, y=P + (1 << 40)) == tgp.EHIP     # as far as its launch


# (offset in elements, row distance) of a tensor of 4 rows of 8 channels beside one at 0, 24: what shares elements
# with it in another way than row by row, and what does not
SHARED = [(0, 8), (0, 16), (0, 25), (0, 32), (1, 24), (7, 24), (-7, 24), (24, 24), (-24, 24), (31, 24), (72, 24), (-72, 24),
          (24, 8), (8, 12), (12, 12), (-8, 16), (40, 16), (17, 25), (79, 8)]
APART = [(0, 24), (8, 24), (16, 24), (-8, 24), (80, 8), (80, 24), (-32, 8), (-80, 24), (96, 24), (8, 48), (-16, 48),
         (88, 24), (8, 25), (9, 24)]


@pytest.mark.parametrize("dtype", [tgp.BF16, tgp.FP32])
def test_tensors_that_overlap(no_launch, dtype):
    """Sharing elements in another way than y (dx) lying on x (dy, x) row by row is refused: rows are
    written while others are read.  Slices that lie between each other's rows are not."""
    e = 2 if dtype == tgp.BF16 else 4

    def elements(at, ld):
        return {at + r * ld + c for r in range(4) for c in range(8)}

    base = elements(0, 24)
    assert all(elements(*t) & base for t in SHARED)
    assert all(t == (0, 24) or not elements(*t) & base for t in APART)
    for at, ld in SHARED + APART:
        want = tgp.EHIP if (at, ld) in APART else tgp.EINVAL    # the launch, skipped here, or the refusal
        p, far = P + at * e, P + (1 << 20)
        for dst, src in (((p, ld), (P, 24)), ((P, 24), (p, ld))):
            for status in (
                    lambda: _fwd(dtype=dtype, x=src[0], ldx=src[1], y=dst[0], ldy=dst[1]),
                    lambda: _bwd(dtype=dtype, dy=src[0], lddy=src[1], x=far, ldx=8, dx=dst[0], lddx=dst[1]),
                    lambda: _bwd(dtype=dtype, dy=far, lddy=8, x=src[0], ldx=src[1], dx=dst[0], lddx=dst[1])):
                tgp.debug_fail_launch(1)
                assert status() == want, (at, ld, tgp.last_error())
                assert want == tgp.EHIP or "overlap" in tgp.last_error()
    tgp.debug_fail_launch(1)
    assert _fwd(dtype=dtype, rows=1, x=P, ldx=8, y=P, ldy=24) == tgp.EHIP        # one row lies on itself
    assert _fwd(dtype=dtype, rows=1, x=P, ldx=8, y=P + e, ldy=24) == tgp.EINVAL
    # what is only read may overlap, and no dx is none
    tgp.debug_fail_launch(1)
    assert _bwd(dtype=dtype, dy=P + e, lddy=9, x=P, ldx=8, dx=P + (1 << 20)) == tgp.EHIP
    tgp.debug_fail_launch(1)
    assert _bwd(dtype=dtype, dy=P, lddy=9, x=P, ldx=8, dx=None, lddx=0) == tgp.EHIP


def test_many_rows_that_overlap(no_launch):
    """By row distances that many rows bring onto each other, and ones whose rows never meet."""
    rows, e = 1 << 24, 2
    assert _fwd(rows=rows, C=8, x=P, ldx=101, y=P + 50 * e, ldy=100) == tgp.EINVAL
    assert _fwd(rows=rows, C=8, x=P, ldx=64, y=P + 16 * e, ldy=128) == tgp.EHIP
    tgp.debug_fail_launch(1)
    assert _fwd(rows=rows, C=8, x=P, ldx=64, y=P + 64 * rows * e, ldy=65) == tgp.EHIP
    assert _fwd(rows=rows, C=8, x=P, ldx=64, y=P + (64 * rows - 65) * e, ldy=65) == tgp.EINVAL


def test_muon_workspace_of_long_lists():
    """Lists that run one after the other share their workspace: no more than the largest asks for."""
    def need(n, r, c):
        return tgp.muon_workspace(tgp.muon_tensors([(r, c, None, None, None)] * n))

    for r, c in ((2048, 18432), (128, 1152), (300, 70)):
        most = need(20, r, c)
        assert need(1, r, c) < need(10, r, c) < most
        assert all(need(n, r, c) == most for n in (21, 40, 41, 100))
    mixed = tgp.muon_tensors([(2048, 4096, None, None, None)] * 30 + [(64, 576, None, None, None)] * 5)
    assert tgp.muon_workspace(mixed) == need(20, 2048, 4096)
