"""Layer norm forward and backward against the 64-bit definition.

Tolerances, fixed before the first run.  A row's sums run over at most C terms
in float32, in trees and short chains: with at most 64 additions behind a term
the mean is off by at most 64 x 2^-24 = 4e-6 of the row's mean magnitude, and
rstd by as much relatively; xhat is then off by EPS32 (|xhat| + A) with A = the
mean of |x - mean|'s and |x|'s ratio to the row's spread.  EPS32 = 1e-5 leaves
a factor of two.  A result stored in bfloat16 may be off by one unit in its
last place (2^-8 of itself) more: half for its rounding, half where the float32
error moves it over a tie.  Column sums: 2^-24 times the additions behind a
term (rows / blocks + the tree, under 1000 at these sizes) of the column's
sum of magnitudes, i.e. 6e-5 at the worst; random signs keep it near its square
root, and 1e-5 of the sum of magnitudes is asked.
"""
import pytest
import torch

import paper_2004_09910_amd as tgp
import train_ops_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu
EPS32 = 1e-5
DT = {"bf16": (tgp.BF16, torch.bfloat16), "fp32": (tgp.FP32, torch.float32)}


def _rows(rows, c, ld, off, dtype, fill=None):
    """A rows x c view at element `off` of a buffer of rows x ld, 16-byte aligned base."""
    buf = torch.full((rows * ld + off + 64,), 7.5, dtype=dtype, device="cuda")
    v = buf[off:off + rows * ld].view(rows, ld)[:, :c] if rows else buf[:0].view(0, c)
    if fill is not None:
        v.copy_(fill)
    return buf, v


def _untouched(buf, view_fn, what):
    """Everything of buf outside the view still holds its fill."""
    keep = torch.ones_like(buf, dtype=torch.bool)
    view_fn(keep)
    assert bool((buf[keep] == 7.5).all()), what


def _inputs(rows, c, seed, spread=1.0, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, c, generator=g) * spread + offset + torch.randn(c, generator=g)
    dy = torch.randn(rows, c, generator=g)
    return x, dy, 1 + 0.2 * torch.randn(c, generator=g), 0.3 * torch.randn(c, generator=g)


def _forward(x, gain, bias, dt, ldx, ldy, offx=0, offy=0, eps=1e-5, stats=True, stream=0):
    code, td = DT[dt]
    rows, c = x.shape
    _, xv = _rows(rows, c, ldx, offx, td, x)
    ybuf, yv = _rows(rows, c, ldy, offy, td)
    g = None if gain is None else gain.cuda()
    b = None if bias is None else bias.cuda()
    st = torch.full((rows, 2), -3.0, device="cuda") if stats else None
    tgp.layer_norm_forward(rows, c, code, xv.data_ptr(), ldx, None if g is None else g.data_ptr(),
                           None if b is None else b.data_ptr(), eps, yv.data_ptr(), ldy,
                           None if st is None else st.data_ptr(), stream)
    torch.cuda.synchronize()
    _untouched(ybuf, lambda k: k[offy:offy + rows * ldy].view(rows, ldy)[:, :c].fill_(False), "y's neighbours")
    return xv, yv, st


def _err(got, want, slack, half):
    d = (got.detach().cpu().double() - want).abs()
    return float((d / (slack + (2.0 ** -8 if half else 0) * want.abs() + 1e-30)).max()) if d.numel() else 0.0


# rows x C: single values, single rows, widths at and around every vector, group
# and block width, long rows, many rows
SHAPES = [(1, 1), (5, 1), (1, 2), (3, 7), (64, 8), (100, 16), (33, 24), (1000, 64), (129, 100),
          (257, 120), (40, 192), (17, 255), (16, 256), (9, 513), (70, 1000), (12, 1024), (5, 2056),
          (3, 4096), (2, 4100), (3, 8200), (1, 16384), (2, 20001), (20000, 24), (4099, 128)]


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,c", SHAPES)
def test_forward_and_backward(rows, c, dt):
    say("layer norm", rows, c, dt)
    code, td = DT[dt]
    x, dy, gain, bias = _inputs(rows, c, rows * 7 + c)
    xv, yv, st = _forward(x, gain, bias, dt, c, c)
    y, mean, rstd = ref.norm_forward(xv.cpu(), gain, bias, 1e-5)
    xd = xv.cpu().double()
    amp = (xd.abs().mean(1) + (xd - mean[:, None]).abs().mean(1)) * rstd
    xhat = (xd - mean[:, None]) * rstd[:, None]
    slack = EPS32 * ((xhat.abs() + amp[:, None]) * gain.double().abs() + bias.double().abs())
    assert _err(yv, y, slack, dt == "bf16") <= 1
    assert float(((st[:, 0].cpu().double() - mean).abs() / (xd.abs().mean(1) + 1e-30)).max()) <= EPS32
    assert float((st[:, 1].cpu().double() / rstd - 1).abs().max()) <= EPS32 * max(1.0, float(amp.max()))
    # backward, from the statistics the forward left
    _, dyv = _rows(rows, c, c, 0, td, dy)
    dxbuf, dxv = _rows(rows, c, c, 0, td)
    dg, db = torch.full((c,), 2.0, device="cuda"), torch.full((c,), -1.0, device="cuda")
    n = tgp.layer_norm_backward_workspace(rows, c, code)
    ws = torch.full((n // 4 + 16,), 9.0, device="cuda")
    args = (rows, c, code, dyv.data_ptr(), c, xv.data_ptr(), c, gain.cuda().data_ptr(), st.data_ptr())
    keep = gain.cuda()
    args = args[:7] + (keep.data_ptr(), st.data_ptr())
    tgp.layer_norm_backward(*args, dxv.data_ptr(), c, dg.data_ptr(), db.data_ptr(), True,
                            ws.data_ptr(), n)
    torch.cuda.synchronize()
    assert bool((ws[(n + 3) // 4:] == 9.0).all()), "past the workspace"
    _untouched(dxbuf, lambda k: k[:rows * c].fill_(False), "dx's neighbours")
    dxr, dgr, dbr = ref.norm_backward(dyv.cpu(), xv.cpu(), gain, st[:, 0].cpu(), st[:, 1].cpu())
    g = (dyv.cpu().double() * gain.double()).abs()
    xh = ((xd - st[:, :1].cpu().double()) * st[:, 1:].cpu().double()).abs()
    # what each term of dx may be off by: float32 sums of g and g xhat, and xhat's own rounding of x - mean
    xe = xh + (xd.abs() * st[:, 1:].cpu().double())
    slack = EPS32 * st[:, 1:].cpu().double() * (
        g + g.mean(1, keepdim=True) + xh * (g * xe).mean(1, keepdim=True) + xe * (g * xh).mean(1, keepdim=True))
    assert _err(dxv, dxr, slack, dt == "bf16") <= 1
    mag_g = (dyv.cpu().double().abs() * xe).sum(0)
    mag_b = dyv.cpu().double().abs().sum(0)
    assert float(((dg.cpu().double() - dgr).abs() / (1e-5 * mag_g + 1e-30)).max()) <= 1
    assert float(((db.cpu().double() - dbr).abs() / (1e-5 * mag_b + 1e-30)).max()) <= 1
    # added to what is there, and the same bits a second time
    dg2, db2 = dg.clone(), db.clone()
    dx2 = torch.empty_like(dxv)
    tgp.layer_norm_backward(*args, dx2.data_ptr(), c, dg2.data_ptr(), db2.data_ptr(), False,
                            ws.data_ptr(), n)
    torch.cuda.synchronize()
    assert torch.equal(dg2, dg + dg) and torch.equal(db2, db + db) and torch.equal(dx2, dxv)
    # either result alone
    dx3 = torch.empty_like(dxv)
    tgp.layer_norm_backward(*args, dx3.data_ptr(), c, None, None, False, None, 0)
    dg3, db3 = torch.zeros_like(dg), torch.zeros_like(db)
    tgp.layer_norm_backward(*args, None, 0, dg3.data_ptr(), db3.data_ptr(), True, ws.data_ptr(), n)
    torch.cuda.synchronize()
    assert torch.equal(dx3, dxv) and torch.equal(dg3, dg) and torch.equal(db3, db)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,c", [(1023, 9), (1024, 72), (1024, 1002), (1025, 1), (1026, 7), (1030, 100), (1100, 255),
                                    (1025, 513), (1025, 1000), (1031, 2056), (1025, 4096)])
def test_rows_around_the_sums_by_columns(rows, c, dt):
    """On both sides of where the gain's and bias's gradients are summed in the one launch."""
    test_forward_and_backward(rows, c, dt)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,c", [(9, 1025), (70, 1501), (33, 2049), (1100, 1501), (1026, 2047), (1030, 2502), (1025, 4095),
                                    (6, 4098), (5, 4097), (3, 8190), (2, 8193)])
def test_long_rows_of_narrow_accesses(rows, c, dt):
    """Rows of more than 1024 accesses of 2 or 4 bytes, up to what registers hold and beyond."""
    test_forward_and_backward(rows, c, dt)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("c,ldx,ldy,offx,offy", [
    (64, 192, 64, 64, 0), (64, 64, 200, 0, 72), (100, 228, 100, 0, 0), (100, 101, 103, 1, 3),
    (24, 25, 24, 5, 0), (256, 260, 264, 4, 8), (1, 3, 2, 1, 1), (2050, 2051, 2050, 0, 1)])
def test_strides_and_alignment(c, ldx, ldy, offx, offy, dt):
    """Channel slices of wider tensors at any element offset: the values of the dense call."""
    say("layer norm slices", c, ldx, ldy, offx, offy, dt)
    code, td = DT[dt]
    rows = 37
    x, dy, gain, bias = _inputs(rows, c, c)
    xv, yv, st = _forward(x, gain, bias, dt, ldx, ldy, offx, offy)
    y, mean, rstd = ref.norm_forward(xv.cpu(), gain, bias, 1e-5)
    xd = xv.cpu().double()
    amp = (xd.abs().mean(1) + (xd - mean[:, None]).abs().mean(1)) * rstd
    slack = EPS32 * ((((xd - mean[:, None]) * rstd[:, None]).abs() + amp[:, None]) * gain.double().abs()
                     + bias.double().abs())
    assert _err(yv, y, slack, dt == "bf16") <= 1
    _, dyv = _rows(rows, c, ldy, offy, td, dy)
    dxbuf, dxv = _rows(rows, c, ldx, offx, td)
    n = tgp.layer_norm_backward_workspace(rows, c, code)
    ws = torch.empty(n // 4 + 4, device="cuda")
    gg, dg, db = gain.cuda(), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    tgp.layer_norm_backward(rows, c, code, dyv.data_ptr(), ldy, xv.data_ptr(), ldx, gg.data_ptr(),
                            st.data_ptr(), dxv.data_ptr(), ldx, dg.data_ptr(), db.data_ptr(), True,
                            ws.data_ptr(), n)
    torch.cuda.synchronize()
    _untouched(dxbuf, lambda k: k[offx:offx + rows * ldx].view(rows, ldx)[:, :c].fill_(False), "dx's neighbours")
    dxr, dgr, dbr = ref.norm_backward(dyv.cpu(), xv.cpu(), gain, st[:, 0].cpu(), st[:, 1].cpu())
    tol = 2.0 ** -8 if dt == "bf16" else 1e-5
    if c > 1:
        assert ref.rel(dxv, dxr) <= tol and ref.rel(dg, dgr) <= 1e-5
    assert ref.rel(db, dbr) <= 1e-5


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("c", [8, 192, 1100])
def test_in_place_and_optional_arguments(c, dt):
    code, td = DT[dt]
    rows = 50
    x, dy, gain, bias = _inputs(rows, c, 3)
    for g, b in ((None, None), (gain, None), (None, bias)):
        xv, yv, st = _forward(x, g, b, dt, c, c)
        y, _, _ = ref.norm_forward(xv.cpu(), g, b, 1e-5)
        assert ref.rel(yv, y) <= (2.0 ** -8 if dt == "bf16" else EPS32)
        _, y2, _ = _forward(x, g, b, dt, c, c, stats=False)
        assert torch.equal(yv, y2)
        z = xv.contiguous().clone()
        keep = [t.cuda() if t is not None else None for t in (g, b)]
        ptr = [t.data_ptr() if t is not None else None for t in keep]
        tgp.layer_norm_forward(rows, c, code, z.data_ptr(), c, ptr[0], ptr[1], 1e-5, z.data_ptr(), c)
        torch.cuda.synchronize()
        assert torch.equal(z, yv)
        d = dy.to(td).cuda()
        n = tgp.layer_norm_backward_workspace(rows, c, code)
        ws = torch.empty(n // 4 + 4, device="cuda")
        got = []
        for place in ("apart", "dy", "x"):
            dd, xx, dx = d.clone(), xv.contiguous().clone(), torch.empty_like(d)
            out = {"apart": dx, "dy": dd, "x": xx}[place]
            dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
            tgp.layer_norm_backward(rows, c, code, dd.data_ptr(), c, xx.data_ptr(), c, ptr[0],
                                    st.data_ptr(), out.data_ptr(), c, dg.data_ptr(), db.data_ptr(),
                                    True, ws.data_ptr(), n)
            torch.cuda.synchronize()
            got.append((out, dg, db))
        dxr, dgr, _ = ref.norm_backward(d.cpu(), xv.cpu(), g, st[:, 0].cpu(), st[:, 1].cpu())
        assert ref.rel(got[0][0], dxr) <= (2.0 ** -8 if dt == "bf16" else EPS32)
        for o in got[1:]:
            assert all(torch.equal(p, q) for p, q in zip(o, got[0]))


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("c", [5, 64, 640, 9000])
def test_constant_and_non_finite_rows(c, dt):
    """A constant row gives the bias (its spread is zero); a row with an
    infinity or NaN is NaN, and its neighbours are as without it."""
    code, td = DT[dt]
    rows = 24
    x, dy, gain, bias = _inputs(rows, c, 11)
    x[3] = 2.5
    x[7] = 0.0
    clean, want, _ = _forward(x, gain, bias, dt, c, c)
    x[9, c // 2] = float("inf")
    x[10, 0] = float("nan")
    x[11, c - 1] = -float("inf")
    xv, yv, st = _forward(x, gain, bias, dt, c, c)
    good = [r for r in range(rows) if r not in (9, 10, 11)]
    assert torch.equal(yv[good], want[good])
    assert bool(torch.isnan(yv[[9, 10, 11]].float()).all())
    for r in (3, 7):
        assert torch.equal(yv[r].cpu(), bias.to(td))
    # large offsets: the variance comes from the differences
    x2, _, _, _ = _inputs(rows, c, 12, spread=0.01, offset=1000.0)
    if dt == "fp32" and c > 5:
        xv, yv, st = _forward(x2, None, None, dt, c, c, eps=0.0)
        _, _, rstd = ref.norm_forward(xv.cpu(), None, None, 0.0)
        assert float((st[:, 1].cpu().double() / rstd - 1).abs().max()) <= 1e-4


def test_zero_rows():
    t = torch.full((8,), 5.0, device="cuda")
    u = torch.full((8,), 6.0, device="cuda")
    tgp.layer_norm_forward(0, 8, tgp.BF16, None, 8, None, None, 1e-5, None, 8)
    assert tgp.layer_norm_backward_workspace(0, 8, tgp.BF16) == 0
    tgp.layer_norm_backward(0, 8, tgp.BF16, None, 8, None, 8, None, None, None, 8, t.data_ptr(),
                            u.data_ptr(), False, None, 0)
    torch.cuda.synchronize()
    assert bool((t == 5).all()) and bool((u == 6).all())
    tgp.layer_norm_backward(0, 8, tgp.BF16, None, 8, None, 8, None, None, None, 8, t.data_ptr(),
                            u.data_ptr(), True, None, 0)
    torch.cuda.synchronize()
    assert bool((t == 0).all()) and bool((u == 0).all())


@pytest.mark.parametrize("c", [6, 96])
def test_gradient_against_differences(c):
    """<dy, y(x + h d) - y(x - h d)> / 2h in 64 bits against <dx, d>, and the same for gain and bias.
    Central differences are off by h^2 (1e-6 relative to second derivatives of order one); the
    kernel's float32 results by 1e-5 of the sums of magnitudes: 1e-4 of those is asked."""
    rows = 12
    x, dy, gain, bias = _inputs(rows, c, 21)
    xv, yv, st = _forward(x, gain, bias, "fp32", c, c)
    n = tgp.layer_norm_backward_workspace(rows, c, tgp.FP32)
    ws = torch.empty(n // 4 + 4, device="cuda")
    d, gg = dy.cuda(), gain.cuda()
    dx, dg, db = torch.empty_like(d), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    tgp.layer_norm_backward(rows, c, tgp.FP32, d.data_ptr(), c, xv.data_ptr(), c, gg.data_ptr(),
                            st.data_ptr(), dx.data_ptr(), c, dg.data_ptr(), db.data_ptr(), True,
                            ws.data_ptr(), n)
    torch.cuda.synchronize()
    h = 1e-3
    gen = torch.Generator().manual_seed(5)

    def loss(x_, gain_, bias_):
        return (dy.double() * ref.norm_forward(x_, gain_, bias_, 1e-5)[0]).sum().item()

    x64, g64, b64 = x.double(), gain.double(), bias.double()
    for k in range(4):
        e, eg, eb = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((rows, c), (c,), (c,)))
        for got, grad, dirn, f in (
                (dx, "x", e, lambda s: loss(x64 + s * e, g64, b64)),
                (dg, "gain", eg, lambda s: loss(x64, g64 + s * eg, b64)),
                (db, "bias", eb, lambda s: loss(x64, g64, b64 + s * eb))):
            num = (f(h) - f(-h)) / (2 * h)
            prod = got.cpu().double() * dirn
            assert abs(num - prod.sum().item()) <= 1e-4 * prod.abs().sum().item() + 1e-9, grad


def test_side_stream_and_graph():
    """On a stream of its own, and captured and replayed with eager work between."""
    rows, c = 3000, 64
    x, dy, gain, bias = _inputs(rows, c, 31)
    s = torch.cuda.Stream()
    xg, dg_, gg, bb = x.bfloat16().cuda(), dy.bfloat16().cuda(), gain.cuda(), bias.cuda()
    y, st, dx = torch.empty_like(xg), torch.empty(rows, 2, device="cuda"), torch.empty_like(xg)
    dgain, dbias = torch.zeros(c, device="cuda"), torch.zeros(c, device="cuda")
    n = tgp.layer_norm_backward_workspace(rows, c, tgp.BF16)
    ws = torch.empty(n // 4 + 4, device="cuda")

    def go(stream):
        tgp.layer_norm_forward(rows, c, tgp.BF16, xg.data_ptr(), c, gg.data_ptr(), bb.data_ptr(), 1e-5,
                               y.data_ptr(), c, st.data_ptr(), stream)
        tgp.layer_norm_backward(rows, c, tgp.BF16, dg_.data_ptr(), c, xg.data_ptr(), c, gg.data_ptr(),
                                st.data_ptr(), dx.data_ptr(), c, dgain.data_ptr(), dbias.data_ptr(),
                                True, ws.data_ptr(), n, stream)

    go(0)
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, st, dx, dgain, dbias)]
    for t in (y, st, dx, dgain, dbias):
        t.zero_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        go(s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (y, st, dx, dgain, dbias)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        for t in (y, st, dx, dgain, dbias):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, st, dx, dgain, dbias)))


def test_micro_batches_add_up():
    """The gradients of m micro-batches, accumulated in the order m..1, are the full batch's."""
    rows, c, m = 4 * 49, 48, 4
    x, dy, gain, bias = _inputs(rows, c, 41)
    xv, yv, st = _forward(x, gain, bias, "fp32", c, c)
    d, gg = dy.cuda(), gain.cuda()
    dx = torch.empty_like(d)
    dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    per = rows // m
    n = tgp.layer_norm_backward_workspace(per, c, tgp.FP32)
    ws = torch.empty(n // 4 + 4, device="cuda")
    for i in range(m - 1, -1, -1):
        sl = slice(i * per, (i + 1) * per)
        tgp.layer_norm_backward(per, c, tgp.FP32, d[sl].data_ptr(), c, xv[sl].data_ptr(), c, gg.data_ptr(),
                                st[sl].data_ptr(), dx[sl].data_ptr(), c, dg.data_ptr(), db.data_ptr(),
                                i == m - 1, ws.data_ptr(), n)
    torch.cuda.synchronize()
    dxr, dgr, dbr = ref.norm_backward(dy, xv.cpu(), gain, st[:, 0].cpu(), st[:, 1].cpu())
    assert ref.rel(dx, dxr) <= 1e-5 and ref.rel(dg, dgr) <= 1e-5 and ref.rel(db, dbr) <= 1e-5


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("c", [24, 1001])
def test_rows_farther_apart_than_32_bits(c, dt):
    """Rows whose byte offsets pass 2^32: three rows 1.2e9 elements apart in one buffer, in and out."""
    say("layer norm, far rows", c, dt)
    code, td = DT[dt]
    ld = 1_200_000_008 if dt == "bf16" else 600_000_004
    x, dy, gain, bias = _inputs(3, c, c)
    buf = torch.empty(2 * ld + c + 8, dtype=td, device="cuda")
    view = buf.as_strided((3, c), (ld, 1))
    view.copy_(x)
    want, _, st = _forward(x, gain, bias, dt, c, c)
    g, b = gain.cuda(), bias.cuda()
    y = torch.empty(3, c, dtype=td, device="cuda")
    tgp.layer_norm_forward(3, c, code, buf.data_ptr(), ld, g.data_ptr(), b.data_ptr(), 1e-5, y.data_ptr(), c)
    torch.cuda.synchronize()
    assert torch.equal(y, _forward(x, gain, bias, dt, c, c)[1]) and torch.equal(view, want)
    n = tgp.layer_norm_backward_workspace(3, c, code)
    ws = torch.empty(n // 4 + 4, device="cuda")
    d = dy.to(td).cuda()
    got = []
    for xp, xl in ((want, c), (buf, ld)):
        dx, dg, db = torch.empty(3, c, dtype=td, device="cuda"), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        tgp.layer_norm_backward(3, c, code, d.data_ptr(), c, xp.data_ptr(), xl, g.data_ptr(), st.data_ptr(),
                                dx.data_ptr(), c, dg.data_ptr(), db.data_ptr(), True, ws.data_ptr(), n)
        torch.cuda.synchronize()
        got.append((dx, dg, db))
    assert all(torch.equal(p, q) for p, q in zip(*got))
    # and written there, in place
    tgp.layer_norm_forward(3, c, code, buf.data_ptr(), ld, g.data_ptr(), b.data_ptr(), 1e-5, buf.data_ptr(), ld)
    torch.cuda.synchronize()
    assert torch.equal(view, y)


def _narrow_rows(c, dt):
    """Rows far from zero: constant ones, and ones whose values vary by little around them."""
    g = torch.Generator().manual_seed(c)
    vals = [12345.678, 1000.1, 100000.3, 0.1, -77777.77, 1e-6, 3.0]
    x = torch.tensor(vals)[:, None].repeat(1, c)
    spread = torch.tensor([2.0 ** -5, 2.0 ** -8, 1.0, 2.0 ** -22, 0.25, 2.0 ** -36, 2.0 ** -3])
    return torch.cat((x, x + spread[:, None] * torch.randn(len(vals), c, generator=g))).to(DT[dt][1]), len(vals)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("c,ldx", [(5, 5), (64, 64), (101, 103), (640, 640), (1000, 1000), (1000, 1001), (2050, 2050),
                                   (4099, 4099), (9000, 9000), (20001, 20001)])
def test_rows_that_vary_little(c, ldx, dt):
    """A constant row of any value is its bias and its own mean, exactly: the first mean is off by some units
    of its last place, all differences are that many, and their sum (under 2^24 units) and quotient are exact.
    Where values vary, x - mean is exact or off by 2^-24 of itself, and its mean by 64 x 2^-24 of the mean
    magnitude of the differences, not of the values: EPS32 of the spread is asked of xhat and of rstd, and of
    the saved mean one rounding, 2^-24 of itself, more."""
    say("layer norm, narrow rows", c, ldx, dt)
    x, n = _narrow_rows(c, dt)
    _, _, gain, bias = _inputs(x.shape[0], c, c)
    xv, yv, st = _forward(x, gain, bias, dt, ldx, c)
    td = DT[dt][1]
    assert torch.equal(yv[:n].cpu(), bias.to(td).expand(n, c))
    assert torch.equal(st[:n, 0].cpu(), x[:n, 0].float())
    y, mean, rstd = ref.norm_forward(xv.cpu(), gain, bias, 1e-5)
    d = (xv.cpu().double() - mean[:, None]) * rstd[:, None]
    slack = EPS32 * ((d.abs() + d.abs().mean(1, keepdim=True)) * gain.double().abs() + bias.double().abs())
    assert _err(yv, y, slack, dt == "bf16") <= 1
    off = (st[:, 0].cpu().double() - mean).abs()
    assert bool((off <= 2.0 ** -24 * mean.abs() * 1.01 + EPS32 * d.abs().mean(1) / rstd).all())
    assert float((st[:, 1].cpu().double() / rstd - 1).abs().max()) <= EPS32


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,c,ld", [
    (1030, 64, 64), (3000, 64, 64), (3000, 8, 12), (1030, 100, 101), (1030, 1500, 1500), (3000, 1100, 1101),   # a wave's rows
    (1030, 4096, 4096), (1100, 2049, 2051), (1030, 4095, 4095), (1030, 3000, 3001),                          # a block's
    (50, 9000, 9000), (1030, 9000, 9000), (50, 4099, 4099), (1030, 4500, 4501)])                             # any row's
def test_in_place_of_every_kernel(rows, c, ld, dt):
    """y on x, dx on dy and dx on x: the bits of the calls with tensors of their own, by every kind of
    kernel, and nothing between the rows touched."""
    say("layer norm in place", rows, c, ld, dt)
    code, td = DT[dt]
    x, dy, gain, bias = _inputs(rows, c, rows + c)
    xv, yv, st = _forward(x, gain, bias, dt, ld, ld)
    g, b = gain.cuda(), bias.cuda()
    buf, z = _rows(rows, c, ld, 0, td, x)
    st2 = torch.empty_like(st)
    tgp.layer_norm_forward(rows, c, code, z.data_ptr(), ld, g.data_ptr(), b.data_ptr(), 1e-5, z.data_ptr(), ld,
                           st2.data_ptr())
    torch.cuda.synchronize()
    assert torch.equal(z, yv) and torch.equal(st2, st)
    _untouched(buf, lambda k: k[:rows * ld].view(rows, ld)[:, :c].fill_(False), "y's neighbours")
    n = tgp.layer_norm_backward_workspace(rows, c, code)
    ws = torch.empty(n // 4 + 4, device="cuda")
    got = []
    for place in ("apart", "dy", "x"):
        bufs = {"apart": _rows(rows, c, ld, 0, td), "dy": _rows(rows, c, ld, 0, td, dy), "x": _rows(rows, c, ld, 0, td, x)}
        dx = bufs[place][1]
        dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        tgp.layer_norm_backward(rows, c, code, bufs["dy"][1].data_ptr(), ld, bufs["x"][1].data_ptr(), ld, g.data_ptr(),
                                st.data_ptr(), dx.data_ptr(), ld, dg.data_ptr(), db.data_ptr(), True, ws.data_ptr(), n)
        torch.cuda.synchronize()
        _untouched(bufs[place][0], lambda k: k[:rows * ld].view(rows, ld)[:, :c].fill_(False), "dx's neighbours")
        got.append((dx, dg, db))
    dxr, dgr, dbr = ref.norm_backward(dy.to(td), xv.cpu(), gain, st[:, 0].cpu(), st[:, 1].cpu())
    assert ref.rel(got[0][0], dxr) <= (2.0 ** -8 if dt == "bf16" else EPS32)
    assert ref.rel(got[0][1], dgr) <= EPS32 and ref.rel(got[0][2], dbr) <= EPS32
    for o in got[1:]:
        assert all(torch.equal(p, q) for p, q in zip(o, got[0]))
