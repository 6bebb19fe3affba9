"""The norms around a residual block against their 64-bit definition.

Tolerances, fixed before the first run.  As for the layer norm, a row's sums run
in float32 trees and short chains of at most 64 additions behind a term, which
leaves fhat and ohat off by EPS32 (|xhat| + A), A the mean magnitude of the row's
values and differences times rstd; EPS32 = 1e-5.  The sum's error goes on into z
times rstd_out, and G's into df.  Each output in bfloat16 may be off by 2^-8 of
itself more.  Sums over rows: EPS32 of the sum of the terms' magnitudes and of
what their factors are off by.
"""
import pytest
import torch

import block_ops_ref as ref
import paper_2004_09910_amd as tgp
from gpu_util import say

pytestmark = pytest.mark.gpu
EPS32 = 1e-5
DT = {"bf16": (tgp.BF16, torch.bfloat16), "fp32": (tgp.FP32, torch.float32)}
VEC = ("scale", "post_gain", "post_bias", "pre_gain", "pre_bias")


def _rows(rows, c, ld, off, dtype, fill=None):
    buf = torch.full((rows * ld + off + 64,), 7.5, dtype=dtype, device="cuda")
    v = buf[off:off + rows * ld].view(rows, ld)[:, :c]
    if fill is not None:
        v.copy_(fill)
    return buf, v


def _untouched(buf, v):
    keep = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(keep, v.shape, v.stride(), v.storage_offset()).fill_(False)
    assert bool((buf[keep] == 7.5).all()), "neighbours"


def _addr(t):
    return None if t is None else t.data_ptr()


def _ld(t):
    return 0 if t is None else t.stride(0)


class Run:
    """One shape's tensors on the device; group 0: no gate."""

    def __init__(self, rows, c, dt, group=0, post=True, vectors=True, seed=0, ld=0, off=0, eps=1e-5):
        g = torch.Generator().manual_seed(seed + 7 * rows + c)
        code, td = DT[dt]
        ld = max(ld, c)
        self.rows, self.c, self.dt, self.td, self.group, self.post, self.eps, self.ld, self.off = (
            rows, c, dt, td, group, post, eps, ld, off)
        self.shape = tgp.residual_shape(rows, c, code, group, post, eps)

        def t(n, values):
            return _rows(n, c, ld, off, td, values)[1]

        self.r = t(rows, 2 * torch.randn(rows, c, generator=g) + torch.randn(c, generator=g))
        self.f = t(rows, torch.randn(rows, c, generator=g) + torch.randn(c, generator=g))
        self.gate = t(rows // group, 1 + 0.3 * torch.randn(rows // group, c, generator=g)) if group else None
        self.dz, self.dout = t(rows, torch.randn(rows, c, generator=g)), t(rows, torch.randn(rows, c, generator=g))
        self.vec = {k: (0.5 + 0.2 * torch.randn(c, generator=g)).cuda() if vectors else None for k in VEC}
        if not post:
            self.vec["post_gain"] = self.vec["post_bias"] = None
        self.params = tgp.residual_params(*[_addr(self.vec[k]) for k in VEC])

    def p(self):
        return [None if self.vec[k] is None else self.vec[k].cpu() for k in VEC]

    def forward(self, out=None, z=True, stats=True, stream=0):
        bufs = []
        if out is None:
            buf, out = _rows(self.rows, self.c, self.ld, self.off, self.td)
            bufs.append((buf, out))
        if z is True:
            buf, z = _rows(self.rows, self.c, self.ld, self.off, self.td)
            bufs.append((buf, z))
        st = torch.full((self.rows, 4), -3.0, device="cuda") if stats else None
        tgp.residual_norm_forward(self.shape, self.params, self.r.data_ptr(), self.ld, self.f.data_ptr(), self.ld,
                                  _addr(self.gate), self.ld, out.data_ptr(), self.ld, _addr(z), self.ld, _addr(st), stream)
        torch.cuda.synchronize()
        for buf, v in bufs:
            _untouched(buf, v)
        return out, z, st

    def backward(self, out, st, dz=True, dout=True, dr=None, df=None, want=VEC, overwrite=True, fill=3.0, dgate=True, stream=0):
        bufs = []
        if dr is None:
            buf, dr = _rows(self.rows, self.c, self.ld, self.off, self.td)
            bufs.append((buf, dr))
        if df is None:
            buf, df = _rows(self.rows, self.c, self.ld, self.off, self.td)
            bufs.append((buf, df))
        dg = None
        if self.group and dgate is True:
            buf, dg = _rows(self.rows // self.group, self.c, self.ld, self.off, self.td)
            bufs.append((buf, dg))
        elif self.group and dgate is not False:
            dg = dgate
        grads = {k: torch.full((self.c,), fill, device="cuda") if k in want and (self.post or "post" not in k) and
                 (dz or "pre" not in k) else None for k in VEC}
        n = tgp.residual_norm_backward_workspace(self.shape)
        ws = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")
        tgp.residual_norm_backward(
            self.shape, self.params, self.dz.data_ptr() if dz else None, self.ld, self.dout.data_ptr() if dout else None,
            self.ld, out.data_ptr() if dz else None, self.ld, self.f.data_ptr(), self.ld, _addr(self.gate), self.ld,
            st.data_ptr(), dr.data_ptr(), self.ld, df.data_ptr(), self.ld, _addr(dg), self.ld,
            tgp.residual_grads(*[_addr(grads[k]) for k in VEC]), overwrite, ws.data_ptr(), n, stream)
        torch.cuda.synchronize()
        assert bool((ws[n:] == 255).all()), "past the workspace"
        for buf, v in bufs:
            _untouched(buf, v)
        return dict(dr=dr, df=df, dgate=dg, **grads)

    def _near(self, got, want, slack, half, what):
        d = (got.detach().cpu().double() - want).abs()
        worst = float((d / (slack + (2.0 ** -8 if half else 0) * want.abs() + 1e-30)).max())
        assert worst <= 1, (what, worst)

    def check(self, pre=True, dout=True):
        say("residual norm", self.rows, self.c, self.dt, "group", self.group, "post", self.post, "pre", pre, "ld", self.ld)
        half = self.dt == "bf16"
        one = torch.ones((), dtype=torch.float64)
        sc = one if self.vec["scale"] is None else self.vec["scale"].cpu().double().abs()
        pg = one if self.vec["post_gain"] is None else self.vec["post_gain"].cpu().double().abs()
        pb = 0 * one if self.vec["post_bias"] is None else self.vec["post_bias"].cpu().double().abs()
        ng = one if self.vec["pre_gain"] is None else self.vec["pre_gain"].cpu().double().abs()
        nb = 0 * one if self.vec["pre_bias"] is None else self.vec["pre_bias"].cpu().double().abs()
        r, f = self.r.cpu().double(), self.f.cpu().double()
        gate = None if self.gate is None else self.gate.cpu()
        q = ref.gate_rows(gate, self.group, self.rows).abs()
        out, z, st = self.forward(z=True if pre else None)
        wo, wz, ws = ref.residual_forward(r, f, gate, self.group, self.p(), self.post, pre, self.eps)

        def amp(t, mean, rstd):
            return (t.abs().mean(1, keepdim=True) + (t - mean).abs().mean(1, keepdim=True)) * rstd

        fh = (f - ws[:, :1]) * ws[:, 1:2] if self.post else f
        af = amp(f, ws[:, :1], ws[:, 1:2]) if self.post else 0 * f[:, :1]
        n = fh * (one if self.vec["post_gain"] is None else self.vec["post_gain"].cpu().double()) + (
            0 if self.vec["post_bias"] is None else self.vec["post_bias"].cpu().double()) if self.post else f
        so = EPS32 * (r.abs() + sc * q * ((fh.abs() + af) * pg + pb))
        self._near(out, wo, so, half, "out")
        if self.post:
            self._near(st[:, 0], ws[:, 0], EPS32 * f.abs().mean(1), False, "mean_f")
            self._near(st[:, 1], ws[:, 1], EPS32 * (1 + af[:, 0]) * ws[:, 1], False, "rstd_f")
        else:
            assert bool((st[:, :2] == 0).all())
        if pre:
            oh = (wo - ws[:, 2:3]) * ws[:, 3:]
            ao = amp(wo, ws[:, 2:3], ws[:, 3:])
            off = (so + so.mean(1, keepdim=True)) * ws[:, 3:]      # of the differences, over the row's spread
            sz = (EPS32 * (oh.abs() + ao) + off + oh.abs() * (oh.abs() * off).mean(1, keepdim=True)) * ng + EPS32 * nb
            self._near(z, wz, sz, half, "z")
        else:
            assert bool((st[:, 2:] == 0).all())
        got = self.backward(out, st, dz=pre, dout=dout)
        # the backward's own inputs: out and the statistics as they were stored
        dz, do = self.dz.cpu().double(), self.dout.cpu().double() if dout else 0 * f
        s64, o64 = st.cpu().double(), out.cpu().double()
        want = ref.residual_backward(self.dz.cpu() if pre else None, self.dout.cpu() if dout else None, out.cpu(), f, gate,
                                     self.group, self.p(), self.post, st.cpu())
        sg = EPS32 * do.abs()
        if pre:
            oh, ao = (o64 - s64[:, 2:3]) * s64[:, 3:], amp(o64, s64[:, 2:3], s64[:, 3:])
            a = dz.abs() * ng
            sg = sg + EPS32 * s64[:, 3:] * (a + a.mean(1, keepdim=True) + (oh.abs() + ao) * (a * (oh.abs() + ao)).mean(1, keepdim=True))
            self._near(got["pre_gain"], want["pre_gain"], EPS32 * (dz.abs() * (oh.abs() + ao)).sum(0), False, "pre_gain")
            self._near(got["pre_bias"], want["pre_bias"], EPS32 * dz.abs().sum(0), False, "pre_bias")
        self._near(got["dr"], want["dr"], sg, half, "dr")
        G = want["dr"].abs()
        if self.post:
            fh, af = (f - s64[:, :1]) * s64[:, 1:2], amp(f, s64[:, :1], s64[:, 1:2])
        sn = sc * q * (sg + EPS32 * G)
        nn = n.abs()
        err = EPS32 * ((fh.abs() + af) * pg + pb) if self.post else EPS32 * nn
        self._near(got["scale"], want["scale"], (q * (sg * nn + G * err) + EPS32 * G * q * nn).sum(0), False, "scale")
        if self.post:
            b, sb = sc * q * G * pg, sn * pg
            x = fh.abs() + af
            sd = s64[:, 1:2] * (sb + sb.mean(1, keepdim=True) + x * (sb * x).mean(1, keepdim=True) +
                                EPS32 * (b + b.mean(1, keepdim=True) + x * (b * x).mean(1, keepdim=True)))
            self._near(got["df"], want["df"], sd, half, "df")
            dn = sc * q * G
            self._near(got["post_gain"], want["post_gain"], (sn * fh.abs() + EPS32 * dn * x).sum(0), False, "post_gain")
            self._near(got["post_bias"], want["post_bias"], (sn + EPS32 * dn).sum(0), False, "post_bias")
        else:
            self._near(got["df"], want["df"], sn, half, "df")
        if gate is not None:
            t = (sc * (sg * nn + G * err + EPS32 * G * nn)).view(-1, self.group, self.c).sum(1)
            self._near(got["dgate"], want["dgate"], t, half, "dgate")
        return out, z, st, got


# rows, C, group: single values, widths at and around every vector, group and block width, gates of one pixel, of
# some, of all, many gates of few pixels and few of many
SHAPES = [(1, 1, 0), (1, 1, 1), (6, 2, 3), (5, 7, 0), (64, 8, 16), (100, 16, 1), (33, 24, 11), (1000, 64, 500),
          (129, 100, 43), (257, 120, 0), (40, 192, 40), (17, 255, 1), (16, 256, 2), (9, 513, 3), (70, 1000, 35),
          (12, 1024, 0), (5, 2056, 5), (3, 4096, 1), (2, 4100, 0), (3, 8200, 3), (2, 16384, 1), (2, 32768, 2),
          (20000, 24, 10000), (20000, 24, 1), (4099, 128, 4099), (6000, 40, 2), (6000, 40, 1500), (3000, 72, 0),
          (4096, 8, 64), (1200, 520, 400)]


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("rows,c,group", SHAPES)
def test_forward_and_backward(rows, c, group, post, dt):
    Run(rows, c, dt, group, post).check()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("rows,c,group", [(37, 48, 0), (40, 130, 8), (1000, 9, 1), (900, 64, 300)])
def test_without_vectors_norm_or_later_stream(rows, c, group, post, dt):
    """No vectors at all; no norm that follows (z, dz NULL); nothing else that reads the stream (dout NULL)."""
    Run(rows, c, dt, group, post, vectors=False).check()
    Run(rows, c, dt, group, post).check(pre=False)
    Run(rows, c, dt, group, post).check(dout=False)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("c,ld,off", [(64, 72, 8), (64, 65, 0), (64, 64, 1), (40, 384, 8), (7, 13, 3), (1100, 1101, 0),
                                      (520, 522, 2), (9000, 9001, 1)])
@pytest.mark.parametrize("group", [0, 1, 10])
def test_strides_and_alignment(c, ld, off, group, dt):
    Run(30, c, dt, group, True, ld=ld, off=off).check()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,c,group", [(50, 64, 0), (60, 100, 1), (60, 136, 20), (8, 1500, 2), (6, 9000, 3), (3000, 32, 1500)])
def test_places(rows, c, group, dt):
    """Outputs on their inputs, row by row: the bits of the calls with tensors of their own."""
    def new():
        return Run(rows, c, dt, group, ld=c + 8)

    a = new()
    out, z, st = a.forward()
    want = a.backward(out, st)
    b = new()
    o2, z2, s2 = b.forward(out=b.r, z=b.f)
    assert torch.equal(o2, out) and torch.equal(z2, z) and torch.equal(s2, st)
    b = new()
    o2, z2, _ = b.forward(out=b.f, z=b.r)
    assert torch.equal(o2, out) and torch.equal(z2, z)
    for dr, df in (("dout", "f"), ("dz", "dout"), ("out", "dz"), ("f", "out")):
        b = new()
        t = dict(dout=b.dout, dz=b.dz, out=out.clone(), f=b.f)
        t["out"] = _rows(rows, c, c + 8, 0, b.td, out)[1]
        got = b.backward(t["out"], st, dr=t[dr], df=t[df], dgate=b.gate if group == 1 else True)
        assert all(torch.equal(got[k], want[k]) for k in want if want[k] is not None), (dr, df)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,c,group", [(50, 64, 0), (60, 100, 20), (6, 9000, 1), (2000, 16, 1000)])
def test_sums_alone_and_added(rows, c, group, dt):
    a = Run(rows, c, dt, group)
    out, _, st = a.forward()
    want = a.backward(out, st)
    for k in VEC:
        got = a.backward(out, st, want=(k,), dgate=False)
        assert torch.equal(got[k], want[k]) and torch.equal(got["df"], want["df"]), k
    none = a.backward(out, st, want=())
    assert torch.equal(none["dr"], want["dr"]) and (not group or torch.equal(none["dgate"], want["dgate"]))
    more = a.backward(out, st, overwrite=False, fill=0.25)
    assert all(torch.equal(more[k], want[k] + 0.25) for k in VEC)
    o2, _, _ = a.forward(z=None, stats=False)
    assert torch.equal(o2, out)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("c", [5, 64, 640, 9000])
def test_constant_and_non_finite_rows(c, dt):
    """A constant row of f adds the post norm's bias; an infinity or NaN in a row of r or f makes that row of z NaN
    and no other."""
    a = Run(12, c, dt, 3)
    a.f[2] = 3.25
    out, z, _ = a.forward()
    v = {k: a.vec[k].cpu().double() for k in VEC}
    want = a.r[2].cpu().double() + v["scale"] * a.gate[0].cpu().double() * v["post_bias"]
    assert float(((out[2].cpu().double() - want).abs() / (want.abs() + 1)).max()) <= (2.0 ** -8 if dt == "bf16" else EPS32)
    for t in (a.r, a.f):
        for bad in (float("inf"), float("nan")):
            old = t[7].clone()
            t[7, c // 2] = bad
            o2, z2, _ = a.forward()
            keep = torch.arange(12) != 7
            assert torch.equal(o2[keep], out[keep]) and torch.equal(z2[keep], z[keep])
            assert bool(torch.isnan(z2[7]).all())
            t[7] = old


def test_zero_rows():
    a = Run(4, 8, "bf16")
    shape = tgp.residual_shape(0, 8, tgp.BF16)
    g = [torch.ones(8, device="cuda") for _ in VEC]
    for overwrite in (False, True):
        tgp.residual_norm_backward(shape, a.params, None, 8, None, 8, None, 8, None, 8, None, 8, None, None, 8, None, 8,
                                   None, 8, tgp.residual_grads(*[t.data_ptr() for t in g]), overwrite, None, 0)
        torch.cuda.synchronize()
        assert all(bool((t == (0.0 if overwrite else 1.0)).all()) for t in g)


@pytest.mark.parametrize("group,post", [(0, True), (5, True), (1, False)])
def test_gradient_against_differences(group, post):
    """The gradients of sum(out dout) + sum(z dz), float32, along random directions, against central differences of
    the 64-bit definition (steps of 1e-5 leave 1e-9)."""
    a = Run(20, 14, "fp32", group, post)
    out, _, st = a.forward()
    got = a.backward(out, st)
    t = {"dr": a.r, "df": a.f, "dgate": a.gate, **{k: a.vec[k] for k in VEC}}
    t = {k: v.cpu().double() for k, v in t.items() if v is not None}
    g = torch.Generator().manual_seed(4)
    dz, dout = a.dz.cpu().double(), a.dout.cpu().double()
    for k in t:
        d = torch.randn(t[k].shape, generator=g, dtype=torch.float64)
        two = []
        for h in (1e-5, -1e-5):
            u = dict(t)
            u[k] = t[k] + h * d
            o, z, _ = ref.residual_forward(u["dr"], u["df"], u.get("dgate"), group, [u.get(n) for n in VEC], post, True, a.eps)
            two.append(float((o * dout).sum() + (z * dz).sum()))
        want = (two[0] - two[1]) / 2e-5
        have = float((got[k].cpu().double() * d).sum())
        size = float(torch.linalg.vector_norm(got[k].cpu().double()) * torch.linalg.vector_norm(d))
        assert abs(have - want) <= 3 * EPS32 * size + 1e-6, (k, have, want)


@pytest.mark.parametrize("rows,c,group", [(300, 64, 0), (300, 72, 100), (4000, 24, 2000), (40, 9000, 4)])
def test_side_stream_and_graph(rows, c, group):
    a = Run(rows, c, "bf16", group)
    out, z, st = a.forward()
    want = a.backward(out, st)
    side = torch.cuda.Stream()
    o2, z2, s2 = a.forward(stream=side.cuda_stream)
    assert torch.equal(o2, out) and torch.equal(z2, z) and torch.equal(s2, st)
    got = a.backward(out, st, stream=side.cuda_stream)
    assert all(torch.equal(got[k], want[k]) for k in want if want[k] is not None)
    new = {k: torch.empty(v.shape, dtype=v.dtype, device="cuda") for k, v in
           dict(out=out, z=z, st=st, dr=out, df=out, **{k: want[k] for k in VEC}).items()}
    dg = torch.empty(rows // group, c, dtype=torch.bfloat16, device="cuda") if group else None
    n = tgp.residual_norm_backward_workspace(a.shape)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        tgp.residual_norm_forward(a.shape, a.params, a.r.data_ptr(), a.ld, a.f.data_ptr(), a.ld, _addr(a.gate), a.ld,
                                  new["out"].data_ptr(), c, new["z"].data_ptr(), c, new["st"].data_ptr(), s)
        tgp.residual_norm_backward(a.shape, a.params, a.dz.data_ptr(), a.ld, a.dout.data_ptr(), a.ld, new["out"].data_ptr(), c,
                                   a.f.data_ptr(), a.ld, _addr(a.gate), a.ld, new["st"].data_ptr(), new["dr"].data_ptr(), c,
                                   new["df"].data_ptr(), c, _addr(dg), c,
                                   tgp.residual_grads(*[new[k].data_ptr() for k in VEC]), True, ws.data_ptr(), n, s)
    for _ in range(3):
        for v in new.values():
            v.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(new["out"], out) and torch.equal(new["z"], z) and torch.equal(new["st"], st)
        assert all(torch.equal(new[k], want[k]) for k in VEC + ("dr", "df"))
        assert dg is None or torch.equal(dg, want["dgate"])
        assert torch.equal(a.forward()[0], out)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("c", [24, 1001])
def test_rows_farther_apart_than_32_bits(c, dt):
    """Rows whose byte offsets pass 2^32: three rows of the stream 1.2e9 elements apart, updated in place.  A wave
    takes such rows one at a time, which adds in another order: each side is off by EPS32 and a rounding."""
    say("residual norm, far rows", c, dt)
    ld = 1_200_000_008 if dt == "bf16" else 600_000_004
    a = Run(3, c, dt, 1)
    want = a.forward()
    back = a.backward(want[0], want[2])
    buf = torch.empty(2 * ld + c + 8, dtype=a.td, device="cuda")
    far = buf.as_strided((3, c), (ld, 1))
    far.copy_(a.r)
    z, st = torch.empty(3, c, dtype=a.td, device="cuda"), torch.empty(3, 4, device="cuda")
    tgp.residual_norm_forward(a.shape, a.params, buf.data_ptr(), ld, a.f.data_ptr(), c, a.gate.data_ptr(), c, buf.data_ptr(),
                              ld, z.data_ptr(), c, st.data_ptr())
    torch.cuda.synchronize()
    tol = 2 * ((2.0 ** -8 if dt == "bf16" else 0) + EPS32)
    assert ref.rel(far, want[0].cpu().double()) <= tol and ref.rel(z, want[1].cpu().double()) <= tol
    assert ref.rel(st, want[2].cpu().double()) <= 2 * EPS32
    far.copy_(want[0])
    st.copy_(want[2])
    n = tgp.residual_norm_backward_workspace(a.shape)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    df, dg = torch.empty(3, c, dtype=a.td, device="cuda"), torch.empty(3, c, dtype=a.td, device="cuda")
    grads = [torch.empty(c, device="cuda") for _ in VEC]
    tgp.residual_norm_backward(a.shape, a.params, a.dz.data_ptr(), c, a.dout.data_ptr(), c, buf.data_ptr(), ld,
                               a.f.data_ptr(), c, a.gate.data_ptr(), c, st.data_ptr(), buf.data_ptr(), ld, df.data_ptr(), c,
                               dg.data_ptr(), c, tgp.residual_grads(*[t.data_ptr() for t in grads]), True, ws.data_ptr(), n)
    torch.cuda.synchronize()
    for t, k in zip([far, df, dg] + grads, ("dr", "df", "dgate") + VEC):
        assert ref.rel(t, back[k].cpu().double()) <= (tol if t.dtype == torch.bfloat16 else 2 * EPS32), k
