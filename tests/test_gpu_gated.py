"""The gated block against its 64-bit definition.

Tolerances, fixed before the first run, as 2-norms relative to the result's.
BF16: a stored bfloat16 is off by 2^-8 of itself at most; y has two such
roundings (h and its own), dx two (dg or du and its own): 2 x 2^-8 plus FP32.
The weights' and biases' gradients take dg, du and h as two bfloat16s, off by
2^-16 at most: 2^-16 + FP32.
FP32 = 5e-6: a product of three-part factors leaves out 3 x 2^-24 of a term, a
float32 sum of K terms in random order some sqrt(K) 2^-24 (K up to 5000 here: 4e-6)
of its terms' 2-norm, which random signs make the result's.
"""
import pytest
import torch

import block_ops_ref as ref
import paper_2004_09910_amd as tgp
from gpu_util import say

pytestmark = pytest.mark.gpu
FP32 = 5e-6
TOL = {"bf16": {"y": 2 * 2.0 ** -8 + FP32, "dx": 2 * 2.0 ** -8 + FP32, "w": 2.0 ** -16 + FP32, "b": 2.0 ** -16 + FP32},
       "fp32": {"y": FP32, "dx": FP32, "w": FP32, "b": FP32}}
DT = {"bf16": (tgp.BF16, torch.bfloat16), "fp32": (tgp.FP32, torch.float32)}
NAMES = ("gate", "up", "down", "b_gate", "b_up", "b_down")


def _view(rows, c, ld, off, dtype, fill=None):
    """A rows x c view at element `off` of a buffer with guard values around it."""
    buf = torch.full((rows * ld + off + 64,), 7.5, dtype=dtype, device="cuda")
    v = buf[off:off + rows * ld].view(rows, ld)[:, :c]
    if fill is not None:
        v.copy_(fill)
    return buf, v


def _untouched(buf, rows, c, ld, off, what):
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep[off:off + rows * ld].view(rows, ld)[:, :c].fill_(False)
    assert bool((buf[keep] == 7.5).all()), what


def _addr(t):
    return None if t is None else t.data_ptr()


class Block:
    def __init__(self, rows, cin, hidden, cout, dt="bf16", act=0, bias=True, seed=0, ldx=0, ldy=0, offx=0, offy=0, offw=0):
        g = torch.Generator().manual_seed(seed + rows + 7 * cin + 31 * hidden)
        code, td = DT[dt]
        self.dt, self.rows, self.cin, self.hidden, self.cout, self.act = dt, rows, cin, hidden, cout, act
        self.ldx, self.ldy, self.offx, self.offy = max(ldx, cin), max(ldy, cout), offx, offy
        self.shape = tgp.gated_shape(cin, hidden, cout, code, act)
        self.w = []
        for r, c in ((hidden, cin), (hidden, cin), (cout, hidden)):
            t = torch.full((r * c + offw + 8,), 7.5, dtype=td, device="cuda")
            t[offw:offw + r * c] = (torch.randn(r * c, generator=g) * (1.5 / c ** 0.5)).cuda()
            self.w.append(t[offw:offw + r * c].view(r, c))
        self.w += [torch.randn(n, generator=g).mul_(0.3).cuda() if bias else None for n in (hidden, hidden, cout)]
        self.xbuf, self.x = _view(rows, cin, self.ldx, offx, td, torch.randn(rows, cin, generator=g))
        self.dybuf, self.dy = _view(rows, cout, self.ldy, offy, td, torch.randn(rows, cout, generator=g))
        self.weights = tgp.gated_weights(*[_addr(t) for t in self.w])

    def _ws(self, backward):
        n = tgp.gated_workspace(self.shape, self.rows, backward)
        return torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda"), n     # NaN, whatever it is read as

    def host(self):
        return [None if t is None else t.cpu() for t in self.w]

    def forward(self, stream=0):
        buf, y = _view(self.rows, self.cout, self.ldy, self.offy, DT[self.dt][1])
        ws, n = self._ws(False)
        if stream:
            torch.cuda.synchronize()
        tgp.gated_forward(self.shape, self.rows, self.weights, self.x.data_ptr(), self.ldx, y.data_ptr(), self.ldy,
                          ws.data_ptr(), n, stream)
        torch.cuda.synchronize()
        assert bool((ws[n:] == 255).all()), "past the workspace"
        _untouched(buf, self.rows, self.cout, self.ldy, self.offy, "y's neighbours")
        return y

    def backward(self, overwrite=True, grads=None, dx="own", want=(True,) * 6, stream=0):
        td = DT[self.dt][1]
        buf, to = _view(self.rows, self.cin, self.ldx, self.offx, td)
        if dx == "x":
            buf, to = self.xbuf, self.x
        elif dx == "dy":
            buf, to = self.dybuf, self.dy
        gbuf = []
        if grads is None:
            for t, use in zip(self.w, want):
                b = None if t is None or not use else torch.full((t.numel() + 64,), 7.5, device="cuda")
                gbuf.append(b)
            grads = [None if b is None else b[:-64].view(t.shape) for b, t in zip(gbuf, self.w)]
        ws, n = self._ws(True)
        if stream:
            torch.cuda.synchronize()
        tgp.gated_backward(self.shape, self.rows, self.weights, self.dy.data_ptr(), self.ldy, self.x.data_ptr(), self.ldx,
                           None if dx is None else to.data_ptr(), self.ldx, tgp.gated_grads(*[_addr(g) for g in grads]),
                           overwrite, ws.data_ptr(), n, stream)
        torch.cuda.synchronize()
        assert bool((ws[n:] == 255).all()), "past the workspace"
        assert all(b is None or bool((b[-64:] == 7.5).all()) for b in gbuf), "past a gradient"
        if dx is not None:
            _untouched(buf, self.rows, self.cin, self.ldx, self.offx, "dx's neighbours")
        return [None if dx is None else to] + list(grads)

    def check(self, more=0.0):
        say("gated", self.rows, self.cin, self.hidden, self.cout, self.dt, self.act, self.ldx, self.ldy, self.offx)
        tol, x, dy, w = {k: v + more for k, v in TOL[self.dt].items()}, self.x.cpu(), self.dy.cpu(), self.host()
        y = self.forward()
        e = ref.rel(y, ref.gated(x, w, self.act))
        assert e <= tol["y"], ("y", e)
        got, want = self.backward(), ref.gated(x, w, self.act, dy)
        for name, a, b in zip(("dx",) + NAMES, got, want):
            e = ref.rel(a, b) if b is not None else 0.0
            assert e <= tol["dx" if name == "dx" else "b" if name.startswith("b_") else "w"], (name, e)
        return y, got


# rows, cin, hidden, cout: ones, odd sizes, sizes around every tile's and stage's, few and many rows
SHAPES = [(1, 1, 1, 1), (1, 8, 8, 8), (2, 3, 5, 7), (1, 256, 1024, 256), (5, 64, 256, 64), (16, 100, 270, 72),
          (17, 72, 96, 40), (31, 128, 64, 128), (32, 64, 520, 1000), (33, 40, 24, 56), (64, 64, 64, 64), (65, 65, 65, 65),
          (100, 16, 1000, 8), (127, 32, 128, 160), (128, 128, 128, 128), (129, 136, 264, 24), (144, 512, 1024, 512),
          (200, 1, 300, 1), (257, 200, 56, 72), (300, 513, 100, 257), (1000, 64, 256, 64), (1001, 24, 40, 24),
          (2049, 128, 72, 136), (4100, 8, 16, 8), (5000, 61, 33, 45),
          (17000, 136, 264, 136), (17001, 129, 257, 100),    # large tiles, odd ends
          (9001, 64, 2000, 72)]                              # (float32) pixels in three parts


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,hidden,cout", SHAPES)
def test_forward_and_backward(rows, cin, hidden, cout, dt):
    Block(rows, cin, hidden, cout, dt, act=(rows + cin) % 2, bias=rows % 3 != 0).check()


# the large tiles of every launch, one and several to a compute unit, and long sums of few tiles in ranges
LARGE = [(8200, 264, 1100, 520), (8190, 500, 264, 500), (2500, 504, 2040, 512), (300, 1016, 4088, 1016),
         (70, 300, 3001, 24), (129, 24, 2500, 300), (4097, 300, 72, 8)]


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,hidden,cout", LARGE)
def test_large_tiles_and_ranges(rows, cin, hidden, cout, dt):
    """As above; sums of K = 8200 terms have a random walk of 90.6 x 2^-24, and 70.7 are in FP32 (K = 5000)."""
    b = Block(rows, cin, hidden, cout, dt, act=rows % 2)
    _, first = b.check(20 * 2.0 ** -24)
    # Added to what is there.  Of pixels in one part this is G + G, exactly.  In two parts, sums c1 and c2, G is
    # fl(c1 + c2) and this fl(fl(G + c1) + c2): three roundings, of values of at most |G|, |G| + |c1| and |2 G|, each off
    # by 2^-24 of them; with |c1| and |c2| about |G| in the 2-norm or less (random signs), 5 |G| 2^-24 of 2 |G|.
    again = [g.clone() for g in first[1:]]
    b.backward(overwrite=False, grads=again)
    for name, g, once in zip(NAMES, again, first[1:]):
        assert ref.rel(g, 2 * once.cpu().double()) <= (2.5 * 2.0 ** -24 if dt == "fp32" else 0.0), name


def test_pixels_in_two_parts_of_one_launch_each():
    """4194374 pixels of few channels; sums of so many terms have a random walk of 2048 x 2^-24."""
    Block((1 << 22) + 70, 8, 72, 8, "bf16").check(2048 * 2.0 ** -24)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [3, 150])
@pytest.mark.parametrize("cin,hidden,cout,ldx,ldy,offx,offy,offw", [
    (64, 128, 64, 72, 80, 0, 8, 0), (64, 128, 64, 65, 67, 0, 0, 0), (64, 128, 64, 64, 64, 1, 3, 0), (40, 64, 48, 48, 56, 8, 8, 1),
    (7, 9, 11, 13, 29, 1, 1, 3), (64, 100, 64, 384, 64, 0, 0, 0), (64, 128, 64, 66, 130, 2, 4, 2)])
def test_strides_and_alignment(rows, cin, hidden, cout, ldx, ldy, offx, offy, offw, dt):
    Block(rows, cin, hidden, cout, dt, 1, True, 5, ldx, ldy, offx, offy, offw).check()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("act", [0, 1])
def test_far_pre_activations(act, dt):
    """Pre-activations from far below to far above where the activation saturates."""
    b = Block(40, 64, 48, 32, dt, act)
    for k in (0, 1):
        b.w[k].mul_(20.0)
    b.check()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,c,hidden", [(5, 32, 64), (140, 72, 100), (700, 64, 130), (300, 33, 47)])
def test_optional_arguments_and_places(rows, c, hidden, dt):
    """dx on x and on dy, gradients added to what is there, and each alone: the bits of the whole call."""
    def new():
        return Block(rows, c, hidden, c, dt, 0, True, 3, c + 8, c + 8)

    want = new().backward()
    for place in ("x", "dy"):
        got = new().backward(dx=place)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), place
    none = new().backward(dx=None)
    assert all(torch.equal(a, b) for a, b in zip(none[1:], want[1:]))
    for k in range(6):
        got = new().backward(dx=None, want=tuple(i == k for i in range(6)))
        assert torch.equal(got[1 + k], want[1 + k]), NAMES[k]
    got = new().backward(want=(False,) * 6)
    assert torch.equal(got[0], want[0])
    grads = [torch.full_like(t, 0.25) for t in want[1:]]
    got = new().backward(overwrite=False, grads=grads)
    assert all(torch.equal(a, b + 0.25) for a, b in zip(got[1:], want[1:]))


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,hidden,cout", [(6, 64, 64, 64), (150, 72, 200, 40), (400, 33, 70, 65)])
def test_non_finite_rows(rows, cin, hidden, cout, dt):
    """An infinity or NaN in a pixel leaves y and dx of every other pixel as they were, bit for bit."""
    b = Block(rows, cin, hidden, cout, dt)
    y, dx = b.forward().clone(), b.backward()[0].clone()
    for bad in (float("inf"), float("nan")):
        for place, t in ((1, b.x), (4, b.dy)):
            old = t.clone()
            t[place, t.shape[1] // 2] = bad
            y2, got = b.forward(), b.backward()
            keep = torch.arange(rows) != place
            assert torch.equal(got[0][keep], dx[keep])
            assert not bool(torch.isfinite(got[0][place]).all())
            if t is b.x:
                assert torch.equal(y2[keep], y[keep]) and not bool(torch.isfinite(y2[place]).all())
            t.copy_(old)


def test_zero_rows():
    b = Block(4, 8, 16, 8)
    grads = [torch.ones_like(t, dtype=torch.float32) for t in b.w]
    g = tgp.gated_grads(*[t.data_ptr() for t in grads])
    for overwrite in (False, True):
        tgp.gated_backward(b.shape, 0, b.weights, None, 8, None, 8, None, 8, g, overwrite, None, 0)
        torch.cuda.synchronize()
        assert all(bool((t == (0.0 if overwrite else 1.0)).all()) for t in grads)


@pytest.mark.parametrize("act", [0, 1])
def test_gradient_against_differences(act):
    """The gradient of sum(y dy), float32, against central differences of the 64-bit block along random directions:
    steps of 1e-4 leave 1e-8 of the third derivative, so what differs is the gradient's own error, FP32 of the
    products' magnitudes."""
    b = Block(30, 12, 20, 9, "fp32", act)
    x, dy, w = b.x.cpu().double(), b.dy.cpu().double(), [t.double() for t in b.host()]
    got = b.backward()
    g = torch.Generator().manual_seed(1)
    for k, t in enumerate([x] + w):
        d = torch.randn(t.shape, generator=g, dtype=torch.float64)
        two = []
        for h in (1e-4, -1e-4):
            args = [x] + list(w)
            args[k] = t + h * d
            two.append(float((ref.gated(args[0], args[1:], act) * dy).sum()))
        want = (two[0] - two[1]) / 2e-4
        have = float((got[k].cpu().double() * d).sum())
        size = float(torch.linalg.vector_norm(got[k].cpu().double()) * torch.linalg.vector_norm(d))
        assert abs(have - want) <= FP32 * size + 1e-6 * abs(want), (k, have, want)


def test_micro_batches_add_up():
    """Gradients of micro-batches, accumulated from the last to the first, are the full batch's."""
    b = Block(4 * 49, 48, 96, 40, "fp32", 1)
    per, m, n = 49, 4, tgp.gated_workspace(b.shape, 49, True)
    grads = [torch.full_like(t, 3.0) for t in b.w]
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dx = torch.empty_like(b.x)
    for i in range(m - 1, -1, -1):
        sl = slice(i * per, (i + 1) * per)
        tgp.gated_backward(b.shape, per, b.weights, b.dy[sl].data_ptr(), 40, b.x[sl].data_ptr(), 48, dx[sl].data_ptr(), 48,
                           tgp.gated_grads(*[t.data_ptr() for t in grads]), i == m - 1, ws.data_ptr(), n)
    torch.cuda.synchronize()
    want = ref.gated(b.x.cpu(), b.host(), 1, b.dy.cpu())
    assert all(ref.rel(a, c) <= FP32 for a, c in zip([dx] + grads, want))


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cin,hidden,cout", [(1, 64, 128, 64), (20, 65, 40, 33), (500, 64, 200, 72), (700, 48, 250, 64),
                                                  (144, 264, 1000, 300)])
def test_side_stream_and_graph(rows, cin, hidden, cout, dt):
    """On another stream, and captured: every replay gives the eager call's bits, with eager calls between."""
    b = Block(rows, cin, hidden, cout, dt)
    y, back = b.forward().clone(), [t.clone() for t in b.backward()]
    side = torch.cuda.Stream()
    assert torch.equal(b.forward(side.cuda_stream), y)
    assert all(torch.equal(p, q) for p, q in zip(b.backward(stream=side.cuda_stream), back))
    out = torch.empty(rows, cout, dtype=DT[dt][1], device="cuda")
    dx = torch.empty(rows, cin, dtype=DT[dt][1], device="cuda")
    grads = [torch.empty(t.shape, device="cuda") for t in b.w]
    n = tgp.gated_workspace(b.shape, rows, False), tgp.gated_workspace(b.shape, rows, True)
    ws = torch.empty(max(n), dtype=torch.uint8, device="cuda")
    g = tgp.gated_grads(*[t.data_ptr() for t in grads])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        tgp.gated_forward(b.shape, rows, b.weights, b.x.data_ptr(), b.ldx, out.data_ptr(), cout, ws.data_ptr(), n[0], s)
        tgp.gated_backward(b.shape, rows, b.weights, b.dy.data_ptr(), b.ldy, b.x.data_ptr(), b.ldx, dx.data_ptr(), cin, g,
                           True, ws.data_ptr(), n[1], s)
    for _ in range(3):
        for t in (out, dx, *grads):
            t.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, y) and all(torch.equal(p, q) for p, q in zip([dx] + grads, back))
        assert torch.equal(b.forward(), y)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("cin", [64, 27])
def test_rows_farther_apart_than_32_bits(cin, dt):
    """Rows whose byte offsets pass 2^32: three rows 1.2e9 elements apart, in and out."""
    say("gated, far rows", cin, dt)
    td = DT[dt][1]
    ld = 1_200_000_008 if dt == "bf16" else 600_000_004
    b = Block(3, cin, 40, cin, dt)
    want_y, want = b.forward().clone(), [t.clone() for t in b.backward()]
    buf = torch.empty(2 * ld + cin + 8, dtype=td, device="cuda")
    far = buf.as_strided((3, cin), (ld, 1))
    far.copy_(b.x)
    small = b.x
    b.x, b.ldx = far, ld
    assert torch.equal(b.forward(), want_y)
    n = tgp.gated_workspace(b.shape, 3, True)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    grads = [torch.empty(t.shape, device="cuda") for t in b.w]
    tgp.gated_backward(b.shape, 3, b.weights, b.dy.data_ptr(), b.ldy, buf.data_ptr(), ld, buf.data_ptr(), ld,
                       tgp.gated_grads(*[t.data_ptr() for t in grads]), True, ws.data_ptr(), n)
    torch.cuda.synchronize()
    assert torch.equal(far, want[0]) and all(torch.equal(p, q) for p, q in zip(grads, want[1:]))
    far.copy_(small)
    out = torch.empty(2 * ld + cin + 8, dtype=td, device="cuda")
    n = tgp.gated_workspace(b.shape, 3, False)
    tgp.gated_forward(b.shape, 3, b.weights, far.data_ptr(), ld, out.data_ptr(), ld, ws.data_ptr(), n)
    torch.cuda.synchronize()
    assert torch.equal(out.as_strided((3, cin), (ld, 1)), want_y)
