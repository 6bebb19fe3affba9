"""Orthogonalised updates and the weights' step against their 64-bit definitions.

Tolerances, fixed before the first run.  momentum: two float32 roundings,
2^-23 of the sum of the terms' magnitudes.  update: bfloat16's rounding is
2^-9 of a value at most; products round their operands to float16, 2^-12 of
an entry, some three of them in each of five steps, each at most doubled by
the steps after it: 15 x 2 x 2^-12 / sqrt(3) if all added up, 4e-3 in norm.
UPDATE = 6e-3 is asked of matrices whose singular values span less than 2^6
(wide random ones, and eight directions with as much noise).  The step's
float32 formulas: a few roundings, 1e-6.
"""
import math

import pytest
import torch

import paper_2004_09910_amd as tgp
import train_ops_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu
UPDATE = 6e-3


def _grad(r, c, seed, strong=8, scale=1e-3):
    g = torch.Generator().manual_seed(seed)
    d = min(strong, r, c)
    u = torch.randn(r, d, generator=g) @ torch.randn(d, c, generator=g) / math.sqrt(max(d, 1))
    return scale * (u + torch.randn(r, c, generator=g))


def _guarded(n, dtype=torch.float32, fill=7.5):
    """n values with 64 guard values after them."""
    return torch.full((n + 64,), fill, dtype=dtype, device="cuda")


def _muon(mats, mu=0.95, nesterov=True, steps=5, eps=1e-7, stream=0, ws_fill=None):
    """mats: (grad, momentum or None).  Returns [(momentum, update)]."""
    dev, rows = [], []
    for g, m in mats:
        r, c = g.shape
        gd = g.cuda().contiguous()
        md = None
        if m is not None:
            md = _guarded(r * c)
            md[:r * c] = m.reshape(-1).cuda()
        o = _guarded(r * c, torch.bfloat16)
        dev.append((gd, md, o, r, c))
        rows.append((r, c, gd.data_ptr(), None if md is None else md.data_ptr(), o.data_ptr()))
    t = tgp.muon_tensors(rows)
    n = tgp.muon_workspace(t)
    ws = torch.full((n + 256,), 255 if ws_fill is None else ws_fill, dtype=torch.uint8, device="cuda")
    tgp.muon_update(t, mu, nesterov, steps, eps, ws.data_ptr(), n, stream)
    torch.cuda.synchronize()
    assert bool((ws[n:] == (255 if ws_fill is None else ws_fill)).all()), "past the workspace"
    out = []
    for gd, md, o, r, c in dev:
        assert bool((o[r * c:] == 7.5).all()), "past the update"
        assert md is None or bool((md[r * c:] == 7.5).all()), "past the momentum"
        out.append((None if md is None else md[:r * c].view(r, c), o[:r * c].view(r, c)))
    return out


SHAPES = [(1, 1), (1, 64), (64, 1), (3, 5), (16, 144), (27, 64), (64, 27), (64, 576), (65, 130), (100, 101),
          (128, 128), (128, 1152), (192, 1000), (256, 256), (300, 70), (513, 2000), (512, 4608),
          (1024, 256), (1, 5000), (5000, 3)]


@pytest.mark.parametrize("r,c", SHAPES)
def test_update_of_one_matrix(r, c):
    say("muon", r, c)
    g, m = _grad(r, c, r + 3 * c), 5 * _grad(r, c, r + 3 * c + 1)
    (mom, o), = _muon([(g, m)])
    mw, ow = ref.muon(g, m, 0.95, True, 5, 1e-7)
    assert float(((mom.cpu().double() - mw).abs() / (0.95 * m.double().abs() + g.double().abs())).max()) <= 2.0 ** -23
    assert ref.rel(o, ow) <= UPDATE
    (_, again), = _muon([(g, m)], ws_fill=0)
    assert torch.equal(o, again)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
@pytest.mark.parametrize("r,c", [(48, 100), (130, 640), (200, 200), (700, 90)])
def test_steps_momentum_and_none(r, c, steps):
    say("muon", r, c, "steps", steps)
    g, m = _grad(r, c, 5), _grad(r, c, 6)
    for mom, nesterov in ((m, True), (m, False), (None, True)):
        (mg, o), = _muon([(g, mom)], mu=0.9, nesterov=nesterov, steps=steps)
        mw, ow = ref.muon(g, mom, 0.9, nesterov, steps, 1e-7)
        assert ref.rel(o, ow) <= UPDATE
        if mom is not None:
            assert ref.rel(mg, mw) <= 2.0 ** -23


def test_singular_values_come_near_one():
    """Wide matrices of full rank: every singular value of the update in the rule's 0.68 .. 1.21."""
    for r, c in ((64, 576), (256, 2304), (300, 60)):
        (_, o), = _muon([(_grad(r, c, 9), None)])
        sv = torch.linalg.svdvals(o.cpu().double())
        assert 0.6 <= float(sv.min()) and float(sv.max()) <= 1.25, (r, c, float(sv.min()), float(sv.max()))


def test_list_of_all_sorts():
    """More matrices than a launch takes, of every size, each as by itself."""
    shapes = [(16, 144), (1, 64), (64, 64), (128, 300), (70, 33), (260, 520), (1, 1)] * 8
    mats = [(_grad(r, c, k, scale=10.0 ** -(k % 9)), _grad(r, c, k + 100)) for k, (r, c) in enumerate(shapes)]
    got = _muon(mats)
    for k in (0, 1, 4, 5, 6, 20, 30, 48, 55):
        (mom, o), = _muon([mats[k]])
        assert torch.equal(o, got[k][1]) and torch.equal(mom, got[k][0]), k


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 1e12, 1e30])
def test_sizes_of_gradients(scale):
    """The update does not depend on the gradient's size, from far under float32's squares to far over
    them (eps = 0)."""
    g = _grad(96, 200, 3, scale=1.0)
    (_, o), = _muon([(g * scale, None)], eps=0.0)
    _, ow = ref.muon(g * scale, None, 0.95, True, 5, 0.0)
    assert ref.rel(o, ow) <= UPDATE


@pytest.mark.parametrize("r,c", [(40, 90), (300, 700), (700, 300)])
def test_zero_and_non_finite(r, c):
    """A zero matrix stays zero; one bad value spoils its own matrix only."""
    g = _grad(r, c, 4)
    for eps in (0.0, 1e-7):
        (_, o), = _muon([(torch.zeros(r, c), None)], eps=eps)
        assert bool((o == 0).all())
    for v in (float("nan"), float("inf"), -float("inf")):
        bad = g.clone()
        bad[r // 2, c // 3] = v
        (_, a), (_, b), (_, d) = _muon([(g, None), (bad, None), (g, None)])
        assert bool(torch.isnan(b.float()).all())
        assert torch.equal(a, d) and bool(torch.isfinite(a.float()).all())


def test_rank_one():
    """A gradient of one direction is that direction's update: u v^T at the one singular value's image.
    What float16 leaves of the other directions (2^-12 of the entries, times 3.4445^5 = 485 through the
    steps, spread over m of them) stays under 0.15 of it in norm."""
    r, c = 128, 512
    gen = torch.Generator().manual_seed(8)
    u, v = torch.randn(r, 1, generator=gen), torch.randn(1, c, generator=gen)
    (_, o), = _muon([(u @ v, None)])
    _, ow = ref.muon(u @ v, None, 0.95, True, 5, 1e-7)
    assert ref.rel(o, ow) <= 0.15


def test_muon_side_stream_and_graph():
    shapes = [(16, 144), (64, 576), (256, 512), (300, 100)]
    g = [_grad(r, c, k).cuda() for k, (r, c) in enumerate(shapes)]
    m0 = [_grad(r, c, k + 9).cuda() for k, (r, c) in enumerate(shapes)]
    m = [t.clone() for t in m0]
    o = [torch.empty(r, c, dtype=torch.bfloat16, device="cuda") for r, c in shapes]
    t = tgp.muon_tensors([(r, c, a.data_ptr(), b.data_ptr(), d.data_ptr())
                          for (r, c), a, b, d in zip(shapes, g, m, o)])
    n = tgp.muon_workspace(t)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def reset():
        for a, b, d in zip(m, m0, o):
            a.copy_(b)
            d.zero_()

    tgp.muon_update(t, 0.95, True, 5, 1e-7, ws.data_ptr(), n)
    torch.cuda.synchronize()
    want = [x.clone() for x in m + o]
    reset()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    tgp.muon_update(t, 0.95, True, 5, 1e-7, ws.data_ptr(), n, s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, m + o))
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tgp.muon_update(t, 0.95, True, 5, 1e-7, ws.data_ptr(), n, torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        reset()
        ws.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, m + o))


@pytest.mark.parametrize("r,c", [(32, 512), (32, 513), (511, 30), (514, 31), (64, 256), (257, 64), (50, 250), (33, 255),
                                 (1728, 30), (64, 864), (16, 1616), (1616, 16)])
def test_update_of_middling_matrices(r, c):
    """On both sides of where one block does a matrix alone."""
    say("muon", r, c)
    g, m = _grad(r, c, r + c), _grad(r, c, 2 * r + c)
    for mom, steps in ((m, 5), (m, 2), (None, 5)):
        (mg, o), = _muon([(g, mom)], steps=steps)
        mw, ow = ref.muon(g, mom, 0.95, True, steps, 1e-7)
        assert ref.rel(o, ow) <= UPDATE
        assert mom is None or ref.rel(mg, mw) <= 2.0 ** -23
    bad = g.clone()
    bad[r // 2, c // 3] = float("nan")
    (_, a), (_, b), (_, d) = _muon([(g, m), (bad, m), (g, m)])
    assert bool(torch.isnan(b.float()).all()) and torch.equal(a, d)
    (_, z), = _muon([(torch.zeros(r, c), None)])
    assert bool((z == 0).all())


@pytest.mark.parametrize("r,c", [(64, 576), (64, 1100), (1100, 64), (128, 640), (256, 1100), (1100, 500)])
def test_two_levels_of_singular_values(r, c):
    """Half of the singular values 20 times the others, a span of 2^4.3: UPDATE, whatever tile an element lies in."""
    say("muon, two levels", r, c)
    gen = torch.Generator().manual_seed(r + c)
    n = min(r, c)
    u, v = (torch.linalg.qr(torch.randn(k, n, generator=gen, dtype=torch.float64))[0] for k in (r, c))
    s = torch.where(torch.arange(n) < n // 2, 1.0, 0.05).double()
    g = ((u * s) @ v.T).float()
    for steps in (4, 5):
        (_, o), = _muon([(g, None)], steps=steps)
        _, ow = ref.muon(g, None, 0.95, True, steps, 1e-7)
        e = ref.rel(o, ow)
        say(steps, "%.1e" % e)
        assert e <= UPDATE


SIZES = [0, 1, 3, 4, 7, 64, 1000, 1024, 1025, 40001, 300000]


@pytest.mark.parametrize("half", [False, True])
def test_weight_step(half):
    gen = torch.Generator().manual_seed(2)
    sizes = SIZES * 6                       # more than a launch takes
    rows, keep = [], []
    for k, n in enumerate(sizes):
        w0 = torch.randn(n, generator=gen)
        o0 = torch.randn(n, generator=gen).bfloat16()
        w = _guarded(n)
        w[:n] = w0.cuda()
        w16 = _guarded(n, torch.bfloat16) if half else None
        o = o0.cuda() if n else torch.zeros(8, dtype=torch.bfloat16, device="cuda")
        rate = 0.01 * (k % 5)
        rows.append((n, w.data_ptr(), w16.data_ptr() if half else None, o.data_ptr(), rate))
        keep.append((w0, o0, w, w16, o, rate))
    tgp.weight_step(tgp.step_tensors(rows), 0.01)
    torch.cuda.synchronize()
    for n, (w0, o0, w, w16, _, rate) in zip(sizes, keep):
        want = ref.weight_step(w0, o0, rate, 0.01)
        assert bool((w[n:] == 7.5).all())
        if n:
            mag = w0.double().abs() + rate * o0.double().abs() + 1e-30
            assert float(((w[:n].cpu().double() - want).abs() / mag).max()) <= 1e-6
        if half:
            assert torch.equal(w16[:n], w[:n].bfloat16()) and bool((w16[n:] == 7.5).all())


@pytest.mark.parametrize("step", [1, 10, 100000])
@pytest.mark.parametrize("half", [False, True])
def test_adamw_step(half, step):
    gen = torch.Generator().manual_seed(3)
    rows, keep = [], []
    sizes = SIZES * 6
    for n in sizes:
        w0, g0, m0 = (torch.randn(n, generator=gen) * s for s in (1.0, 1e-2, 1e-2))
        v0 = 1e-4 * torch.rand(n, generator=gen)
        dev = []
        for t in (w0, g0, m0, v0):
            b = _guarded(n)
            b[:n] = t.cuda()
            dev.append(b)
        w16 = _guarded(n, torch.bfloat16) if half else None
        rows.append((n, dev[0].data_ptr(), w16.data_ptr() if half else None, dev[1].data_ptr(),
                     dev[2].data_ptr(), dev[3].data_ptr()))
        keep.append(((w0, g0, m0, v0), dev, w16))
    tgp.adamw_step(tgp.adamw_tensors(rows), 1e-2, 0.9, 0.99, 1e-8, 1e-3, step)
    torch.cuda.synchronize()
    for n, ((w0, g0, m0, v0), dev, w16) in zip(sizes, keep):
        w, m, v = ref.adamw(w0, g0, m0, v0, 1e-2, 0.9, 0.99, 1e-8, 1e-3, step)
        for b in dev:
            assert bool((b[n:] == 7.5).all())
        assert ref.rel(dev[0][:n], w) <= 1e-6 and ref.rel(dev[2][:n], m) <= 1e-6 and ref.rel(dev[3][:n], v) <= 1e-6
        if half:
            assert torch.equal(w16[:n], dev[0][:n].bfloat16()) and bool((w16[n:] == 7.5).all())


def test_bfloat16_copies_round_to_even_and_keep_nan():
    vals = [1.0, 1.00390625, 1.01171875, -1.00390625, float("inf"), -float("inf"), float("nan"), 3.4e38, 0.0, 1e-40]
    n = len(vals)
    w = torch.tensor(vals, device="cuda")
    o = torch.zeros(16, dtype=torch.bfloat16, device="cuda")
    w16 = torch.zeros(16, dtype=torch.bfloat16, device="cuda")
    tgp.weight_step(tgp.step_tensors([(n, w.data_ptr(), w16.data_ptr(), o.data_ptr(), 0.5)]), 0.0)
    torch.cuda.synchronize()
    want = torch.tensor(vals).bfloat16()
    got = w16[:n].cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(got[ok], want[ok]) and bool((w16[n:] == 0).all())


def test_failed_launches_are_reported():
    """A launch that fails (injected) ends the call with EHIP; the next call is whole."""
    g = _grad(200, 300, 1)
    (_, want), = _muon([(g, None)])
    gd = g.cuda()
    o = torch.empty(200, 300, dtype=torch.bfloat16, device="cuda")
    t = tgp.muon_tensors([(200, 300, gd.data_ptr(), None, o.data_ptr())])
    n = tgp.muon_workspace(t)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for k in (1, 2, 4):
        tgp.debug_fail_launch(k)
        with pytest.raises(tgp.TgpError) as e:
            tgp.muon_update(t, 0.95, True, 5, 1e-7, ws.data_ptr(), n)
        assert e.value.status == tgp.EHIP and "muon_update" in tgp.last_error()
        tgp.debug_fail_launch(0)
    tgp.muon_update(t, 0.95, True, 5, 1e-7, ws.data_ptr(), n)
    torch.cuda.synchronize()
    assert torch.equal(o, want)
    tgp.debug_fail_launch(1)
    with pytest.raises(tgp.TgpError):
        tgp.weight_step(tgp.step_tensors([(64, gd.data_ptr(), None, o.data_ptr(), 0.0)]), 0.0)
    tgp.debug_fail_launch(0)


@pytest.mark.parametrize("r,c", [(4096, 131072), (131000, 4001)])
def test_matrices_of_half_a_billion_values(r, c):
    """Offsets that pass 32 bits.  A matrix of signs u v^T is one singular direction, whose value 1 one step
    takes to a + b + c = 0.7010: every entry becomes its sign times 0.7010 / sqrt(r c), within bfloat16's
    rounding and float16's of a few products (2^-8 + 2^-9)."""
    say("muon", r, c)
    g = torch.Generator(device="cuda").manual_seed(1)
    u = torch.randint(0, 2, (r, 1), device="cuda", generator=g, dtype=torch.int8) * 2 - 1
    v = torch.randint(0, 2, (1, c), device="cuda", generator=g, dtype=torch.int8) * 2 - 1
    grad = (u * v).float()
    o = torch.empty(r, c, dtype=torch.bfloat16, device="cuda")
    t = tgp.muon_tensors([(r, c, grad.data_ptr(), None, o.data_ptr())])
    n = tgp.muon_workspace(t)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    tgp.muon_update(t, 0.0, False, 1, 0.0, ws.data_ptr(), n)
    torch.cuda.synchronize()
    want = sum(ref.NS) / math.sqrt(r * c)
    off = (o.float() * grad / want - 1).abs().max().item()
    assert off <= 2.0 ** -8 + 2.0 ** -9, off


def test_weight_step_past_32_bits():
    """Two billion values: more bytes than 32 bits count, more blocks than a launch takes."""
    n = (1 << 31) + 4099
    w = torch.ones(n, device="cuda")
    o = torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda")
    o[-1], o[1 << 31] = 1.0, 2.0
    tgp.weight_step(tgp.step_tensors([(n, w.data_ptr(), None, o.data_ptr(), 0.25)]), 0.0)
    torch.cuda.synchronize()
    assert w[-1].item() == 0.75 and w[1 << 31].item() == 0.5
    w[-1] = w[1 << 31] = 0.875
    assert bool((w == 0.875).all())


# Of matrices whose singular values are anything, what is left (as parts of the update's norm): bfloat16's rounding
# of the result, 2^-9 / sqrt(3) x 1.5 = 1.7e-3; float16's of the products' left operands, which turns X by at most
# |E P^-1| a product, E being 2^-12 / sqrt(3) of P's entries: 1.4e-4 x a^2 / 0.68 = 2.4e-3 for two steps at once, twice;
# of X where two steps are left, times their a^2 in directions that U lacks: 1.4e-4 x 11.9 = 1.7e-3; and of X before
# that, where P's diagonal stands for P (three steps left): half of 1.4e-4 x a^3 = 2.9e-3 at most.  In quadrature 5.1e-3;
# the sum of the largest two and half the others, 8e-3, is asked.
ANY_SPECTRUM = 8e-3


def _spectrum(kind, m, n, gen):
    """A matrix of m x n with the singular values that `kind` names, in random directions."""
    def ortho(k):
        return torch.linalg.qr(torch.randn(k, min(k, min(m, n)), generator=gen, dtype=torch.float64))[0]

    r = min(m, n)
    k = torch.arange(r, dtype=torch.float64)
    if kind == "cells":     # four rows at a time are one direction
        g = torch.zeros(m, n, dtype=torch.float64)
        for i in range(0, m, 4):
            g[i:i + 4] = torch.randn(min(4, m - i), 1, generator=gen, dtype=torch.float64) @ torch.randn(
                1, n, generator=gen, dtype=torch.float64)
        return g.float()
    if kind == "rows":      # half of the rows are zero
        g = torch.randn(m, n, generator=gen)
        g[::2] = 0
        return g
    s = {"flat": k * 0 + 1, "squares": (k + 1) ** -2, "decades": 10.0 ** (-4 * k / max(r - 1, 1)),
         "2^9": 2.0 ** (-9 * k / max(r - 1, 1)), "2^11": 2.0 ** (-11 * k / max(r - 1, 1)),
         "2^14": 2.0 ** (-14 * k / max(r - 1, 1)), "one of 2000": torch.where(k == 0, 2000.0, 1.0).double(),
         "rank 1": (k < 1).double(), "rank 8": (k < 8).double(), "half rank": (k < (r + 1) // 2).double()}[kind]
    return ((ortho(m) * s) @ ortho(n).T).float()


@pytest.mark.parametrize("kind", ["flat", "squares", "decades", "2^9", "2^11", "2^14", "one of 2000", "rank 1", "rank 8",
                                  "half rank", "cells", "rows"])
def test_any_spectrum(kind):
    """By one block (up to 64 rows), by tiles one step at a time and two, whole and transposed, and a list of all."""
    shapes = [(16, 144), (30, 32), (64, 256), (64, 64), (200, 60), (256, 256), (300, 500), (64, 576), (130, 700),
              (256, 2304), (1152, 128)]
    gen = torch.Generator().manual_seed(len(kind) * 7 + ord(kind[0]))
    mats = [(_spectrum(kind, r, c, gen), None) for r, c in shapes]
    got = _muon(mats)
    for (g, _), (_, o), (r, c) in zip(mats, got, shapes):
        _, ow = ref.muon(g, None, 0.95, True, 5, 1e-7)
        e = ref.rel(o, ow)
        say(kind, r, c, "%.1e" % e)
        assert e <= ANY_SPECTRUM


@pytest.mark.parametrize("steps", [3, 4, 6, 7])
@pytest.mark.parametrize("kind", ["squares", "rank 1", "half rank", "flat"])
def test_any_spectrum_of_other_steps(kind, steps):
    """As above; with each step beyond five what X's rounding left out is multiplied by a or a^2 once more where P is
    near one, which turns X by up to 1.4e-4 x a^2: twice the tolerance."""
    gen = torch.Generator().manual_seed(steps)
    shapes = [(24, 200), (64, 200), (250, 250), (128, 640), (640, 128)]
    mats = [(_spectrum(kind, r, c, gen), None) for r, c in shapes]
    for (g, _), (_, o), (r, c) in zip(mats, _muon(mats, steps=steps), shapes):
        _, ow = ref.muon(g, None, 0.95, True, steps, 1e-7)
        e = ref.rel(o, ow)
        say(kind, r, c, steps, "%.1e" % e)
        assert e <= ANY_SPECTRUM * (1 if steps < 6 else 2)


def _muon64(grad, momentum, steps):
    """The definition in 64 bits on the device (plain products; contiguous operands)."""
    m = 0.95 * momentum.double() + grad.double()
    u = grad.double() + 0.95 * m
    x = u.T.contiguous() if u.shape[0] > u.shape[1] else u
    x = x / (torch.linalg.vector_norm(x) + 1e-7)
    for _ in range(steps):
        a = x @ x.T.contiguous()
        x = ref.NS[0] * x + (ref.NS[1] * a + ref.NS[2] * (a @ a)) @ x
    return m, (x.T if u.shape[0] > u.shape[1] else x)


@pytest.mark.parametrize("shapes", [
    # P X in tiles of 128 columns, two steps at a time and one
    [(1024, 4096)], [(1024, 2600), (700, 2000)], [(2048, 2048)],
    # P in more blocks than two a CU
    [(2500, 2100)],
    # P X in tiles of 192 columns, X X^T in ranges of tiles of 64 x 64 or (2048 x 18432) 128 x 128
    [(1024, 9216)], [(9216, 1024)], [(2048, 18432)],
    # X X^T whole in tiles of 128 x 128, P X one step at a time in tiles of 192; all sorts in one list
    [(4096, 4100), (300, 5000), (40, 40), (1000, 1001)],
], ids=lambda s: "+".join("%dx%d" % t for t in s))
@pytest.mark.parametrize("strong", [8, 0])
def test_large_matrices(shapes, strong):
    """Every kind of tile with all five steps: eight strong directions in noise (UPDATE), and of rank 8
    (ANY_SPECTRUM)."""
    say("muon, large", shapes, strong)
    g = torch.Generator(device="cuda").manual_seed(len(shapes) + strong)

    def grad(r, c):
        d = min(8, r, c)
        t = torch.randn(r, d, device="cuda", generator=g) @ torch.randn(d, c, device="cuda", generator=g) / math.sqrt(8)
        return 1e-3 * (t + torch.randn(r, c, device="cuda", generator=g) if strong else t)

    grads, moms = [grad(r, c) for r, c in shapes], [5 * grad(r, c) for r, c in shapes]
    if not strong:
        moms = [-2 * t for t in grads]      # the same eight directions
    news = [t.clone() for t in moms]
    out = [torch.empty(r, c, dtype=torch.bfloat16, device="cuda") for r, c in shapes]
    t = tgp.muon_tensors([(r, c, a.data_ptr(), b.data_ptr(), o.data_ptr())
                          for (r, c), a, b, o in zip(shapes, grads, news, out)])
    n = tgp.muon_workspace(t)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for steps in (5, 2):
        for a, b in zip(news, moms):
            a.copy_(b)
        tgp.muon_update(t, 0.95, True, steps, 1e-7, ws.data_ptr(), n)
        torch.cuda.synchronize()
        for a, b, m, o in zip(grads, moms, news, out):
            mw, ow = _muon64(a, b, steps)
            e = float(torch.linalg.vector_norm(o.double() - ow) / torch.linalg.vector_norm(ow))
            say(tuple(a.shape), steps, "%.1e" % e)
            assert float(torch.linalg.vector_norm(m.double() - mw) / torch.linalg.vector_norm(mw)) <= 2.0 ** -22
            assert e <= (UPDATE if strong else ANY_SPECTRUM)
            del mw, ow


def test_long_lists_share_their_workspace():
    """More tiled matrices than a list takes, of sizes that lie differently in each list's workspace, with
    whole ones among them: every matrix as by itself, twice over in one workspace."""
    shapes = [(128, 300), (300, 128), (64, 700), (260, 520), (16, 144), (130, 130), (90, 200), (500, 65), (64, 64)] * 6
    mats = [(_grad(r, c, k, scale=10.0 ** -(k % 5)), _grad(r, c, k + 100)) for k, (r, c) in enumerate(shapes)]
    got = _muon(mats)
    again = _muon(mats, ws_fill=0)
    for k, (a, b) in enumerate(zip(got, again)):
        assert torch.equal(a[1], b[1]) and torch.equal(a[0], b[0]), k
    for k in range(0, len(mats), 5):
        (mom, o), = _muon([mats[k]])
        assert torch.equal(o, got[k][1]) and torch.equal(mom, got[k][0]), k
