"""AdamW with 8-bit states against its 64-bit definition.

Codes and exponents are decided in float64 on both sides and have to be equal.
The weight: float32 of formulas with some ten roundings, m and v not stored in
between: 1e-6 of |w| and of the step's size; its bfloat16 copy is the rounding of
the float32 that is stored, exactly."""
import pytest
import torch

import block_ops_ref as ref
import paper_2004_09910_amd as tgp
from gpu_util import say

pytestmark = pytest.mark.gpu
K = dict(rate=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, decay=1e-4, step=7, seed=0x123456789abcdef)
FILL = 7.5


class State:
    """A list of tensors with guard values after each buffer; host copies beside them."""

    def __init__(self, sizes, half=True, seed=0, fresh=False, grads=None):
        g = torch.Generator().manual_seed(seed)
        self.sizes, self.half, self.t = sizes, half, []
        for k, n in enumerate(sizes):
            nb = -(-n // 128)
            grad = torch.randn(n, generator=g) * torch.exp(2 * torch.randn(n, generator=g)) * 10.0 ** -(k % 9)
            if grads is not None:
                grad = grads[k]
            w = torch.randn(n, generator=g)
            m = torch.randint(0, 256, (n,), generator=g).to(torch.uint8)
            m = torch.where((m & 127) == 127, m - 1, m)
            r = torch.randint(0, 127, (n,), generator=g).to(torch.uint8)
            e = torch.randint(90, 125, (nb, 2), generator=g).to(torch.uint8)
            if fresh:
                m, r, e = m * 0, r * 0, e * 0
            dev = {}
            for name, v, fill in (("w", w, FILL), ("grad", grad, FILL), ("m", m, 201), ("r", r, 202), ("e", e.view(-1), 203)):
                b = torch.full((v.numel() + 64,), fill, dtype=v.dtype, device="cuda")
                b[:v.numel()] = v.cuda()
                dev[name] = b
            if half:
                dev["w16"] = torch.full((n + 64,), FILL, dtype=torch.bfloat16, device="cuda")
            self.t.append((dict(w=w, grad=grad, m=m, r=r, e=e), dev))
        self.list = tgp.adamw8_tensors([
            (n, d["w"].data_ptr(), d["w16"].data_ptr() if half else None, d["grad"].data_ptr(), d["m"].data_ptr(),
             d["r"].data_ptr(), d["e"].data_ptr()) for n, (_, d) in zip(sizes, self.t)])

    def step(self, stream=0, **kw):
        a = dict(K, **kw)
        tgp.adamw8_step(self.list, a["rate"], a["beta1"], a["beta2"], a["eps"], a["decay"], a["step"], a["seed"], stream)

    def check(self, host=None, **kw):
        a = dict(K, **kw)
        torch.cuda.synchronize()
        for k, (n, (h, d)) in enumerate(zip(self.sizes, self.t)):
            w, m, r, e = ref.adamw8(h["w"], h["grad"], h["m"], h["r"], h["e"], k, **a)
            got = d["w"][:n].cpu()
            fine = torch.isfinite(w)
            tol = 1e-6 * (w.abs() + h["w"].double().abs() + a["rate"] * 4)
            assert bool(((got.double() - w).abs() <= tol)[fine].all()), (k, n)
            assert torch.equal(torch.isfinite(got), fine)
            assert torch.equal(d["m"][:n].cpu() & torch.where((m & 127) == 127, 127, 255).to(torch.uint8), m), (k, n)
            assert torch.equal(d["r"][:n].cpu(), r) and torch.equal(d["e"][:e.numel()].cpu().view(-1, 2), e), (k, n)
            if self.half:
                assert torch.equal(d["w16"][:n].cpu().nan_to_num(7.0), got.bfloat16().nan_to_num(7.0))
                assert bool((d["w16"][n:] == FILL).all())
            assert bool((d["w"][n:] == FILL).all() and (d["m"][n:] == 201).all() and (d["r"][n:] == 202).all())
            assert bool((d["e"][2 * -(-n // 128):] == 203).all())
            h.update(w=got, m=m, r=r, e=e)


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("sizes", [[1], [5], [127], [128], [129], [1000, 2048, 2049], [4096, 1, 130001], [7] * 120])
def test_steps(sizes, half):
    """Some steps one after the other, each from the states that the one before left."""
    say("adamw8", sizes[:4], half)
    s = State(sizes, half, seed=len(sizes) + sizes[0])
    for step in (7, 8, 9):
        s.step(step=step, seed=step * 77)
        s.check(step=step, seed=step * 77)


def test_fresh_states_and_first_step():
    s = State([300, 64, 2050], fresh=True)
    for step in (1, 2):
        s.step(step=step, decay=0.0)
        s.check(step=step, decay=0.0)


def test_betas_and_sizes_of_gradients():
    """From far under float32's squares to its largest values, and betas of 0."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn(640, generator=g)
    grads = [x * s for s in (1e-42, 1e-30, 1e-19, 1.0, 1e19, 1e30, 3e37)] + [x * 0, x * torch.exp(20 * torch.randn(640, generator=g))]
    for b1, b2 in ((0.9, 0.999), (0.0, 0.0), (0.5, 0.99999)):
        s = State([640] * len(grads), grads=grads, fresh=True)
        for step in (1, 2, 3):
            s.step(step=step, beta1=b1, beta2=b2, seed=step)
            s.check(step=step, beta1=b1, beta2=b2, seed=step)


def test_non_finite_gradients():
    """An infinity or NaN makes its own value NaN, its codes the NaN code, and nothing else."""
    x = torch.randn(400, generator=torch.Generator().manual_seed(5))
    x[3], x[150], x[399] = float("inf"), float("nan"), float("-inf")
    s = State([400], grads=[x], fresh=True)
    s.step()
    s.check()
    m, r = s.t[0][1]["m"][:400].cpu(), s.t[0][1]["r"][:400].cpu()
    bad = ~torch.isfinite(x)
    assert torch.equal((m & 127) == 127, bad) and torch.equal(r == 127, bad)
    assert torch.equal(torch.isnan(s.t[0][1]["w"][:400].cpu()), bad)


def test_rounding_is_unbiased():
    """Over seeds the mean of what is kept is the value: beta1 = beta2 = 0, so that m and v are g and g^2.
    With N seeds the mean is off by at most 5 standard deviations, half a code's distance / sqrt(N) each (a code's
    distance is an eighth of the value at most), and by the random bits' own 2^-17 of a distance."""
    x = torch.randn(4096, generator=torch.Generator().manual_seed(9)).abs() + 0.1
    seeds = 400
    sm, sr = torch.zeros(4096, dtype=torch.float64), torch.zeros(4096, dtype=torch.float64)
    s = State([4096], grads=[x], fresh=True)
    for k in range(seeds):
        s.step(beta1=0.0, beta2=0.0, rate=0.0, seed=k)
        d = s.t[0][1]
        e = d["e"][:64].cpu().view(-1, 2)
        sm += ref.adamw8_decode(d["m"][:4096].cpu(), e[:, 0])
        sr += ref.adamw8_decode(d["r"][:4096].cpu(), e[:, 1])
    for t in (sm, sr):
        off = (t / seeds / x.double() - 1).abs()
        assert float(off.max()) <= 5 * 0.125 / 2 / seeds ** 0.5
        assert float((t / seeds / x.double() - 1).mean().abs()) <= 5 * 0.125 / 2 / (seeds * 4096) ** 0.5


def test_states_that_change_by_less_than_a_code_move():
    """A gradient that has shrunk: root decays to it, as sqrt(v) of the float32 step does, though a step is a
    fiftieth of a code's distance."""
    n, beta2 = 4096, 0.99
    g = torch.full((n,), 1e-3)
    s = State([n], grads=[g], fresh=True)
    d = s.t[0][1]
    d["r"][:n], d["e"][1:64:2] = 0x70, 127    # 128 x 2^-7 = 1
    v = 1.0
    for step in range(1, 301):
        s.step(beta2=beta2, step=step, seed=step, rate=0.0)
        v = beta2 * v + (1 - beta2) * 1e-6
    got = ref.adamw8_decode(d["r"][:n].cpu(), d["e"][:64].cpu().view(-1, 2)[:, 1])
    # the mean root stays on its path but for what the spread adds: codes are 1/8 apart at most and the spread that
    # 1 / (1 - beta2) steps of rounding leave is under one distance, so root's mean is at most 1/8 of v^0.5 off
    assert abs(float(got.mean()) / v ** 0.5 - 1) <= 0.125, (float(got.mean()), v ** 0.5)


def test_list_is_its_tensors_and_places_matter():
    """A tensor's step depends on its place in the list by its random bits alone; the same call gives the same bits."""
    sizes = [3000, 3000]
    a, b = State(sizes, seed=1), State(sizes, seed=1)
    a.step()
    b.step()
    torch.cuda.synchronize()
    for (_, p), (_, q) in zip(a.t, b.t):
        assert all(torch.equal(p[k], q[k]) for k in p)
    x = torch.randn(3000, generator=torch.Generator().manual_seed(2))
    c = State(sizes, grads=[x, x], fresh=True)
    c.step(step=1)
    torch.cuda.synchronize()
    assert not torch.equal(c.t[0][1]["m"][:3000], c.t[1][1]["m"][:3000])


def test_side_stream_and_graph():
    """Captured, every replay takes one more step from the states it finds, as eager calls do."""
    sizes = [5000, 130, 2048]
    a, b = State(sizes, seed=4), State(sizes, seed=4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step(side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    a.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(torch.cuda.current_stream().cuda_stream)
    b.step()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        b.step()
        torch.cuda.synchronize()
        for (_, p), (_, q) in zip(a.t, b.t):
            assert all(torch.equal(p[k], q[k]) for k in p)


@pytest.mark.parametrize("place", [1, 5])
def test_more_tensors_than_a_launch_and_large_ones(place):
    sizes = [33] * 50 + [2048 * 300 + 77]
    s = State(sizes, seed=place)
    s.step()
    s.check()
