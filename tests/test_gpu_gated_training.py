"""GatedPipeline, the gated blocks, the norms around them and the 8-bit step put
together, against torch's float64 autograd of the same network on the CPU."""
import importlib.util
import math
import os

import pytest
import torch
import torch.nn.functional as F

import block_ops_ref as ref
from gpu_util import say
from paper_2004_09910_amd.training import GatedPipeline
from workloads import specs
from workloads.specs import BF16, CONV1X1, CONV3X3, DWCONV3X3, FP32, Layer, Net

pytestmark = pytest.mark.gpu
MATRICES = ("gate", "up", "down")


def _net():
    return Net("gated-tiny", (Layer(CONV3X3, 8, 16), Layer(DWCONV3X3, 16, 16, relu=False, bias=False),
                              Layer(CONV1X1, 16, 24), Layer(CONV3X3, 24, 8, relu=False)), 8, 12, 12)


def _norm(h, eps, gain, bias):
    mean = h.mean(1, keepdim=True)
    var = (h - mean).square().mean(1, keepdim=True)
    return (h - mean) / torch.sqrt(var + eps) * gain[:, None, None] + bias[:, None, None]


def _leaf(t):
    return None if t is None else t.double().cpu().requires_grad_()


def _reference(sess, x, target):
    """Output and leaves with their gradients by autograd in float64 (NCHW)."""
    P, norms, blocks = {}, [], []
    for idx, p in sess.params.items():
        L = sess.net.layers[idx]
        w = p["w"].double().cpu()
        w = w.reshape(L.cout, 1, 3, 3) if L.kind == DWCONV3X3 else w.permute(0, 3, 1, 2).contiguous()
        P[idx] = (w.requires_grad_(), _leaf(p["b"]))
    xin = x.double().cpu().permute(0, 3, 1, 2).contiguous().requires_grad_()
    h = xin
    for j, (lo, hi) in enumerate(sess.bounds):
        q = {k: _leaf(sess.norms[j][k]) for k in ("gain", "bias")}
        b = {k: _leaf(sess.blocks[j][k]) for k in MATRICES + sess.VECTORS}
        t = _norm(h, sess.eps, q["gain"], q["bias"])
        g, u = (F.conv2d(t, b[k][:, :, None, None], b["b_" + k]) for k in ("gate", "up"))
        a = F.silu(g) if sess.act == 0 else F.gelu(g)
        f = F.conv2d(a * u, b["down"][:, :, None, None], b["b_down"])
        r = h + b["scale"][:, None, None] * _norm(f, sess.eps, b["post_gain"], b["post_bias"])
        h = _norm(r, sess.eps, b["pre_gain"], b["pre_bias"])
        norms.append(q)
        blocks.append(b)
        for idx in range(lo, hi):
            L = sess.net.layers[idx]
            h = F.conv2d(h, P[idx][0], P[idx][1], padding=0 if L.kind == CONV1X1 else 1,
                         groups=L.cout if L.kind == DWCONV3X3 else 1)
            h = h.relu() if L.relu else h
    (h - target.double().cpu().permute(0, 3, 1, 2)).square().mean().backward()
    return h, xin, P, norms, blocks


def _close(got, want, what, tol=1e-4):
    e = ref.rel(got, want)
    assert e <= tol, (what, e)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("mode", [specs.CKPT_ALWAYS, specs.CKPT_NEVER])
def test_gradients_and_step_of_a_gated_pipeline(mode, act):
    """float32, three partitions, four micro-batches.  1e-4 of a gradient's norm: sums of at most a few hundred
    float32 terms in some 25 operators one after the other, each off by some 5e-6 of its norm at most."""
    say("gated pipeline, mode", mode, "act", act)
    torch.manual_seed(1)
    sess = GatedPipeline(_net(), FP32, n=3, ratio=3, act=act, scale=0.5, balance=[1, 2, 1])
    for q in sess.norms:
        q["gain"].copy_(1 + 0.2 * torch.randn_like(q["gain"]))
        q["bias"].copy_(0.2 * torch.randn_like(q["bias"]))
    for b in sess.blocks:
        for k in sess.VECTORS:
            b[k].add_(0.2 * torch.randn_like(b[k]))
    sess.plan(8, 4, mode)
    x = torch.randn(8, 12, 12, 8, device="cuda")
    t = torch.randn(8, 12, 12, 8, device="cuda")
    y64, x64, P, norms, blocks = _reference(sess, x, t)
    for repeat in range(2):       # the accumulators start anew
        y = sess.forward(x)
        dx = torch.empty_like(x)
        sess.backward((y - t) * (2.0 / y.numel()), dx)
    torch.cuda.synchronize()
    _close(y, y64.detach().permute(0, 2, 3, 1), "y")
    _close(dx, x64.grad.permute(0, 2, 3, 1), "dx")
    for idx, (w, b) in P.items():
        L = sess.net.layers[idx]
        _close(sess.params[idx]["dw"], w.grad.reshape(L.cout, 9) if L.kind == DWCONV3X3 else w.grad.permute(0, 2, 3, 1), idx)
        if b is not None:
            _close(sess.params[idx]["db"], b.grad, idx)
    for j in range(3):
        for k in ("gain", "bias"):
            _close(sess.norms[j]["d" + k], norms[j][k].grad, (j, k))
        for k in MATRICES + sess.VECTORS:
            _close(sess.blocks[j]["d_" + k], blocks[j][k].grad, (j, k))
    # the step of the blocks' tensors from these gradients: states and weights
    before = [{k: b["w_" + k].clone().cpu() for k in MATRICES + sess.VECTORS} for b in sess.blocks]
    sess.update(decay=0.01)
    torch.cuda.synchronize()
    place = 0
    for b, old in zip(sess.blocks, before):
        for k in MATRICES + sess.VECTORS:
            n = old[k].numel()
            zeros = torch.zeros(n, dtype=torch.uint8)
            # the call takes the rate and the decay as float32
            w, m, r, ex = ref.adamw8(old[k].reshape(-1), b["d_" + k].reshape(-1).cpu(), zeros, zeros,
                                     torch.zeros(-(-n // 128), 2, dtype=torch.uint8), place, 1e-3, 0.9, 0.95, 1e-8, 0.01, 1, 1)
            _close(b["w_" + k].reshape(-1), w, (place, k), 1e-6)
            assert torch.equal(b["m_" + k].cpu(), m) and torch.equal(b["root_" + k].cpu(), r), (place, k)
            assert torch.equal(b["exps_" + k].cpu().view(-1, 2), ex), (place, k)
            place += 1
    sess.close()


def test_bfloat16_weights_follow_their_masters():
    torch.manual_seed(2)
    sess = GatedPipeline(_net(), BF16, n=2, balance=[2, 2])
    sess.plan(4, 2, specs.CKPT_ALWAYS)
    x, t = (torch.randn(4, 12, 12, 8, device="cuda").bfloat16() for _ in range(2))
    first = [{k: b[k].clone() for k in MATRICES} for b in sess.blocks]
    for _ in range(3):
        sess.train_step(x, t)
    torch.cuda.synchronize()
    for b, f in zip(sess.blocks, first):
        for k in MATRICES:
            assert torch.equal(b[k], b["w_" + k].bfloat16()) and not torch.equal(b[k], f[k])
    sess.close()


def test_steps_on_a_side_stream():
    """The same three steps on the default stream and on another: every call takes the current stream, so nothing
    differs, bit by bit."""
    got = []
    for side in (False, True):
        torch.manual_seed(3)
        sess = GatedPipeline(_net(), BF16, n=2, balance=[1, 3])
        sess.plan(4, 2, specs.CKPT_EXCEPT_LAST)
        x, t = (torch.randn(4, 12, 12, 8, device="cuda").bfloat16() for _ in range(2))
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream() if side else torch.cuda.current_stream()):
            for _ in range(3):
                sess.train_step(x, t)
        torch.cuda.synchronize()
        got.append([b["w_" + k].clone() for b in sess.blocks for k in MATRICES + sess.VECTORS])
        sess.close()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_gradients_after_a_new_partition():
    torch.manual_seed(4)
    sess = GatedPipeline(_net(), FP32, n=1, balance=[4])
    sess.plan(8, 4, specs.CKPT_ALWAYS)
    x, t = (torch.randn(8, 12, 12, 8, device="cuda") for _ in range(2))
    sess.train_step(x, t)
    sess.balance_by_time(2, 3, specs.CKPT_ALWAYS)
    sess.plan(8, 4, specs.CKPT_ALWAYS)
    y64, x64, _, _, blocks = _reference(sess, x, t)
    y = sess.forward(x)
    dx = torch.empty_like(x)
    sess.backward((y - t) * (2.0 / y.numel()), dx)
    torch.cuda.synchronize()
    _close(y, y64.detach().permute(0, 2, 3, 1), "y")
    _close(dx, x64.grad.permute(0, 2, 3, 1), "dx")
    for j, b in enumerate(blocks):
        for k in MATRICES + sess.VECTORS:
            _close(sess.blocks[j]["d_" + k], b[k].grad, (j, k))
    sess.update()
    sess.close()


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_the_example_runs(dtype):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_norm_stack.py")
    spec = importlib.util.spec_from_file_location("train_norm_stack", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses = ex.train(3, dtype, log=None, gated=2)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
