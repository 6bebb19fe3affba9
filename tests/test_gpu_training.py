"""The stage tasks, the norms between them and the update, put together
(paper_2004_09910_amd/training.py), against torch's float64 autograd of the
same network on the CPU, and a run whose loss falls."""
import math

import pytest
import torch
import torch.nn.functional as F

import train_ops_ref as ref
from gpu_util import say
from paper_2004_09910_amd.training import NormPipeline
from workloads import specs
from workloads.specs import BF16, CONV1X1, CONV3X3, DWCONV3X3, FP32, Layer, Net

pytestmark = pytest.mark.gpu


def _net():
    return Net("norm-tiny", (Layer(CONV3X3, 8, 16), Layer(DWCONV3X3, 16, 16, relu=False, bias=False),
                             Layer(CONV1X1, 16, 24), Layer(CONV3X3, 24, 8, relu=False)), 8, 12, 12)


def _reference(sess, x, target):
    """Loss, output and gradients by autograd in float64 (NCHW)."""
    P, leaves = {}, []
    for idx, p in sess.params.items():
        L = sess.net.layers[idx]
        w = p["w"].double().cpu()
        w = w.reshape(L.cout, 1, 3, 3) if L.kind == DWCONV3X3 else w.permute(0, 3, 1, 2).contiguous()
        w.requires_grad_()
        b = None if p["b"] is None else p["b"].double().cpu().requires_grad_()
        P[idx] = (w, b)
    N = [(q["gain"].double().cpu().requires_grad_(), q["bias"].double().cpu().requires_grad_()) for q in sess.norms]
    xin = x.double().cpu().permute(0, 3, 1, 2).contiguous().requires_grad_()
    h = xin
    for j, (lo, hi) in enumerate(sess.bounds):
        mean = h.mean(1, keepdim=True)
        var = (h - mean).square().mean(1, keepdim=True)
        h = (h - mean) / torch.sqrt(var + sess.eps) * N[j][0][:, None, None] + N[j][1][:, None, None]
        for idx in range(lo, hi):
            L = sess.net.layers[idx]
            h = F.conv2d(h, P[idx][0], P[idx][1], padding=0 if L.kind == CONV1X1 else 1,
                         groups=L.cout if L.kind == DWCONV3X3 else 1)
            h = h.relu() if L.relu else h
    t = target.double().cpu().permute(0, 3, 1, 2)
    loss = (h - t).square().mean()
    loss.backward()
    return loss.item(), h, xin, P, N


@pytest.mark.parametrize("mode", [specs.CKPT_ALWAYS, specs.CKPT_EXCEPT_LAST, specs.CKPT_NEVER])
def test_gradients_of_a_normalised_pipeline(mode):
    """float32, three partitions, four micro-batches.  Sums of a few hundred float32 terms in each of
    four layers and three norms: 1e-4 of a gradient's norm, as the parity tests ask of float32 runs."""
    say("normalised pipeline, mode", mode)
    torch.manual_seed(1)
    sess = NormPipeline(_net(), FP32, n=3, balance=[1, 2, 1])
    for q in sess.norms:
        q["gain"].copy_(1 + 0.2 * torch.randn_like(q["gain"]))
        q["bias"].copy_(0.2 * torch.randn_like(q["bias"]))
    sess.plan(8, 4, mode)
    x = torch.randn(8, 12, 12, 8, device="cuda")
    t = torch.randn(8, 12, 12, 8, device="cuda")
    loss, y64, x64, P, N = _reference(sess, x, t)
    y = sess.forward(x)
    dx = torch.empty_like(x)
    sess.backward((y - t) * (2.0 / y.numel()), dx)
    torch.cuda.synchronize()
    assert ref.rel(y, y64.detach().permute(0, 2, 3, 1)) <= 1e-4
    assert ref.rel(dx, x64.grad.permute(0, 2, 3, 1)) <= 1e-4
    for idx, (w, b) in P.items():
        L = sess.net.layers[idx]
        want = w.grad.reshape(L.cout, 9) if L.kind == DWCONV3X3 else w.grad.permute(0, 2, 3, 1)
        assert ref.rel(sess.params[idx]["dw"], want) <= 1e-4, idx
        if b is not None:
            assert ref.rel(sess.params[idx]["db"], b.grad) <= 1e-4, idx
    for q, (gain, bias) in zip(sess.norms, N):
        assert ref.rel(q["dgain"], gain.grad) <= 1e-4 and ref.rel(q["dbias"], bias.grad) <= 1e-4
    # the update of every parameter from these gradients
    before = {idx: (p["master"].clone(), None if p["b"] is None else p["b"].clone()) for idx, p in sess.params.items()}
    sess.update()
    torch.cuda.synchronize()
    for idx, p in sess.params.items():
        w0, b0 = before[idx]
        g = p["dw"].double().cpu()
        if sess.net.layers[idx].kind == DWCONV3X3:
            want = ref.adamw(w0.cpu(), g, torch.zeros(1), torch.zeros(1), 1e-3, 0.9, 0.95, 1e-8, 0.0, 1)[0]
            assert ref.rel(p["master"], want) <= 1e-6
        else:
            r, c = w0.shape[0], w0.numel() // w0.shape[0]
            o = ref.muon(g.reshape(r, c), torch.zeros(r, c), 0.95, True, 5, 1e-7)[1].reshape(w0.shape)
            step = p["master"].double().cpu() - w0.double().cpu() * (1 - sess.decay)
            # the update's tolerance (test_gpu_weight_update.py), and float32's of the weights beside it
            assert ref.rel(step, -0.02 * math.sqrt(max(1.0, r / c)) * o) <= 6e-3 + 1e-4
        if b0 is not None:
            want = ref.adamw(b0.cpu(), p["db"].cpu(), torch.zeros(1), torch.zeros(1), 1e-3, 0.9, 0.95, 1e-8, 0.0, 1)[0]
            assert ref.rel(p["b"], want) <= 1e-6
    sess.close()


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_training_lowers_the_loss(dtype):
    """The example's task in both types: the mean loss of the last five of 30 steps is under half of that
    of the first two."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_norm_stack.py")
    spec = importlib.util.spec_from_file_location("train_norm_stack", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    losses = ex.train(30, dtype, log=None)
    say("losses", [round(v, 3) for v in losses])
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-5:]) / 5 < 0.5 * sum(losses[:2]) / 2


def test_bfloat16_weights_follow_their_masters():
    torch.manual_seed(2)
    sess = NormPipeline(_net(), BF16, n=2, balance=[2, 2])
    sess.plan(4, 2, specs.CKPT_ALWAYS)
    x = torch.randn(4, 12, 12, 8, device="cuda").bfloat16()
    t = torch.randn(4, 12, 12, 8, device="cuda").bfloat16()
    for _ in range(3):
        sess.train_step(x, t)
    torch.cuda.synchronize()
    for p in sess.params.values():
        assert torch.equal(p["w"], p["master"].bfloat16())
    sess.close()


def test_gradients_after_a_new_partition():
    """balance_by_time between two steps, to more partitions: outputs and the norms' gradients are those of the
    new partition's network (tolerance as above)."""
    torch.manual_seed(3)
    sess = NormPipeline(_net(), FP32, n=1, balance=[4])
    sess.plan(8, 4, specs.CKPT_ALWAYS)
    x, t = (torch.randn(8, 12, 12, 8, device="cuda") for _ in range(2))
    sess.train_step(x, t)
    for n in (4, 2):
        sess.balance_by_time(2, n, specs.CKPT_ALWAYS)
        sess.plan(8, 4, specs.CKPT_ALWAYS)
        say("partition", sess.balance)
        _, y64, x64, _, N = _reference(sess, x, t)
        y = sess.forward(x)
        dx = torch.empty_like(x)
        sess.backward((y - t) * (2.0 / y.numel()), dx)
        torch.cuda.synchronize()
        assert ref.rel(y, y64.detach().permute(0, 2, 3, 1)) <= 1e-4
        assert ref.rel(dx, x64.grad.permute(0, 2, 3, 1)) <= 1e-4
        for q, (gain, bias) in zip(sess.norms, N):
            assert ref.rel(q["dgain"], gain.grad) <= 1e-4 and ref.rel(q["dbias"], bias.grad) <= 1e-4
        sess.update()
    sess.close()


def _reference_skips(sess, x, gout):
    """As _reference, of a network with pools and skips, from the output's gradient: output, input, layers'
    (weight, bias) and norms, with their gradients."""
    P, N, skips = {}, [], {}
    for idx, p in sess.params.items():
        L = sess.net.layers[idx]
        w = p["w"].double().cpu()
        w = w.reshape(L.cout, 1, 3, 3) if L.kind == DWCONV3X3 else w.permute(0, 3, 1, 2).contiguous()
        P[idx] = (w.requires_grad_(), None if p["b"] is None else p["b"].double().cpu().requires_grad_())
    for q in sess.norms:
        N.append(tuple(q[k].double().cpu().requires_grad_() for k in ("gain", "bias")))
    xin = x.double().cpu().permute(0, 3, 1, 2).contiguous().requires_grad_()
    h = xin
    for (lo, hi), (gain, bias) in zip(sess.bounds, N):
        mean = h.mean(1, keepdim=True)
        var = (h - mean).square().mean(1, keepdim=True)
        h = (h - mean) / torch.sqrt(var + sess.eps) * gain[:, None, None] + bias[:, None, None]
        for idx in range(lo, hi):
            L = sess.net.layers[idx]
            if L.prologue == specs.PRO_MAXPOOL2:
                h = F.max_pool2d(h, 2)
            elif L.prologue == specs.PRO_UPCAT2:
                h = torch.cat((F.interpolate(h, scale_factor=2, mode="nearest"), skips[L.pop_id]), 1)
            h = F.conv2d(h, P[idx][0], P[idx][1], padding=0 if L.kind == CONV1X1 else 1,
                         groups=L.cout if L.kind == DWCONV3X3 else 1)
            h = h.relu() if L.relu else h
            if L.stash_id >= 0:
                skips[L.stash_id] = h
    h.backward(gout.double().cpu().permute(0, 3, 1, 2))
    return h, xin, P, N


def _compare_skips(sess, x, dy, tol):
    h, xin, P, N = _reference_skips(sess, x, dy)
    y = sess.forward(x)
    dx = torch.empty_like(x)
    sess.backward(dy, dx)
    torch.cuda.synchronize()
    assert ref.rel(y, h.detach().permute(0, 2, 3, 1)) <= tol
    assert ref.rel(dx, xin.grad.permute(0, 2, 3, 1)) <= tol
    for idx, (w, b) in P.items():
        L = sess.net.layers[idx]
        want = w.grad.reshape(L.cout, 9) if L.kind == DWCONV3X3 else w.grad.permute(0, 2, 3, 1)
        assert ref.rel(sess.params[idx]["dw"], want) <= tol, idx
        if b is not None:
            assert ref.rel(sess.params[idx]["db"], b.grad) <= tol, idx
    for q, (gain, bias) in zip(sess.norms, N):
        assert ref.rel(q["dgain"], gain.grad) <= tol and ref.rel(q["dbias"], bias.grad) <= tol


def _skip_net():
    return Net("norm-unet", (Layer(CONV3X3, 8, 16, stash_id=0),
                             Layer(CONV3X3, 16, 24, prologue=specs.PRO_MAXPOOL2),
                             Layer(CONV3X3, 24, 24),
                             Layer(CONV3X3, 40, 16, prologue=specs.PRO_UPCAT2, pop_id=0),
                             Layer(CONV1X1, 16, 8, relu=False)), 8, 12, 12)


@pytest.mark.parametrize("mode", [specs.CKPT_ALWAYS, specs.CKPT_NEVER])
@pytest.mark.parametrize("balance", [[1, 2, 2], [2, 2, 1], [3, 2]])
def test_gradients_of_a_network_with_skips(balance, mode):
    """A small U-Net in float32, its skip within a partition, across one and from a partition's last layer:
    1e-4 of each gradient's norm, as above."""
    say("normalised U-Net", balance, mode)
    torch.manual_seed(4)
    sess = NormPipeline(_skip_net(), FP32, n=len(balance), balance=balance)
    for q in sess.norms:
        q["gain"].copy_(1 + 0.2 * torch.randn_like(q["gain"]))
        q["bias"].copy_(0.2 * torch.randn_like(q["bias"]))
    sess.plan(8, 4, mode)
    x, dy = torch.randn(8, 12, 12, 8, device="cuda"), 1e-3 * torch.randn(8, 12, 12, 8, device="cuda")
    _compare_skips(sess, x, dy, 1e-4)
    sess.close()


def test_bfloat16_gradients():
    """Layers without ReLU, so that no decision hangs on a rounding: each of some ten tensors between x and dx (outputs,
    norms, gradients of both) is rounded to bfloat16, 2^-9 / sqrt(3) x 1.5 of its norm a time, and a gradient sees up to twenty
    of them: 20^1/2 x 1.7e-3 = 7.6e-3; twice that is asked."""
    torch.manual_seed(5)
    sess = NormPipeline(Net("norm-chain", (Layer(CONV3X3, 16, 32, relu=False), Layer(DWCONV3X3, 32, 32, relu=False, bias=False),
                                           Layer(CONV1X1, 32, 24, relu=False), Layer(CONV3X3, 24, 16, relu=False)), 16, 12, 12),
                        BF16, n=3, balance=[1, 2, 1])
    for q in sess.norms:
        q["gain"].copy_(1 + 0.2 * torch.randn_like(q["gain"]))
        q["bias"].copy_(0.2 * torch.randn_like(q["bias"]))
    sess.plan(8, 4, specs.CKPT_ALWAYS)
    x, dy = torch.randn(8, 12, 12, 16, device="cuda").bfloat16(), (1e-3 * torch.randn(8, 12, 12, 16, device="cuda")).bfloat16()
    _compare_skips(sess, x, dy, 1.5e-2)
    sess.close()
