"""GatedPipeline's bookkeeping, without a GPU: its buffers live on the CPU and
the calls that would launch are recorded in place of being made."""
import types

import pytest
import torch

import paper_2004_09910_amd as tgp
from paper_2004_09910_amd import training
from paper_2004_09910_amd.training import GatedPipeline
from workloads.specs import BF16, CKPT_ALWAYS, CONV1X1, CONV3X3, FP32, Layer, Net

LAUNCHES = ("layer_norm_forward", "layer_norm_backward", "stage_forward", "stage_backward_recompute", "grad_accumulate",
            "muon_update", "weight_step", "adamw_step", "gated_forward", "gated_backward", "residual_norm_forward",
            "residual_norm_backward", "adamw8_step")


def _net():
    return Net("widths", (Layer(CONV3X3, 8, 16), Layer(CONV1X1, 16, 24), Layer(CONV1X1, 24, 40),
                          Layer(CONV3X3, 40, 8, relu=False)), 8, 6, 6)


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name in LAUNCHES:
            return lambda *a: self.calls.append((name, a))
        return getattr(tgp, name)

    def named(self, name):
        return [a for n, a in self.calls if n == name]


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(training, "tgp", r)
    monkeypatch.setattr(tgp, "bind_workspace", lambda h, ws, nbytes: None)   # CPU memory is at 64 bytes
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0))
    return r


def _run(sess, r):
    x = torch.zeros(4, 6, 6, 8, dtype=training.TORCH_DT[sess.dtype])
    r.calls.clear()
    sess.forward(x)
    sess.backward(torch.zeros_like(x), torch.zeros_like(x))
    sess.update()


def _check(sess, r):
    """Every block of a forward and backward works on its own parameters, gradients and widths, overwriting at the
    first micro-batch and adding at the others; the step takes each of them once."""
    _run(sess, r)
    m, n = sess.m, sess.n
    widths = [sess.part_in_shape(j)[0] for j in range(1, n + 1)]
    forward, backward = r.named("gated_forward"), r.named("gated_backward")
    assert len(forward) == len(backward) == m * n
    for k, a in enumerate(forward):
        b, c = sess.blocks[k % n], widths[k % n]
        shape, weights = a[0], a[2]
        assert (shape.cin, shape.hidden, shape.cout, shape.dtype) == (c, b["hidden"], c, sess.dtype)
        assert [getattr(weights, q) for q in ("gate", "up", "down", "b_gate", "b_up", "b_down")] == [
            b[q].data_ptr() for q in ("gate", "up", "down", "b_gate", "b_up", "b_down")]
        assert a[4] == a[6] == c
    for k, a in enumerate(backward):
        b, c = sess.blocks[n - 1 - k % n], widths[n - 1 - k % n]
        assert a[0].cin == c and a[9].gate == b["d_gate"].data_ptr() and a[9].b_down == b["d_b_down"].data_ptr()
        assert a[10] == (k < n)          # overwrites at the first micro-batch
    for a in r.named("residual_norm_backward"):
        assert a[2] == a[13] and a[4] is None          # the stream's gradient over what the stage left
    assert len(r.named("residual_norm_forward")) == len(r.named("residual_norm_backward")) == m * n
    (step,) = r.named("adamw8_step")
    got = sorted((d.count, d.w, d.grad, d.exps) for d in step[0])
    want = sorted((b["w_" + k].numel(), b["w_" + k].data_ptr(), b["d_" + k].data_ptr(), b["exps_" + k].data_ptr())
                  for b in sess.blocks for k in ("gate", "up", "down") + sess.VECTORS)
    assert got == want
    assert step[6] == step[7] == sess.updates


@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_blocks_follow_a_new_partition(monkeypatch, recorder, dtype):
    sess = GatedPipeline(_net(), dtype, n=3, ratio=3, balance=[1, 1, 2], device="cpu")
    sess.plan(4, 2, CKPT_ALWAYS)
    _check(sess, recorder)
    sess.blocks[0]["b_up"].fill_(3.0)
    sess.blocks[2]["scale"].fill_(5.0)        # the boundary before layer 2
    for balance, kept in (([2, 1, 1], 1), ([2, 2], 1), ([1, 1, 1, 1], 2)):
        monkeypatch.setattr(tgp, "balance_by_time", lambda h, ws, nb, it, n, st, b=balance: (
            tgp.set_partition(h, n, b), (list(b), [1.0] * 4))[1])
        sess.balance_by_time(2, len(balance), CKPT_ALWAYS)
        recorder.calls.clear()
        with pytest.raises(RuntimeError):     # the dropped plan is not run
            sess.forward(torch.zeros(4, 6, 6, 8))
        assert not recorder.calls
        sess.plan(4, 2, CKPT_ALWAYS)
        _check(sess, recorder)
        assert bool((sess.blocks[0]["b_up"] == 3).all()) and bool((sess.blocks[kept]["scale"] == 5).all())
    sess.close()


def test_micro_batches_cover_the_buffers(recorder):
    """Rows of the block's input, output and stream and of the statistics: each buffer once, from end to end."""
    sess = GatedPipeline(_net(), FP32, n=2, balance=[1, 3], device="cpu")
    sess.plan(4, 2, CKPT_ALWAYS)
    _run(sess, recorder)
    for j in (1, 2):
        c = sess.xn[j - 1].shape[3]
        calls = recorder.named("gated_forward")[j - 1::2]
        assert len(calls) == 2
        for t, place in ((sess.t[j - 1], 3), (sess.f[j - 1], 5)):
            at = t.data_ptr()
            for a in calls:
                assert a[place] == at
                at += a[1] * 4 * c
            assert at == t.data_ptr() + t.numel() * 4
        calls = recorder.named("residual_norm_forward")[j - 1::2]
        for t, place, each in ((sess.f[j - 1], 4, 4 * c), (sess.r[j - 1], 8, 4 * c), (sess.xn[j - 1], 10, 4 * c),
                               (sess.stats4[j - 1], 12, 16)):
            at = t.data_ptr()
            for a in calls:
                assert a[place] == at
                at += a[0].rows * each
            assert at == t.data_ptr() + t.numel() * 4
    sess.close()


def test_the_inputs_gradient_is_the_callers_wish(recorder):
    """Without dx the first norm computes none, and nothing is summed for it."""
    sess = GatedPipeline(_net(), FP32, n=2, balance=[2, 2], device="cpu")
    sess.plan(4, 2, CKPT_ALWAYS)
    x = torch.zeros(4, 6, 6, 8)
    sess.forward(x)
    recorder.calls.clear()
    sess.backward(x.clone())
    at = [a[9] for a in recorder.named("layer_norm_backward")]
    assert at[1::2] == [None, None] and None not in at[::2]
    sess.close()
