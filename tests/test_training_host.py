"""NormPipeline's bookkeeping, without a GPU: its buffers live on the CPU and
the calls that would launch are recorded in place of being made."""
import types

import pytest
import torch

import paper_2004_09910_amd as tgp
from paper_2004_09910_amd import training
from paper_2004_09910_amd.training import NormPipeline
from workloads.specs import CKPT_ALWAYS, CONV1X1, CONV3X3, FP32, Layer, Net


def _net():
    return Net("widths", (Layer(CONV3X3, 8, 16), Layer(CONV1X1, 16, 24), Layer(CONV1X1, 24, 40),
                          Layer(CONV3X3, 40, 8, relu=False)), 8, 6, 6)


class Recorder:
    """Stands for the library in training.py: what launches is noted, the rest is the library's."""

    LAUNCHES = ("layer_norm_forward", "layer_norm_backward", "stage_forward", "stage_backward_recompute",
                "grad_accumulate", "muon_update", "weight_step", "adamw_step")

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name in self.LAUNCHES:
            return lambda *a: self.calls.append((name, a))
        return getattr(tgp, name)


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(training, "tgp", r)
    monkeypatch.setattr(tgp, "bind_workspace", lambda h, ws, nbytes: None)   # CPU memory is at 64 bytes
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0))
    return r


def _repartition(monkeypatch, sess, balance):
    """balance_by_time with the outcome `balance`, as no times can be taken here."""
    def chosen(h, ws, nbytes, iters, n, stream):
        tgp.set_partition(h, n, balance)
        return list(balance), [1.0] * len(sess.net.layers)
    monkeypatch.setattr(tgp, "balance_by_time", chosen)
    assert sess.balance_by_time(2, len(balance), CKPT_ALWAYS)[0] == list(balance)


def _check_calls(sess, r):
    """Every norm of a forward, backward and update works on vectors of its channels."""
    sizes = {q[k].data_ptr(): q[k].numel() for q in sess.norms for k in ("gain", "bias", "dgain", "dbias")}
    want = [sess.part_in_shape(j)[0] for j in range(1, sess.n + 1)]
    assert [q["gain"].numel() for q in sess.norms] == want
    r.calls.clear()
    x, y = torch.zeros(4, 6, 6, 8), torch.zeros(4, 6, 6, 8)
    sess.forward(x)
    sess.backward(y, torch.zeros_like(x))
    sess.update()
    seen = 0
    for name, a in r.calls:
        if name == "layer_norm_forward":
            assert sizes[a[5]] == sizes[a[6]] == a[1]
            seen += 1
        elif name == "layer_norm_backward":
            assert sizes[a[7]] == sizes[a[11]] == sizes[a[12]] == a[1]
            seen += 1
        elif name == "adamw_step":
            counts = {d.w: d.count for d in a[0]}
            assert all(counts[q[k].data_ptr()] == q[k].numel() for q in sess.norms for k in ("gain", "bias"))
            assert len(counts) == sum(p["b"] is not None for p in sess.params.values()) + 2 * sess.n
    assert seen == 2 * sess.n * sess.m


def test_norms_follow_a_new_partition(monkeypatch, recorder):
    """Partitions that move to boundaries of other widths, and more and fewer of them: norms, accumulators and
    the optimiser's list have the new boundaries' channels; a norm whose boundary stays keeps its values."""
    sess = NormPipeline(_net(), FP32, n=3, balance=[1, 1, 2], device="cpu")
    sess.plan(4, 2, CKPT_ALWAYS)
    _check_calls(sess, recorder)
    sess.norms[0]["gain"].fill_(3.0)
    sess.norms[2]["bias"].fill_(5.0)          # the boundary before layer 2
    for balance, kept in (([2, 1, 1], 1), ([2, 2], 1), ([1, 1, 1, 1], 2)):
        _repartition(monkeypatch, sess, balance)
        sess.plan(4, 2, CKPT_ALWAYS)
        _check_calls(sess, recorder)
        assert bool((sess.norms[0]["gain"] == 3).all()) and bool((sess.norms[kept]["bias"] == 5).all())
    sess.close()


def test_a_dropped_plan_is_not_run(monkeypatch, recorder):
    """After a new partition and before its plan nothing is launched."""
    sess = NormPipeline(_net(), FP32, n=2, balance=[2, 2], device="cpu")
    x = torch.zeros(4, 6, 6, 8)
    with pytest.raises(RuntimeError):
        sess.forward(x)
    sess.plan(4, 2, CKPT_ALWAYS)
    sess.forward(x)
    _repartition(monkeypatch, sess, [1, 2, 1])
    recorder.calls.clear()
    for call in (lambda: sess.forward(x), lambda: sess.backward(x), lambda: sess.train_step(x, x)):
        with pytest.raises(RuntimeError):
            call()
    assert not recorder.calls
    sess.close()
