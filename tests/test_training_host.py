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


def _wrong(good):
    """Tensors that are not the planned one: more and fewer samples, other extents, channels first, another type, a
    slice of a wider tensor, another device."""
    b, h, w, c = good.shape
    return [torch.zeros(b + 2, h, w, c), torch.zeros(b - 2, h, w, c), torch.zeros(b, h + 1, w, c), torch.zeros(b, h, w, c + 1),
            torch.zeros(b, c, h, w), torch.zeros(b, c, h, w).permute(0, 2, 3, 1), good.double(), good.bfloat16(),
            torch.zeros(b, h, w, 2 * c)[..., :c], good.to("meta"), good[0]]


def test_tensors_that_do_not_fit_the_plan(recorder):
    """Refused before the first launch: the calls read raw addresses by the plan's sizes."""
    net = Net("ends", (Layer(CONV3X3, 8, 16), Layer(CONV1X1, 16, 24, relu=False)), 8, 6, 10)
    sess = NormPipeline(net, FP32, n=2, balance=[1, 1], device="cpu")
    sess.plan(4, 2, CKPT_ALWAYS)
    x, y = torch.zeros(4, 6, 10, 8), torch.zeros(4, 6, 10, 24)
    for bad in _wrong(x):
        with pytest.raises(ValueError, match="^x "):
            sess.forward(bad)
        with pytest.raises(ValueError, match="^x "):
            sess.train_step(bad, y)
    assert not recorder.calls
    sess.forward(x)
    recorder.calls.clear()
    for bad in _wrong(y):
        with pytest.raises(ValueError, match="^dy "):
            sess.backward(bad)
    for bad in _wrong(x):
        with pytest.raises(ValueError, match="^dx "):
            sess.backward(y, bad)
    for shape in ((4, 6, 10, 1), (1, 6, 10, 24), (24,), (6, 6, 10, 24)):     # what torch would broadcast, or not
        with pytest.raises(ValueError, match="^target "):
            sess.train_step(x, torch.zeros(shape))
    assert not recorder.calls
    sess.backward(y, x.clone())
    sess.train_step(x, y.bfloat16())
    assert recorder.calls
    sess.close()


def test_backward_needs_its_forward(recorder):
    """The plan's buffers hold nothing before the first forward."""
    sess = NormPipeline(_net(), FP32, n=2, balance=[2, 2], device="cpu")
    for _ in range(2):
        sess.plan(4, 2, CKPT_ALWAYS)
        x = torch.zeros(4, 6, 6, 8)
        recorder.calls.clear()
        with pytest.raises(RuntimeError):
            sess.backward(x)
        assert not recorder.calls
        sess.forward(x)
        sess.backward(x)
    sess.close()


def test_micro_batches_cover_the_buffers(recorder):
    """The forward's rows of x, xn and statistics, of all micro-batches: each buffer once, from end to end."""
    sess = NormPipeline(_net(), FP32, n=2, balance=[1, 3], device="cpu")
    sess.plan(6, 3, CKPT_ALWAYS)
    x = torch.zeros(6, 6, 6, 8)
    sess.forward(x)
    for j, src in ((1, x), (2, sess.out[0])):
        c = src.shape[3]
        calls = [a for name, a in recorder.calls if name == "layer_norm_forward" and a[1] == c]
        assert len(calls) == 3
        for t, place, each in ((src, 3, 4 * c), (sess.xn[j - 1], 8, 4 * c), (sess.stats[j - 1], 10, 8)):
            at = t.data_ptr()
            for a in calls:
                assert a[place] == at
                at += a[0] * each
            assert at == t.data_ptr() + t.numel() * 4
    sess.close()
