"""Training of a pipeline whose partitions read normalised inputs: the stage
tasks, the layer norms between them and the update of what they learn, as a
program puts them together.

    x_i^j = f^j(norm^j(x_i^{j-1})),   j = 1..n,  for each micro-batch i

Layer norm is per pixel, so the split into micro-batches does not change the
gradients (which batch norm would), and its backward adds each micro-batch's
dgain and dbias to accumulators in the stages' own order i = m..1.  After the
last accumulation the weight matrices take momentum and the orthogonalised
update, biases, gains and depthwise weights AdamW; bfloat16 networks keep
float32 master weights and get the rounded copies that their layers read.

Torch provides device memory, streams and the loss (a squared error).
"""
from __future__ import annotations

import math

import torch

import paper_2004_09910_amd as tgp
from workloads import specs
from workloads.specs import BF16, DWCONV3X3

from .harness import TORCH_DT, Session


class NormPipeline(Session):
    """A Session (network, partitions, bound parameters) with a layer norm before
    every partition and an optimiser.  A new partition (balance_by_time) takes
    effect with the plan() that has to follow it: a norm whose boundary stays
    keeps its values and its optimiser's states, the others start anew."""

    def __init__(self, net: specs.Net, dtype: int, n: int, eps: float = 1e-5, **kw):
        super().__init__(net, dtype, n=n, **kw)
        self.eps = eps
        self.norms, self.norm_at = [], []     # of each partition, and its first layer
        self._optimiser()
        self._match_norms()

    # ------------------------------------------------------------- optimiser

    def _match_norms(self):
        """Norms for the network's present partition, and the list of what AdamW updates."""
        self._set_bounds()
        at = [lo for lo, _ in self.bounds]
        old = dict(zip(self.norm_at, self.norms))
        self.norms, self.norm_at = [], at
        for j, lo in enumerate(at, 1):
            c = self.part_in_shape(j)[0]
            # gain, bias and AdamW's two states of each
            self.norms.append(old.get(lo) or {
                k: torch.full((c,), float(k == "gain"), device=self.device)
                for k in ("gain", "bias", "dgain", "dbias", "gain_m", "gain_v", "bias_m", "bias_v")})
        self.adam = tgp.adamw_tensors(self.vectors + [
            (q[k].numel(), q[k].data_ptr(), None, q["d" + k].data_ptr(), q[k + "_m"].data_ptr(), q[k + "_v"].data_ptr())
            for q in self.norms for k in ("gain", "bias")])

    def _optimiser(self, rate=0.02, weight_decay=0.01):
        muon, step = [], []
        self.vectors = []    # AdamW's tensors but the norms'
        self.state = []      # keeps the buffers behind the lists alive

        def zeros(like, dtype=torch.float32):
            t = torch.zeros(like.shape, dtype=dtype, device=self.device)
            self.state.append(t)
            return t

        def vector(w, w16, grad):
            self.vectors.append((w.numel(), w.data_ptr(), None if w16 is None else w16.data_ptr(),
                                 grad.data_ptr(), zeros(w).data_ptr(), zeros(w).data_ptr()))

        for idx, p in self.params.items():
            w16 = p["w"] if self.dtype == BF16 else None
            w = p["w"].float() if self.dtype == BF16 else p["w"]
            self.state.append(w)
            p["master"] = w
            if self.net.layers[idx].kind == DWCONV3X3:
                vector(w, w16, p["dw"])
            else:
                rows, cols = w.shape[0], w.numel() // w.shape[0]
                o = zeros(w, torch.bfloat16)
                muon.append((rows, cols, p["dw"].data_ptr(), zeros(w).data_ptr(), o.data_ptr()))
                step.append((w.numel(), w.data_ptr(), None if w16 is None else w16.data_ptr(),
                             o.data_ptr(), rate * math.sqrt(max(1.0, rows / cols))))
            if p["b"] is not None:
                vector(p["b"], None, p["db"])
        self.muon, self.step = tgp.muon_tensors(muon), tgp.step_tensors(step)
        self.decay = rate * weight_decay
        self.updates = 0
        self.muon_ws = torch.empty(max(tgp.muon_workspace(self.muon), 256), dtype=torch.uint8,
                                   device=self.device)

    def update(self, mu=0.95, ns_steps=5, adam_rate=1e-3):
        """One step of all parameters from the accumulated gradients."""
        s = torch.cuda.current_stream().cuda_stream
        self.updates += 1
        tgp.muon_update(self.muon, mu, True, ns_steps, 1e-7, self.muon_ws.data_ptr(),
                        self.muon_ws.numel(), s)
        tgp.weight_step(self.step, self.decay, s)
        tgp.adamw_step(self.adam, adam_rate, 0.9, 0.95, 1e-8, 0.0, self.updates, s)

    # ------------------------------------------------------------- forward, backward

    def plan(self, B: int, m: int, mode: int, lanes: int = 1) -> int:
        need = super().plan(B, m, mode, lanes)
        self._match_norms()
        dt = TORCH_DT[self.dtype]

        def buf(j):
            c, h, w = self.part_in_shape(j)
            return torch.empty((B, h, w, c), dtype=dt, device=self.device)

        h, w = self.net.out_hw()
        # per partition: its normalised input, its statistics, and the gradient
        # of what it reads; `out[j]` is what partition j writes
        self.xn = [buf(j) for j in range(1, self.n + 1)]
        self.dxn = [buf(j) for j in range(1, self.n + 1)]
        self.stats = [torch.empty((t.numel() // t.shape[3], 2), device=self.device) for t in self.xn]
        self.out = [buf(j) for j in range(2, self.n + 1)]
        self.out.append(torch.empty((B, h, w, self.net.out_channels()), dtype=dt, device=self.device))
        self.x = None     # the last forward's input
        ws = [tgp.layer_norm_backward_workspace(t.numel() // t.shape[3] // m, t.shape[3], self.dtype)
              for t in self.xn]
        self.norm_ws = torch.empty(max(ws + [256]), dtype=torch.uint8, device=self.device)
        return need

    def _planned(self):
        if self.ws is None:
            raise RuntimeError("plan() has to come first, again after a new partition or layer times")

    def _fits(self, name, t, like, raw=True):
        """t as the plan has it: the shape of its buffer `like` and, where its address is taken (raw), the
        type, layout and device."""
        if t.shape != like.shape:
            raise ValueError(f"{name} is {tuple(t.shape)}, the plan has {tuple(like.shape)} (NHWC)")
        if raw and (t.dtype != like.dtype or t.device != like.device or not t.is_contiguous()):
            raise ValueError(f"{name} is {t.dtype} on {t.device}, strides {t.stride()}; the plan has {like.dtype} on "
                             f"{like.device}, contiguous")

    def _rows(self, t, i):
        """Micro-batch i of a full-batch tensor (or of its pixels): address, pixels, channels."""
        per = t.shape[0] // self.m
        part = t[(i - 1) * per:i * per]
        return part.data_ptr(), part.numel() // t.shape[-1], t.shape[-1]

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """All F_{i,j}, each after its norm; returns the network's output (full batch)."""
        self._planned()
        self._fits("x", x, self.xn[0])
        s = torch.cuda.current_stream().cuda_stream
        self.x = x
        for i in range(1, self.m + 1):
            for j in range(1, self.n + 1):
                src, rows, c = self._rows(x if j == 1 else self.out[j - 2], i)
                dst = self._rows(self.xn[j - 1], i)[0]
                q = self.norms[j - 1]
                tgp.layer_norm_forward(rows, c, self.dtype, src, c, q["gain"].data_ptr(),
                                       q["bias"].data_ptr(), self.eps, dst, c,
                                       self._rows(self.stats[j - 1], i)[0], s)
                tgp.stage_forward(self.h, j, i, self.checkpointed(i), dst,
                                  self._rows(self.out[j - 1], i)[0], s)
        return self.out[-1]

    def backward(self, dy: torch.Tensor, dx: torch.Tensor = None) -> None:
        """F' and B of every task in the order i = m..1, each followed by its
        norm's backward; the gradients are left in the accumulators, and the
        input's in dx (if given)."""
        self._planned()
        if self.x is None:
            raise RuntimeError("forward() has to come first")
        self._fits("dy", dy, self.out[-1])
        if dx is not None:
            self._fits("dx", dx, self.x)
        s = torch.cuda.current_stream().cuda_stream
        for i in range(self.m, 0, -1):
            for j in range(self.n, 0, -1):
                # the gradient of partition j's output: the loss's, or what the
                # norm of partition j + 1 wrote over the gradient it read
                src = self._rows(dy if j == self.n else self.dxn[j], i)[0]
                g, rows, c = self._rows(self.dxn[j - 1], i)
                tgp.stage_backward_recompute(self.h, j, i, src, g, s)
                tgp.grad_accumulate(self.h, j, i, i == self.m, s)
                x = self._rows(self.x if j == 1 else self.out[j - 2], i)[0]
                q = self.norms[j - 1]
                to = g if j > 1 else (None if dx is None else self._rows(dx, i)[0])
                tgp.layer_norm_backward(rows, c, self.dtype, g, c, x, c, q["gain"].data_ptr(),
                                        self._rows(self.stats[j - 1], i)[0], to, c,
                                        q["dgain"].data_ptr(), q["dbias"].data_ptr(), i == self.m,
                                        self.norm_ws.data_ptr(), self.norm_ws.numel(), s)

    def train_step(self, x: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        """Forward, mean squared error, backward, update; returns the loss (on the device).
        x, and what forward and backward take, are contiguous NHWC tensors of the planned batch in the
        network's type; ValueError otherwise, before anything runs."""
        self._planned()
        self._fits("x", x, self.xn[0])
        self._fits("target", target, self.out[-1], raw=False)
        y = self.forward(x)
        err = y.float() - target.float()
        self.backward((err * (2.0 / err.numel())).to(y.dtype))
        self.update()
        return err.square().mean()
