"""Layer normalisation over channels and the update of a network's weights, as cases to be timed and compared.

Four operators that a training program calls between and after the stage tasks of a pipeline:

  norm_fwd   y = gain (x - mean) rstd + bias over the channels of each pixel, with the rows' statistics
  norm_bwd   its gradients: dx, and the gain's and bias's summed over all pixels
  muon       momentum, and the orthogonalised update of every weight matrix by Newton-Schulz products
  update     the weights' step: w (1 - decay) - rate O for the matrices, AdamW for vectors (or for everything)

Tensors are NHWC: a row is a pixel, weights are [cout][kh kw cin].  Sizes are those of the U-Net, cell and stack
workloads.  Where `own` is false the operators run in plain torch operations in float32, rounded once at the end.
"""
import math

import torch

own = False

EPS = 1e-5                       # layer norm
NS = (3.4445, -4.7750, 2.0315)   # the Newton-Schulz quintic a x + b x^3 + c x^5
NS_STEPS, NS_EPS = 5, 1e-7
MU = 0.95                        # momentum
RATE, DECAY = 0.02, 0.0002       # of the matrices' step: learning rate, learning rate x weight decay
ADAM = {"rate": 1e-3, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "decay": 1e-5, "step": 10}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------- the cases

def _norm(name, op, rows, c, dtype, ldx=0, ldy=0):
    """`rows` pixels of `c` channels; ldx, ldy: channels of the tensor that x (with dx) and y (with dy) are
    slices of, where not their own."""
    d = {"op": op, "rows": rows, "c": c, "dtype": dtype, "ldx": max(ldx, c), "ldy": max(ldy, c)}
    return dict(d, name=name) if name else d


def _mats(name, op, shapes, dtype="bf16", rule="muon"):
    """shapes: "rows x cols" of each weight matrix, with a bias of `rows` values each; dtype: of the network."""
    d = {"op": op, "shapes": ",".join("%dx%d" % s for s in shapes), "dtype": dtype}
    if op == "update":
        d["rule"] = rule
    return dict(d, name=name) if name else d


def _stack(layers, c):
    return [(c, 9 * c)] * layers


def _unet(levels, base):
    """The weight matrices of a U-Net with two 3x3 layers a level and a one-channel head."""
    ch = [base << k for k in range(levels)]
    s = []
    for k, c in enumerate(ch):
        s += [(c, 9 * (ch[k - 1] if k else base)), (c, 9 * c)]
    for k in range(levels - 2, -1, -1):
        s += [(ch[k], 9 * (ch[k + 1] + ch[k])), (ch[k], 9 * ch[k])]
    return s + [(1, base)]


def listed():
    return [
        # One image at the deep end of the 5-level U-Net (12 x 12 pixels of 1024 channels), as a program that
        # answers for one image normalises it: latency.
        _norm("norm-fwd-b1", "norm_fwd", 144, 1024, "bf16"),
        # A micro-batch of the U-Net's first level, 4 x 192 x 192 x 64: the ordinary large, narrow tensor.
        _norm("norm-fwd-unet0", "norm_fwd", 4 * 192 * 192, 64, "bf16"),
        # A cropped image batch of 3 x 45 x 61 pixels and 100 channels in float32, its result written into its
        # place in a concatenated tensor.
        _norm("norm-fwd-ragged", "norm_fwd", 3 * 45 * 61, 100, "fp32", ldy=228),
        # One image of 56 x 56 through one layer's norm, backward: latency.
        _norm("norm-bwd-b1", "norm_bwd", 56 * 56, 64, "bf16"),
        # A micro-batch of the 18-cell workload, 4 x 56 x 56 x 256.
        _norm("norm-bwd-cells", "norm_bwd", 4 * 56 * 56, 256, "bf16"),
        # A micro-batch of the 6-level U-Net's first level, 2 x 256 x 256 x 128, its input a slice of the
        # concatenated tensor of 384 channels: the largest.
        _norm("norm-bwd-unet6", "norm_bwd", 2 * 256 * 256, 128, "bf16", ldx=384),
        # The weights of the 4-layer, 16-channel float32 stack: what a toy pays for its step.
        _mats("muon-stack", "muon", _stack(4, 16), "fp32"),
        # The pointwise weights of 18 cells at 256 channels: many small square matrices.
        _mats("muon-cells", "muon", [(256, 256)] * 18),
        # Every weight of the 5-level U-Net at 64 channels, 31 million in 19 matrices from 1 x 64 to 1024 x 9216:
        # the step of the headline network.
        _mats("muon-unet5", "muon", _unet(5, 64)),
        # One 3 x 3 layer of 2048 channels at the deep end of the 6-level U-Net: the largest products.
        _mats("muon-deep", "muon", [(2048, 9 * 2048)]),
        # The step of the stack's weights and biases.
        _mats("update-stack", "update", _stack(4, 16), "fp32"),
        # The step of all of the 5-level U-Net's weights and biases, with the bfloat16 copies that the layers read.
        _mats("update-unet5", "update", _unet(5, 64)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _flops(rows, cols, steps=NS_STEPS):
    """Products of `steps` Newton-Schulz steps of one matrix, symmetric ones at half: one step at a time, or two
    at a time on the m x m side where that is less."""
    m, n = float(min(rows, cols)), float(max(rows, cols))
    pairs, odd = divmod(steps, 2)
    return min(steps * (3 * m * m * n + m ** 3), pairs * (3 * m * m * n + 5 * m ** 3) + odd * (3 * m * m * n + m ** 3))


def draw(rng):
    op = rng.choice(("norm_fwd", "norm_bwd", "norm_fwd", "norm_bwd", "muon", "muon", "update"))
    if op.startswith("norm"):
        dtype = rng.choice(("bf16", "bf16", "fp32"))
        c = _log(rng, 1, 4096)
        if c > 16 and rng.random() < 0.6:
            c = (c + 7) // 8 * 8
        most = 2 * 256 * 256 * 128 // (1 if dtype == "bf16" else 2)
        rows = _log(rng, 1, min(1 << 19, max(1, most // c)))
        wide = lambda: c + (_log(rng, 1, 512) if rng.random() < 0.3 else 0)  # noqa: E731
        return _norm(None, op, rows, c, dtype, wide(), wide())
    most = 0.9 * _flops(2048, 9 * 2048)
    shapes, work, size = [], 0.0, 0
    for _ in range(rng.choice((1, 2, 3, 4, 6, 8, 12))):
        taps = rng.choice((1, 9, 9))
        r, c = _log(rng, 1, 2048), _log(rng, 1, 2048)
        if rng.random() < 0.5:
            r, c = (r + 15) // 16 * 16, (c + 15) // 16 * 16
        f, e = _flops(r, taps * c), r * taps * c
        if not shapes or (work + f <= most and size + e <= 32 << 20):
            shapes, work, size = shapes + [(r, taps * c)], work + f, size + e
    return _mats(None, op, shapes, rng.choice(("bf16", "bf16", "fp32")), rng.choice(("muon", "adamw")))


# ---------------------------------------------------------------- inputs

def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def _flat(sizes):
    """Offsets of tensors of these sizes in one buffer, each at a multiple of 64 values, and the buffer's size."""
    at, offs = 0, []
    for s in sizes:
        offs.append(at)
        at += (s + 63) // 64 * 64
    return offs, at


def _gaps(buf, offs, sizes):
    """buf with zeros between its tensors: what lies there belongs to none and stays zero."""
    used = torch.zeros_like(buf)
    for o, n in zip(offs, sizes):
        used[o:o + n] = 1
    return buf * used


def _gradients(shapes, offs, total, g, noise):
    """Weight gradients of the sort a batch gives: a few strong directions in broadband noise, every matrix of a
    size of its own."""
    buf = torch.zeros(total, device="cuda")
    for k, ((r, c), o) in enumerate(zip(shapes, offs)):
        d = min(8, r, c)
        u = torch.randn(r, d, device="cuda", generator=g) / math.sqrt(d)
        v = torch.randn(d, c, device="cuda", generator=g)
        t = u @ v + noise * torch.randn(r, c, device="cuda", generator=g)
        buf[o:o + r * c] = t.reshape(-1) * (1e-3 * 1.5 ** -(k % 7))
    return buf


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = {"case": case}
    if case["op"].startswith("norm"):
        rows, c, dt = case["rows"], case["c"], DT[case["dtype"]]

        def tensor(ld):
            return torch.empty(rows, ld, dtype=dt, device="cuda")[:, :c]

        def normal(*shape):
            return torch.randn(*shape, device="cuda", generator=g)

        # a layer's output: every channel its own spread and offset
        s["x"] = tensor(case["ldx"])
        s["x"].copy_(normal(rows, c) * normal(c).abs().add_(0.2) + 0.5 * normal(c))
        s["gain"], s["bias"] = 1 + 0.1 * normal(c), 0.1 * normal(c)
        if case["op"] == "norm_fwd":
            s["y"], s["stats"] = tensor(case["ldy"]), torch.empty(rows, 2, device="cuda")
        else:
            xf = s["x"].float()
            mean = xf.mean(1, keepdim=True)
            var = (xf - mean).square().mean(1, keepdim=True)
            s["stats"] = torch.cat((mean, (var + EPS).rsqrt()), 1).contiguous()
            s["dy"] = tensor(case["ldy"])
            s["dy"].copy_(normal(rows, c) * 1e-2)
            s["dx"] = tensor(case["ldx"])
            s["dgain"], s["dbias"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        if own:
            import paper_2004_09910_amd as tgp
            if case["op"] == "norm_bwd":
                n = tgp.layer_norm_backward_workspace(rows, c, tgp.BF16 if case["dtype"] == "bf16" else tgp.FP32)
                s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
        return s
    shapes = _shapes(case)
    offs, total = _flat([r * c for r, c in shapes])
    s.update(shapes=shapes, offs=offs, total=total)
    s["grad"] = _gradients(shapes, offs, total, g, 1.0)
    if case["op"] == "muon":
        s["momentum"] = _gradients(shapes, offs, total, g, 0.3) * 8
        s["o"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
        if own:
            import paper_2004_09910_amd as tgp
            s["list"] = tgp.muon_tensors([
                (r, c, s["grad"][o:].data_ptr(), s["momentum"][o:].data_ptr(), s["o"][o:].data_ptr())
                for (r, c), o in zip(shapes, offs)])
            s["ws"] = torch.empty(tgp.muon_workspace(s["list"]), dtype=torch.uint8, device="cuda")
        return s
    # weights, biases and what the step keeps beside them; an update is orthogonal rows of 1 / sqrt(cols)
    voffs, vtotal = _flat([r for r, _ in shapes])
    s.update(voffs=voffs, vtotal=vtotal)
    half = case["dtype"] == "bf16"
    s["w"] = torch.zeros(total, device="cuda")
    s["o"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    for (r, c), o in zip(shapes, offs):
        s["w"][o:o + r * c] = math.sqrt(2 / c) * torch.randn(r * c, device="cuda", generator=g)
        s["o"][o:o + r * c] = torch.randn(r * c, device="cuda", generator=g) / math.sqrt(max(r, c))
    s["w16"] = s["w"].bfloat16() if half else None
    rows = [r for r, _ in shapes]
    s["b"] = _gaps(0.1 * torch.randn(vtotal, device="cuda", generator=g), voffs, rows)
    s["db"] = _gaps(1e-3 * torch.randn(vtotal, device="cuda", generator=g), voffs, rows)
    both = [("b", "db", voffs, rows, vtotal)]
    if case["rule"] == "adamw":
        both.append(("w", "grad", offs, [r * c for r, c in shapes], total))
    for w, _, of, sizes, n in both:
        s[w + "_m"] = _gaps(1e-3 * torch.randn(n, device="cuda", generator=g), of, sizes)
        s[w + "_v"] = _gaps(1e-6 * torch.rand(n, device="cuda", generator=g) + 1e-8, of, sizes)
    if own:
        import paper_2004_09910_amd as tgp

        def at(name, o):
            return s[name][o:].data_ptr() if s[name] is not None else None

        s["adam"] = tgp.adamw_tensors([
            (n, at(w, o), at("w16", o) if w == "w" else None, at(grad, o), at(w + "_m", o), at(w + "_v", o))
            for w, grad, of, sizes, _ in both for o, n in zip(of, sizes)])
        if case["rule"] == "muon":
            s["list"] = tgp.step_tensors([
                (r * c, at("w", o), at("w16", o), at("o", o), _rate(r, c)) for (r, c), o in zip(shapes, offs)])
    return s


def _rate(r, c):
    """A matrix's learning rate: larger where it has more rows than columns."""
    return RATE * math.sqrt(max(1.0, r / c))


# ---------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2004_09910_amd as tgp
    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "norm_fwd":
        x, y = s["x"], s["y"]
        tgp.layer_norm_forward(case["rows"], case["c"], tgp.BF16 if case["dtype"] == "bf16" else tgp.FP32,
                               x.data_ptr(), case["ldx"], s["gain"].data_ptr(), s["bias"].data_ptr(), EPS,
                               y.data_ptr(), case["ldy"], s["stats"].data_ptr(), stream)
        return {"y": y, "stats": s["stats"]}
    if case["op"] == "norm_bwd":
        tgp.layer_norm_backward(case["rows"], case["c"], tgp.BF16 if case["dtype"] == "bf16" else tgp.FP32,
                                s["dy"].data_ptr(), case["ldy"], s["x"].data_ptr(), case["ldx"],
                                s["gain"].data_ptr(), s["stats"].data_ptr(), s["dx"].data_ptr(), case["ldx"],
                                s["dgain"].data_ptr(), s["dbias"].data_ptr(), True, s["ws"].data_ptr(),
                                s["ws"].numel(), stream)
        return {"dx": s["dx"], "dgain": s["dgain"], "dbias": s["dbias"]}
    if case["op"] == "muon":
        tgp.muon_update(s["list"], MU, True, NS_STEPS, NS_EPS, s["ws"].data_ptr(), s["ws"].numel(), stream)
        return {"momentum": s["momentum"], "o": s["o"]}
    if case["rule"] == "muon":
        tgp.weight_step(s["list"], DECAY, stream)
    tgp.adamw_step(s["adam"], ADAM["rate"], ADAM["beta1"], ADAM["beta2"], ADAM["eps"], ADAM["decay"], ADAM["step"],
                   stream)
    return _updated(s)


def _updated(s):
    return {k: s[k] for k in ("w", "w16", "b", "b_m", "b_v", "w_m", "w_v") if s.get(k) is not None}


def _run_plain(s):
    case = s["case"]
    if case["op"] == "norm_fwd":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = ((d * d).mean(1, keepdim=True) + EPS).rsqrt()
        return {"y": (d * rstd * s["gain"] + s["bias"]).to(s["x"].dtype), "stats": torch.cat((mean, rstd), 1)}
    if case["op"] == "norm_bwd":
        dy, rstd = s["dy"].float(), s["stats"][:, 1:]
        xhat = (s["x"].float() - s["stats"][:, :1]) * rstd
        g = dy * s["gain"]
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        return {"dx": dx.to(s["x"].dtype), "dgain": (dy * xhat).sum(0), "dbias": dy.sum(0)}
    if case["op"] == "muon":
        s["momentum"].mul_(MU).add_(s["grad"])
        u = s["grad"] + MU * s["momentum"]
        a, b, c = NS
        for rows, cols in dict.fromkeys(s["shapes"]):    # equal matrices as one batch
            at = [o for shape, o in zip(s["shapes"], s["offs"]) if shape == (rows, cols)]
            x = torch.stack([u[o:o + rows * cols] for o in at]).view(-1, rows, cols)
            x = x.mT if rows > cols else x
            x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + NS_EPS)
            for _ in range(NS_STEPS):
                p = x @ x.mT
                x = a * x + (b * p + c * (p @ p)) @ x
            for o, v in zip(at, (x.mT if rows > cols else x).bfloat16()):
                s["o"][o:o + rows * cols].view(rows, cols).copy_(v)
        return {"momentum": s["momentum"], "o": s["o"]}
    if case["rule"] == "muon":
        for (rows, cols), o in zip(s["shapes"], s["offs"]):
            w = s["w"][o:o + rows * cols]
            w.mul_(1 - DECAY).sub_(_rate(rows, cols) * s["o"][o:o + rows * cols].float())
    else:
        _adam_plain(s["w"], s["grad"], s["w_m"], s["w_v"])
    if s["w16"] is not None:
        s["w16"].copy_(s["w"])
    _adam_plain(s["b"], s["db"], s["b_m"], s["b_v"])
    return _updated(s)


def _adam_plain(w, g, m, v):
    k = ADAM
    m.mul_(k["beta1"]).add_(g * (1 - k["beta1"]))
    v.mul_(k["beta2"]).add_(g * g * (1 - k["beta2"]))
    mhat = m / (1 - k["beta1"] ** k["step"])
    vhat = v / (1 - k["beta2"] ** k["step"])
    w.mul_(1 - k["decay"]).sub_(k["rate"] * mhat / (vhat.sqrt() + k["eps"]))


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["op"].startswith("norm"):
        n, e = case["rows"] * case["c"], 2 if case["dtype"] == "bf16" else 4
        if case["op"] == "norm_fwd":     # x in, y and statistics out
            return {"bytes": 2 * n * e + 8 * case["rows"] + 8 * case["c"], "flops": 8 * n}
        return {"bytes": 3 * n * e + 8 * case["rows"] + 12 * case["c"], "flops": 14 * n}
    shapes = _shapes(case)
    n, v = sum(r * c for r, c in shapes), sum(r for r, _ in shapes)
    if case["op"] == "muon":             # gradient and momentum in, momentum and update out
        return {"bytes": 14 * n, "flops": sum(_flops(r, c) for r, c in shapes)}
    half = 2 if case["dtype"] == "bf16" else 0
    adam = 28 * v                        # w, m, v in and out, the gradient in
    return {"bytes": adam + n * ((28 if case["rule"] == "adamw" else 10) + half), "flops": 16 * (n + v)}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "norm_fwd":
        x = s["x"].to(f64)
        var, mean = torch.var_mean(x, dim=1, unbiased=False)
        rstd = 1 / torch.sqrt(var + EPS)
        y = torch.addcmul(s["bias"].to(f64), (x - mean[:, None]) * rstd[:, None], s["gain"].to(f64))
        return {"y": y, "stats": torch.stack((mean, rstd), 1)}
    if case["op"] == "norm_bwd":
        # the Jacobian of one row, J = rstd (I - 1 1^T / c - xhat xhat^T / c), applied to gain * dy
        mean, rstd = s["stats"].to(f64).unbind(1)
        dy = s["dy"].to(f64)
        xhat = (s["x"].to(f64) - mean[:, None]) * rstd[:, None]
        g = dy * s["gain"].to(f64)
        along = (g * xhat).sum(1) / case["c"]
        dx = (g - (g.sum(1) / case["c"])[:, None] - along[:, None] * xhat) * rstd[:, None]
        return {"dx": dx, "dgain": torch.einsum("rc,rc->c", dy, xhat), "dbias": dy.sum(0)}
    if case["op"] == "muon":
        m = MU * s["momentum"].to(f64) + s["grad"].to(f64)
        u = s["grad"].to(f64) + MU * m
        out = torch.zeros(s["total"], dtype=f64, device="cuda")
        for (r, c), o in zip(s["shapes"], s["offs"]):
            x = u[o:o + r * c].reshape(r, c)
            x = x / (torch.linalg.matrix_norm(x) + NS_EPS)
            for _ in range(NS_STEPS):    # x (a + b x^T x + c (x^T x)^2), from the shorter side
                if r > c:
                    q = x.T @ x
                    x = NS[0] * x + NS[1] * (x @ q) + NS[2] * (x @ q @ q)
                else:
                    q = x @ x.T
                    x = NS[0] * x + NS[1] * (q @ x) + NS[2] * (q @ (q @ x))
            out[o:o + r * c] = x.reshape(-1)
        return {"momentum": m, "o": out}
    k, got = ADAM, {}

    def adam(w, g):
        m = k["beta1"] * s[w + "_m"].to(f64) + (1 - k["beta1"]) * s[g].to(f64)
        v = k["beta2"] * s[w + "_v"].to(f64) + (1 - k["beta2"]) * s[g].to(f64) ** 2
        step = m / (1 - k["beta1"] ** k["step"]) / (torch.sqrt(v / (1 - k["beta2"] ** k["step"])) + k["eps"])
        got.update({w: s[w].to(f64) * (1 - k["decay"]) - k["rate"] * step, w + "_m": m, w + "_v": v})

    adam("b", "db")
    if case["rule"] == "adamw":
        adam("w", "grad")
    else:
        rate = torch.zeros(s["total"], dtype=f64, device="cuda")
        for (r, c), o in zip(s["shapes"], s["offs"]):
            rate[o:o + r * c] = _rate(r, c)
        got["w"] = s["w"].to(f64) * (1 - DECAY) - rate * s["o"].to(f64)
    if s["w16"] is not None:
        got["w16"] = got["w"]
    return got
