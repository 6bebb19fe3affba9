"""Gated feed-forward blocks, the norms around a residual block, and AdamW with 8-bit states, as cases to be timed and
compared.

Five calls that a training program makes between and after the stage tasks of a pipeline of residual blocks:

  gated_fwd  y = (act(x Wg^T + bg) * (x Wu^T + bu)) Wd^T + bd over the channels of each pixel
  gated_bwd  its gradients: dx, and those of the three weight matrices and their biases; it starts from x
  res_fwd    out = r + scale gate norm(f) and z = norm(out): what stands between two blocks
  res_bwd    its gradients: of r, f and the gate, and of the scale, gains and biases over all pixels
  adamw8     AdamW over every weight, its states kept as 8-bit floats with a power of two per 128 values

Tensors are NHWC: a row is a pixel, weights are [cout][cin].  Sizes are those of the U-Net, cell and stack workloads.
Where `own` is false the operators run in plain torch operations in float32 (the 8-bit states' roundings in float64),
rounded once at the end.
"""
import math

import torch

own = False

EPS = 1e-5                       # layer norm
BLOCK = 128                      # values of the 8-bit states that share a power of two
ADAM = {"rate": 1e-3, "beta1": 0.9, "beta2": 0.99, "eps": 1e-8, "decay": 1e-5, "step": 10, "seed": 0x1234567890ab}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------- the cases

def _gated(name, op, rows, cin, hidden, cout, dtype, act="silu", bias=True, ldx=0, ldy=0):
    """`rows` pixels from `cin` to `cout` channels; ldx, ldy: channels of the tensor that x (with dx) and y (with
    dy) are slices of, where not their own."""
    d = {"op": op, "rows": rows, "cin": cin, "hidden": hidden, "cout": cout, "dtype": dtype, "act": act, "bias": bias,
         "ldx": max(ldx, cin), "ldy": max(ldy, cout)}
    return dict(d, name=name) if name else d


def _res(name, op, images, pixels, c, dtype, gate="none", post=True, scale=True, ldr=0, ldf=0):
    """`images` of `pixels` pixels of `c` channels; gate: "none", "image" (a row of channels for each) or "pixel";
    post: whether the block's output is normalised; ldr, ldf: channels of the tensor that the stream (r, out and their
    gradients) and the block's output (with its gradient) are slices of."""
    d = {"op": op, "images": images, "pixels": pixels, "c": c, "dtype": dtype, "gate": gate, "post": post,
         "scale": scale, "ldr": max(ldr, c), "ldf": max(ldf, c)}
    return dict(d, name=name) if name else d


def _adam(name, shapes, dtype="bf16"):
    """shapes: "rows x cols" of each weight matrix, with a bias of `rows` values each; dtype: of the network."""
    d = {"op": "adamw8", "shapes": ",".join("%dx%d" % s for s in shapes), "dtype": dtype}
    return dict(d, name=name) if name else d


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
        # One pixel through a block of the 18-cell workload's width: what a program that answers for one position at
        # a time pays, latency and the weights' bytes.
        _gated("gated-fwd-pixel", "gated_fwd", 1, 256, 1024, 256, "bf16"),
        # A micro-batch of the 18-cell workload, 4 x 56 x 56 x 256, four hidden channels for each.
        _gated("gated-fwd-cells", "gated_fwd", 4 * 56 * 56, 256, 1024, 256, "bf16"),
        # A cropped image batch of 3 x 45 x 61 pixels and 100 channels in float32, from 100 to 72 channels, the result
        # written into its place in a concatenated tensor.
        _gated("gated-fwd-ragged", "gated_fwd", 3 * 45 * 61, 100, 270, 72, "fp32", act="gelu", ldy=200),
        # One image at the deep end of the 5-level U-Net, 12 x 12 pixels of 1024 channels, backward.
        _gated("gated-bwd-b1", "gated_bwd", 144, 1024, 2048, 1024, "bf16"),
        # A micro-batch of the U-Net's first level, 4 x 192 x 192 x 64: many pixels, few channels.
        _gated("gated-bwd-unet0", "gated_bwd", 4 * 192 * 192, 64, 256, 64, "bf16", act="gelu"),
        # A micro-batch of 4 x 32 x 32 pixels of 1024 channels at the deep end of the 6-level U-Net: the largest.
        _gated("gated-bwd-deep", "gated_bwd", 4 * 32 * 32, 1024, 4096, 1024, "bf16", bias=False),
        # One image at the deep end of the 5-level U-Net between two blocks: latency.
        _res("res-fwd-b1", "res_fwd", 1, 144, 1024, "bf16", post=False, scale=False),
        # A micro-batch of the U-Net's first level, its gate one value for each channel of an image.
        _res("res-fwd-unet0", "res_fwd", 4, 192 * 192, 64, "bf16", gate="image"),
        # A micro-batch of the 18-cell workload, a gate at every pixel.
        _res("res-bwd-cells", "res_bwd", 4, 56 * 56, 256, "bf16", gate="pixel"),
        # A micro-batch of the 6-level U-Net's first level, 2 x 256 x 256 x 128, its stream a slice of the concatenated
        # tensor of 384 channels.
        _res("res-bwd-unet6", "res_bwd", 2, 256 * 256, 128, "bf16", gate="image", ldr=384),
        # The step of the 4-layer, 16-channel float32 stack's weights and biases: what a toy pays.
        _adam("adamw8-stack", [(16, 144)] * 4, "fp32"),
        # The step of all 31 million weights and the biases of the 5-level U-Net, with the bfloat16 copies.
        _adam("adamw8-unet5", _unet(5, 64)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _products(case):
    """Operations of the products of one pass, 2 a multiply-add."""
    unit = 2.0 * case["rows"] * case["hidden"]
    return unit * (2 * case["cin"] + case["cout"]) if case["op"] == "gated_fwd" else \
        unit * (6 * case["cin"] + 2 * case["cout"])


def draw(rng):
    op = rng.choice(("gated_fwd", "gated_fwd", "gated_bwd", "gated_bwd", "res_fwd", "res_bwd", "adamw8"))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    if op == "adamw8":
        shapes, size = [], 0
        for _ in range(rng.choice((1, 2, 4, 8, 12, 60))):
            r, c = _log(rng, 1, 2048), _log(rng, 1, 2048) * rng.choice((1, 9))
            if not shapes or size + r * c <= 30 << 20:
                shapes, size = shapes + [(r, c)], size + r * c
        return _adam(None, shapes, dtype)

    def channels(hi):
        c = _log(rng, 1, hi)
        return (c + 7) // 8 * 8 if c > 16 and rng.random() < 0.6 else c

    def wide(c):
        return c + (_log(rng, 1, 512) if rng.random() < 0.3 else 0)

    if op.startswith("res"):
        c = channels(4096)
        most = max(1, 2 * 256 * 256 * 128 // (1 if dtype == "bf16" else 2) // c)
        images = _log(rng, 1, min(64, most))
        return _res(None, op, images, _log(rng, 1, min(1 << 18, max(1, most // images))), c, dtype,
                    rng.choice(("none", "image", "pixel")), rng.random() < 0.7, rng.random() < 0.7, wide(c), wide(c))
    top = 0.9 * _products(listed()[5])
    while True:
        cin, hidden = channels(1024), channels(4096)
        cout = cin if rng.random() < 0.6 else channels(1024)
        case = _gated(None, op, _log(rng, 1, 4 * 192 * 192), cin, hidden, cout, dtype, rng.choice(("silu", "gelu")),
                      rng.random() < 0.6, wide(cin), wide(cout))
        cost = _products(case) * (6 if dtype == "fp32" else 1)
        if cost <= top and case["rows"] * max(hidden, cin, cout) <= 4 * 192 * 192 * 512:
            return case


# ---------------------------------------------------------------- inputs

def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def _flat(sizes):
    """Offsets of tensors of these sizes in one buffer, each at a multiple of BLOCK values, and the buffer's size."""
    at, offs = 0, []
    for s in sizes:
        offs.append(at)
        at += (s + BLOCK - 1) // BLOCK * BLOCK
    return offs, at


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    s = {"case": case}
    if case["op"] == "adamw8":
        return _prepare_adam(s, normal, g)
    dt = DT[case["dtype"]]

    def tensor(rows, c, ld, values=None):
        t = torch.empty(rows, ld, dtype=dt, device="cuda")[:, :c]
        return t if values is None else t.copy_(values)

    if case["op"].startswith("gated"):
        rows, cin, hidden, cout = (case[k] for k in ("rows", "cin", "hidden", "cout"))
        # a normalised input, and weights that keep its size
        s["x"] = tensor(rows, cin, case["ldx"], normal(rows, cin))
        for k, r, c in (("gate", hidden, cin), ("up", hidden, cin), ("down", cout, hidden)):
            s["w_" + k] = (normal(r, c) * (1.5 / math.sqrt(c))).to(dt)
            s["b_" + k] = 0.1 * normal(r) if case["bias"] else None
        if case["op"] == "gated_fwd":
            s["y"] = tensor(rows, cout, case["ldy"])
        else:
            s["dy"] = tensor(rows, cout, case["ldy"], 1e-2 * normal(rows, cout))
            s["dx"] = tensor(rows, cin, case["ldx"])
            for k in ("w_gate", "w_up", "w_down", "b_gate", "b_up", "b_down"):
                s["d" + k] = None if s[k] is None else torch.empty(s[k].shape, device="cuda")
        if own:
            import paper_2004_09910_amd as tgp
            s["shape"] = tgp.gated_shape(cin, hidden, cout, tgp.BF16 if case["dtype"] == "bf16" else tgp.FP32,
                                         tgp.ACT_SILU if case["act"] == "silu" else tgp.ACT_GELU)
            names = ("w_gate", "w_up", "w_down", "b_gate", "b_up", "b_down")
            s["weights"] = tgp.gated_weights(*[_at(s[k]) for k in names])
            if case["op"] == "gated_bwd":
                s["grads"] = tgp.gated_grads(*[_at(s["d" + k]) for k in names])
            n = tgp.gated_workspace(s["shape"], rows, case["op"] == "gated_bwd")
            s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
        return s
    c, rows = case["c"], case["images"] * case["pixels"]
    s["group"] = {"none": 0, "image": case["pixels"], "pixel": 1}[case["gate"]]
    # a stream that has grown over some blocks, and a block's output of a size and offset of its own in every channel
    r = 3 * normal(rows, c) + normal(c)
    f = normal(rows, c) * normal(c).abs().add_(0.2) + 0.5 * normal(c)
    s["f"] = tensor(rows, c, case["ldf"], f)
    s["gate"] = tensor(rows // s["group"], c, c, 1 + 0.3 * normal(rows // s["group"], c)) if s["group"] else None
    s["scale"] = 0.3 * normal(c) if case["scale"] else None
    for k in ("post", "pre"):
        there = k == "pre" or case["post"]
        s[k + "_gain"], s[k + "_bias"] = (1 + 0.1 * normal(c), 0.1 * normal(c)) if there else (None, None)
    if case["op"] == "res_fwd":
        s["r"], s["out"] = tensor(rows, c, case["ldr"], r), tensor(rows, c, case["ldr"])
        s["z"], s["stats"] = tensor(rows, c, c), torch.zeros(rows, 4, device="cuda")
    else:
        # what the forward left
        s["r"] = r
        got = _res_forward(s)
        s["out"], s["stats"] = tensor(rows, c, case["ldr"], got["out"]), got["stats"]
        s["dz"] = tensor(rows, c, c, 1e-2 * normal(rows, c))
        s["dout"] = tensor(rows, c, case["ldr"], 1e-2 * normal(rows, c))
        s["dr"], s["df"] = tensor(rows, c, case["ldr"]), tensor(rows, c, case["ldf"])
        s["dgate"] = None if s["gate"] is None else torch.empty_like(s["gate"])
        for k in ("scale", "post_gain", "post_bias", "pre_gain", "pre_bias"):
            s["d" + k] = None if s[k] is None else torch.empty(c, device="cuda")
        del s["r"]
    if own:
        import paper_2004_09910_amd as tgp
        s["shape"] = tgp.residual_shape(rows, c, tgp.BF16 if case["dtype"] == "bf16" else tgp.FP32, s["group"],
                                        case["post"], EPS)
        names = ("scale", "post_gain", "post_bias", "pre_gain", "pre_bias")
        s["params"] = tgp.residual_params(*[_at(s[k]) for k in names])
        if case["op"] == "res_bwd":
            s["grads"] = tgp.residual_grads(*[_at(s["d" + k]) for k in names])
            n = tgp.residual_norm_backward_workspace(s["shape"])
            s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    return s


def _at(t):
    return None if t is None else t.data_ptr()


def _prepare_adam(s, normal, g):
    case = s["case"]
    sizes = [n for r, c in _shapes(case) for n in (r * c, r)]
    offs, total = _flat(sizes)
    used = torch.zeros(total, device="cuda")
    for o, n in zip(offs, sizes):
        used[o:o + n] = 1    # what lies between two tensors belongs to none and stays zero
    s["w"] = 0.05 * normal(total) * used
    s["w16"] = s["w"].bfloat16() if case["dtype"] == "bf16" else None
    # gradients whose size differs from value to value and from block to block, and states of earlier ones
    size = 1e-3 * torch.exp(1.5 * normal(total)) * torch.exp(2 * normal(total // BLOCK)).repeat_interleave(BLOCK) * used
    s["grad"] = size * normal(total)
    m, r = 0.3 * size * normal(total), size * (0.3 + torch.rand(total, device="cuda", generator=g))
    s["exps"] = torch.empty(total // BLOCK, 2, dtype=torch.uint8, device="cuda")
    for k, (name, v) in enumerate((("m", m), ("r", r))):
        e = torch.frexp(v.view(-1, BLOCK).abs().amax(1)).exponent.long() + 126    # 127 + floor(log2)
        e = torch.where(v.view(-1, BLOCK).abs().amax(1) > 0, e.clamp(1, 254), torch.zeros_like(e))
        s["exps"][:, k] = e.to(torch.uint8)
        s[name] = (v.double().view(-1, BLOCK) * _pow2(134 - e)[:, None]).float().reshape(-1).to(torch.float8_e4m3fn)
    sizes_of = [(n, o, k) for k, (n, o) in enumerate(zip(sizes, offs))]
    if own:
        import paper_2004_09910_amd as tgp
        s["list"] = tgp.adamw8_tensors([
            (n, s["w"][o:].data_ptr(), None if s["w16"] is None else s["w16"][o:].data_ptr(), s["grad"][o:].data_ptr(),
             s["m"][o:].data_ptr(), s["r"][o:].data_ptr(), s["exps"][o // BLOCK:].data_ptr())
            for n, o, _ in sizes_of])
    else:
        # every value's place in its tensor, and its tensor's key
        s["index"] = torch.zeros(total, dtype=torch.int64, device="cuda")
        s["key"] = torch.zeros(total, dtype=torch.int64, device="cuda")
        for n, o, k in sizes_of:
            s["index"][o:o + n] = torch.arange(n, device="cuda")
            s["key"][o:o + n] = _key(k)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2004_09910_amd as tgp
    case, stream = s["case"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "gated_fwd":
        tgp.gated_forward(s["shape"], case["rows"], s["weights"], s["x"].data_ptr(), case["ldx"], s["y"].data_ptr(),
                          case["ldy"], s["ws"].data_ptr(), s["ws"].numel(), stream)
        return {"y": s["y"]}
    if case["op"] == "gated_bwd":
        tgp.gated_backward(s["shape"], case["rows"], s["weights"], s["dy"].data_ptr(), case["ldy"], s["x"].data_ptr(),
                           case["ldx"], s["dx"].data_ptr(), case["ldx"], s["grads"], True, s["ws"].data_ptr(),
                           s["ws"].numel(), stream)
        return _present(s, "dx", "dw_gate", "dw_up", "dw_down", "db_gate", "db_up", "db_down")
    if case["op"] == "res_fwd":
        c = case["c"]
        tgp.residual_norm_forward(s["shape"], s["params"], s["r"].data_ptr(), case["ldr"], s["f"].data_ptr(),
                                  case["ldf"], _at(s["gate"]), c, s["out"].data_ptr(), case["ldr"], s["z"].data_ptr(),
                                  c, s["stats"].data_ptr(), stream)
        return _present(s, "out", "z", "stats")
    if case["op"] == "res_bwd":
        c = case["c"]
        tgp.residual_norm_backward(s["shape"], s["params"], s["dz"].data_ptr(), c, s["dout"].data_ptr(), case["ldr"],
                                   s["out"].data_ptr(), case["ldr"], s["f"].data_ptr(), case["ldf"], _at(s["gate"]), c,
                                   s["stats"].data_ptr(), s["dr"].data_ptr(), case["ldr"], s["df"].data_ptr(),
                                   case["ldf"], _at(s["dgate"]), c, s["grads"], True, s["ws"].data_ptr(),
                                   s["ws"].numel(), stream)
        return _present(s, "dr", "df", "dgate", "dscale", "dpost_gain", "dpost_bias", "dpre_gain", "dpre_bias")
    k = ADAM
    tgp.adamw8_step(s["list"], k["rate"], k["beta1"], k["beta2"], k["eps"], k["decay"], k["step"], k["seed"], stream)
    return _present(s, "w", "w16", "m", "r", "exps")


def _present(s, *names):
    return {k: s[k] for k in names if s.get(k) is not None}


def _run_plain(s):
    return {"gated_fwd": _gated_forward, "gated_bwd": _gated_backward, "res_fwd": _res_forward,
            "res_bwd": _res_backward, "adamw8": _adam_step}[s["case"]["op"]](s)


def _linear(x, w, b):
    y = x @ w.float().T
    return y if b is None else y + b


def _act(g, kind):
    """act(g) and act'(g)."""
    if kind == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _gated_forward(s):
    x = s["x"].float()
    a, _ = _act(_linear(x, s["w_gate"], s["b_gate"]), s["case"]["act"])
    h = a * _linear(x, s["w_up"], s["b_up"])
    return {"y": _linear(h, s["w_down"], s["b_down"]).to(s["x"].dtype)}


def _gated_backward(s):
    x, dy = s["x"].float(), s["dy"].float()
    a, slope = _act(_linear(x, s["w_gate"], s["b_gate"]), s["case"]["act"])
    u = _linear(x, s["w_up"], s["b_up"])
    dh = dy @ s["w_down"].float()
    dg, du = dh * u * slope, dh * a
    got = {"dx": (dg @ s["w_gate"].float() + du @ s["w_up"].float()).to(s["x"].dtype),
           "dw_gate": dg.T @ x, "dw_up": du.T @ x, "dw_down": dy.T @ (a * u)}
    if s["b_gate"] is not None:
        got.update(db_gate=dg.sum(0), db_up=du.sum(0), db_down=dy.sum(0))
    return got


def _normalise(x):
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = ((d * d).mean(1, keepdim=True) + EPS).rsqrt()
    return d * rstd, mean, rstd


def _gate(s):
    """The gate of every pixel, with the scale; 1 where there is none."""
    t = 1.0 if s["gate"] is None else s["gate"].float().repeat_interleave(s["group"], 0)
    return t if s["scale"] is None else t * s["scale"]


def _res_forward(s):
    n, post = s["f"].float(), s["case"]["post"]
    stats = torch.zeros(n.shape[0], 4, device="cuda")
    if post:
        n, stats[:, :1], stats[:, 1:2] = _normalise(n)
        n = n * s["post_gain"] + s["post_bias"]
    out = s["r"].float() + _gate(s) * n
    z, stats[:, 2:3], stats[:, 3:] = _normalise(out)
    z = z * s["pre_gain"] + s["pre_bias"]
    return {"out": out.to(s["f"].dtype), "z": z.to(s["f"].dtype), "stats": stats}


def _norm_back(g, xhat, rstd):
    return rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))


def _res_backward(s):
    dt, st = s["f"].dtype, s["stats"]
    dz, out, f = s["dz"].float(), s["out"].float(), s["f"].float()
    xhat = (out - st[:, 2:3]) * st[:, 3:]
    got = {"dpre_gain": (dz * xhat).sum(0), "dpre_bias": dz.sum(0)}
    g = s["dout"].float() + _norm_back(dz * s["pre_gain"], xhat, st[:, 3:])
    got["dr"] = g.to(dt)
    fhat = (f - st[:, :1]) * st[:, 1:2] if s["case"]["post"] else f
    n = fhat * s["post_gain"] + s["post_bias"] if s["case"]["post"] else f
    dn = _gate(s) * g
    if s["scale"] is not None:
        got["dscale"] = (g * n if s["gate"] is None else
                         g * n * s["gate"].float().repeat_interleave(s["group"], 0)).sum(0)
    if s["gate"] is not None:
        t = g * n if s["scale"] is None else g * n * s["scale"]
        got["dgate"] = t.view(-1, s["group"], t.shape[1]).sum(1).to(dt)
    if s["case"]["post"]:
        got.update(dpost_gain=(dn * fhat).sum(0), dpost_bias=dn.sum(0))
        dn = _norm_back(dn * s["post_gain"], fhat, st[:, 1:2])
    got["df"] = dn.to(dt)
    return got


def _pow2(k):
    """2^k in float64, for whole numbers k."""
    return ((k + 1023) << 52).view(torch.float64)


LOW = 0xffffffff


def _mix(x):
    """A mixing of 32 bits (in int64): multiplications by odd parts of the golden ratio and of sqrt 3."""
    x = x ^ (x >> 16)
    x = (x * 0x9e3779b1) & LOW
    x = x ^ (x >> 15)
    x = (x * 0xbb67ae85) & LOW
    return x ^ (x >> 16)


def _key(k):
    """The key of tensor k of a list."""
    seed = ADAM["seed"]
    return _mix((seed & LOW) ^ _mix(((seed >> 32) + _mix(k + 1)) & LOW))


def _decode(codes, exps):
    return codes.float().double().view(-1, BLOCK) * _pow2(exps.long() - 134)[:, None]


def _adam_step(s):
    k, f64 = ADAM, torch.float64
    b1, b2 = k["beta1"], k["beta2"]
    g = s["grad"].to(f64).view(-1, BLOCK)
    m = b1 * _decode(s["m"], s["exps"][:, 0]) + (1 - b1) * g
    r = torch.sqrt(b2 * _decode(s["r"], s["exps"][:, 1]).square() + (1 - b2) * (g * g))
    step = (m / (1 - b1 ** k["step"])) / (r / math.sqrt(1 - b2 ** k["step"]) + k["eps"])
    s["w"].copy_((s["w"].view(-1, BLOCK).to(f64) * (1 - k["decay"]) - k["rate"] * step).view(-1))
    if s["w16"] is not None:
        s["w16"].copy_(s["w"])
    bits = _mix(s["index"] ^ s["key"]).view(-1, BLOCK)
    for col, name, v, u in ((0, "m", m, bits & 0xffff), (1, "r", r, bits >> 16)):
        most = v.abs().amax(1)
        e = (torch.frexp(most).exponent.long() + 126).clamp(1, 254) * (most > 0)
        t = v.abs() * _pow2(134 - e)[:, None]
        ulp = _pow2((torch.frexp(t).exponent.long() - 1).clamp(min=-6) - 3)
        q = torch.floor(t / ulp + (u.to(f64) + 0.5) * 2.0 ** -16)
        if name == "r":
            q = torch.where(v > 0, q.clamp(min=1), q)    # a root that is not zero stays so
        s[name].copy_((torch.sign(v) * q * ulp).view(-1).float())
        s["exps"][:, col] = e.to(torch.uint8)
    return _present(s, "w", "w16", "m", "r", "exps")


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    e = 2 if case.get("dtype") == "bf16" else 4
    if case["op"].startswith("gated"):
        rows, cin, hidden, cout = (case[k] for k in ("rows", "cin", "hidden", "cout"))
        w, b = hidden * (2 * cin + cout), (2 * hidden + cout) * case["bias"]
        if case["op"] == "gated_fwd":
            return {"bytes": e * (rows * (cin + cout) + w) + 4 * b, "flops": _products(case)}
        return {"bytes": e * (rows * (2 * cin + cout) + w) + 4 * (w + 2 * b), "flops": _products(case)}
    if case["op"] == "adamw8":
        n = sum(r * c + r for r, c in _shapes(case))
        return {"bytes": n * (16 + (2 if case["dtype"] == "bf16" else 0)) + n // 32, "flops": 30 * n}
    rows, c = case["images"] * case["pixels"], case["c"]
    gates = {"none": 0, "image": case["images"], "pixel": rows}[case["gate"]]
    if case["op"] == "res_fwd":      # r, f and the gate in; out, z and statistics out
        return {"bytes": e * c * (4 * rows + gates) + 16 * rows, "flops": 20 * rows * c}
    return {"bytes": e * c * (6 * rows + 2 * gates) + 16 * rows, "flops": 40 * rows * c}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("gated"):
        return _exact_gated(s)
    return _exact_adam(s) if case["op"] == "adamw8" else _exact_res(s)


def _exact_gated(s):
    case, f64 = s["case"], torch.float64
    x, wg, wu, wd = (s[k].to(f64) for k in ("x", "w_gate", "w_up", "w_down"))
    bg, bu, bd = (torch.zeros((), dtype=f64, device="cuda") if s[k] is None else s[k].to(f64)
                  for k in ("b_gate", "b_up", "b_down"))
    g, u = torch.matmul(x, wg.t()).add_(bg), torch.matmul(x, wu.t()).add_(bu)
    if case["act"] == "silu":
        p = torch.sigmoid(g)
        slope = p + g * p * torch.sigmoid(-g)
    else:
        p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        slope = p + g * torch.exp(-(g * g) / 2) / math.sqrt(2 * math.pi)
    act = g * p
    if case["op"] == "gated_fwd":
        return {"y": torch.matmul(act * u, wd.t()).add_(bd)}
    dy = s["dy"].to(f64)
    dh = torch.matmul(dy, wd)
    got = {"dw_down": torch.matmul(dy.t(), act * u)}
    dg, du = slope.mul_(u).mul_(dh), act.mul_(dh)
    got.update(dx=torch.matmul(torch.cat((dg, du), 1), torch.cat((wg, wu), 0)),
               dw_gate=torch.matmul(dg.t(), x), dw_up=torch.matmul(du.t(), x))
    if case["bias"]:
        got.update(db_gate=dg.sum(0), db_up=du.sum(0), db_down=dy.sum(0))
    return got


def _exact_res(s):
    case, f64 = s["case"], torch.float64
    images, pixels, c = case["images"], case["pixels"], case["c"]

    def of(name, fill):
        return torch.full((), fill, dtype=f64, device="cuda") if s.get(name) is None else s[name].to(f64)

    def field(t):    # images x pixels x channels
        return t.to(f64).reshape(images, pixels, c)

    def moments(t):
        var, mean = torch.var_mean(t, dim=2, unbiased=False, keepdim=True)
        return mean, 1 / torch.sqrt(var + EPS)

    f = field(s["f"])
    q = of("gate", 1.0)
    if q.dim():
        q = q.view(images, -1, c)    # a row for the image, or for each of its pixels
    if case["op"] == "res_fwd":
        stats = torch.zeros(images, pixels, 4, dtype=f64, device="cuda")
        n = f
        if case["post"]:
            stats[..., :1], stats[..., 1:2] = moments(f)
            n = (f - stats[..., :1]) * stats[..., 1:2] * of("post_gain", 1) + of("post_bias", 0)
        out = field(s["r"]) + of("scale", 1) * q * n
        stats[..., 2:3], stats[..., 3:] = moments(out)
        z = (out - stats[..., 2:3]) * stats[..., 3:] * of("pre_gain", 1) + of("pre_bias", 0)
        return {"out": out.view(-1, c), "z": z.view(-1, c), "stats": stats.view(-1, 4)}
    m1, r1, m2, r2 = s["stats"].to(f64).view(images, pixels, 4).split(1, 2)
    dz, dout = field(s["dz"]), field(s["dout"])
    ohat = (field(s["out"]) - m2) * r2
    a = dz * of("pre_gain", 1)
    g = dout + r2 * a - r2 * (a.sum(2, keepdim=True) + ohat * (a * ohat).sum(2, keepdim=True)) / c
    got = {"dr": g.view(-1, c), "dpre_gain": (dz * ohat).sum((0, 1)), "dpre_bias": dz.sum((0, 1))}
    fhat = (f - m1) * r1 if case["post"] else f
    n = fhat * of("post_gain", 1) + of("post_bias", 0)
    gn = g * n
    if case["scale"]:
        got["dscale"] = (gn * q).sum((0, 1))
    if q.dim():
        got["dgate"] = of("scale", 1) * (gn.sum(1) if case["gate"] == "image" else gn.view(-1, c))
    dn = of("scale", 1) * q * g
    if case["post"]:
        got["dpost_gain"], got["dpost_bias"] = (dn * fhat).sum((0, 1)), dn.sum((0, 1))
        b = dn * of("post_gain", 1)
        dn = r1 * b - r1 * (b.sum(2, keepdim=True) + fhat * (b * fhat).sum(2, keepdim=True)) / c
    got["df"] = dn.view(-1, c)
    return got


def _exact_adam(s):
    k, f64 = ADAM, torch.float64
    # every value of a positive 8-bit float of 4 exponent and 3 mantissa bits, in order
    grid = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).to(f64)
    total = s["w"].numel()
    old = []
    for name, col in (("m", 0), ("r", 1)):
        size = torch.exp2(s["exps"][:, col].to(f64) - 134).repeat_interleave(BLOCK)
        old.append(s[name].to(torch.float32).to(f64) * size)
    g = s["grad"].to(f64)
    m = (1 - k["beta1"]) * g + old[0] * k["beta1"]
    v = (1 - k["beta2"]) * g.square() + old[1].square() * k["beta2"]
    den = torch.sqrt(v / (1 - k["beta2"] ** k["step"])) + k["eps"]
    w = (1 - k["decay"]) * s["w"].to(f64) - k["rate"] / (1 - k["beta1"] ** k["step"]) * (m / den)
    got = {"w": w, "exps": torch.zeros_like(s["exps"])}
    if s["w16"] is not None:
        got["w16"] = w
    sizes = [n for r, c in _shapes(s["case"]) for n in (r * c, r)]
    bits = torch.zeros(total, dtype=torch.int64, device="cuda")
    for j, (n, o) in enumerate(zip(sizes, _flat(sizes)[0])):
        bits[o:o + n] = _mix(torch.arange(n, device="cuda") ^ _key(j))
    for name, col, value, u in (("m", 0, m, bits % 65536), ("r", 1, v.sqrt(), bits // 65536)):
        most = value.abs().view(-1, BLOCK).amax(1)
        e = torch.where(most > 0, torch.floor(torch.log2(most.clamp(min=2.0 ** -1000))).clamp(-126, 127) + 127, 0 * most)
        t = value.abs() * torch.exp2(134 - e).repeat_interleave(BLOCK)
        at = torch.searchsorted(grid, t, right=True) - 1
        below, above = grid[at], grid[(at + 1).clamp(max=126)]
        share = (t - below) / torch.where(above > below, above - below, above + 1)
        q = torch.where(share >= 1 - (u + 0.5) / 65536, above, below)
        if name == "r":
            q = torch.where((value > 0) & (q == 0), grid[1], q)
        got[name] = torch.copysign(q, value)
        got["exps"][:, col] = e.to(torch.uint8)
    return got
