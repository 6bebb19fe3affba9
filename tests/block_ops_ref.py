"""Plain 64-bit definitions of the gated block, the norms around a residual
block and AdamW with 8-bit states, for the tests of their kernels (torch on the
CPU; they follow the formulas of the header and nothing of the library)."""
import math

import torch

F64 = torch.float64
E4M3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).to(F64)   # 0 .. 448
M32 = 0xffffffff


def act(g, kind):
    """act(g), act'(g)."""
    if kind == 0:
        p = torch.sigmoid(g)
        return g * p, p + g * p * (1 - p)
    p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def gated(x, w, kind, dy=None):
    """x: rows x cin; w: gate, up, down, b_gate, b_up, b_down (biases may be None).  Returns y, or with dy the
    gradients of x and of w in its order (None for biases that are None)."""
    wg, wu, wd, bg, bu, bd = (None if t is None else t.to(F64) for t in w)
    x = x.to(F64)
    zero = torch.zeros((), dtype=F64)
    g = x @ wg.T + (zero if bg is None else bg)
    u = x @ wu.T + (zero if bu is None else bu)
    a, slope = act(g, kind)
    if dy is None:
        return (a * u) @ wd.T + (zero if bd is None else bd)
    dy = dy.to(F64)
    dh = dy @ wd
    dg, du = dh * u * slope, dh * a
    return [dg @ wg + du @ wu, dg.T @ x, du.T @ x, dy.T @ (a * u)] + [
        None if b is None else t.sum(0) for b, t in ((bg, dg), (bu, du), (bd, dy))]


def normalise(x, eps):
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    return (x - mean) * rstd, mean, rstd


def _or(t, value):
    return torch.full((), value, dtype=F64) if t is None else t.to(F64)


def gate_rows(gate, group, rows):
    return torch.ones((), dtype=F64) if gate is None else gate.to(F64).repeat_interleave(group, 0)


def residual_forward(r, f, gate, group, p, post, pre, eps):
    """p: scale, post_gain, post_bias, pre_gain, pre_bias.  Returns out, z (None without pre), stats."""
    r, f = r.to(F64), f.to(F64)
    stats = torch.zeros(r.shape[0], 4, dtype=F64)
    n = f
    if post:
        n, stats[:, :1], stats[:, 1:2] = normalise(f, eps)
        n = n * _or(p[1], 1) + _or(p[2], 0)
    out = r + _or(p[0], 1) * gate_rows(gate, group, len(r)) * n
    z = None
    if pre:
        z, stats[:, 2:3], stats[:, 3:] = normalise(out, eps)
        z = z * _or(p[3], 1) + _or(p[4], 0)
    return out, z, stats


def norm_back(g, xhat, rstd):
    return rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))


def residual_backward(dz, dout, out, f, gate, group, p, post, stats):
    """Returns a dict of dr, df, dgate, scale, post_gain, post_bias, pre_gain, pre_bias."""
    f, st = f.to(F64), stats.to(F64)
    got = {}
    g = torch.zeros_like(f) if dout is None else dout.to(F64)
    if dz is not None:
        dz = dz.to(F64)
        ohat = (out.to(F64) - st[:, 2:3]) * st[:, 3:]
        g = g + norm_back(dz * _or(p[3], 1), ohat, st[:, 3:])
        got.update(pre_gain=(dz * ohat).sum(0), pre_bias=dz.sum(0))
    fhat = (f - st[:, :1]) * st[:, 1:2] if post else f
    n = fhat * _or(p[1], 1) + _or(p[2], 0) if post else f
    q = gate_rows(gate, group, len(f))
    dn = _or(p[0], 1) * q * g
    got.update(dr=g, scale=(g * q * n).sum(0))
    if gate is not None:
        got["dgate"] = (_or(p[0], 1) * g * n).view(-1, group, f.shape[1]).sum(1)
    got["df"] = dn
    if post:
        got.update(post_gain=(dn * fhat).sum(0), post_bias=dn.sum(0),
                   df=norm_back(dn * _or(p[1], 1), fhat, st[:, 1:2]))
    return got


def mix(x):
    x = x ^ (x >> 16)
    x = x * 0x9e3779b1 & M32
    x = x ^ (x >> 15)
    x = x * 0xbb67ae85 & M32
    return x ^ (x >> 16)


def adamw8_bits(count, place, seed):
    """The 32 random bits of every value."""
    key = mix((seed & M32) ^ mix((seed >> 32) + mix(place + 1) & M32))
    i = torch.arange(count, dtype=torch.int64)
    return mix((i & M32) ^ ((key + 0x9e3779b1 * (i >> 32)) & M32))


def adamw8_decode(codes, exps):
    """What the codes stand for (codes: count bytes; exps: a byte a block)."""
    e = exps.to(F64).repeat_interleave(128)[:codes.numel()]
    return codes.view(torch.float8_e4m3fn).to(torch.float32).to(F64) * torch.exp2(e - 134)


def adamw8_encode(v, u, root):
    """Codes and exponent bytes of v by the 16 random bits u of each value."""
    n = v.numel()
    fine = torch.isfinite(v)
    a = torch.where(fine, v.abs(), torch.zeros_like(v))
    top = torch.nn.functional.pad(a, (0, -n % 128)).view(-1, 128).amax(1)
    e = torch.where(top > 0, (torch.frexp(top).exponent + 126).clamp(1, 254), torch.zeros_like(top).int())
    t = a * torch.exp2(134 - e.to(F64)).repeat_interleave(128)[:n]
    at = torch.searchsorted(E4M3, t, right=True) - 1
    up = E4M3[at + 1] - E4M3[at]
    at = at + ((t - E4M3[at]) / up + (u.to(F64) + 0.5) / 65536 >= 1)
    if root:
        at = torch.where(a > 0, at.clamp(min=1), at)
    code = torch.where(fine, at, torch.full_like(at, 127)) + 128 * (torch.signbit(v) & fine)
    return code.to(torch.uint8), e.to(torch.uint8)


def adamw8(w, g, m, r, exps, place, rate, beta1, beta2, eps, decay, step, seed):
    """m, r: codes; exps: blocks x 2.  Returns w, m, r, exps after the step."""
    w, g = w.to(F64), g.to(F64)
    mv = beta1 * adamw8_decode(m, exps[:, 0]) + (1 - beta1) * g
    rv = torch.sqrt(beta2 * adamw8_decode(r, exps[:, 1]) ** 2 + (1 - beta2) * (g * g))
    w = w * (1 - decay) - rate * (mv / (1 - beta1 ** step)) / (rv / math.sqrt(1 - beta2 ** step) + eps)
    bits = adamw8_bits(w.numel(), place, seed)
    mc, me = adamw8_encode(mv, bits & 0xffff, False)
    rc, re = adamw8_encode(rv, bits >> 16, True)
    return w, mc, rc, torch.stack((me, re), 1)


def rel(got, want):
    """2-norm of the difference over the 2-norm of `want`."""
    d = torch.linalg.vector_norm(got.detach().cpu().to(F64) - want).item()
    n = torch.linalg.vector_norm(want).item()
    return d / n if n else (0.0 if d == 0 else math.inf)
