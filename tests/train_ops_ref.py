"""Plain 64-bit definitions of the layer norm, the orthogonalised update and
the weights' step, for the tests of their kernels (torch on the CPU; the loops
follow the formulas of the header and nothing of the library)."""
import math

import torch

F64 = torch.float64
NS = (3.4445, -4.7750, 2.0315)


def norm_forward(x, gain, bias, eps):
    """x: rows x C.  Returns y, mean, rstd."""
    x = x.to(F64)
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1 / torch.sqrt(var + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gain is not None:
        y = y * gain.to(F64)
    if bias is not None:
        y = y + bias.to(F64)
    return y, mean, rstd


def norm_backward(dy, x, gain, mean, rstd):
    """Returns dx, dgain, dbias."""
    dy, x, mean, rstd = (t.to(F64) for t in (dy, x, mean, rstd))
    xhat = (x - mean[:, None]) * rstd[:, None]
    g = dy if gain is None else dy * gain.to(F64)
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def muon(grad, momentum, mu, nesterov, steps, eps):
    """Returns the new momentum (None without one) and the update."""
    g = grad.to(F64)
    m, u = None, g
    if momentum is not None:
        m = mu * momentum.to(F64) + g
        u = g + mu * m if nesterov else m
    flip = u.shape[0] > u.shape[1]
    x = u.T if flip else u
    norm = torch.linalg.matrix_norm(x)
    x = x / (norm + eps) if norm + eps != 0 else torch.zeros_like(x)
    for _ in range(steps):
        a = x @ x.T
        x = NS[0] * x + (NS[1] * a + NS[2] * a @ a) @ x
    return m, (x.T if flip else x)


def weight_step(w, update, rate, decay):
    return w.to(F64) * (1 - decay) - rate * update.to(F64)


def adamw(w, g, m, v, rate, beta1, beta2, eps, decay, step):
    w, g, m, v = (t.to(F64) for t in (w, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    den = torch.sqrt(v / (1 - beta2 ** step)) + eps
    return w * (1 - decay) - rate * (m / (1 - beta1 ** step)) / den, m, v


def rel(got, want):
    """2-norm of the difference over the 2-norm of `want`."""
    d = torch.linalg.vector_norm(got.detach().cpu().to(F64) - want).item()
    n = torch.linalg.vector_norm(want).item()
    return d / n if n else (0.0 if d == 0 else math.inf)
