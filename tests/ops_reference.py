"""Plain 64-bit evaluations of the operators that the tests compare the kernels with,
written from their formulas with torch's elementary operations (on any device)."""

import math

import torch

COEF = (3.4445, -4.7750, 2.0315)


def newton_schulz(g, steps=5, coef=COEF, eps=1e-7):
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t().contiguous()
    x = x / (torch.sqrt((x * x).sum()) + eps)
    a, b, c = coef
    for _ in range(steps):
        gram = x @ x.t().contiguous()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if tall else x


def muon_step(x, g, m, lr, momentum, weight_decay=0.0, nesterov=True, scale="rms", steps=5,
              coef=COEF, eps=1e-7, grad_scale=1.0, wd=True):
    """(x, m) after the step, from fp32 scalars as the C interface takes them."""
    f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    mu, lr, lam, gs = f32(momentum), f32(lr), f32(weight_decay), f32(grad_scale)
    g = g.double() * gs
    m = mu * m.double() + (1.0 - mu) * g
    u = mu * m + (1.0 - mu) * g if nesterov else m
    rows, cols = u.shape
    s = {"rms": 0.2 * math.sqrt(max(rows, cols)), "spectral": math.sqrt(max(1.0, rows / cols)),
         "unit": 1.0}[scale]
    o = newton_schulz(u, steps, coef, eps)
    return x.double() * (1.0 - lr * lam * wd) - lr * s * o, m


def relative(a, b):
    """2-norm of a - b over that of b."""
    a, b = a.double(), b.double()
    n = float(torch.linalg.vector_norm(b))
    d = float(torch.linalg.vector_norm(a - b))
    return d / n if n else d


def cross_entropy(hidden, table, targets, ignore=-100, reduction="mean"):
    """(mean, loss, grad_hidden, grad_table, size_hidden, size_table): the sizes are the
    gradients' sums with every term's magnitude, what their rounding errors go by."""
    h, w = hidden.double(), table.double()
    keep = targets != ignore
    rows = keep.nonzero()[:, 0]
    h, t = h[rows], targets[rows].long()
    z = h @ w.t().contiguous()
    top = z.max(dim=1, keepdim=True).values if len(rows) else z[:, :1]
    lse = torch.log(torch.exp(z - top).sum(dim=1, keepdim=True)) + top
    loss = torch.zeros(len(targets), dtype=torch.float64, device=hidden.device)
    loss[rows] = (lse - z.gather(1, t[:, None]))[:, 0]
    count = max(1, len(rows))
    q = torch.exp(z - lse)
    q.scatter_add_(1, t[:, None], torch.full_like(lse, -1.0))
    if reduction == "mean":
        q = q / count
    gh, sh = torch.zeros_like(hidden.double()), torch.zeros_like(hidden.double())
    gh[rows], sh[rows] = q @ w, q.abs() @ w.abs()
    qt = q.t().contiguous()
    return loss.sum() / count, loss, gh, qt @ h, sh, qt.abs() @ h.abs()
