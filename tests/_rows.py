"""64-bit forms of layer norm and of 8-bit checkpoints, and how far a correct fp32 kernel may be from them (torch, CPU or GPU; no code of
the library)."""
import math

import torch

U32 = 2.0 ** -24                     # half a step of fp32, relative
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}   # smallest positive number
# Additions that a sum over a row or over the rows may take one after another, and the few operations around it: a lane adds up to 64
# elements, six exchanges follow; over rows a lane adds its share, then 6 exchanges, 4 waves, 16 and 64 partial sums.
N_ROW, N_ROWS = 80, 300


def half_step(t, dtype):
    """Rounding to dtype: half a step relative to the value, half the smallest number near zero."""
    return t.abs() * (torch.finfo(dtype).eps / 2) + TINY[dtype] / 2


def pack64(x):
    """(q int8, b uint8) by the definition: frexp and powers from a table, all in 64 bits."""
    rows, c = x.shape
    v = torch.zeros((rows, -(-c // 32) * 32), dtype=torch.float64, device=x.device)
    v[:, :c] = x.double()
    v = v.view(rows, -1, 32)
    fine = torch.isfinite(v).all(2, keepdim=True)
    v0 = torch.where(fine, v, torch.zeros_like(v))
    _, ex = torch.frexp(v0.abs().amax(2, keepdim=True))
    b = (ex.long() - 1 + 127).clamp(min=1)                # largest in [2^(ex-1), 2^ex)
    b = torch.where(v0.abs().amax(2, keepdim=True) == 0, torch.ones_like(b), b)
    q = torch.round(v0 / steps(x.device)[b]).clamp(-127, 127)
    q = torch.where((q == 0) & (v0 != 0), torch.sign(v0), q)
    b = torch.where(fine, b, torch.full_like(b, 255))
    return q.to(torch.int8).view(rows, -1)[:, :c].contiguous(), b.to(torch.uint8).view(rows, -1)


def steps(device):
    return torch.tensor([2.0 ** (b - 133) for b in range(255)] + [float("nan")], dtype=torch.float64, device=device)


def unpack64(q, b):
    return q.double() * steps(q.device)[b.long()].repeat_interleave(32, 1)[:, :q.shape[1]]


def fwd64(x, w, b, eps, relu, res):
    """(y, stats, tolerance of y before its rounding, tolerance of stats)"""
    x = x.double()
    w = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    m = x.mean(1, keepdim=True)
    var = (x - m).square().mean(1, keepdim=True)
    r = (var + eps) ** -0.5
    pre = (x - m) * r * w + b + (0 if res is None else res.double())
    y = torch.where(pre < 0, torch.zeros_like(pre), pre) if relu else pre
    a = N_ROW * U32
    dm = a * x.abs().mean(1, keepdim=True)                       # the mean's sum
    dr = r * (a + dm.square() * r.square() / 2)                  # half of the sum of squares' error, a root, a quotient
    dy = w.abs() * ((x - m).abs() * dr + r * (dm + 4 * U32 * (x.abs() + m.abs()))) + 4 * U32 * (
        ((x - m) * r * w).abs() + b.abs() + (0 if res is None else res.double().abs()))
    return y, torch.cat([m, r], 1), dy, torch.cat([dm, dr], 1) + 1e-38


def bwd64(dout, x, stats, w, gate):
    """(dx, dweight, dbias, dresidual) and the tolerances of the first three before a rounding; gate: bool or None"""
    x, g = x.double(), dout.double()
    m, r = stats.double()[:, :1], stats.double()[:, 1:]
    w = torch.ones(x.shape[1], dtype=torch.float64, device=x.device) if w is None else w.double()
    if gate is not None:
        g = torch.where(gate, g, torch.zeros_like(g))
    xh, h = (x - m) * r, g * w
    c1, c2 = h.mean(1, keepdim=True), (h * xh).mean(1, keepdim=True)
    dx = r * (h - c1 - xh * c2)
    a = N_ROW * U32
    exh = r * U32 * (x.abs() + m.abs()) + 2 * U32 * xh.abs()
    ec1 = a * h.abs().mean(1, keepdim=True)
    ec2 = a * (h * xh).abs().mean(1, keepdim=True) + (h.abs() * exh).mean(1, keepdim=True)
    edx = r * (ec1 + xh.abs() * ec2 + exh * c2.abs() + 4 * U32 * (h.abs() + c1.abs() + (xh * c2).abs()))
    an = N_ROWS * U32
    edw = (g.abs() * exh).sum(0) + an * (g * xh).abs().sum(0)
    return (dx, (g * xh).sum(0), g.sum(0), g), (edx, edw + 1e-38, an * g.abs().sum(0) + 1e-38)


def within(got, want, tol, dtype=None):
    """got is `want` but for tol and, given a dtype, one rounding to it (of a value that may be off by tol)."""
    got = got.double()
    if dtype is not None:
        tol = tol + half_step(want.abs() + tol, dtype)
        # rounding takes a value from half a step above the type's largest on to infinity
        most = torch.finfo(dtype).max
        over = torch.isinf(got) & (want.abs() + tol >= most + 2.0 ** math.floor(math.log2(most)) * torch.finfo(dtype).eps / 2)
        got = torch.where(over & (torch.sign(got) == torch.sign(want)), want, got)
    off = (got - want).abs() - tol
    assert got.shape == want.shape and not torch.isnan(got).any()
    worst = off.max().item() if off.numel() else -1.0
    assert worst <= 0, f"{(off > 0).sum().item()} of {off.numel()} beyond, worst by {worst:.3g} of {tol.flatten()[off.argmax()].item():.3g}"
