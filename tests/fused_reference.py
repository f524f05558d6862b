"""64-bit results of the operators of exo_fused.h, each with a bound of what rounding may do to it.

A value is a pair (value, bound) of fp64 tensors.  The bounds count roundings: half a step (2^-8 bf16, 2^-11 fp16, relative, and 2^-25 of
fp16's gradual underflow) wherever the operator rounds to 16 bits, and for a sum of K products in fp32 K * 2^-23 of the sum of their
magnitudes (the tensor core may truncate).  Functions of fp32 arguments get 2^-18 relative: exponentials by ex2 and quotients by approximate
reciprocals are good to some 2^-21.
"""
import math

import torch

FUNCTION = 2.0 ** -18


def half_step(dtype):
    return torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 2.0 ** -24


def smallest(dtype):
    return 2.0 ** -25 if dtype == torch.float16 else 0.0


def exactly(t):
    t = t.double()
    return t, torch.zeros_like(t)


def rounded(a, dtype):
    v, e = a
    return v, e + half_step(dtype) * (v.abs() + e) + smallest(dtype)


def product(a, b):
    """Elementwise."""
    (v, e), (w, f) = a, b
    return v * w, v.abs() * f + e * w.abs() + e * f


def plus(a, b):
    return a[0] + b[0], a[1] + b[1]


def matmul(a, b):
    (v, e), (w, f) = a, b
    m = (v.abs() + e) @ (w.abs() + f)
    return v @ w, m - v.abs() @ w.abs() + v.shape[1] * 2.0 ** -23 * m


def turned(a):
    return a[0].t(), a[1].t()


def rows(a, at):
    return a[0][at], a[1][at]


ACTS = {
    "silu": lambda z: z * torch.sigmoid(z),
    "gelu": lambda z: z * 0.5 * torch.erfc(-z / math.sqrt(2.0)),
    "gelu_tanh": lambda z: z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)),
}


def activation(name, z):
    """act and its derivative.  Both derivatives are bounded: |act'| < 1.13 and |act''| < 1 for all three."""
    v = z[0].detach().clone().requires_grad_()
    a = ACTS[name](v)
    slope, = torch.autograd.grad(a.sum(), v)
    a = a.detach()
    # (a sigmoid's own error scales with the argument)
    return (a, 1.13 * z[1] + FUNCTION * a.abs()), (slope, z[1] + FUNCTION * (1.0 + z[0].abs() * slope.abs()))


def ffn(x, gate_up, down, act, dy=None):
    """{"y": ...} and with dy the gradients too, from 16-bit tensors."""
    dt, F = x.dtype, down.shape[1]
    X, Wg, Wu, Wd = exactly(x), exactly(gate_up[:F]), exactly(gate_up[F:]), exactly(down)
    g, u = matmul(X, turned(Wg)), matmul(X, turned(Wu))
    h = rounded(product(activation(act, g)[0], u), dt)
    out = {"y": rounded(matmul(h, turned(Wd)), dt)}
    if dy is None:
        return out
    dY = exactly(dy)
    g, u = rounded(g, dt), rounded(u, dt)          # as saved
    a, slope = activation(act, g)
    dh = matmul(dY, Wd)
    dg, du, h = (rounded(t, dt) for t in (product(product(dh, u), slope), product(dh, a), product(a, u)))
    dx = plus(matmul(dg, Wg), matmul(du, Wu))
    m = (dg[0].abs() + dg[1]) @ Wg[0].abs() + (du[0].abs() + du[1]) @ Wu[0].abs()
    out["dx"] = rounded((dx[0], dx[1] + 2 * F * 2.0 ** -23 * m), dt)   # one sum of 2 F products
    dgu = [matmul(turned(t), X) for t in (dg, du)]
    out["dgate_up"] = torch.cat([t[0] for t in dgu]), torch.cat([t[1] for t in dgu])
    out["ddown"] = matmul(turned(dY), h)
    return out


def ce(x, w, target, smoothing=0.0, ignore=-100, dloss=None, kept=True):
    """{"loss", "lse"} and with dloss the gradients too."""
    dt, V = x.dtype, w.shape[0]
    l, e = matmul(exactly(x), turned(exactly(w)))
    worst = e.amax(1)
    lse = torch.logsumexp(l, 1)
    # exponentials, their sum in fp32 over the columns, the logarithm, and the sum with the largest logit
    sure = worst + 2 * FUNCTION + V * 2.0 ** -23 / 16 + 2.0 ** -23 * (lse.abs() + l.abs().amax(1))
    taken = (target >= 0) & (target < V) & (target != ignore)
    at = torch.where(taken, target, 0)
    hit = l.gather(1, at[:, None])[:, 0]
    mean = l.mean(1)
    loss = torch.where(taken, lse - (1 - smoothing) * hit - smoothing * mean, 0.0)
    bound = sure + worst + 4 * 2.0 ** -24 * (lse.abs() + hit.abs()) + smoothing * V * 2.0 ** -23 * l.abs().mean(1)
    out = {"loss": (loss, torch.where(taken, bound, 0.0)), "lse": (lse, sure)}
    if dloss is None:
        return out
    r = torch.where(taken, dloss.double(), 0.0)
    p = torch.exp(l - lse[:, None])
    off = p * (torch.expm1(e + sure[:, None]) + FUNCTION + 2.0 ** -22 * (l - lse[:, None]).abs())
    if kept:   # the exponential was rounded to 16 bits, relative to the largest of its part
        off = off + p * half_step(dt) + smallest(dt) * p.amax(1, keepdim=True)
    hot = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    d = r[:, None] * (p - (1 - smoothing) * hot - smoothing / V)
    eps = 2.0 ** -23 * (p + hot + smoothing / V)
    # the gradient is rounded at a scale where the largest |dloss| is 2^13 or more
    step = smallest(dt) * r.abs().amax() / 2.0 ** 13
    d = (d, r.abs()[:, None] * (off + eps) + half_step(dt) * (d.abs() + r.abs()[:, None] * off) + step)
    out["dx"] = rounded(matmul(d, exactly(w)), dt)
    out["dw"] = matmul(turned(d), exactly(x))
    return out


def quantized(x):
    """(codes, scales) as fp32 arithmetic has them."""
    x = x.float().cpu()
    scale = (x.abs().amax(1) if x.shape[1] else torch.zeros(x.shape[0])) / torch.full((x.shape[0],), 127.0)
    safe = torch.where(scale > 0, scale, torch.ones_like(scale))
    codes = torch.where((scale > 0)[:, None], torch.round(x / safe[:, None]).clamp(-127, 127), torch.zeros_like(x))
    return codes.to(torch.int8), scale


def check(got, want, what=""):
    """|got - value| <= bound everywhere."""
    v, e = want
    got = got.double().to(v.device)
    over = (got - v).abs() - e
    assert torch.isfinite(got).all(), what
    worst = over.argmax()
    assert (over <= 0).all(), (what, "off by", (got - v).abs().flatten()[worst].item(), "allowed", e.flatten()[worst].item())
