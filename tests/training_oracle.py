"""The operators of a training step in 64 bits, from their definitions, and how far fp32 arithmetic may be off.

A bound counts roundings: half a step of the output's type relative to the value, and for a sum of K products in fp32, in whatever order, two
roundings of 2^-24 per term relative to the sum of the magnitudes (the matrix cores may cut where they do not round).
"""
import torch

from operator_oracle import U32, half_step


def product(a, b):
    """(a @ b, bound of it in fp32) of stored matrices."""
    a, b = a.double(), b.double().contiguous()
    return a @ b, 2 * (a.shape[1] + 16) * U32 * (a.abs() @ b.abs())


def stored(value, bound, dtype):
    """The bound of a value rounded to a type."""
    return bound + half_step(dtype) * (value.abs() + bound)


def silu(g):
    """(silu, its slope): g / (1 + e^-g), s (1 + g (1 - s))."""
    s = torch.sigmoid(g)
    return g * s, s * (1 + g * (1 - s))


def ffn_forward(x, wg, wu):
    """{name: (value, bound)} of gate, up and hidden."""
    (g, eg), (u, eu) = product(x, wg), product(x, wu)
    a, _ = silu(g)
    h = a * u
    # the slope of silu lies in (-0.1, 1.1); the exponential is off by |g| roundings and a few, the rest by a few
    eh = 1.1 * eg * (u.abs() + eu) + a.abs() * eu + (16 + 2 * g.abs()) * U32 * h.abs()
    return {"gate": (g, eg), "up": (u, eu), "hidden": (h, eh)}


def ffn_gates(dy, wd, gate, up):
    """{name: (value, bound)} of dgate and dup from gate and up as stored."""
    dh, e = product(dy, wd.double().t())
    g, u = gate.double(), up.double()
    s = torch.sigmoid(g)
    a, slope = silu(g)
    few = (24 + 4 * g.abs()) * U32
    size = s * (1 + g.abs() * (1 - s)) * u.abs()
    return {"dgate": (dh * u * slope, e * u.abs() * slope.abs() + few * size * (dh.abs() + e)), "dup": (dh * a, e * a.abs() + few * a.abs() * (dh.abs() + e))}


def head_logits(x, w):
    return product(x, w.double().t())


def head_loss(x, w, ids):
    """{name: (value, bound)} of loss and lse."""
    z, e = head_logits(x, w)
    v = w.shape[0]
    lse = torch.logsumexp(z, 1)
    span = (lse[:, None] - z).abs().amax(1)
    # a logit's error goes through the sum of exponentials with a weight of at most one; chains of at most 400 roundings
    bound = e.amax(1) + (400 + 4 * span) * U32 + 4 * U32 * lse.abs()
    rows = ((ids >= 0) & (ids < v)).nonzero()[:, 0]
    at = ids[rows].long()
    loss, off = torch.zeros_like(lse), torch.zeros_like(lse)
    loss[rows] = lse[rows] - z[rows, at]
    off[rows] = bound[rows] + e[rows, at] + 2 * U32 * (lse[rows].abs() + z[rows, at].abs())
    return {"loss": (loss, off), "lse": (lse, bound)}


def head_gradients(x, w, ids, lse, dloss, scale):
    """{name: (value, bound)} of dx and dw from a stored lse."""
    z, e = head_logits(x, w)
    far = (z - lse.double()[:, None]).abs()
    p = torch.exp(z - lse.double()[:, None])
    return _head_gradients(x, w, ids, dloss, scale, p, p * torch.expm1(e + (8 + 4 * far) * U32))


def head_gradients_of_one_pass(x, w, ids, dloss, scale):
    """The same where the backward pass's logits have the bits of those that lse was taken of: an error d of the logits moves p by
    p (d - sum p d), at most 2 p (1 - p) max |d|, and half as much again for what that moves in turn; the rest is the rounding of lse and
    of the exponential."""
    z, e = head_logits(x, w)
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = torch.exp(z - lse)
    assert float(e.max()) < 0.1
    return _head_gradients(x, w, ids, dloss, scale, p, 3 * p * (1 - p) * e.amax(1, keepdim=True) + p * (16 + 4 * (z - lse).abs() + 2 * lse.abs()) * U32)


def _head_gradients(x, w, ids, dloss, scale, p, ep):
    v = w.shape[0]
    rows = ((ids >= 0) & (ids < v)).nonzero()[:, 0]
    weight = torch.zeros(len(ids), 1, dtype=torch.float64, device=x.device)
    weight[rows, 0] = dloss.double()[rows] if dloss is not None else 1.0
    hot = torch.zeros_like(p)
    hot[rows, ids[rows].long()] = 1
    dz = (p - hot) * weight
    edz = ep * weight.abs() + 4 * U32 * (p + hot) * weight.abs()
    edz = edz + half_step(x.dtype) * (dz.abs() + edz)
    scale = abs(scale), scale
    out = {}
    for name, a, ea, b in (("dx", dz, edz, w.double()), ("dw", dz.t().contiguous(), edz.t().contiguous(), x.double())):
        value, bound = product(a, b)
        out[name] = (scale[1] * value, scale[0] * (bound * 1.01 + ea @ b.abs()) + 4 * U32 * (scale[1] * value).abs())
    return out


def clip(grads, max_norm, eps):
    """(norm, the factor)."""
    norm = float(sum(g.double().square().sum() for g in grads)) ** 0.5
    return norm, min(1.0, max_norm / (norm + eps)) if norm + eps > 0 and max_norm != float("inf") else 1.0
