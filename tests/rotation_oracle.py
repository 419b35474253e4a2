"""Norm and rotation of heads in 64 bits on the CPU, and how far 16-bit outputs may be from it.

u is the unit roundoff of the 16-bit type.  Inputs are exact; a result is rounded once.  In 32 bits on the way: the sum of a head's squares (at most
20 additions one after the other, 2^-24 each, halved by the root), root, weight: together below 2^-19 relative; cosine and sine: the part of a
turn 2^-25 turns, the series 2^-23: below 2^-20 absolutely.  So, with |z| the values of a pair,

  |y - Y|    <= u |Y| + 2^-18 (|z_a| + |z_b|)
  |dx - dX|  <= u |dX| + 2^-16 r (|w| (|dy_a| + |dy_b|) + |x r| mean(|w| (|dy_a| + |dy_b|) |x r|))      (two sums of a head, each as above)
  |dw - dW|  <= u |dW| + (n 2^-24 + 2^-16) sum (|dy_a| + |dy_b|) |x r|                                  (n terms one after the other)

and 2^-25 for the subnormal numbers of float16.
"""
import torch

from attention_oracle import TINY, UNIT


def parts(x, rot, pairs):
    """[..., d] -> first and second values of the pairs, and the rest."""
    if pairs == "halves":
        return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]
    return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]


def whole(a, b, rest, pairs):
    both = torch.cat([a, b], -1) if pairs == "halves" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([both, rest], -1)


def angles(freqs, positions, axis_of=None):
    """[tokens, 1, rot / 2]"""
    positions = positions.cpu().double()
    if positions.dim() == 1:
        positions = positions[None]
    freqs = freqs.cpu()
    which = torch.zeros(len(freqs), dtype=torch.long) if axis_of is None else axis_of.cpu().long().clamp(max=len(positions) - 1)
    return (positions[which].t() * freqs)[:, None]


def rotation(x, weight, angle, eps, pairs, dy=None):
    """(values, bounds) of y and, with dy, dx and dw (None without a weight).  x [tokens, heads, d]."""
    u, tiny = UNIT[x.dtype], TINY[x.dtype]
    x = x.cpu().double().detach().requires_grad_(dy is not None)
    w = None if weight is None else weight.cpu().double().detach().requires_grad_(dy is not None)
    rot = 2 * angle.shape[-1]
    inverse = torch.ones(()).double() if w is None else (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    z = x if w is None else x * inverse * w
    a, b, rest = parts(z, rot, pairs)
    y = whole(a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos(), rest, pairs)

    def spread(t):                              # |t_a| + |t_b| at both
        a, b, rest = parts(t.detach().abs(), rot, pairs)
        return whole(a + b, a + b, rest, pairs)
    out = {"y": (y.detach(), u * y.detach().abs() + 2.0 ** -18 * spread(z) + tiny)}
    if dy is None:
        return out
    dy = dy.cpu().double()
    got = torch.autograd.grad(y, [x] if w is None else [x, w], dy)
    size, inverse = spread(dy), inverse.detach()
    if w is None:
        out["dx"] = got[0], u * got[0].abs() + 2.0 ** -16 * size + tiny
        return out
    unit, weighted = (x.detach() * inverse).abs(), w.detach().abs() * size
    out["dx"] = got[0], u * got[0].abs() + 2.0 ** -16 * inverse * (weighted + unit * (weighted * unit).mean(-1, keepdim=True)) + tiny
    n = x.shape[0] * x.shape[1]
    out["dw"] = got[1], u * got[1].abs() + (n * 2.0 ** -24 + 2.0 ** -16) * (size * unit).sum((0, 1)) + tiny
    return out
