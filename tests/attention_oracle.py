"""Attention in 64 bits on the CPU, and how far 16-bit operands and outputs may be from it.

u is the unit roundoff of the 16-bit type.  The kernels round probabilities and dS once (relative error u each, subnormal numbers of
float16 2^-25 absolutely), every output once, and hold everything else in 32 bits, whose errors (2^-24 times the number of terms)
are far below u at the sizes tested: half a u more on every term covers them.  So, elementwise,

  |o - O|    <= u |O|  + 1.5 u sum_j P_j |v_j|
  |dv - dV|  <= u |dV| + 1.5 u sum_i P_i |do_i|
  |ds - dS|  <= 1.5 u |dS| + 0.5 u P sum |do||v| + P |delta D|,  |delta D| <= sum |do| |o - O| (D comes from the rounded o)
  |dq - dQ|  <= u |dQ| + scale sum_j |ds - dS| |k_j|,  dK likewise
"""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def heads_first(x, heads):
    """[B, L, Hkv, d] -> [B, heads, L, d] in 64 bits, key/value heads repeated."""
    x = x.detach().double().cpu().transpose(1, 2)
    return x.repeat_interleave(heads // x.shape[1], 1)


def attention(q, k, v, keep, scale, dtype, do=None):
    """(values, bounds) of o, lse and, with do, dq, dk, dv.  keep: [B, Lq, Lk] truth values; k and v at keys that no row keeps do not matter."""
    u, tiny, H, Hkv = UNIT[dtype], TINY[dtype], q.shape[2], k.shape[2]
    K, V, Q = heads_first(k, H), heads_first(v, H), heads_first(q, H)
    keep = keep.cpu()
    used = keep.any(1)[:, None, :, None]
    K, V = torch.where(used, K, torch.zeros_like(K)), torch.where(used, V, torch.zeros_like(V))
    S = (Q @ K.transpose(2, 3) * scale).masked_fill(~keep[:, None], -math.inf)
    lse = torch.logsumexp(S, 3)
    P = torch.exp(S - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[..., None])
    O = P @ V
    seen = keep[:, None].double()
    o_off = u * O.abs() + 1.5 * u * (P @ V.abs()) + tiny * (seen @ V.abs() + 1)
    back = lambda x: x.transpose(1, 2)  # noqa: E731
    shared = lambda x: back(x.view(x.shape[0], Hkv, H // Hkv, *x.shape[2:]).sum(2))  # noqa: E731
    out = {"o": (back(O), back(o_off)), "lse": (lse, 1e-5 + 1e-5 * lse.abs())}
    if do is None:
        return out
    G = heads_first(do, H)
    D = (G * O).sum(3, keepdim=True)
    dP = G @ V.transpose(2, 3)
    dS = P * (dP - D)
    s_off = 1.5 * u * dS.abs() + P * (0.5 * u * (G.abs() @ V.abs().transpose(2, 3)) + (G.abs() * o_off).sum(3, keepdim=True)) + tiny * seen
    dQ, dK, dV = dS @ K * scale, dS.transpose(2, 3) @ Q * scale, P.transpose(2, 3) @ G
    out["dq"] = back(dQ), back(u * dQ.abs() + scale * (s_off @ K.abs()) + tiny)
    k_off, v_off = scale * (s_off.transpose(2, 3) @ Q.abs()), 1.5 * u * (P.transpose(2, 3) @ G.abs()) + tiny * (seen.transpose(2, 3) @ G.abs())
    dK, dV = shared(dK), shared(dV)
    out["dk"] = dK, u * dK.abs() + shared(k_off) + tiny
    out["dv"] = dV, u * dV.abs() + shared(v_off) + tiny
    return out


def check(got, want, where):
    values, off = want
    got = got.detach().double().cpu()
    assert got.shape == values.shape, where
    finite = torch.isfinite(values)
    assert torch.equal(got[~finite], values[~finite]), where
    over = ((got - values).abs() - off)[finite]
    assert not torch.isnan(over).any(), where
    assert over.numel() == 0 or over.max() <= 0, (where, over.max().item())
