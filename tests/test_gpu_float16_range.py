"""Float16 between its smallest numbers and its largest: probabilities far below a row's largest, gradients through the gated block from below
the normal numbers to beyond the largest."""
import math

import pytest

from test_gpu_attention import everything, tensors
from test_gpu_attention import run as run_cross
from test_gpu_ffn import act_of
from test_gpu_ffn import run as run_ffn
from test_gpu_ffn import tensors as block

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


@pytest.mark.parametrize("apart", [13.0, 16.0, 18.0])
@pytest.mark.parametrize("Lq,H,d,Lk", [(1, 2, 64, 4096), (40, 1, 64, 4096), (130, 1, 128, 1500), (300, 70, 64, 700)])
def test_probabilities_far_below_the_largest(M, Lq, H, d, Lk, apart):
    """One key takes nearly all of the softmax and its values are zero, so that the others' small probabilities make the result.  A probability is
    kept to u of its size or to 2^-25 of 2^-7 of the row's largest: o is off by u |O| + 1.5 u sum P |v| + 2^-32 sum |v|, and 2^-25."""
    import torch
    from attention_oracle import attention, check
    u = 2.0 ** -11
    t = tensors((1, Lq, H, d), (1, Lk, H, d), torch.float16, 37, train=False)
    t["q"], t["k"] = t["q"] / 16, t["k"] / 16
    t["q"][..., 0], t["k"][..., 0] = 1.0, 0.0
    t["v"] = t["v"].abs() * 16
    t["k"][:, Lk // 3, :, 0], t["v"][:, Lk // 3] = apart, 0.0
    run_cross(M, t, scale=1.0)
    want = attention(t["q"], t["k"], t["v"], everything(1, Lq, Lk), 1.0, torch.float16)
    O, V = want["o"][0], t["v"].double().cpu()
    off = 2.5 * u * O + 2.0 ** -32 * V.sum(1, keepdim=True) + 2.0 ** -25          # (V >= 0: sum P |v| is O)
    check(t["o"], (O, off), apart)
    check(t["lse"], want["lse"], apart)


def gradients(t, act):
    """The gated block's gradients in 64 bits."""
    x, wg, wu, wd, dy = (t[n].detach().double().cpu() for n in ("x", "w_gate", "w_up", "w_down", "dy"))
    g, up = x @ wg.t(), x @ wu.t()
    a, da = act_of(act, g)
    dh = dy @ wd
    dg, du = dh * up * da, dh * a
    return {"dx": dg @ wg + du @ wu, "dw_gate": dg.t() @ x, "dw_up": du.t() @ x, "dw_down": dy.t() @ (a * up)}


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu", "sigmoid"])
@pytest.mark.parametrize("rows,K,F,J", [(600, 256, 520, 264), (50, 72, 136, 64), (3000, 264, 1400, 200)])
@pytest.mark.parametrize("by", [-18, -16, -11, 5])
def test_gradients_of_the_gated_block(M, rows, K, F, J, by, act, dtype):
    """dy from 2^-18 to 2^5.  In the 2-norm g, u, dg or du and the result are rounded to at most u / 2 each, g's counting up to twice (its way
    through the activation): 1.5 u covers their root of squares; half a unit of the subnormal numbers on every element of dx and of the result."""
    import torch
    from attention_oracle import TINY, UNIT
    dt = getattr(torch, dtype)
    t = block(rows, K, F, J, dt, 41)
    # values that float16 holds exactly after the scaling: what is measured is the way from dy on
    t["dy"] = ((t["dy"].float() * 64).round() / 64).clamp(-4, 4) if by > -14 else t["dy"].float().sign()
    t["dy"] = (t["dy"] * 2.0 ** by).to(dt)
    run_ffn(M, t, act)
    for name, want in gradients(t, act).items():
        got = t[name].double().cpu()
        off = (got - want).norm()
        assert off <= 1.5 * UNIT[dt] * want.norm() + TINY[dt] * want.numel() ** 0.5, (name, (off / want.norm()).item(), (off / UNIT[dt] / want.norm()).item())


def test_gradients_beyond_the_largest(M):
    """dg lies beyond float16's largest number, the gradients that are made of it do not."""
    import torch
    t = block(70, 64, 8, 64, torch.float16, 43)
    t["x"], t["w_gate"], t["w_up"], t["dy"] = t["x"] * 2.0 ** -8, t["w_gate"] * 2.0 ** -4, t["w_up"] * 2.0 ** 16, t["dy"] * 2.0 ** 7
    run_ffn(M, t, "silu")
    for name, want in gradients(t, "silu").items():
        assert want.abs().max() < 65504
        got = t[name].double().cpu()
        assert (got - want).norm() <= 1.5 * 2.0 ** -11 * want.norm() + 2.0 ** -25 * want.numel() ** 0.5, name


@pytest.mark.parametrize("fill", [0.0, math.inf, math.nan])
def test_gradients_of_odd_rows(M, fill):
    """Rows of zeros, infinities or NaN in dy leave the other rows' dx alone (off by at most 144 terms of half a unit of the subnormal numbers times
    weights below 1/2, and by the roundings of dg and du of at most 2^-12: 2^-18 covers both); zeros alone give zeros."""
    import torch
    for rows in (20, 200):
        t = block(rows, 64, 72, 40, torch.float16, 47)
        t["dy"] *= 2.0 ** -14
        want = gradients(t, "silu")["dx"]
        t["dy"][3] = fill
        run_ffn(M, t, "silu")
        clean = [r for r in range(rows) if r != 3]
        assert ((t["dx"].double().cpu() - want)[clean].abs().max() <= 2.0 ** -18)
        assert not t["dx"][3].any() if fill == 0 else not torch.isfinite(t["dx"][3]).any()
    t["dy"].zero_()
    run_ffn(M, t, "silu")
    for name in ("dx", "dw_gate", "dw_up", "dw_down"):
        assert not t[name].any(), name
