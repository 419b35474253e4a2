"""Float16 through the attention kernels of eight waves: shapes whose plans take them forward, for dQ and for dK and dV, every size of head
and every kind of mask that they are built for."""
import math

import pytest

from test_gpu_attention import compare, everything, run, tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


def masks(masking, B, Lk):
    import torch
    kw, keep = {}, torch.ones(B, Lk, dtype=torch.bool)
    if masking in ("lens", "both"):
        lens = torch.tensor([Lk - 5, 0, Lk, 1, 700][:B], dtype=torch.int32)
        kw["kv_lens"] = lens.cuda()
        keep &= torch.arange(Lk) < lens[:, None]
    if masking in ("mask", "both"):
        mask = torch.rand(B, Lk, generator=torch.Generator().manual_seed(5)) < 0.4
        mask[:, 64:160] = False
        kw["key_mask"] = mask.cuda()
        keep &= mask
    return kw, keep


@pytest.mark.parametrize("masking", ["none", "lens", "mask", "both"])
@pytest.mark.parametrize("shape", [(1, 270, 70, 200, 70, 64), (1, 260, 33, 1601, 33, 72), (3, 130, 40, 1100, 20, 128)])
def test_forward(M, shape, masking):
    import torch
    B, Lq, H, Lk, Hkv, d = shape
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), torch.float16, 13, train=False)
    kw, keep = masks(masking, B, Lk)
    t["k"][~keep.cuda()] = math.nan
    t["v"][~keep.cuda()] = math.inf
    run(M, t, **kw)
    compare(t, keep[:, None].expand(B, Lq, Lk), (shape, masking))


@pytest.mark.parametrize("masking", ["none", "lens", "mask"])
@pytest.mark.parametrize("shape", [(1, 600, 48, 1030, 48, 128), (1, 1100, 40, 1030, 40, 64), (2, 130, 72, 300, 9, 64), (2, 130, 72, 300, 9, 120)])
def test_backward(M, shape, masking):
    import torch
    B, Lq, H, Lk, Hkv, d = shape
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), torch.float16, 17)
    kw, keep = masks(masking, B, Lk)
    run(M, t, **kw)
    compare(t, keep[:, None].expand(B, Lq, Lk), (shape, masking))


@pytest.mark.parametrize("gradients", ["small", "rising", "large"])
@pytest.mark.parametrize("shape", [(1, 600, 48, 1030, 48, 128), (1, 1100, 40, 1030, 40, 64)])
def test_gradients_of_all_sizes(M, shape, gradients):
    """As three roundings of at most u / 2 each allow in the 2-norm, and half a unit of the subnormal numbers on every element of the result."""
    import torch
    from attention_oracle import TINY, UNIT, attention
    B, Lq, H, Lk, Hkv, d = shape
    dt = torch.float16
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), dt, 19)
    t["q"], t["k"], scale = t["q"] / 16, t["k"] / 16, 256 * d ** -0.5
    up = lambda n: torch.exp2(torch.linspace(-8, 0, n, device="cuda").round())[None, :, None, None]  # noqa: E731
    if gradients == "small":
        t["do"] = t["do"] * 2.0 ** -11
    elif gradients == "large":
        t["do"] = t["do"] * 2.0 ** 8
    else:
        t["do"], t["v"] = (t["do"] * up(Lq)).to(dt), (t["v"] * up(Lk)).to(dt)
    run(M, t, scale=scale)
    want = attention(t["q"], t["k"], t["v"], everything(B, Lq, Lk), scale, dt, t["do"])
    for name in ("dq", "dk", "dv"):
        value = want[name][0]
        off = (t[name].double().cpu() - value).norm()
        assert off <= 1.5 * UNIT[dt] * value.norm() + TINY[dt] * value.numel() ** 0.5, (name, (off / value.norm()).item())
