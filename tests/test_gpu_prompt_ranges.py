"""Attention of packed prompts where its ranges end: D and dS of a handful of keys."""
import pytest

from test_gpu_prompt_attention import run, tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("beside", [0, 20000])
def test_D_of_few_keys_that_weigh_the_same(M, beside, dtype):
    """All keys' values are ones and all dO the same, queries are orthogonal to keys: dP is one number B, P is 1 / n, dS is P (B - D) = 0, and what D is off by shows alone.
    Alone and beside a sequence over so many keys, with which blocks have eight waves.

    In float16's forward pass the sum is n 2^7 and its logarithm, below 16, off by a unit of 2^-20; twice it is multiplied and rounded, 2^-23 of 4: 2^-20 and 2^-21 of
    a power of two, times ln 2 below 2^-20 of P.  An exponential is off by 2^-23, and D is n / 2 additions in each of two lanes and one, 2^-24 each: 2^-21 for n up to
    16.  So |B - D| <= B (2^-20 + 2^-21 + 2^-22), which dS and the results of n terms have as they have P; their own roundings are below 2^-7 of that."""
    import torch
    d, dt, B = 128, getattr(torch, dtype), 128.0 * 128
    lens = [7, 9, 11, 14, 16, 3] if beside else list(range(2, 17))
    t = tensors(lens + [1500] * (beside > 0), lens + [beside] * (beside > 0), 2, 1, d, dt, 77)
    t["q"][..., :64], t["k"][..., 64:] = 0, 0
    t["v"].fill_(1.0)
    t["do"].fill_(128.0)
    run(M, t, causal=False)
    at = 0
    for n in lens:
        one = slice(at, at + n)
        at += n
        off = 1.01 * B * (2.0 ** -20 + 2.0 ** -21 + 2.0 ** -22) * d ** -0.5
        k, q = t["k"][one].double().abs().sum(0, keepdim=True) / n, t["q"][one].double().abs().sum((0, 1), keepdim=True) / n
        for name, bound in (("dq", off * k), ("dk", off * q)):
            far = t[name][one].double().abs() - bound - 2.0 ** -25
            assert (far <= 0).all(), (n, name, far.max().item(), (t[name][one].double().abs() / (bound + 2.0 ** -25)).max().item())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_dS_of_up_to_16_keys_one_by_one(M, dtype):
    """Keys are unit vectors, so that a value of dQ is one dS times the scale, and of V and dO one value is not zero, so that dP is exact: dS goes into dQ as two
    operands and is off by u^2 and by what errors in 32 bits add, and its result is rounded once, to u.

    P is off by 2^-19 (scores below 8 and their products with log2 e below 2^-21 of a power of two, lse, the logarithm of a sum of up to 2^11, 2^-20), D by that and 16
    additions, 2^-20.  Float16 has steps of 2^-24 below its normal numbers."""
    import torch
    d, dt = 64, getattr(torch, dtype)
    u, scale = torch.finfo(dt).eps / 2, d ** -0.5
    lens = [16, 9, 13, 2, 15, 7] * 8
    t = tensors(lens, lens, 4, 2, d, dt, 101)
    at = 0
    for n in lens:
        t["k"][at:at + n] = torch.eye(n, d, device="cuda")[:, None].to(dt)
        at += n
    t["q"] *= 3
    t["v"][..., 1:], t["do"][..., 1:] = 0, 0
    run(M, t, kv=False, causal=False)
    at = 0
    for b, n in enumerate(lens):
        one = slice(at, at + n)
        at += n
        q, do, v = (t[x][one].double().cpu().transpose(0, 1) for x in ("q", "do", "v"))
        P = (q[..., :n] * scale).softmax(2)
        dP = do[..., :1] * v[..., 0].repeat_interleave(2, 0)[:, None]
        D = (P * dP).sum(2, keepdim=True)
        dS = P * (dP - D)
        off = (u + 1.01 * u * u) * dS.abs() + 1.01 * P * (2.0 ** -19 * (dP - D).abs() + (2.0 ** -19 + 2.0 ** -20) * (P * dP.abs()).sum(2, keepdim=True))
        far = (t["dq"][one].double().cpu().transpose(0, 1)[..., :n] - dS * scale).abs() - off * scale - 2.0 ** -25
        assert (far <= 0).all(), (b, n, int((far > 0).sum()), far.max().item())
