"""Float16 at its smallest numbers: probabilities far below a row's largest."""
import pytest

from test_gpu_attention import everything, tensors
from test_gpu_attention import run as run_cross

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
