"""Keys as far apart as a call may have them: a tile spans nearly 2^31 bytes."""
import pytest

from test_gpu_attention import compare, everything, run, tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("masking", ["none", "mask"])
@pytest.mark.parametrize("Lq", [1, 150])
def test_longest_token_stride(Lq, masking):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as M
    Lk, H, d, far = 131, 2, 128, 1 << 24
    t = tensors((1, Lq, H, d), (1, Lk, H, d), torch.bfloat16, 59, train=Lq > 1)
    pool = torch.empty((Lk - 1) * far + 4 * H * d, dtype=torch.bfloat16, device="cuda")
    for i, n in enumerate(("k", "v") + (("dk", "dv") if Lq > 1 else ())):
        y = torch.as_strided(pool, (1, Lk, H, d), (0, far, d, 1), i * H * d)
        y.copy_(t[n])
        t[n] = y
    keep, kw = everything(1, Lq, Lk), {}
    if masking == "mask":
        keep = (torch.arange(Lk) % 3 != 1).view(1, 1, Lk).expand(1, Lq, Lk)
        kw["key_mask"] = keep[:, 0].cuda()
    run(M, t, **kw)
    compare(t, keep, (Lq, masking))
