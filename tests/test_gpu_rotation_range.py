"""Norm and rotation of heads whose squares pass what 32 bits hold, which bfloat16's values can, and of heads far below eps."""
import pytest

from test_gpu_qk_rotate import compare, run, tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("d,rot", [(32, 32), (64, 64), (80, 32), (128, 128), (256, 64)])
def test_heads_of_far_apart_sizes(M, d, rot, pairs):
    """Beside each other in a wave: 2^-100 (the norm is eps's), ordinary, 2^59 to 2^110 (squares that pass 2^128 or not), and a head of one value of 2^62 among ordinary ones."""
    import torch
    t = tensors(13, 5, 3, d, rot, torch.bfloat16, 51)
    sizes = (2.0 ** torch.tensor([-100.0, 0, 59, 60, 61, 62, 63, 64, 80, 110, 0, -20, 96])).to(torch.bfloat16).cuda()
    for n in ("q", "k"):
        t[n][:, ::2] *= sizes[:, None, None]
    t["q"][3, 1, 7], t["k"][10, 1, 20] = 2.0 ** 62, -2.0 ** 62
    run(M, t, pairs=pairs)
    compare(t, (d, rot), pairs)
    assert t["q_out"][2:10].float().square().mean(2).min() > 0.1


def test_heads_that_are_not_finite_beside_far_ones(M):
    """Stay in their head."""
    import math

    import torch
    t = tensors(4, 4, 2, 64, 64, torch.bfloat16, 52, train=False)
    t["q"] *= 2.0 ** 70
    run(M, t)
    compare(t, "far")
    clean = t["q_out"].clone()
    t["q"][1, 2, 5], t["q"][2, 0, 9] = math.inf, math.nan
    run(M, t)
    others = torch.ones(4, 4, dtype=torch.bool)
    others[1, 2] = others[2, 0] = False
    assert torch.equal(t["q_out"][others.cuda()], clean[others.cuda()])
    assert not torch.isfinite(t["q_out"][1, 2, 5]) and torch.isnan(t["q_out"][2, 0]).all()
