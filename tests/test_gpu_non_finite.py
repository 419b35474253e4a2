"""Infinities and NaN in what a row does not see: rows past a tree's nodes."""
import math

import pytest

from test_gpu_tree_attention import build, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


def put(t, b, p, page, k=None, v=None):
    """Position p of sequence b in the pool of pages, not in t's k and v."""
    if k is not None:
        t["pool"][t["table"][b, p // page], 0, p % page] = k
    if v is not None:
        t["pool"][t["table"][b, p // page], 1, p % page] = v


TREES = [  # nodes, H, Hkv, d, lengths: one, two, four and eight waves with rows of their own, keys in pieces and not
    (5, 4, 1, 64, [70, 300]), (6, 4, 1, 128, [6000, 411]), (3, 8, 8, 40, [900, 20]), (40, 2, 2, 128, [100, 129]), (50, 3, 3, 64, [5000, 3000]), (100, 1, 1, 96, [77, 2100]),
    (140, 72, 36, 64, [300, 40])]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("n,H,Hkv,d,lens", TREES)
def test_rows_past_the_nodes(M, n, H, Hkv, d, lens, dtype):
    """They give zeros and lse -inf whatever the cache and their own queries hold; the other rows see the cache as it is."""
    import torch
    t = build(2, n, H, Hkv, d, 16, lens, getattr(torch, dtype), seed=n)
    counts = [n - 2, 0]
    for b in range(2):
        put(t, b, 3, 16, v=math.nan)
        put(t, b, lens[b] - 1, 16, k=-math.inf, v=math.inf)
    t["q"][:, n - 1] = math.nan
    run(M, t, counts)
    for b, c in enumerate(counts):
        assert not t["o"][b, c:].any() and (t["lse"][b, :, c:] == -math.inf).all()
        assert torch.isnan(t["o"][b, :c]).all()
