"""Infinities and NaN in what a row does not see, and in what it sees: rows past the nodes, nodes that no row sees, the last key,
padded columns, rows without keys; gates near the largest numbers."""
import math

import pytest

from test_gpu_attention import everything
from test_gpu_attention import compare as compare_cross
from test_gpu_attention import run as run_cross
from test_gpu_attention import tensors
from test_gpu_tree_attention import build, compare, keeps, random_tree, run

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


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("n,H,Hkv,d,lens", TREES + [(9, 2, 1, 32, [0, 63]), (64, 1, 1, 64, [63, 64]), (70, 2, 2, 128, [31, 500]), (200, 2, 1, 80, [130, 1])])
@pytest.mark.parametrize("counted", ["all", "fewer"])
def test_nodes_that_no_row_sees(M, n, H, Hkv, d, lens, counted, dtype):
    """Their keys and values reach no row: pruned branches, the nodes that only rows past the count would see, and padding without a count."""
    import torch
    sees = random_tree(2, n, n)
    unseen = sorted({1, n // 3, n // 2, min(n - 1, 64), n - 1})
    counts = None if counted == "all" else [n - 1, n // 2 + 1]
    for j in unseen:
        sees[:, :, j] = False
    if counts:
        for b, c in enumerate(counts):
            sees[b, c:] = True
    t = build(2, n, H, Hkv, d, 16, lens, getattr(torch, dtype), seed=n, sees=sees)
    for b in range(2):
        for i, j in enumerate(unseen):
            put(t, b, lens[b] + j, 16, k=(math.nan, math.inf, -math.inf)[i % 3], v=(math.inf, math.nan, -math.inf)[i % 3])
    run(M, t, counts)
    compare(t, keeps(t, counts), (n, counts))


@pytest.mark.parametrize("n,used,H,Hkv,lens", [(700, 30, 2, 2, [100, 70]), (1024, 1, 2, 1, [64, 5]), (600, 599, 1, 1, [0, 33]), (64, 20, 32, 8, [500, 129])])
def test_room_that_is_not_used(M, n, used, H, Hkv, lens):
    """Rows and nodes past those used are left empty by their bits alone, without a count; their cache slots hold anything."""
    import torch
    sees = random_tree(2, n, 5)
    sees[:, used:], sees[:, :, used:] = False, False
    t = build(2, n, H, Hkv, 64, 16, lens, torch.bfloat16, seed=n, sees=sees)
    for b in range(2):
        for j in range(used, n):
            put(t, b, lens[b] + j, 16, k=math.nan, v=math.nan if j % 2 else math.inf)
    run(M, t)
    compare(t, keeps(t), (n, used))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("B,Lq,H,Lk,Hkv,d", [(1, 1, 4, 33, 2, 64), (2, 1, 4, 5001, 1, 128), (2, 50, 1, 95, 1, 40), (2, 130, 3, 65, 3, 32), (1, 700, 2, 1601, 1, 128), (1, 270, 70, 200, 70, 64)])
@pytest.mark.parametrize("masking", ["none", "lens"])
def test_infinite_values_of_the_last_key(M, B, Lq, H, Lk, Hkv, d, masking, dtype):
    """An infinity in a value that counts comes out as it is, in its own column."""
    import torch
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), getattr(torch, dtype), 23, train=False)
    lens, kw = torch.full((B,), Lk), {}
    if masking == "lens":
        lens = torch.tensor([Lk - 2, Lk // 2 + 1][:B])
        kw["kv_lens"] = lens.to(torch.int32).cuda()
    t["q"] /= 4                                         # (probabilities stay in the range of 16 bits)
    for b in range(B):
        t["v"][b, lens[b] - 1, :, 3], t["v"][b, lens[b] - 1, :, d - 1] = math.inf, -math.inf
        t["v"][b, lens[b]:], t["k"][b, lens[b]:] = math.nan, math.nan
    run_cross(M, t, **kw)
    compare_cross(t, (torch.arange(Lk) < lens[:, None])[:, None].expand(B, Lq, Lk), "last key")


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("d", [8, 24, 32, 40, 64, 80, 128])
@pytest.mark.parametrize("Lq", [1, 40, 200])
@pytest.mark.parametrize("masking", ["none", "mask", "tree"])
def test_keys_at_minus_infinity(M, Lq, d, masking, dtype):
    """Positive queries on a key that holds -inf: its score is -inf and its probability 0, whatever the head size."""
    import torch
    dt, B, H, Lk = getattr(torch, dtype), 2, 2, 130
    if masking == "tree":
        t = build(B, Lq, H, 1, d, 16, [Lk, Lk], dt, seed=d)
        t["q"] = t["q"].abs()
        for p in (0, 7, 70, Lk - 1):
            t["k"][:, p, :, :8] = -math.inf
            for b in range(B):
                put(t, b, p, 16, k=t["k"][b, p].cuda())
        run(M, t)
        return compare(t, keeps(t), d)
    t = tensors((B, Lq, H, d), (B, Lk, 1, d), dt, 29, train=False)
    t["q"] = t["q"].abs()
    t["k"][:, [0, 7, 70, Lk - 1], :, :8] = -math.inf
    keep = torch.ones(B, Lk, dtype=torch.bool)
    if masking == "mask":
        keep[:, 5:60] = False
    run_cross(M, t, **({"key_mask": keep.cuda()} if masking == "mask" else {}))
    compare_cross(t, keep[:, None].expand(B, Lq, Lk), d)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("B,Lq,H,Lk,Hkv,d", [(2, 1, 4, 200, 2, 64), (2, 3, 8, 3000, 1, 64), (3, 50, 1, 150, 1, 80), (2, 140, 2, 333, 2, 128), (2, 700, 48, 300, 24, 64)])
def test_rows_without_keys(M, B, Lq, H, Lk, Hkv, d, dtype):
    """A batch whose mask is empty gives zeros, lse -inf and zero gradients also where its queries are infinite or NaN."""
    import torch
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), getattr(torch, dtype), 31)
    keep = torch.ones(B, Lk, dtype=torch.bool)
    keep[1] = False
    t["q"][1, :, 0], t["q"][1, Lq // 2] = math.inf, math.nan
    run_cross(M, t, key_mask=keep.cuda())
    for name in ("o", "dq", "dk", "dv"):
        assert not t[name][1].any(), name
    assert (t["lse"][1] == -math.inf).all()
    t = {n: x[:1] for n, x in t.items()}
    compare_cross(t, everything(1, Lq, Lk), "the others")


@pytest.mark.parametrize("rows", [40, 200])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_large_gates(M, act, rows):
    """Gates of up to 2^72, whose squares and cubes are beyond 32 bits: the activations are the identity or 0 there, with slopes of 1 and 0."""
    import torch
    from test_gpu_ffn import run as run_ffn
    from test_gpu_ffn import tensors as block
    t = block(rows, 64, 72, 40, torch.bfloat16, 53)
    t["x"], t["w_up"], t["dy"] = t["x"] * 2.0 ** 70, t["w_up"] * 2.0 ** -70, t["dy"] * 2.0 ** -60
    run_ffn(M, t, act)
    x, wg, wu, wd, dy = (t[n].double().cpu() for n in ("x", "w_gate", "w_up", "w_down", "dy"))
    g, up = x @ wg.t(), x @ wu.t()
    dh, on = dy @ wd, (g > 0).double()
    dg, du = dh * up * on, dh * g * on
    want = {"y": (g * on * up) @ wd.t(), "dx": dg @ wg + du @ wu, "dw_gate": dg.t() @ x, "dw_up": du.t() @ x, "dw_down": dy.t() @ (g * on * up)}
    assert all(value.abs().max() < 2.0 ** 127 for value in want.values())
    for name, value in want.items():                    # (four roundings of at most u / 2 each, in the 2-norm)
        assert (t[name].double().cpu() - value).norm() <= 1.5 * 2.0 ** -8 * value.norm(), name


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("Lq,H,Hkv,Lk,d", [(5, 2, 2, 70, 64), (33, 3, 1, 100, 128), (700, 24, 24, 300, 128), (65, 2, 2, 2000, 32), (1100, 40, 40, 270, 64)])
def test_infinite_gradient_of_the_last_row(M, Lq, H, Hkv, Lk, d, dtype):
    """It comes out as it is in the values' gradients, in its own column: dV = P^T dO."""
    import torch
    from attention_oracle import attention, check
    t = tensors((1, Lq, H, d), (1, Lk, Hkv, d), getattr(torch, dtype), 61)
    t["q"] /= 4
    t["do"][:, -1, -1, 5] = math.inf
    run_cross(M, t)
    want = attention(t["q"], t["k"], t["v"], everything(1, Lq, Lk), d ** -0.5, t["q"].dtype, t["do"])
    assert torch.isinf(want["dv"][0]).any()
    check(t["dv"], want["dv"], (Lq, d))
