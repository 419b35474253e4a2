"""Cross attention, forward and backward, against a plain 64-bit form (attention_oracle.py): lengths from none to several tiles, odd ones,
shared heads, layouts, masks that leave rows empty, what masked keys hold, pieces, streams, graphs."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


def tensors(shape_q, shape_k, dtype, seed, train=True):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    B, Lq, H, d = shape_q
    t = {"q": r(*shape_q), "k": r(*shape_k), "v": r(*shape_k), "o": torch.full(shape_q, math.nan, dtype=dtype, device="cuda"),
         "lse": torch.full((B, H, Lq), math.nan, device="cuda")}
    if train:
        t["do"] = r(*shape_q)
        t |= {n: torch.full_like(t[n[1]], math.nan) for n in ("dq", "dk", "dv")}
    return t


def run(M, t, **kw):
    import torch
    a = M.attn(t["q"], t["k"], t["v"], t["o"], lse=t["lse"], **kw)
    # whatever the workspace holds before a call does not matter
    a.use_workspace(torch.full((M.mmee_attn_workspace(a, "do" in t),), 255, dtype=torch.uint8, device="cuda"))
    M.mmee_attn_forward(a)
    if "do" in t:
        M.mmee_attn_backward(a, M.attn_grads(t["do"], t["dq"], t["dk"], t["dv"]))
    torch.cuda.synchronize()


def compare(t, keep, where, scale=None):
    from attention_oracle import attention, check
    want = attention(t["q"], t["k"], t["v"], keep, scale or t["q"].shape[3] ** -0.5, t["q"].dtype, t.get("do"))
    for name, value in want.items():
        check(t[name], value, (where, name))


def everything(B, Lq, Lk):
    import torch
    return torch.ones(B, Lq, Lk, dtype=torch.bool)


SHAPES = [  # B, Lq, H, Lk, Hkv, d
    (1, 1, 1, 1, 1, 8), (2, 1, 4, 33, 2, 32), (1, 3, 6, 64, 1, 40), (3, 5, 2, 31, 2, 64), (1, 31, 8, 65, 8, 72), (2, 17, 4, 127, 2, 128),
    (1, 65, 1, 129, 1, 128), (2, 130, 3, 63, 3, 16), (1, 257, 2, 300, 2, 96), (1, 40, 16, 200, 2, 120), (2, 33, 12, 513, 4, 24), (1, 128, 5, 256, 1, 56)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(M, shape, dtype):
    import torch
    B, Lq, H, Lk, Hkv, d = shape
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), getattr(torch, dtype), hash(shape) % 1000)
    run(M, t)
    compare(t, everything(B, Lq, Lk), shape)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", [(4, 1, 4, 200, 2, 64), (3, 37, 8, 150, 2, 80), (5, 140, 2, 333, 2, 128), (4, 9, 6, 96, 6, 32)])
@pytest.mark.parametrize("masking", ["lens", "mask", "both", "shared mask"])
def test_masks(M, shape, masking, dtype):
    """Lengths (none, one, more than there are, negative) and masks (whole batches of them empty); masked keys hold infinities, NaN and the
    type's lowest value, which reach no result; gradients at masked keys are zero."""
    import torch
    B, Lq, H, Lk, Hkv, d = shape
    dt = getattr(torch, dtype)
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), dt, 7)
    kw, keep = {}, torch.ones(B, Lk, dtype=torch.bool)
    if masking in ("lens", "both"):
        lens = torch.tensor(([0, 1, Lk + 50, -3, 67] * B)[:B], dtype=torch.int32)
        kw["kv_lens"] = lens.cuda()
        keep &= torch.arange(Lk) < lens[:, None]
    if masking != "lens":
        mask = torch.rand(B, Lk, generator=torch.Generator().manual_seed(3)) < 0.5
        mask[B - 1] = False
        mask[0, 64:128] = False
        if masking == "shared mask":
            mask = mask[:1].expand(B, Lk)
        kw["key_mask"] = mask.cuda() if masking == "mask" else mask.to(torch.uint8).cuda() if masking == "both" else mask[:1].cuda().expand(B, Lk)
        keep &= mask
    for fill, at in ((math.nan, 0), (math.inf, 1), (-math.inf, 2), (torch.finfo(dt).min, 3)):
        dead = ~keep & (torch.arange(Lk) % 4 == at)
        t["k"][dead.cuda()] = fill
        t["v"][dead.cuda()] = fill
    run(M, t, **kw)
    compare(t, keep[:, None].expand(B, Lq, Lk), (shape, masking))
    assert not t["dk"][~keep.cuda()].any() and not t["dv"][~keep.cuda()].any()
    empty = ~keep.any(1)
    assert empty.any() or masking == "shared mask"
    assert not t["o"][empty.cuda()].any() and not t["dq"][empty.cuda()].any() and (t["lse"][empty.cuda()] == -math.inf).all()


@pytest.mark.parametrize("layout", ["heads first", "fused kv", "fused qkv", "broadcast keys", "broadcast batch", "sliced"])
def test_layouts(M, layout):
    import torch
    B, Lq, H, Lk, Hkv, d, dt = 2, 50, 4, 90, 2, 64, torch.bfloat16
    if layout == "fused qkv":
        Lq = Lk
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), dt, 11)
    shift = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    if layout == "heads first":
        t |= {n: shift(t[n]) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")}
    elif layout == "fused kv":
        kv, dkv = torch.stack([t["k"], t["v"]], 2), torch.full((B, Lk, 2, Hkv, d), math.nan, dtype=dt, device="cuda")
        t |= {"k": kv[:, :, 0], "v": kv[:, :, 1], "dk": dkv[:, :, 0], "dv": dkv[:, :, 1]}
    elif layout == "fused qkv":
        x, dx = torch.cat([t["q"], t["k"], t["v"]], 2), torch.full((B, Lk, H + 2 * Hkv, d), math.nan, dtype=dt, device="cuda")
        for p, y in (("", x), ("d", dx)):
            t |= {p + "q": y[:, :, :H], p + "k": y[:, :, H:H + Hkv], p + "v": y[:, :, H + Hkv:]}
    elif layout == "broadcast keys":
        t["k"] = t["k"][:, :1].expand(B, Lk, Hkv, d)
    elif layout == "broadcast batch":
        t["k"], t["v"], t["do"] = t["k"][:1].expand(B, -1, -1, -1), t["v"][:1].expand(B, -1, -1, -1), t["do"][:1, :, :1].expand(B, -1, H, -1)
    else:
        wide = torch.full((B, Lk, Hkv, d + 24), math.nan, dtype=dt, device="cuda")
        wide[..., 8:8 + d] = t["k"]
        t["k"] = wide[..., 8:8 + d]
        out = torch.full((B, Lq, H, d + 8), 5.0, dtype=dt, device="cuda")
        t["o"] = out[..., 8:]
    run(M, t)
    compare(t, everything(B, Lq, Lk), layout)
    if layout == "sliced":
        assert (out[..., :8] == 5.0).all()


@pytest.mark.parametrize("shape", [(1, 1, 4, 5000, 1, 128), (1, 8, 8, 3001, 1, 64), (1, 150, 1, 2500, 1, 32), (1, 700, 8, 40, 1, 128)])
def test_pieces(M, shape):
    """Few rows over many keys and the other way round: the work is cut into pieces that are joined."""
    import torch
    B, Lq, H, Lk, Hkv, d = shape
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), torch.float16, 5)
    run(M, t)
    compare(t, everything(B, Lq, Lk), shape)
    lens = torch.tensor([Lk // 3], dtype=torch.int32)
    run(M, t, kv_lens=lens.cuda())
    compare(t, (torch.arange(Lk) < lens[:, None])[:, None].expand(B, Lq, Lk), shape)


@pytest.mark.parametrize("masking", ["none", "lens", "mask", "both"])
@pytest.mark.parametrize("shape", [(1, 270, 70, 200, 70, 64), (1, 260, 33, 1601, 33, 72), (3, 130, 40, 1100, 20, 128), (4, 40, 3, 1300, 3, 64), (5, 20, 2, 1700, 1, 32)])
def test_many_blocks(M, shape, masking):
    """Tiles of 256 rows, alone and with the keys in pieces, and batches whose lengths (none and one among them) share the pieces."""
    import torch
    B, Lq, H, Lk, Hkv, d = shape
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), torch.bfloat16, 13, train=False)
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
    t["k"][~keep.cuda()] = math.nan
    t["v"][~keep.cuda()] = math.inf
    run(M, t, **kw)
    compare(t, keep[:, None].expand(B, Lq, Lk), (shape, masking))


@pytest.mark.parametrize("masking", ["none", "lens", "mask"])
@pytest.mark.parametrize("shape", [(1, 600, 48, 1030, 48, 128), (2, 130, 72, 300, 9, 64), (2, 130, 72, 300, 9, 120)])
def test_many_blocks_backward(M, shape, masking):
    """Gradients over tiles of 256 rows or keys, alone and in pieces."""
    import torch
    B, Lq, H, Lk, Hkv, d = shape
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), torch.bfloat16, 17)
    kw, keep = {}, torch.ones(B, Lk, dtype=torch.bool)
    if masking == "lens":
        lens = torch.tensor([Lk - 5, 100][:B], dtype=torch.int32)
        kw["kv_lens"] = lens.cuda()
        keep &= torch.arange(Lk) < lens[:, None]
    elif masking == "mask":
        keep = torch.rand(B, Lk, generator=torch.Generator().manual_seed(6)) < 0.4
        kw["key_mask"] = keep.cuda()
    run(M, t, **kw)
    compare(t, keep[:, None].expand(B, Lq, Lk), (shape, masking))


def test_nothing_to_do(M):
    import torch
    t = tensors((2, 5, 2, 64), (2, 0, 1, 64), torch.bfloat16, 1)
    run(M, t)
    assert not t["o"].any() and not t["dq"].any() and (t["lse"] == -math.inf).all()
    t = tensors((2, 0, 2, 64), (2, 70, 1, 64), torch.bfloat16, 1)
    run(M, t)
    assert not t["dk"].any() and not t["dv"].any()


def test_scores_far_apart(M):
    """Scores that span hundreds, rising along the keys so that every tile raises the maximum; one row's scores all equal."""
    import torch
    t = tensors((1, 64, 2, 64), (1, 700, 1, 64), torch.bfloat16, 2)
    t["k"] = (t["k"].float().sign() * 0 + torch.linspace(0, 6, 700, device="cuda")[None, :, None, None]).to(torch.bfloat16)
    t["q"] = t["q"].abs()
    t["q"][0, 5] = 0
    run(M, t)
    compare(t, everything(1, 64, 700), "rising")


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", [(1, 1024, 2, 2048, 1, 64), (1, 700, 1, 2048, 1, 128), (1, 300, 40, 260, 40, 128)])
@pytest.mark.parametrize("gradients", ["small", "rising", "large"])
def test_gradients_of_all_sizes(M, shape, gradients, dtype):
    """dS far below float16's normal numbers, or thousands, or rising along rows and keys.  In the 2-norm three roundings of relative
    error at most u / 2 each reach dQ and dK (dS, the output, and O in D), two reach dV: 1.5 u covers them, and half a unit of the subnormal
    numbers on every element of the result."""
    import torch
    from attention_oracle import UNIT, TINY, attention
    B, Lq, H, Lk, Hkv, d = shape
    dt = getattr(torch, dtype)
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


def test_scale(M):
    import torch
    t = tensors((1, 20, 2, 32), (1, 50, 2, 32), torch.float16, 2)
    run(M, t, scale=0.7)
    compare(t, everything(1, 20, 50), "scale", scale=0.7)


def test_differences(M):
    """<gradient, w> against the difference quotient of the 64-bit loss sum(o * do) along w; the kernel's gradients may be off by
    what their bounds allow, elements' errors adding up as their absolute values at the worst."""
    import torch
    from attention_oracle import attention
    B, Lq, H, Lk, Hkv, d, eps = 1, 9, 4, 37, 2, 32, 1e-5
    t = tensors((B, Lq, H, d), (B, Lk, Hkv, d), torch.float16, 9)
    run(M, t)
    keep, scale = everything(B, Lq, Lk), d ** -0.5
    want = attention(t["q"], t["k"], t["v"], keep, scale, torch.float16, t["do"])
    x = {n: t[n].double().cpu() for n in ("q", "k", "v")}
    for n in x:
        w = torch.randn(x[n].shape, generator=torch.Generator().manual_seed(4), dtype=torch.float64)
        loss = [(attention(**{**x, n: x[n] + s * eps * w}, keep=keep, scale=scale, dtype=torch.float16)["o"][0] * t["do"].double().cpu()).sum().item() for s in (1, -1)]
        slope = (loss[0] - loss[1]) / (2 * eps)
        got = (t["d" + n].double().cpu() * w).sum().item()
        assert abs(got - slope) <= (want["d" + n][1] * w.abs()).sum().item() + 1e-6 * abs(slope) + 1e-6, n


def test_offsets_beyond_32_bits(M):
    """Batches that lie more than 2^32 elements apart."""
    import torch
    B, Lq, H, Lk, d, far = 2, 3, 2, 70, 64, (1 << 32) + 4096
    t = tensors((B, Lq, H, d), (B, Lk, H, d), torch.bfloat16, 3)
    pool = torch.empty(far + 2 * Lk * H * d, dtype=torch.bfloat16, device="cuda")
    for n, at in (("k", 0), ("v", Lk * H * d)):
        y = torch.as_strided(pool, (B, Lk, H, d), (far, H * d, d, 1), at)
        y.copy_(t[n])
        t[n] = y
    run(M, t)
    compare(t, everything(B, Lq, Lk), "far")


def test_stream_and_repeats(M):
    """On a stream of the caller's, behind work that is still running; the same bits every time."""
    import torch
    t = tensors((2, 300, 4, 64), (2, 500, 2, 64), torch.bfloat16, 6)
    run(M, t)
    first = {n: t[n].clone() for n in ("o", "lse", "dq", "dk", "dv")}
    stream = torch.cuda.Stream()
    late = {n: t[n].clone() for n in ("q", "k", "v")}
    M.mmee_set_stream(stream.cuda_stream)
    try:
        for n in late:
            t[n].zero_()
        for n in first:
            t[n].fill_(math.nan)
        torch.cuda.synchronize()
        a = M.attn(t["q"], t["k"], t["v"], t["o"], lse=t["lse"])
        a.use_workspace(torch.empty(M.mmee_attn_workspace(a, True), dtype=torch.uint8, device="cuda"))
        g = M.attn_grads(t["do"], t["dq"], t["dk"], t["dv"])
        with torch.cuda.stream(stream):
            torch.cuda._sleep(20_000_000)
            for n in late:
                t[n].copy_(late[n])
        M.mmee_attn_forward(a)
        M.mmee_attn_backward(a, g)
        stream.synchronize()
    finally:
        M.mmee_set_stream(None)
    for n in first:
        assert torch.equal(t[n], first[n]), n


def test_graph(M):
    """Captured once, replayed on other inputs with eager work in between."""
    import torch
    t = tensors((1, 40, 4, 64), (1, 900, 1, 64), torch.bfloat16, 8)
    run(M, t)
    a = M.attn(t["q"], t["k"], t["v"], t["o"], lse=t["lse"])
    a.use_workspace(torch.empty(M.mmee_attn_workspace(a, True), dtype=torch.uint8, device="cuda"))
    g = M.attn_grads(t["do"], t["dq"], t["dk"], t["dv"])
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    M.mmee_set_stream(stream.cuda_stream)
    try:
        with torch.cuda.graph(graph, stream=stream):
            M.mmee_attn_forward(a)
            M.mmee_attn_backward(a, g)
    finally:
        M.mmee_set_stream(None)
    for seed in (1, 2, 3):
        new = tensors((1, 40, 4, 64), (1, 900, 1, 64), torch.bfloat16, seed)
        for n in ("q", "k", "v", "do"):
            t[n].copy_(new[n])
        graph.replay()
        torch.cuda.synchronize()
        run(M, new)
        for n in ("o", "lse", "dq", "dk", "dv"):
            assert torch.equal(t[n], new[n]), (seed, n)
