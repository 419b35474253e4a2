"""Appending keys and values to a paged cache, with norms and rotation, against a plain 64-bit form: packed and even batches, counts, positions,
pages that end inside a sequence's tokens, pages that are not there, layouts, what stays untouched, streams, graphs, and the tree attention that reads it."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


def tensors(lens, held, H, Hkv, d, rot, page, dtype, seed, norm=True, starts=True, extra=0):
    """lens new tokens behind held cached ones of each sequence; `extra` tokens of no sequence behind them."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)  # noqa: E731
    T, B = sum(lens) + extra, len(lens)
    width = max(-(-(n + max(0, c)) // page) for n, c in zip(lens, held))
    x = r(T, H + 2 * Hkv, d)
    t = {"q": x[:, :H], "k": x[:, H:H + Hkv], "v": x[:, H + Hkv:], "q_out": torch.full((T, H, d), 3.0, dtype=dtype, device="cuda")}
    pool = torch.full((B * width + 3, 2, page, Hkv, d), -5.0, dtype=dtype, device="cuda")
    t["k_pages"], t["v_pages"] = pool[:, 0], pool[:, 1]
    t["page_table"] = torch.randperm(B * width + 3, generator=g, device="cuda")[:B * width].to(torch.int32).view(B, width)
    t["cache_lens"] = torch.tensor(held, dtype=torch.int32, device="cuda")
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    t["starts"] = torch.tensor(at, dtype=torch.int32, device="cuda") if starts else None
    t["counts"] = None
    t["freqs"] = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).cuda() if rot else None
    t["positions"] = t["axis_of"] = None
    for n in ("q", "k"):
        t[n + "_weight"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dtype) if norm else None
    if not H:
        t["q"] = t["q_out"] = t["q_weight"] = None
    return t


def call(M, t, **kw):
    return M.cache_append(**{n: t[n] for n in ("k", "v", "k_pages", "v_pages", "page_table", "cache_lens", "starts", "counts", "q", "q_out", "freqs", "positions", "axis_of",
                                               "q_weight", "k_weight")}, **kw)


def expected(t, lens, pairs="halves", eps=1e-6):
    """(values, bounds) of q_out and the pages: what was there, and, token by token, what is put there."""
    import torch
    from rotation_oracle import angles, rotation
    k, v = t["k_pages"].cpu().double(), t["v_pages"].cpu().double()
    q = t["q_out"].cpu().double() if t["q"] is not None else None
    off_k, off_q = torch.zeros_like(k), None if q is None else torch.zeros_like(q)
    P, page = k.shape[:2]
    held, table = t["cache_lens"].tolist(), t["page_table"].tolist()
    at = 0
    for b, n in enumerate(lens):
        for j in range(n):
            token = at + j
            if t["counts"] is not None and j >= int(t["counts"][b]):
                continue
            place = max(0, held[b]) + j
            where = torch.tensor([place]) if t["positions"] is None else t["positions"][..., token:token + 1].cpu()
            angle = torch.zeros(1, 1, 0, dtype=torch.float64) if t["freqs"] is None else angles(t["freqs"], where, t["axis_of"])
            if q is not None:
                y, off = rotation(t["q"][token:token + 1], t["q_weight"], angle, eps, pairs)["y"]
                q[token], off_q[token] = y[0], off[0]
            to = table[b][place // page] if place // page < len(table[b]) else -1
            if 0 <= to < P:
                y, off = rotation(t["k"][token:token + 1], t["k_weight"], angle, eps, pairs)["y"]
                k[to, place % page], off_k[to, place % page] = y[0], off[0]
                v[to, place % page] = t["v"][token].cpu().double()
        at += n
    out = {"k_pages": (k, off_k), "v_pages": (v, torch.zeros_like(v))}
    return out if q is None else out | {"q_out": (q, off_q)}


def run_and_compare(M, t, lens, where, **kw):
    import torch
    from attention_oracle import check
    want = expected(t, lens, kw.get("pairs", "halves"))
    M.mmee_cache_append_forward(call(M, t, **kw))
    torch.cuda.synchronize()
    for name, value in want.items():
        check(t[name], value, (where, name))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("lens,held,H,Hkv,d,rot,page", [
    ([1], [0], 1, 1, 8, 0, 1), ([1], [37], 32, 8, 128, 128, 16), ([1] * 5, [0, 15, 16, 17, 200], 4, 2, 64, 64, 16), ([3, 0, 1, 40, 0], [5, 9, 63, 60, 2], 6, 3, 80, 32, 32),
    ([70, 1, 17], [0, 100, 31], 0, 2, 96, 96, 64), ([0, 5], [3, 3], 2, 2, 256, 64, 8), ([9, 9], [7, 1], 3, 1, 24, 16, 4), ([100], [1], 12, 12, 64, 64, 128)])
def test_shapes(M, lens, held, H, Hkv, d, rot, page, dtype):
    import torch
    for norm in (True, False):
        for pairs in ("halves", "neighbours"):
            t = tensors(lens, held, H, Hkv, d, rot, page, getattr(torch, dtype), len(lens) + d, norm=norm)
            run_and_compare(M, t, lens, (lens, d, norm, pairs), pairs=pairs)


def test_many_sequences(M):
    """More of them than a wave looks at in one go, empty ones among them; tokens of no sequence before and behind."""
    import torch
    lens = [i * 7 % 4 for i in range(300)]
    t = tensors(lens, [i * 3 % 40 for i in range(300)], 2, 1, 32, 32, 16, torch.bfloat16, 5, extra=6)
    t["starts"] += 2
    before = t["q_out"].clone()
    shifted = dict(t)
    shifted |= {n: t[n][2:-4] for n in ("q", "k", "v", "q_out")}
    want = expected(shifted, lens)
    M.mmee_cache_append_forward(call(M, t))
    torch.cuda.synchronize()
    from attention_oracle import check
    for name, value in want.items():
        check(shifted[name], value, name)
    assert torch.equal(t["q_out"][:2], before[:2]) and torch.equal(t["q_out"][-4:], before[-4:])


def test_even_batches_counts_and_bad_pages(M):
    """As many tokens of every sequence, of which only some count; pages outside the pool and positions past the table are not written."""
    import torch
    B, n = 6, 5
    t = tensors([n] * B, [0, 14, 30, -4, 16, 3], 4, 2, 64, 64, 16, torch.float16, 3, starts=False)
    t["counts"] = torch.tensor([5, 0, -1, 3, 9, 1], dtype=torch.int32, device="cuda")
    run_and_compare(M, t, [n] * B, "counts")
    t = tensors([n] * B, [0, 14, 30, 12, 16, 3], 4, 2, 64, 64, 16, torch.float16, 4, starts=False)
    t["page_table"][1, 1], t["page_table"][2, 2], t["page_table"][3, 0] = -1, 2 ** 30, t["k_pages"].shape[0]
    t["page_table"] = t["page_table"][:, :2]
    t["page_table"][5, 0] = -2 ** 31
    run_and_compare(M, t, [n] * B, "bad pages")
    t["cache_lens"][:] = 2 ** 31 - 3
    run_and_compare(M, t, [n] * B, "past every table")


@pytest.mark.parametrize("axes", [1, 3])
def test_positions(M, axes):
    """Positions of their own: drafted trees, images."""
    import torch
    lens = [7, 12, 1]
    t = tensors(lens, [3, 20, 0], 4, 4, 64, 48, 16, torch.bfloat16, 6)
    t["positions"] = torch.randint(-50, 70000, (axes, 20) if axes > 1 else (20,), generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()
    t["axis_of"] = (torch.arange(24) % 3).to(torch.uint8).cuda() if axes > 1 else None
    run_and_compare(M, t, lens, axes)


def test_starts_out_of_order_stay_within(M):
    """Starts that do not ascend, and beyond the tokens: pages that no sequence holds stay as they were, whatever else is written."""
    import torch
    lens = [4, 4, 4, 4]
    t = tensors(lens, [0, 0, 0, 0], 2, 1, 32, 32, 16, torch.bfloat16, 7)
    for starts in ([9, 3, 12, 1, 16], [0, -5, 100, 8, 4], [-2 ** 31, 2 ** 31 - 1, 0, 5, 2 ** 31 - 1]):
        t["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        M.mmee_cache_append_forward(call(M, t))
        torch.cuda.synchronize()
    free = torch.ones(t["k_pages"].shape[0], dtype=torch.bool)
    free[t["page_table"].cpu().long().flatten()] = False
    assert free.any() and (t["v_pages"][free.cuda()] == -5.0).all() and (t["k_pages"][free.cuda()] == -5.0).all()


def test_streams_and_graphs(M):
    """A decoding step captured once and replayed as the lengths grow."""
    import torch
    from attention_oracle import check
    B = 5
    t = tensors([1] * B, [30, 0, 15, 7, 31], 4, 2, 64, 64, 16, torch.bfloat16, 8, starts=False)
    t["page_table"] = torch.arange(B * 3, dtype=torch.int32, device="cuda").view(B, 3)
    t["k_pages"], t["v_pages"] = (torch.zeros(B * 3, 16, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    M.mmee_set_stream(stream.cuda_stream)
    try:
        c = call(M, t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            M.mmee_cache_append_forward(c)
        for step in range(4):
            want = expected(t, [1] * B)
            torch.cuda.synchronize()
            with torch.cuda.stream(stream):
                graph.replay()
            stream.synchronize()
            for name, value in want.items():
                check(t[name], value, (step, name))
            t["cache_lens"] += 1
            t["q"].add_(0.25)
            t["k"].neg_()
    finally:
        M.mmee_set_stream(None)


def test_tree_attention_reads_what_was_appended(M):
    """Single tokens and trees: appended, then attended to through the same table, against 64-bit attention over the same pages."""
    import torch
    from attention_oracle import attention, check
    B, n, H, Hkv, d, page = 3, 9, 8, 2, 64, 16
    t = tensors([n] * B, [0, 40, 23], H, Hkv, d, d, page, torch.bfloat16, 9, starts=False)
    t["k_pages"].normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    t["v_pages"].normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    depth = torch.tensor([0, 1, 1, 2, 2, 2, 3, 3, 4])
    t["positions"] = (t["cache_lens"].cpu()[:, None] + depth).to(torch.int32).flatten().cuda()
    t["counts"] = torch.tensor([9, 4, 9], dtype=torch.int32, device="cuda")
    M.mmee_cache_append_forward(call(M, t))
    sees = torch.tril(torch.ones(n, n, dtype=torch.bool)) & (torch.rand(n, n, generator=torch.Generator().manual_seed(3)) < 0.5) | torch.eye(n, dtype=torch.bool)
    bits = (sees.long() << torch.arange(n)).sum(1).expand(B, n).contiguous()[..., None].cuda()
    o = torch.full((B, n, H, d), math.nan, dtype=torch.bfloat16, device="cuda")
    q = t["q_out"].view(B, n, H, d)
    a = M.tree_attn(q, t["k_pages"], t["v_pages"], t["page_table"], t["cache_lens"], bits, o, node_counts=t["counts"])
    a.use_workspace(torch.empty(M.mmee_tree_attn_workspace(a), dtype=torch.uint8, device="cuda"))
    M.mmee_tree_attn_forward(a)
    torch.cuda.synchronize()
    for b in range(B):
        held, count = int(t["cache_lens"][b]), int(t["counts"][b])
        k, v = (t[name][t["page_table"][b].long()].flatten(0, 1)[None, :held + count] for name in ("k_pages", "v_pages"))
        keep = torch.cat([torch.ones(count, held, dtype=torch.bool), sees[:count, :count]], 1)
        check(o[b:b + 1, :count], attention(q[b:b + 1, :count], k, v, keep[None], d ** -0.5, torch.bfloat16)["o"], b)
        assert not o[b, count:].any()
