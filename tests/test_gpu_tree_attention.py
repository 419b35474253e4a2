"""Tree attention over a paged cache against a plain 64-bit form: trees from one node to many, pages that end inside a tile, odd lengths,
shared pages, rows that see nothing, bad page numbers, long contexts, offsets beyond 32 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2604_03446_amd as mod
    return mod


def words_of(sees):
    """[B, n, n] truth values -> int64 bit patterns."""
    import torch
    B, n, _ = sees.shape
    w = (n + 63) // 64
    bits = torch.zeros(B, n, w * 64, dtype=torch.long)
    bits[:, :, :n] = sees
    return (bits.view(B, n, w, 64) << torch.arange(64)).sum(-1)


def random_tree(B, n, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    sees = torch.zeros(B, n, n, dtype=torch.bool)
    for b in range(B):
        for i in range(n):
            if i and torch.rand((), generator=g) < 0.9:
                sees[b, i] = sees[b, int(torch.randint(0, i, (), generator=g))]
            sees[b, i, i] = True
    return sees


def build(B, n, H, Hkv, d, page, lens, dtype, seed=0, spare=3, sees=None, fill=math.nan):
    """Tensors of a call; cache positions that no sequence holds are `fill`."""
    import torch
    g = torch.Generator().manual_seed(seed)
    width = max((l + n + page - 1) // page for l in lens) + 1
    pages = B * width + spare
    pool = torch.full((pages, 2, page, Hkv, d), fill, dtype=dtype)
    table = torch.randperm(pages, generator=g)[:B * width].view(B, width).to(torch.int32)
    k, v = (torch.randn(B, max(lens) + n, Hkv, d, generator=g).to(dtype) for _ in range(2))
    for b, l in enumerate(lens):
        for p in range(l + n):
            pool[table[b, p // page], 0, p % page] = k[b, p]
            pool[table[b, p // page], 1, p % page] = v[b, p]
    t = {"q": torch.randn(B, n, H, d, generator=g).to(dtype).cuda(), "pool": pool.cuda(), "table": table.cuda(), "k": k, "v": v,
         "lens": torch.tensor(lens, dtype=torch.int32).cuda(), "sees": random_tree(B, n, seed) if sees is None else sees,
         "o": torch.full((B, n, H, d), math.nan, dtype=dtype).cuda(), "lse": torch.full((B, H, n), math.nan).cuda()}
    t["k_pages"], t["v_pages"] = t["pool"][:, 0], t["pool"][:, 1]
    return t


def run(M, t, counts=None, **kw):
    import torch
    a = M.tree_attn(t["q"], t["k_pages"], t["v_pages"], t["table"], t["lens"], words_of(t["sees"]).cuda(), t["o"], lse=t["lse"],
                    node_counts=None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda(), **kw)
    a.use_workspace(torch.full((M.mmee_tree_attn_workspace(a),), 255, dtype=torch.uint8, device="cuda"))
    M.mmee_tree_attn_forward(a)
    torch.cuda.synchronize()


def keeps(t, counts=None):
    import torch
    B, n, L = t["q"].shape[0], t["q"].shape[1], t["k"].shape[1]
    keep = torch.zeros(B, n, L, dtype=torch.bool)
    for b, l in enumerate(t["lens"].tolist()):
        c = n if counts is None else max(0, min(n, counts[b]))
        keep[b, :c, :l] = True
        keep[b, :c, l:l + c] = t["sees"][b, :c, :c]
    return keep


def compare(t, keep, where):
    from attention_oracle import attention, check
    want = attention(t["q"], t["k"], t["v"], keep, t["q"].shape[3] ** -0.5, t["q"].dtype)
    for name in ("o", "lse"):
        check(t[name], want[name], (where, name))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("n,H,Hkv,d,page,lens", [
    (1, 1, 1, 32, 16, [0]), (1, 4, 1, 64, 1, [5, 64]), (7, 8, 2, 128, 16, [100, 3, 57]), (8, 4, 4, 64, 32, [64, 31, 33]), (13, 4, 1, 96, 64, [127, 0]),
    (33, 2, 2, 128, 16, [95, 129]), (63, 8, 2, 80, 128, [40, 200]), (64, 1, 1, 40, 16, [63, 64, 65]), (65, 2, 1, 64, 8, [1, 120]), (100, 4, 2, 128, 16, [300]),
    (150, 1, 1, 8, 4, [77]), (200, 2, 1, 64, 256, [513, 20])])
def test_trees(M, n, H, Hkv, d, page, lens, dtype):
    import torch
    t = build(len(lens), n, H, Hkv, d, page, lens, getattr(torch, dtype), seed=n)
    run(M, t)
    compare(t, keeps(t), (n, page))


@pytest.mark.parametrize("n,counts", [(9, [9, 0, 1, 40, -2]), (70, [70, 64, 65, 3, 0])])
def test_node_counts(M, n, counts):
    """Fewer nodes than there is room for: what lies behind them counts for nothing; rows past the count give zeros."""
    import torch
    t = build(5, n, 4, 2, 64, 16, [33, 64, 0, 90, 10], torch.bfloat16, seed=2)
    for b, c in enumerate(counts):
        for p in range(int(t["lens"][b]) + max(0, min(n, c)), int(t["lens"][b]) + n):
            t["pool"][t["table"][b, p // 16], :, p % 16] = math.nan
    run(M, t, counts)
    compare(t, keeps(t, counts), counts)


def test_rows_that_see_nothing(M):
    """An empty ancestor row over an empty cache; a row that does not see itself; bits past the nodes do not matter."""
    import torch
    sees = random_tree(2, 5, 1)
    sees[:, 2] = False
    sees[0, 3, 3] = False
    t = build(2, 5, 2, 1, 64, 16, [0, 40], torch.float16, sees=sees)
    run(M, t)
    compare(t, keeps(t), "nothing")
    assert not t["o"][0, 2].any() and (t["lse"][0, :, 2] == -math.inf).all()
    first = t["o"].clone()
    words = words_of(sees) | torch.tensor(-1 << 5)
    a = M.tree_attn(t["q"], t["k_pages"], t["v_pages"], t["table"], t["lens"], words.cuda(), t["o"])
    a.use_workspace(torch.empty(M.mmee_tree_attn_workspace(a), dtype=torch.uint8, device="cuda"))
    M.mmee_tree_attn_forward(a)
    assert torch.equal(t["o"], first)


@pytest.mark.parametrize("n,H", [(4, 2), (40, 4)])
def test_pages_that_are_not_there(M, n, H):
    """Positions of pages outside the pool count as masked; lengths beyond the table are clamped."""
    import torch
    t = build(2, n, H, 1, 64, 16, [100, 100], torch.bfloat16, seed=4)
    t["table"][0, 2] = -1
    t["table"][1, 1] = t["pool"].shape[0]
    t["table"][1, 3] = 0x7fffffff
    run(M, t)
    keep = keeps(t)
    keep[0, :, 32:48] = False
    keep[1, :, 16:32] = False
    keep[1, :, 48:64] = False
    compare(t, keep, "pages")
    narrow = dict(t, table=t["table"][:, :4].contiguous(), o=t["o"].clone(), lse=t["lse"].clone())
    narrow["table"][:] = torch.arange(8, dtype=torch.int32).view(2, 4)
    narrow["pool"] = torch.randn_like(t["pool"].float()).to(torch.bfloat16)
    narrow["k_pages"], narrow["v_pages"] = narrow["pool"][:, 0], narrow["pool"][:, 1]
    narrow["k"] = narrow["pool"][:8, 0].reshape(2, 64, 1, 64).cpu()
    narrow["v"] = narrow["pool"][:8, 1].reshape(2, 64, 1, 64).cpu()
    run(M, narrow)
    compare(narrow, torch.ones(2, n, 64, dtype=torch.bool), "clamped")


@pytest.mark.parametrize("n,H,Hkv", [(1, 8, 1), (16, 4, 1), (60, 8, 2)])
def test_long_contexts_in_pieces(M, n, H, Hkv):
    import torch
    t = build(2, n, H, Hkv, 64, 128, [6000, 411], torch.float16, seed=6)
    run(M, t)
    compare(t, keeps(t), n)


@pytest.mark.parametrize("n,H,Hkv,d,page,lens", [
    (140, 72, 36, 64, 16, [300, 40]), (70, 16, 4, 128, 128, [4000, 700]), (9, 8, 2, 64, 32, [1500, 0, 3000, 1, 511]), (50, 6, 3, 96, 64, [0, 2500, 64])])
def test_many_blocks(M, n, H, Hkv, d, page, lens):
    """Tiles of 256 rows, alone and in pieces; batches whose contexts (none and one among them) share the pieces."""
    import torch
    t = build(len(lens), n, H, Hkv, d, page, lens, torch.bfloat16, seed=n)
    run(M, t)
    compare(t, keeps(t), (n, lens))


@pytest.mark.parametrize("page", [1, 2, 8, 64])
@pytest.mark.parametrize("n,H,Hkv,d,counts", [(40, 8, 2, 128, [40, 17, 0]), (3, 4, 1, 64, [3, 1, 2]), (20, 4, 2, 64, [5, 20, 20]), (5, 6, 6, 32, [4, 5, 1])])
def test_long_tables(M, n, H, Hkv, d, counts, page):
    """Contexts of many pages, fewer nodes than there is room for, a page of the middle that is not there."""
    import torch
    t = build(3, n, H, Hkv, d, page, [1200, 900, 1037], torch.bfloat16, seed=page)
    t["table"][1, 512 // page] = -5
    run(M, t, counts)
    keep = keeps(t, counts)
    keep[1, :, 512 // page * page:(512 // page + 1) * page] = False
    compare(t, keep, (n, page))


def test_shared_pages_and_strides(M):
    """Sequences that begin with the same pages; heads before tokens inside a page; a table with room behind its rows."""
    import torch
    t = build(2, 6, 4, 2, 64, 16, [64, 64], torch.bfloat16, seed=3)
    t["table"][1, :4] = t["table"][0, :4]
    t["k"][1, :64], t["v"][1, :64] = t["k"][0, :64], t["v"][0, :64]
    pool = t["pool"].transpose(2, 3).contiguous().transpose(2, 3)
    t["k_pages"], t["v_pages"] = pool[:, 0], pool[:, 1]
    wide = torch.full((2, t["table"].shape[1] + 5), -7, dtype=torch.int32, device="cuda")
    wide[:, :-5] = t["table"]
    t["table"] = wide[:, :-5]
    run(M, t)
    compare(t, keeps(t), "shared")


def test_offsets_beyond_32_bits(M):
    """A pool of more than 2^32 elements; the sequence's pages lie at both of its ends."""
    import torch
    n, Hkv, d, page = 5, 8, 128, 64
    t = build(1, n, 8, Hkv, d, page, [200], torch.bfloat16, seed=8)
    size = 2 * page * Hkv * d
    pages = (1 << 32) // size + 10
    pool = torch.empty(pages, 2, page, Hkv, d, dtype=torch.bfloat16, device="cuda")
    table = t["table"].clone()
    for j in range(table.shape[1]):
        to = j if j % 2 else pages - 1 - j
        pool[to] = t["pool"][int(t["table"][0, j])]
        table[0, j] = to
    t |= {"pool": pool, "table": table, "k_pages": pool[:, 0], "v_pages": pool[:, 1]}
    run(M, t)
    compare(t, keeps(t), "far")


def test_nothing_to_do(M):
    import torch
    t = build(1, 3, 2, 1, 64, 16, [0], torch.bfloat16)
    run(M, t, [0])
    assert not t["o"].any() and (t["lse"] == -math.inf).all()
