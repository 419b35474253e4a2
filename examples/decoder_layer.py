"""One decoder layer checks a tree of drafted tokens: what the planner says of its chains, and the chains run.

The layer is three chains of two matrix products: attention of the drafted tokens over the cache (I = tokens, L = cache),
cross attention to an encoder's states (I = tokens, L = encoder's length), and a gated feed-forward block.  For each of them
the program asks for the mapping with the least energy on an accelerator, then runs the chain on this GPU, on a stream of its own:

    python3 examples/decoder_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_03446_amd as M  # noqa: E402  (after torch, whose HIP runtime it uses)
from inputs import CONFIGS  # noqa: E402


class Layer:
    """Weights of a layer of `heads` query heads over `kv_heads` shared ones, and the buffers of a step of `batch` trees of `nodes` tokens."""

    def __init__(self, batch, nodes, heads, kv_heads, head_dim, hidden, dtype=torch.bfloat16, seed=0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        width = heads * head_dim
        weight = lambda rows, cols: (torch.randn(rows, cols, generator=gen, device="cuda") * cols ** -0.5).to(dtype)  # noqa: E731
        empty = lambda *shape: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        self.batch, self.nodes, self.heads, self.kv_heads, self.head_dim, self.hidden, self.width, self.dtype = batch, nodes, heads, kv_heads, head_dim, hidden, width, dtype
        self.w_qkv = weight((heads + 2 * kv_heads) * head_dim, width)
        self.w_self_out, self.w_cross_q, self.w_cross_out = (weight(width, width) for _ in range(3))
        self.w_gate, self.w_up, self.w_down = weight(hidden, width), weight(hidden, width), weight(width, hidden)
        self.tree_out, self.cross_out = empty(batch, nodes, heads, head_dim), empty(batch, nodes, heads, head_dim)
        self.ffn_hidden, self.ffn_out = empty(batch * nodes, hidden), empty(batch * nodes, width)

    def _run(self, args, size, call):
        args.use_workspace(torch.empty(size, dtype=torch.uint8, device="cuda"))
        call(args)

    def step(self, x, k_pages, v_pages, page_table, cache_lens, ancestors, enc_k, enc_v, enc_lens):
        """x [batch, nodes, width] -> the layer's output; the drafted tokens' keys and values go into the cache behind what it holds.
        The library's stream (mmee_set_stream) has to be torch's current one."""
        B, n, H, Hkv, d = self.batch, self.nodes, self.heads, self.kv_heads, self.head_dim
        norm = lambda t: torch.nn.functional.layer_norm(t.float(), (self.width,)).to(self.dtype)  # noqa: E731
        qkv = (norm(x) @ self.w_qkv.t()).view(B, n, H + 2 * Hkv, d)
        place = cache_lens[:, None].long() + torch.arange(n, device="cuda")
        page = page_table.gather(1, place // k_pages.shape[1]).long()
        k_pages[page, place % k_pages.shape[1]] = qkv[:, :, H:H + Hkv]
        v_pages[page, place % k_pages.shape[1]] = qkv[:, :, H + Hkv:]
        tree = M.tree_attn(qkv[:, :, :H], k_pages, v_pages, page_table, cache_lens, ancestors, self.tree_out)
        self._run(tree, M.mmee_tree_attn_workspace(tree), M.mmee_tree_attn_forward)
        x = x + self.tree_out.view(B, n, -1) @ self.w_self_out.t()

        q = (norm(x) @ self.w_cross_q.t()).view(B, n, H, d)
        cross = M.attn(q, enc_k, enc_v, self.cross_out, kv_lens=enc_lens)
        self._run(cross, M.mmee_attn_workspace(cross), M.mmee_attn_forward)
        x = x + self.cross_out.view(B, n, -1) @ self.w_cross_out.t()

        block = M.ffn(norm(x).view(B * n, -1), self.w_gate, self.w_up, self.w_down, self.ffn_out, self.ffn_hidden)
        self._run(block, M.mmee_ffn_workspace(block), M.mmee_ffn_forward)
        return x + self.ffn_out.view(B, n, -1)


def plan(batch, nodes, heads, head_dim, hidden, cache, encoder, hw):
    """The least-energy mappings of the layer's chains on an accelerator: [(name, Result)]."""
    chain = lambda many, I, K, L, J, softmax: dict(batch=many, I=I, K=K, L=L, J=J, word_bytes=2, tiling_mode=1, c_softmax=softmax)  # noqa: E731
    chains = {"tree attention": chain(batch * heads, nodes, head_dim, cache, head_dim, 10),
              "cross attention": chain(batch * heads, nodes, head_dim, encoder, head_dim, 10),
              "feed-forward": chain(1, batch * nodes, heads * head_dim, hidden, heads * head_dim, 0)}
    return [(name, M.mmee_chain_search_multi(c, hw, [M.OBJ_ENERGY])[0]) for name, c in chains.items()]


def inputs(layer, cache, encoder, page=16, seed=1):
    """A batch in the middle of decoding: caches of different lengths in pages in no order, random trees, padded encoder states."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, n, Hkv, d, dtype = layer.batch, layer.nodes, layer.kv_heads, layer.head_dim, layer.dtype
    r = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(dtype)  # noqa: E731
    width = -(-(cache + n) // page)
    sees = torch.eye(n, dtype=torch.bool).repeat(B, 1, 1)
    host = torch.Generator().manual_seed(seed)
    for i in range(1, n):
        parent = torch.randint(0, i, (B,), generator=host)
        sees[:, i] |= sees[torch.arange(B), parent]
    bits = torch.zeros(B, n, -(-n // 64) * 64, dtype=torch.long)
    bits[:, :, :n] = sees
    return dict(x=r(B, n, layer.width), k_pages=r(B * width, page, Hkv, d), v_pages=r(B * width, page, Hkv, d),
                page_table=torch.randperm(B * width, generator=gen, device="cuda").to(torch.int32).view(B, width),
                cache_lens=torch.randint(cache // 2, cache + 1, (B,), generator=gen, device="cuda").to(torch.int32),
                ancestors=(bits.view(B, n, -1, 64) << torch.arange(64)).sum(-1).cuda(), enc_k=r(B, encoder, Hkv, d), enc_v=r(B, encoder, Hkv, d),
                enc_lens=torch.randint(1, encoder + 1, (B,), generator=gen, device="cuda").to(torch.int32))


def main():
    batch, nodes, heads, kv_heads, head_dim, hidden, cache, encoder = 8, 24, 12, 4, 64, 3072, 512, 300
    for name, r in plan(batch, nodes, heads, head_dim, hidden, cache, encoder, CONFIGS["bert"]["hw"]):
        m = r.best
        print("%-16s tiles %s, loops %s, levels %s, %s: %.3g pJ, %d DRAM words an instance" % (
            name, list(m.xG), "".join("iklj"[o] for o in m.order), list(m.level), "fused" if m.fused else "unfused", r.cost.energy_pj, r.cost.da_words))
    layer = Layer(batch, nodes, heads, kv_heads, head_dim, hidden)
    batch_in = inputs(layer, cache, encoder)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    M.mmee_set_stream(stream.cuda_stream)               # once for all calls
    with torch.cuda.stream(stream):
        y = layer.step(**batch_in)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(20):
            y = layer.step(**batch_in)
        end.record()
    end.synchronize()
    M.mmee_set_stream(None)
    print("a step of %d trees of %d tokens: %.3f ms, output %s, finite: %s" % (batch, nodes, begin.elapsed_time(end) / 20, tuple(y.shape), bool(torch.isfinite(y).all())))


if __name__ == "__main__":
    main()
