"""One decoder layer takes in a batch of prompts, then checks a tree of drafted tokens: what the planner says of its chains, and the chains run.

The layer is three chains of two matrix products: attention of a prompt over itself (I = L = tokens) or of the drafted tokens over the
cache (I = tokens, L = cache), cross attention to an encoder's states (I = tokens, L = encoder's length), and a gated feed-forward block.  For each of
them the program asks for the mapping with the least energy on an accelerator, then runs the chain on this GPU, on a stream of its own:

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

    def __init__(self, batch, nodes, heads, kv_heads, head_dim, hidden, dtype=torch.bfloat16, seed=0, base=None):
        """base: of the frequencies by which queries and keys are rotated, after a norm of each head; None: neither."""
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        width = heads * head_dim
        weight = lambda rows, cols: (torch.randn(rows, cols, generator=gen, device="cuda") * cols ** -0.5).to(dtype)  # noqa: E731
        empty = lambda *shape: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        self.batch, self.nodes, self.heads, self.kv_heads, self.head_dim, self.hidden, self.width, self.dtype = batch, nodes, heads, kv_heads, head_dim, hidden, width, dtype
        self.w_qkv = weight((heads + 2 * kv_heads) * head_dim, width)
        self.w_self_out, self.w_cross_q, self.w_cross_out = (weight(width, width) for _ in range(3))
        self.w_gate, self.w_up, self.w_down = weight(hidden, width), weight(hidden, width), weight(width, hidden)
        self.freqs = self.q_weight = self.k_weight = None
        if base is not None:
            self.freqs = (base ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)).cuda()
            self.q_weight, self.k_weight = ((1 + 0.1 * torch.randn(head_dim, generator=gen, device="cuda")).to(dtype) for _ in range(2))
        self.tree_out, self.cross_out = empty(batch, nodes, heads, head_dim), empty(batch, nodes, heads, head_dim)

    def _run(self, args, size, call):
        args.use_workspace(torch.empty(size, dtype=torch.uint8, device="cuda"))
        call(args)

    def _norm(self, t):
        return torch.nn.functional.layer_norm(t.float(), (self.width,)).to(self.dtype)

    def prompt(self, x, starts, k_pages, v_pages, page_table, cache_lens, enc_k, enc_v, enc_starts):
        """x [tokens, width], packed prompts that begin at starts -> the layer's output; their keys and values go into the cache, whose cache_lens are 0.
        enc_k, enc_v: the encoder's states of each prompt, packed likewise, from enc_starts on."""
        T, H, Hkv, d = x.shape[0], self.heads, self.kv_heads, self.head_dim
        qkv = (self._norm(x) @ self.w_qkv.t()).view(T, H + 2 * Hkv, d)
        q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        if self.freqs is not None:
            at = torch.arange(T, device="cuda", dtype=torch.int32)
            positions = at - starts[torch.bucketize(at, starts, right=True) - 1]
            q_turned, k_turned = torch.empty_like(q), torch.empty_like(k)
            M.mmee_qk_rotate_forward(M.qk_rotate(q, k, q_turned, k_turned, self.freqs, positions, q_weight=self.q_weight, k_weight=self.k_weight))
            q, k = q_turned, k_turned
        M.mmee_cache_append_forward(M.cache_append(k, v, k_pages, v_pages, page_table, cache_lens, starts=starts))
        out = torch.empty(T, H, d, dtype=self.dtype, device="cuda")
        own = M.prompt_attn(q, k, v, out, starts)
        self._run(own, M.mmee_prompt_attn_workspace(own), M.mmee_prompt_attn_forward)
        x = x + out.view(T, -1) @ self.w_self_out.t()

        q = (self._norm(x) @ self.w_cross_q.t()).view(T, H, d)
        cross = M.prompt_attn(q, enc_k, enc_v, out, starts, kv_starts=enc_starts, causal=False)
        self._run(cross, M.mmee_prompt_attn_workspace(cross), M.mmee_prompt_attn_forward)
        x = x + out.view(T, -1) @ self.w_cross_out.t()
        return x + self._feed_forward(x)

    def _feed_forward(self, x):
        hidden, out = (torch.empty(x.shape[0], n, dtype=self.dtype, device="cuda") for n in (self.hidden, self.width))
        block = M.ffn(self._norm(x), self.w_gate, self.w_up, self.w_down, out, hidden)
        self._run(block, M.mmee_ffn_workspace(block), M.mmee_ffn_forward)
        return out

    def step(self, x, k_pages, v_pages, page_table, cache_lens, ancestors, enc_k, enc_v, enc_lens, positions=None):
        """x [batch, nodes, width] -> the layer's output; the drafted tokens' keys and values go into the cache behind what it holds.  positions int32
        [batch * nodes]: of the nodes in their sequences, which have branches; wanted where they are rotated.
        The library's stream (mmee_set_stream) has to be torch's current one."""
        B, n, H, Hkv, d = self.batch, self.nodes, self.heads, self.kv_heads, self.head_dim
        norm = self._norm
        qkv = (norm(x) @ self.w_qkv.t()).view(B * n, H + 2 * Hkv, d)
        q = qkv[:, :H]
        rotation = {}
        if self.freqs is not None:
            rotation = dict(q=q, q_out=torch.empty_like(q), freqs=self.freqs, positions=positions, q_weight=self.q_weight, k_weight=self.k_weight)
            q = rotation["q_out"]
        M.mmee_cache_append_forward(M.cache_append(qkv[:, H:H + Hkv], qkv[:, H + Hkv:], k_pages, v_pages, page_table, cache_lens, **rotation))
        tree = M.tree_attn(q.view(B, n, H, d), k_pages, v_pages, page_table, cache_lens, ancestors, self.tree_out)
        self._run(tree, M.mmee_tree_attn_workspace(tree), M.mmee_tree_attn_forward)
        x = x + self.tree_out.view(B, n, -1) @ self.w_self_out.t()

        q = (norm(x) @ self.w_cross_q.t()).view(B, n, H, d)
        cross = M.attn(q, enc_k, enc_v, self.cross_out, kv_lens=enc_lens)
        self._run(cross, M.mmee_attn_workspace(cross), M.mmee_attn_forward)
        x = x + self.cross_out.view(B, n, -1) @ self.w_cross_out.t()

        return x + self._feed_forward(x.view(B * n, -1)).view(B, n, -1)


def plan(batch, nodes, heads, head_dim, hidden, cache, encoder, hw):
    """The least-energy mappings of the layer's chains on an accelerator: [(name, Result)]."""
    chain = lambda many, I, K, L, J, softmax: dict(batch=many, I=I, K=K, L=L, J=J, word_bytes=2, tiling_mode=1, c_softmax=softmax)  # noqa: E731
    chains = {"prompt": chain(batch * heads, cache, head_dim, cache, head_dim, 10),
              "tree attention": chain(batch * heads, nodes, head_dim, cache, head_dim, 10),
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


def prompts(layer, lens, enc_lens, page=16, room=64, seed=2):
    """Prompts of these lengths, packed, the encoder's states of each, and an empty cache with room for so many tokens more."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    Hkv, d, B = layer.kv_heads, layer.head_dim, len(lens)
    r = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(layer.dtype)  # noqa: E731
    starts = lambda of: torch.tensor([0] + of, device="cuda").cumsum(0).to(torch.int32)  # noqa: E731
    width = -(-(max(lens) + room) // page)
    return dict(x=r(sum(lens), layer.width), starts=starts(lens), k_pages=r(B * width, page, Hkv, d), v_pages=r(B * width, page, Hkv, d),
                page_table=torch.randperm(B * width, generator=gen, device="cuda").to(torch.int32).view(B, width),
                cache_lens=torch.zeros(B, dtype=torch.int32, device="cuda"), enc_k=r(sum(enc_lens), Hkv, d), enc_v=r(sum(enc_lens), Hkv, d), enc_starts=starts(enc_lens))


def main():
    batch, nodes, heads, kv_heads, head_dim, hidden, cache, encoder = 8, 24, 12, 4, 64, 3072, 512, 300
    for name, r in plan(batch, nodes, heads, head_dim, hidden, cache, encoder, CONFIGS["bert"]["hw"]):
        m = r.best
        print("%-16s tiles %s, loops %s, levels %s, %s: %.3g pJ, %d DRAM words an instance" % (
            name, list(m.xG), "".join("iklj"[o] for o in m.order), list(m.level), "fused" if m.fused else "unfused", r.cost.energy_pj, r.cost.da_words))
    layer = Layer(batch, nodes, heads, kv_heads, head_dim, hidden)
    batch_in = inputs(layer, cache, encoder)
    lens = [cache * (i + 1) // batch for i in range(batch)]
    rotated = Layer(batch, nodes, heads, kv_heads, head_dim, hidden, base=10000.0)
    prompt_in = prompts(rotated, lens, [encoder - 7 * i for i in range(batch)])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    M.mmee_set_stream(stream.cuda_stream)               # once for all calls
    with torch.cuda.stream(stream):
        rotated.prompt(**prompt_in)
        prompt_begin, prompt_end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        prompt_begin.record()
        z = rotated.prompt(**prompt_in)
        prompt_end.record()
        y = layer.step(**batch_in)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(20):
            y = layer.step(**batch_in)
        end.record()
    end.synchronize()
    M.mmee_set_stream(None)
    print("%d prompts of %d to %d tokens: %.3f ms, output %s, finite: %s" % (
        batch, lens[0], lens[-1], prompt_begin.elapsed_time(prompt_end), tuple(z.shape), bool(torch.isfinite(z).all())))
    print("a step of %d trees of %d tokens: %.3f ms, output %s, finite: %s" % (batch, nodes, begin.elapsed_time(end) / 20, tuple(y.shape), bool(torch.isfinite(y).all())))


if __name__ == "__main__":
    main()
